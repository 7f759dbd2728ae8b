// Class log probabilities: the top's candidates, rows in registers, wide rows and their parts, the entry points (see logprob.cuh).
#include "logprob.cuh"

namespace {

// ---- the top: candidates of a warp ---------------------------------------------------------------------------------------------------------------------

// A warp's candidates: `count` keys in shared memory.  After a sort they are the k best so far; limit: the k-th best's key (0: fewer than k yet), above: its value.
struct Candidates {
  u64* list;
  int count;
  u64 limit;
  float above;
};
// Keeps the best k, in order.
__device__ __noinline__ void sort_candidates(Candidates& c, int k) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  const int count = c.count;
  const u64 a = lane < count ? c.list[lane] : 0, b = lane + 32 < count ? c.list[lane + 32] : 0;
  int ra = 0, rb = 0;
  for (int i = 0; i < count; ++i) { const u64 o = c.list[i]; ra += o > a; rb += o > b; }
  __syncwarp();
  if (a && ra < k) c.list[ra] = a;
  if (b && rb < k) c.list[rb] = b;
  __syncwarp();
  c.count = min(k, count);
  if (c.count == k) { c.limit = c.list[k - 1]; c.above = key_value(c.limit); }
}
// Puts down the lanes' keys that are better than the limit (0: none).
__device__ __noinline__ void put_candidates(Candidates& c, u64 key, int k) {
  const unsigned yes = __ballot_sync(0xffffffffu, key > c.limit);
  if (!yes) return;
  if (key > c.limit) c.list[c.count + __popc(yes & ((1u << (threadIdx.x & 31)) - 1))] = key;
  c.count += __popc(yes);
  if (c.count > LIST - 32) sort_candidates(c, k);
}
// The lane's place among the lanes' maxima.  The k-th largest has k values at least that are not below it: what is below it is not among the best k.
__device__ __noinline__ int rank_of_lanes(float mine) {
  const int lane = threadIdx.x & 31;
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < 32; ++i) { const float o = __shfl_sync(0xffffffffu, mine, i); rank += o > mine || (o == mine && i < lane); }
  return rank;
}

// ---- rows in the registers of a team of lanes ----------------------------------------------------------------------------------------------------------

// A row is on LANES lanes with up to W words each: word i of lane l is word i LANES + l of the row.
template <class T, bool PAIRS, int LANES, int W, int MODE>
__global__ void __launch_bounds__(32 * WARPS) team_kernel(const Args a) {
  using Wd = typename Word<T, PAIRS>::type;
  constexpr int NW = Word<T, PAIRS>::n, TEAMS = 32 * WARPS / LANES;
  __shared__ u64 lists[MODE == FORWARD && LANES == 32 ? WARPS * LIST : 1];
  const int lane = threadIdx.x % LANES, CW = a.C / NW;
  for (long long row0 = (long long)blockIdx.x * TEAMS; row0 < a.n; row0 += (long long)gridDim.x * TEAMS) {
    const long long at = row0 + threadIdx.x / LANES;
    const bool have = at < a.n;
    const long long row = have ? at : a.n - 1;                       // a team without a row goes along with the last one
    const Wd* const x = reinterpret_cast<const Wd*>(static_cast<const T*>(a.x) + row * a.ld) + lane;
    float v[W][NW];
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll
      for (int e = 0; e < NW; ++e) v[i][e] = -INFINITY;
      if (i * LANES + lane < CW) unpack<T>(x[i * LANES], v[i]);
    }
    const int label = label_of(a, row);
    RowResult r;
    if (MODE != GRAD) {
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if (i * LANES >= CW) continue;
#pragma unroll
        for (int e = 0; e < NW; ++e) m = max_nan(m, v[i][e]);
      }
      const float mine = m;
#pragma unroll
      for (int d = LANES / 2; d; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
      // (words behind the row are masked classes: they add nothing but one each to others)
      RowSums sum;
      const float m8 = m * (1.f / CUT);
      int words = 0;
#pragma unroll
      for (int i = 0; i < W; i += 2 / NW) {
        if (i * LANES >= CW) continue;
        words += 2 / NW;
        if constexpr (NW == 2) sum.add2(v[i][0], v[i][1], m8);
        else sum.add2(v[i][0], v[i + 1][0], m8);
      }
      float s = sum.both(sum.s), q = sum.both(sum.q), others = sum.both(sum.others);
#pragma unroll
      for (int d = LANES / 2; d; d >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, d);
        q += __shfl_xor_sync(0xffffffffu, q, d);
        others += __shfl_xor_sync(0xffffffffu, others, d);
      }
      r = row_result({m, s + ((float)(words * NW * LANES - 1) - others), -CUT * q}, !(m < INFINITY));
      if (lane == 0 && have) {
        if (a.logprob) a.logprob[row] = label < 0 ? 0.f : log_p(to_f32<T>(static_cast<const T*>(a.x)[row * a.ld + label]), r);
        if (a.entropy) a.entropy[row] = r.H;
        if (a.stats) a.stats[row] = make_float2(r.m, r.l);
      }
      if (MODE == FORWARD && a.k > 0) {
        if (LANES == 32) {
          Candidates top = {lists + (threadIdx.x >> 5) * LIST, 0, 0, -INFINITY};
          const float known = mine != mine ? -INFINITY : mine;
          const int rank = rank_of_lanes(known);
          const float floor = __shfl_sync(0xffffffffu, known, __ffs(__ballot_sync(0xffffffffu, rank == a.k - 1)) - 1);
#pragma unroll
          for (int i = 0; i < W; ++i) {
            if (i * LANES >= CW) continue;
#pragma unroll
            for (int e = 0; e < NW; ++e)
              if (__any_sync(0xffffffffu, v[i][e] >= floor)) put_candidates(top, v[i][e] >= floor ? key_of(v[i][e], (i * LANES + lane) * NW + e) : 0, a.k);
          }
          sort_candidates(top, a.k);
          if (lane < a.k && have) write_top(a, row, lane, lane < top.count ? top.list[lane] : 0, r);
          __syncwarp();
        } else {
          // the team's best, k times
          for (int t = 0; t < a.k; ++t) {
            float best = -INFINITY;
            int where = -1;
#pragma unroll
            for (int i = 0; i < W; ++i) {
              if (i * LANES >= CW) continue;
#pragma unroll
              for (int e = 0; e < NW; ++e) if (v[i][e] > best) { best = v[i][e]; where = i * NW + e; }
            }
            int cls = where < 0 ? 0x7fffffff : ((where / NW) * LANES + lane) * NW + where % NW;
            const int own = cls;
#pragma unroll
            for (int d = LANES / 2; d; d >>= 1) {
              const float o = __shfl_xor_sync(0xffffffffu, best, d);
              const int oc = __shfl_xor_sync(0xffffffffu, cls, d);
              if (o > best || (o == best && oc < cls)) { best = o; cls = oc; }
            }
            const bool none = cls == 0x7fffffff;
            if (lane == 0 && have) {
              if (a.top_logprob) a.top_logprob[row * a.k + t] = none ? -INFINITY : log_p(best, r);
              if (a.top_class) a.top_class[row * a.k + t] = none ? -1 : cls;
            }
            if (own != cls) where = -1;
#pragma unroll
            for (int i = 0; i < W; ++i) {
              if (i * LANES >= CW) continue;
#pragma unroll
              for (int e = 0; e < NW; ++e) if (where == i * NW + e) v[i][e] = -INFINITY;
            }
          }
        }
      }
    } else {
      const float2 ml = a.stats_in[row];
      r = {ml.x, ml.y, a.entropy_in ? a.entropy_in[row] : 0.f};
    }
    if (MODE != FORWARD) {
      const GradRow gr = grad_row(a, row, label, r);
      const bool special = have && label >= 0 && label / NW % LANES == lane;       // this lane has the label's word
      const float at = special ? to_f32<T>(static_cast<const T*>(a.x)[row * a.ld + label]) : 0.f;
      __syncwarp();                              // the label's logit has been read before its place is written
      Wd* const dx = reinterpret_cast<Wd*>(static_cast<T*>(a.dx) + row * a.ld_dx) + lane;
#pragma unroll
      for (int i = 0; i < W; i += 2 / NW) {
        if (i * LANES >= CW) continue;
        float y[2];
        if constexpr (NW == 2) {
          grad_of2(gr, v[i][0], v[i][1], y, y + 1);
          if (have && i * LANES + lane < CW) dx[i * LANES] = pack<T>(y);
        } else {
          grad_of2(gr, v[i][0], v[i + 1][0], y, y + 1);
          if (have && i * LANES + lane < CW) dx[i * LANES] = from_f32<T>(y[0]);
          if (have && (i + 1) * LANES + lane < CW) dx[(i + 1) * LANES] = from_f32<T>(y[1]);
        }
      }
      if (special) static_cast<T*>(a.dx)[row * a.ld_dx + label] = from_f32<T>(grad_of_label(gr, at));
    }
  }
}

// ---- many classes: a warp or a block to a row or a part of one ----------------------------------------------------------------------------------------

// Vectors of 16 bytes over the classes [begin, end) of a row, on the row's own 16-byte grid: the first and the last may be cut.
template <class T>
struct Span {
  static constexpr int V = 16 / (int)sizeof(T);
  const T* row;
  int shift, end, begin;                        // elements of the grid in front of the row
  __device__ __forceinline__ Span(const T* r, int b, int e) : row(r), shift((int)((reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T))), end(e), begin(b) {}
  __device__ __forceinline__ int first() const { return (begin + shift) / V; }
  __device__ __forceinline__ int last() const { return (end + shift + V - 1) / V; }         // one behind
  __device__ __forceinline__ int column(int v) const { return v * V - shift; }
  template <int HOW>
  __device__ __forceinline__ Vec<T, V> load(int v) const {
    const int c = column(v);
    Vec<T, V> r;
    if (c >= begin && c + V <= end) return load_vec<Vec<T, V>, HOW>(row + c);
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = c + i >= begin && c + i < end ? row[c + i] : from_f32<T>(-INFINITY);
    return r;
  }
};

// Largest element of a vector; a NaN is larger than all.
__device__ __forceinline__ float vector_max(const Vec<float, 4>& r) { return max_nan(max_nan(r.v[0], r.v[1]), max_nan(r.v[2], r.v[3])); }
__device__ __forceinline__ float vector_max(const Vec<__nv_bfloat16, 8>& r) {
  const __nv_bfloat162* const h = reinterpret_cast<const __nv_bfloat162*>(&r);
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float vector_max(const Vec<__half, 8>& r) {
  const __half2* const h = reinterpret_cast<const __half2*>(&r);
  const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(__low2float(m), __high2float(m));
}

// A vector's 16 bytes as pairs.
template <class T, int V>
__device__ __forceinline__ void to_pairs(const Vec<T, V>& r, F2 (&x)[V / 2]) {
#pragma unroll
  for (int i = 0; i < V; i += 2) x[i / 2] = f2(to_f32<T>(r.v[i]), to_f32<T>(r.v[i + 1]));
}

// The best k of a row of a warp by way of candidates, batch after batch: where more values than a list takes are as large as the k-th of the threads' maxima.
template <class T>
__device__ __noinline__ void stream_candidates(Candidates& c, const Span<T> span, int v0, int step, int k) {
  constexpr int V = Span<T>::V;
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (; v0 < span.last(); v0 += step) {
    const int v = v0 + lane, at = span.column(v);
    float most = -INFINITY;
    if (v < span.last()) most = vector_max(span.template load<LOAD_PLAIN>(v));
    if (!__any_sync(0xffffffffu, !(most <= c.above))) continue;
#pragma unroll 1
    for (int i = 0; i < V; ++i)
      put_candidates(c, v < span.last() && at + i >= span.begin && at + i < span.end ? key_of(to_f32<T>(span.row[at + i]), at + i) : 0, k);
    sort_candidates(c, k);
  }
  sort_candidates(c, k);
}

__device__ __forceinline__ void copy_async(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

constexpr int block_warps(int wpr) { return wpr == 1 ? WARPS : wpr; }
// WPR warps to a row or a part of one: a block to itself, or eight rows of a warp each in a block.  Thread t has the vectors t, t + 32 WPR, ... of it.
template <class T, bool TOP, int WPR, bool WITH_GRAD>
__global__ void __launch_bounds__(32 * block_warps(WPR), 4 * WARPS / block_warps(WPR)) stream_kernel(const Args a) {
  constexpr int V = 16 / (int)sizeof(T), U = 4, AHEAD = 2, TEAM = 32 * WPR, PLACES = LIST * WPR, BW = block_warps(WPR), SHARES = BW / WPR;
  __shared__ u64 lists[TOP ? BW * LIST : 1];
  __shared__ u64 best[TOP ? SHARES * MAX_TOP : 1];
  __shared__ float warp_top[TOP ? BW * MAX_TOP : 1];
  __shared__ float2 warp_sums[BW];
  __shared__ float warp_max[BW], warp_rest[BW];
  __shared__ int warp_same[BW], counts[SHARES], owners[SHARES];
  __shared__ unsigned chosen[BW];
  __shared__ uint8_t who[TOP ? 32 * BW : 1];
  __shared__ Vec<T, V> ahead[AHEAD * U * 32 * BW];
  early_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = warp / WPR, mine = threadIdx.x % TEAM, w0 = share * WPR;     // w0: the team's first warp
  const auto sync = [] { if (WPR == 1) __syncwarp(); else __syncthreads(); };
  const long long units = a.n * a.parts, stride = (long long)gridDim.x * SHARES;
  for (long long unit = (long long)blockIdx.x * SHARES + share; unit < units; unit += stride) {
    const long long row = a.parts == 1 ? unit : unit / a.parts;
    const int part = a.parts == 1 ? 0 : (int)(unit - row * a.parts);
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    const int begin = part * a.part_len, end = a.C - begin < a.part_len ? a.C : begin + a.part_len;
    const Span<T> span(x, begin, end);
    const int first = span.first(), last = span.last();
    float m = -INFINITY;
    F2 s2 = f2(0.f, 0.f), t2 = s2;
    // Batches ahead, by asynchronous copies into places of the thread's own.  The first and the last vector of a span may be cut: those come by element.
    int place = 0;
    const T* from = x + span.column(first + mine);
    const auto fetch = [&](int v0) {
      Vec<T, V>* const to = &ahead[place * U * (32 * BW) + threadIdx.x];
      if (v0 > first && v0 + U * TEAM < last) {
#pragma unroll
        for (int u = 0; u < U; ++u) copy_async(to + u * (32 * BW), from + u * TEAM * V);
      } else if (v0 < last) {
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
          const int v = v0 + u * TEAM + mine;
          if (v > first && v < last - 1) copy_async(to + u * (32 * BW), from + u * TEAM * V);
          else if (v < last) to[u * (32 * BW)] = span.template load<LOAD_PLAIN>(v);
          else {
            Vec<T, V> none;
#pragma unroll
            for (int i = 0; i < V; ++i) none.v[i] = from_f32<T>(-INFINITY);
            to[u * (32 * BW)] = none;
          }
        }
      }
      from += U * TEAM * V;
      asm volatile("cp.async.commit_group;" ::: "memory");
      place = place + 1 == AHEAD ? 0 : place + 1;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(first + i * U * TEAM);
    for (int v0 = first; v0 < last; v0 += U * TEAM) {
      asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
      Vec<T, V> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = load_vec<Vec<T, V>>(&ahead[(place * U + u) * (32 * BW) + threadIdx.x]);
      float now = m;
#pragma unroll
      for (int u = 0; u < U; ++u) now = max_nan(now, vector_max(raw[u]));
      fetch(v0 + AHEAD * U * TEAM);              // into the place of this batch, which has been read
      const float d = fmaxf(m - now, LEAST), f = ex2(d * LOG2E);       // (nothing before: both sums are 0)
      const F2 d2 = f2(d, d), g2 = f2(f, f), minus = f2(-now, -now), log2e = f2(LOG2E, LOG2E);
      t2 = mul(fma(s2, d2, t2), g2);
      s2 = mul(s2, g2);
      m = now;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        F2 v[V / 2];
        to_pairs<T, V>(raw[u], v);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          float p, q;
          split(add(v[i], minus), &p, &q);
          const F2 e = f2(fmaxf(p, LEAST), fmaxf(q, LEAST));
          split(mul(e, log2e), &p, &q);
          const F2 w = f2(ex2(p), ex2(q));
          s2 = add(s2, w);
          t2 = fma(w, e, t2);
        }
      }
    }
    // The team's maximum, the first thread that has it, and the sums without that thread's.
    float most = m, s, t, lo, hi;
#pragma unroll
    for (int d = 16; d; d >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (WPR > 1) {
      if (lane == 0) warp_max[warp] = most;
      sync();
      most = warp_max[w0];
#pragma unroll
      for (int w = 1; w < WPR; ++w) most = max_nan(most, warp_max[w0 + w]);
    }
    const bool bad = !(most < INFINITY), none = most == -INFINITY;
    split(s2, &lo, &hi); s = lo + hi;
    split(t2, &lo, &hi); t = lo + hi;
    const float d = fmaxf(m - most, LEAST), f = ex2(d * LOG2E);
    t = f * fmaf(s, d, t);
    s *= f;
    const unsigned have = __ballot_sync(0xffffffffu, m == most);
    int owner = __ffs(have) - 1;
    if (WPR > 1) {
      int w = 0;
      while (w < WPR - 1 && warp_max[w0 + w] != most) ++w;
      if (w0 + w == warp) { if (lane == owner) s = 0.f; if (lane == 0) owners[share] = owner; }
      owner = w * 32;                            // its lane comes with the sums
    } else if (lane == owner) s = 0.f;
#pragma unroll
    for (int k = 16; k; k >>= 1) { s += __shfl_xor_sync(0xffffffffu, s, k); t += __shfl_xor_sync(0xffffffffu, t, k); }
    if (WPR > 1) {
      if (lane == 0) warp_sums[warp] = make_float2(s, t);
      sync();
      s = t = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) { s += warp_sums[w0 + w].x; t += warp_sums[w0 + w].y; }
      owner += owners[share];
    }
    // That thread's vectors again, by all, without what equals the maximum.
    float rest = 0.f;
    int same = 0;
    if (!bad && !none) {
      for (int v = first + owner + mine * TEAM; v < last; v += TEAM * TEAM) {
        const Vec<T, V> r = span.template load<LOAD_PLAIN>(v);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float y = to_f32<T>(r.v[i]);
          if (y == most) ++same;
          else rest += ex2(fmaxf(y - most, LEAST) * LOG2E);
        }
      }
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, k);
    same = __reduce_add_sync(0xffffffffu, same);
    if (WPR > 1) {
      if (lane == 0) { warp_rest[warp] = rest; warp_same[warp] = same; }
      sync();
      rest = 0.f;
      same = 0;
#pragma unroll
      for (int w = 0; w < WPR; ++w) { rest += warp_rest[w0 + w]; same += warp_same[w0 + w]; }
    }
    const Sums sums = {most, s + rest + (float)(same - 1), t};
    const RowResult r = row_result(sums, bad);
    const int label = a.parts == 1 ? label_of(a, row) : -1;
    if (mine == 0) {
      if (a.parts == 1) write_row<T>(a, row, label, r);
      else a.part[unit] = none ? make_float4(-INFINITY, 0.f, 0.f, bad) : make_float4(sums.m, sums.s, sums.t, bad);
    }
    if (TOP) {
      // The k-th largest of the threads' maxima.
      const float known = m != m ? -INFINITY : m;
      const int rank = rank_of_lanes(known);
      if (rank < a.k) warp_top[warp * MAX_TOP + rank] = known;
      if (mine == 0) counts[share] = 0;
      sync();
      float kth = warp_top[warp * MAX_TOP + a.k - 1];
      if (WPR > 1) {
        int head = 0;
        for (int i = 0; i < a.k; ++i) {
          const float h = lane < WPR && head < a.k ? warp_top[(w0 + lane) * MAX_TOP + head] : -INFINITY;
          kth = h;
#pragma unroll
          for (int k = WPR / 2; k; k >>= 1) kth = fmaxf(kth, __shfl_xor_sync(0xffffffffu, kth, k));
          kth = __shfl_sync(0xffffffffu, kth, 0);
          const unsigned has = __ballot_sync(0xffffffffu, lane < WPR && head < a.k && h == kth);
          if (lane == __ffs(has) - 1) ++head;
        }
      }
      const unsigned look = __ballot_sync(0xffffffffu, m != m || (m >= kth && m > -INFINITY));
      if (WPR > 1) {
        if (lane == 0) chosen[warp] = look;
        sync();
      }
      u64* const list = lists + w0 * LIST;
      // Those threads' numbers in a row, then their vectors, all at once.
      int before = 0, threads = 0;
#pragma unroll
      for (int w = 0; w < WPR; ++w) {
        const int c = __popc(WPR > 1 ? chosen[w0 + w] : look);
        if (w0 + w < warp) before += c;
        threads += c;
      }
      if (look >> lane & 1) who[w0 * 32 + before + __popc(look & ((1u << lane) - 1))] = (uint8_t)mine;
      sync();
      const int each = (last - first + TEAM - 1) / TEAM;
      for (int f = mine; f < threads * each; f += TEAM) {
        const int j = f / threads, v = first + who[w0 * 32 + f - j * threads] + j * TEAM;
        if (v >= last) continue;
        const Vec<T, V> got = span.template load<LOAD_PLAIN>(v);
        if (vector_max(got) < kth) continue;
        for (int i = 0; i < V; ++i) {
          const float y = to_f32<T>(got.v[i]);
          if (y >= kth && y > -INFINITY) {
            const int to = atomicAdd(&counts[share], 1);
            if (to < PLACES) list[to] = key_of(y, span.column(v) + i);
          }
        }
      }
      sync();
      const int count = counts[share];
      u64* const out = best + share * MAX_TOP;
      if (count <= PLACES) {
        if (mine < MAX_TOP) out[mine] = 0;
        sync();
        for (int j = mine; j < count; j += TEAM) {
          const u64 key = list[j];
          int place = 0;
          for (int i = 0; i < count; ++i) place += list[i] > key;
          if (place < a.k) out[place] = key;
        }
        sync();
      } else {
        sync();
        Candidates c = {lists + warp * LIST, 0, 0, -INFINITY};
        stream_candidates<T>(c, span, first + (warp - w0) * 32, TEAM, a.k);
        if (lane >= c.count && lane < a.k) c.list[lane] = 0;
        sync();
        if (warp == w0) {
          // the lists' heads, the best of them taken k times
          int head = 0;
          u64 h = lane < WPR ? list[lane * LIST] : 0;
          for (int i = 0; i < a.k; ++i) {
            const uint32_t up = __reduce_max_sync(0xffffffffu, (uint32_t)(h >> 32));
            const uint32_t down = __reduce_max_sync(0xffffffffu, (uint32_t)(h >> 32) == up ? (uint32_t)h : 0u);
            const u64 top = ((u64)up << 32) | down;
            if (lane == 0) out[i] = top;
            if (top && h == top) { ++head; h = head < a.k ? list[lane * LIST + head] : 0; }
          }
        }
        sync();
      }
      if (mine < a.k) {
        if (a.parts == 1) write_top(a, row, mine, out[mine], r);
        else a.part_top[unit * a.k + mine] = out[mine];
      }
    }
    if (WITH_GRAD) {
      sync();                                    // the label's logit has been read before its place is written
      const GradRow gr = grad_row(a, row, label, r);
      T* const dx = static_cast<T*>(a.dx) + row * a.ld_dx;
      const bool alike = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(x)) & 15) == 0;
      // from the end, which the caches have had last
      for (int v = last - 1 - mine; v >= first; v -= TEAM) {
        const Vec<T, V> in = span.template load<LOAD_PLAIN>(v);
        const int c = span.column(v);
        Vec<T, V> out;
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          float y, z;
          grad_of2(gr, to_f32<T>(in.v[i]), to_f32<T>(in.v[i + 1]), &y, &z);
          out.v[i] = from_f32<T>(y);
          out.v[i + 1] = from_f32<T>(z);
        }
        if (label >= c && label < c + V) {
#pragma unroll
          for (int i = 0; i < V; ++i) if (c + i == label) out.v[i] = from_f32<T>(grad_of_label(gr, to_f32<T>(in.v[i])));
        }
        if (alike && c >= 0 && c + V <= a.C) store_vec_once(dx + c, out);
        else
#pragma unroll
          for (int i = 0; i < V; ++i) if (c + i >= 0 && c + i < a.C) dx[c + i] = out.v[i];
      }
    }
    sync();
  }
}

// The parts of a row: a block to a row.  Sums by a tree in a fixed order, the top by the heads of the parts' lists.
constexpr int JOIN_THREADS = 128;
template <class T>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const Args a) {
  __shared__ u64 lists[MAX_PARTS * MAX_TOP];
  early_start();
  const int lane = threadIdx.x & 31;
  for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
    const u64* const top = a.part_top + row * a.parts * a.k;
    for (int i = threadIdx.x; i < a.parts * a.k; i += JOIN_THREADS) lists[i] = top[i];
    __syncthreads();
    if (threadIdx.x < 32) {
      const float4* const part = a.part + row * a.parts;
      Sums sums = {-INFINITY, 0.f, 0.f};
      bool bad = false;
      for (int i = lane; i < a.parts; i += 32) {
        const float4 o = part[i];
        join(sums, {o.x, o.y, o.z});
        bad |= o.w != 0.f;
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        const Sums o = {__shfl_down_sync(0xffffffffu, sums.m, d), __shfl_down_sync(0xffffffffu, sums.s, d), __shfl_down_sync(0xffffffffu, sums.t, d)};
        if (lane < d) join(sums, o);
      }
      sums = {__shfl_sync(0xffffffffu, sums.m, 0), __shfl_sync(0xffffffffu, sums.s, 0), __shfl_sync(0xffffffffu, sums.t, 0)};
      const RowResult r = row_result(sums, __any_sync(0xffffffffu, bad));
      const int label = label_of(a, row);
      if (lane == 0) write_row<T>(a, row, label, r);
      if (a.k) {
        int head0 = 0, head1 = 0;
        u64 h0 = lane < a.parts ? lists[lane * a.k] : 0, h1 = lane + 32 < a.parts ? lists[(lane + 32) * a.k] : 0, keep = 0;
        for (int i = 0; i < a.k; ++i) {
          const u64 mine = h0 > h1 ? h0 : h1;
          const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
          const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32) == hi ? (uint32_t)mine : 0u);
          const u64 best = ((u64)hi << 32) | lo;
          if (lane == i) keep = best;
          if (best && h0 == best) { ++head0; h0 = head0 < a.k ? lists[lane * a.k + head0] : 0; }
          else if (best && h1 == best) { ++head1; h1 = head1 < a.k ? lists[(lane + 32) * a.k + head1] : 0; }
        }
        if (lane < a.k) write_top(a, row, lane, keep, r);
      }
    }
    __syncthreads();
  }
}

// The gradient of many classes: a warp to GRAD_VECTORS x 32 vectors of a row.
constexpr int GRAD_VECTORS = 4;
template <class T>
__global__ void __launch_bounds__(256) grad_kernel(const Args a, int chunks) {
  constexpr int V = 16 / (int)sizeof(T);
  early_start();
  const int lane = threadIdx.x & 31;
  const long long units = a.n * chunks;
  for (long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); unit < units; unit += (long long)gridDim.x * 8) {
    const long long row = unit / chunks;
    const int chunk = (int)(unit - row * chunks);
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    T* const dx = static_cast<T*>(a.dx) + row * a.ld_dx;
    const Span<T> span(x, 0, a.C);
    const int v0 = chunk * (GRAD_VECTORS * 32) + lane;
    Vec<T, V> in[GRAD_VECTORS];
#pragma unroll
    for (int u = 0; u < GRAD_VECTORS; ++u) if (v0 + u * 32 < span.last()) in[u] = span.template load<LOAD_ONCE>(v0 + u * 32);
    const float2 ml = a.stats_in[row];
    const GradRow gr = grad_row(a, row, label_of(a, row), {ml.x, ml.y, a.entropy_in ? a.entropy_in[row] : 0.f});
    const bool alike = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(x)) & 15) == 0;
#pragma unroll
    for (int u = 0; u < GRAD_VECTORS; ++u) {
      const int v = v0 + u * 32;
      if (v >= span.last()) continue;
      const int c = span.column(v);
      Vec<T, V> out;
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        float y, z;
        grad_of2(gr, to_f32<T>(in[u].v[i]), to_f32<T>(in[u].v[i + 1]), &y, &z);
        out.v[i] = from_f32<T>(y);
        out.v[i + 1] = from_f32<T>(z);
      }
      if (gr.label >= c && gr.label < c + V) {
#pragma unroll
        for (int i = 0; i < V; ++i) if (c + i == gr.label) out.v[i] = from_f32<T>(grad_of_label(gr, to_f32<T>(in[u].v[i])));
      }
      if (alike && c >= 0 && c + V <= a.C) store_vec_once(dx + c, out);
      else
#pragma unroll
        for (int i = 0; i < V; ++i) if (c + i >= 0 && c + i < a.C) dx[c + i] = out.v[i];
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------------------------

// Rows in tiles: where there are enough of them, and enough elements, for the tiles to be on all SMs.  Tiles / registers, 16 384 x 47 fp32 6.2 / 4.1 us with the gradient, 65 536 8.8 / 9.8; 8 192 x 300 8.2 / 7.2,
// 16 384 10.3 / 12.3; top 5, 8 192 x 47 6.7 / 5.2, 16 384 6.7 / 7.7; 2 048 x 300 7.2 / 6.6, 4 096 8.0 / 10.3; 2 048 x 1 000 9.2 / 8.2, 4 096 11.4 / 13.4.
constexpr int TILE_ROWS = 4096;
constexpr int64_t TILE_ELEMENTS_LEAST = 1 << 21, TILE_ELEMENTS_TOP = 3 << 18;
inline bool by_tile(const Args& a, int ts, bool grad) {
  return a.n >= TILE_ROWS && a.C <= tile_classes(ts, grad, a.k) && a.n * a.C >= (a.k ? TILE_ELEMENTS_TOP : TILE_ELEMENTS_LEAST);
}
// 16-bit rows that begin at even elements everywhere.
inline bool in_pairs(const Args& a, int ts, bool grad) {
  const auto even = [](const void* p, long long ld) { return rows_aligned(p, 4) && ld % 2 == 0; };
  return ts == 2 && a.C % 2 == 0 && even(a.x, a.ld) && (!grad || even(a.dx, a.ld_dx));
}

// How a row of many classes is split: into as many parts as give every SM four blocks, but none shorter than 8 192 classes (4 096: 1 x 20 000 bf16 5.7 -> 4.7 us, 10 x 250 000 8.2 -> 9.8, with the top 10 14.6 -> 19.5).
constexpr int ENOUGH_WARPS = 148 * 32, ENOUGH_BLOCKS = 148 * 4, PART_MIN = 8192;
inline int parts_of(int64_t n, int C) {
  if (n >= ENOUGH_BLOCKS || C < 2 * PART_MIN) return 1;
  const int64_t want = (ENOUGH_BLOCKS + n - 1) / n, most = C / PART_MIN;
  return (int)std::min<int64_t>(std::min<int64_t>(want, most), MAX_PARTS);
}

struct Space { size_t part, top, stats, entropy, bytes; };
Space space_of(int64_t n, int C, int k) {
  Space s = {};
  if (C < 2 * PART_MIN) return s;
  const size_t rows = (size_t)std::min<int64_t>(n, ENOUGH_BLOCKS - 1), parts = std::min<size_t>(rows * MAX_PARTS, (size_t)ENOUGH_BLOCKS + rows);   // n * ceil(E / n) < E + n
  size_t at = 0;
  const auto take = [&](size_t b) { const size_t here = at; at += (b + 255) / 256 * 256; return here; };
  s.part = take(parts * sizeof(float4));
  s.stats = take(rows * sizeof(float2));
  s.entropy = take(rows * sizeof(float));
  s.top = take(parts * (size_t)k * sizeof(u64));
  s.bytes = n > 0 ? at : 0;
  return s;
}

template <class T, bool PAIRS, int MODE>
void launch_team(Launches& enqueue, const Args& a) {
  const int words = a.C / Word<T, PAIRS>::n;
  const auto go = [&](auto lanes, auto w) {
    constexpr int L = decltype(lanes)::value, W = decltype(w)::value, TEAMS = 32 * WARPS / L;
    enqueue(team_kernel<T, PAIRS, L, W, MODE>, dim3((unsigned)std::min<int64_t>((a.n + TEAMS - 1) / TEAMS, 1 << 30)), 32 * WARPS, 0, a);
  };
  using std::integral_constant;
  if (words <= 64) go(integral_constant<int, 8>(), integral_constant<int, 8>());
  else if (words <= 128) go(integral_constant<int, 8>(), integral_constant<int, 16>());
  else if (words <= 512) go(integral_constant<int, 32>(), integral_constant<int, 16>());
  else if constexpr (!PAIRS) go(integral_constant<int, 32>(), integral_constant<int, 32>());
}
template <class T>
void launch_grad(Launches& enqueue, const Args& a, int sms) {
  constexpr int V = 16 / (int)sizeof(T);
  const int chunks = ((a.C + 2 * V - 2) / V + GRAD_VECTORS * 32 - 1) / (GRAD_VECTORS * 32);     // vectors of a row wherever it begins
  enqueue(grad_kernel<T>, dim3((unsigned)std::min<int64_t>((a.n * chunks + 7) / 8, (int64_t)sms * 64)), 256, 0, a, chunks);
}
// The smallest team, of 1, 2, 4 or 8 warps, with which there are enough warps: what comes behind a row's pass is latency, and more rows at once hide it.  (2 000 x 120 001 bf16, top 10: 2 warps 159 us, 4 129.)
template <class T, bool TOP, bool WITH_GRAD>
void launch_stream(Launches& enqueue, const Args& a) {
  const auto go = [&](auto wpr) {
    constexpr int WPR = decltype(wpr)::value, BW = block_warps(WPR), SHARES = BW / WPR;
    enqueue(stream_kernel<T, TOP, WPR, WITH_GRAD>, dim3((unsigned)std::min<int64_t>((a.n * a.parts + SHARES - 1) / SHARES, 1 << 30)), 32 * BW, 0, a);
  };
  const int64_t rows = a.n * a.parts;
  if (rows >= ENOUGH_WARPS) go(std::integral_constant<int, 1>());
  else if (rows * 2 >= ENOUGH_WARPS) go(std::integral_constant<int, 2>());
  else if (rows * 4 >= ENOUGH_WARPS) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 8>());
}

enum { GIVEN_WEIGHTS = 1, GIVEN_STATS = 2 };

// Everything that the three entry points share.  what: 0, or the gradient in the same call (GIVEN_WEIGHTS), or from what an earlier call left (GIVEN_STATS).
int class_call(Args a, int32_t type, int what, int in_place_ok, void* workspace, int64_t workspace_bytes, cudaStream_t st, int dev, int sms) {
  const int ts = row_type_size(type);
  const Space sp = what == GIVEN_STATS ? Space{} : space_of(a.n, a.C, a.k);
  const int64_t n = a.n;
  const bool grad = what != 0, in_place = grad && in_place_ok && a.dx == a.x && a.ld_dx == a.ld;
  const size_t nb = (size_t)n;
  const Region outs[] = {grad ? region_of_rows(a.dx, n, a.ld_dx, a.C, ts) : region_of(nullptr, 0), region_of(a.logprob, nb * 4), region_of(a.entropy, nb * 4), region_of(a.stats, nb * 8),
                         region_of(a.top_logprob, nb * a.k * 4), region_of(a.top_class, nb * a.k * 8), region_of(a.status, 4)};
  const Region ins[] = {in_place ? region_of(nullptr, 0) : region_of_rows(a.x, n, a.ld, a.C, ts), region_of(a.labels, nb * 8), region_of(a.grad_logprob, nb * 4),
                        region_of(a.grad_entropy, nb * 4), region_of(a.stats_in, nb * 8), region_of(a.entropy_in, nb * 4)};
  const bool pairs = in_pairs(a, ts, grad), team = a.C <= TEAM_CLASSES;
  a.parts = team ? 1 : parts_of(n, a.C);
  const int64_t need = what != GIVEN_STATS && a.parts > 1 ? (int64_t)sp.bytes : 0;
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) || !workspace_ok(workspace, workspace_bytes, need, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  a.part_len = a.parts == 1 ? a.C : (int)(((int64_t)a.C + a.parts - 1) / a.parts);
  Launches enqueue = {st};
  with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    if (team) {
      const auto with = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        if (by_tile(a, ts, grad)) {
          if constexpr (std::is_same_v<T, float>) logprob_rows_f32(enqueue, a, MODE);
          else if constexpr (std::is_same_v<T, __nv_bfloat16>) logprob_rows_bf16(enqueue, a, MODE, pairs);
          else logprob_rows_f16(enqueue, a, MODE, pairs);
          return;
        }
        if constexpr (sizeof(T) == 2) { if (pairs) { launch_team<T, true, MODE>(enqueue, a); return; } }
        launch_team<T, false, MODE>(enqueue, a);
      };
      if (what == GIVEN_STATS) with(std::integral_constant<int, GRAD>());
      else if (what == GIVEN_WEIGHTS) with(std::integral_constant<int, TRAIN>());
      else with(std::integral_constant<int, FORWARD>());
      return 0;
    }
    if (what == GIVEN_STATS) { launch_grad<T>(enqueue, a, sms); return 0; }
    if (a.parts == 1) {
      if (what == GIVEN_WEIGHTS) launch_stream<T, false, true>(enqueue, a);
      else if (a.k) launch_stream<T, true, false>(enqueue, a);
      else launch_stream<T, false, false>(enqueue, a);
      return 0;
    }
    char* const ws = static_cast<char*>(workspace);
    a.part = reinterpret_cast<float4*>(ws + sp.part);
    a.part_top = reinterpret_cast<u64*>(ws + sp.top);
    if (grad) {
      if (!a.stats) a.stats = reinterpret_cast<float2*>(ws + sp.stats);
      if (!a.entropy) a.entropy = reinterpret_cast<float*>(ws + sp.entropy);
      a.stats_in = a.stats; a.entropy_in = a.entropy;
    }
    if (a.k) launch_stream<T, true, false>(enqueue, a);
    else launch_stream<T, false, false>(enqueue, a);
    enqueue(join_kernel<T>, dim3((unsigned)std::min<int64_t>(n, 1 << 20)), JOIN_THREADS, 0, a);
    if (grad) launch_grad<T>(enqueue, a, sms);
    return 0;
  });
  return enqueue.done("class log probabilities");
}

bool class_shape_ok(int64_t n, int32_t classes) { return n >= 0 && n < (1ll << 31) && classes >= 1; }
bool class_args_ok(int64_t n, int32_t classes, const void* x, int64_t ld, int32_t type, const int64_t* labels, const void* status) {
  const int ts = row_type_size(type);
  return ts && class_shape_ok(n, classes) && ld >= classes && rows_fit(n, ld, 4) && rows_aligned(labels, 8) && rows_aligned(status, 4) && (n == 0 || (x && rows_aligned(x, ts)));
}

}  // namespace

extern "C" int64_t taurus_class_logprob_workspace(int64_t n, int32_t classes, int32_t k) {
  if (!class_shape_ok(n, classes) || k < 0) return TAURUS_ERR_INVALID_ARG;
  if (classes > TAURUS_MAX_CLASSES || k > MAX_TOP) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)space_of(n, classes, k).bytes;
}

extern "C" int taurus_class_logprob(int64_t n, int32_t classes, const void* logits, int64_t ld, int32_t type, const int64_t* labels, float* logprob, float* entropy,
                                    float* stats, int32_t k, float* top_logprob, int64_t* top_class, void* workspace, int64_t workspace_bytes, int32_t* status,
                                    void* cuda_stream) {
  if (!class_args_ok(n, classes, logits, ld, type, labels, status) || k < 0 || !rows_aligned(logprob, 4) || !rows_aligned(entropy, 4) || !rows_aligned(stats, 8) ||
      !rows_aligned(top_logprob, 4) || !rows_aligned(top_class, 8))
    return TAURUS_ERR_INVALID_ARG;
  if (classes > TAURUS_MAX_CLASSES || k > MAX_TOP) return TAURUS_ERR_UNSUPPORTED;
  if (n == 0) return TAURUS_OK;
  if ((logprob && !labels) || (k > 0 && !top_logprob && !top_class)) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  Args a = {};
  a.n = n; a.C = classes; a.x = logits; a.ld = ld; a.labels = reinterpret_cast<const long long*>(labels); a.logprob = logprob; a.entropy = entropy;
  a.stats = reinterpret_cast<float2*>(stats); a.k = k; a.top_logprob = k ? top_logprob : nullptr; a.top_class = k ? reinterpret_cast<long long*>(top_class) : nullptr; a.status = status;
  return class_call(a, type, 0, 0, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream), dev, sms);
}

extern "C" int taurus_class_logprob_train(int64_t n, int32_t classes, const void* logits, int64_t ld, int32_t type, const int64_t* labels, const float* grad_logprob,
                                          const float* grad_entropy, float* logprob, float* entropy, float* stats, void* grad_logits, int64_t ld_grad, void* workspace,
                                          int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  if (!class_args_ok(n, classes, logits, ld, type, labels, status) || ld_grad < classes || !rows_fit(n, ld_grad, 4) || !rows_aligned(logprob, 4) || !rows_aligned(entropy, 4) ||
      !rows_aligned(stats, 8) || !rows_aligned(grad_logprob, 4) || !rows_aligned(grad_entropy, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (classes > TAURUS_MAX_CLASSES) return TAURUS_ERR_UNSUPPORTED;
  if (n == 0) return TAURUS_OK;
  if (!grad_logits || !rows_aligned(grad_logits, row_type_size(type)) || ((logprob || grad_logprob) && !labels) || (!grad_logprob && !grad_entropy)) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  Args a = {};
  a.n = n; a.C = classes; a.x = logits; a.ld = ld; a.labels = reinterpret_cast<const long long*>(labels); a.logprob = logprob; a.entropy = entropy;
  a.stats = reinterpret_cast<float2*>(stats); a.grad_logprob = grad_logprob; a.grad_entropy = grad_entropy; a.dx = grad_logits; a.ld_dx = ld_grad; a.status = status;
  return class_call(a, type, GIVEN_WEIGHTS, 1, workspace, workspace_bytes, static_cast<cudaStream_t>(cuda_stream), dev, sms);
}

extern "C" int taurus_class_logprob_grad(int64_t n, int32_t classes, const void* logits, int64_t ld, int32_t type, const int64_t* labels, const float* stats, const float* entropy,
                                         const float* grad_logprob, const float* grad_entropy, void* grad_logits, int64_t ld_grad, int32_t* status, void* cuda_stream) {
  if (!class_args_ok(n, classes, logits, ld, type, labels, status) || ld_grad < classes || !rows_fit(n, ld_grad, 4) || !rows_aligned(stats, 8) || !rows_aligned(entropy, 4) ||
      !rows_aligned(grad_logprob, 4) || !rows_aligned(grad_entropy, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (classes > TAURUS_MAX_CLASSES) return TAURUS_ERR_UNSUPPORTED;
  if (n == 0) return TAURUS_OK;
  if (!stats || !grad_logits || !rows_aligned(grad_logits, row_type_size(type)) || (grad_logprob && !labels) || (grad_entropy && !entropy) || (!grad_logprob && !grad_entropy))
    return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  Args a = {};
  a.n = n; a.C = classes; a.x = logits; a.ld = ld; a.labels = reinterpret_cast<const long long*>(labels); a.stats_in = reinterpret_cast<const float2*>(stats); a.entropy_in = entropy;
  a.grad_logprob = grad_logprob; a.grad_entropy = grad_entropy; a.dx = grad_logits; a.ld_dx = ld_grad; a.status = status;
  return class_call(a, type, GIVEN_STATS, 1, nullptr, 0, static_cast<cudaStream_t>(cuda_stream), dev, sms);
}
