#pragma once
// Class log probabilities of short rows (see logprob.cuh): tiles of rows in shared memory, of one element type for each file that includes this.
#include "logprob.cuh"

namespace {

// ---- few classes: a thread to a row of a tile in shared memory ---------------------------------------------------------------------------------------

// How a tile of rows lies in global memory: single elements | 16-byte vectors over rows without gaps | vectors within rows of a pitch.
enum { TILE_ELEMENTS = 0, TILE_FLAT = 1, TILE_VECTORS = 2 };
// Brings a tile of `rows` rows of C words in and out.  P: words of a row in shared memory.
template <class W>
struct Tile {
  static constexpr int V = 16 / (int)sizeof(W);
  int rows, C, P, vectors;
  unsigned by_C, by_vectors;
  __device__ __forceinline__ unsigned div(unsigned f, unsigned by) const { return by ? __umulhi(f, by) : f; }     // f < 2^16
  // The places of a vector's words: those that reach into the next row are P - C further.  (Rows shorter than a vector: any number of rows further.)
  __device__ __forceinline__ void places(int f, int (&at)[V]) const {
    const int row = div(f, by_C), col = f - row * C;
    if (C >= V) {
#pragma unroll
      for (int i = 0; i < V; ++i) at[i] = row * P + col + i + (col + i >= C ? P - C : 0);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) { const int r = div(f + i, by_C); at[i] = r * P + f + i - r * C; }
    }
  }
  __device__ __forceinline__ void load(W* sm, const W* x, long long ld, int mode) const {
    if (mode == TILE_ELEMENTS) {
      for (int f = threadIdx.x; f < rows * C; f += (int)blockDim.x) { const int row = div(f, by_C), col = f - row * C; sm[row * P + col] = x[row * ld + col]; }
      return;
    }
    const bool flat = mode == TILE_FLAT;
    const int words = rows * C, total = flat ? words / V : rows * vectors;
    for (int v0 = threadIdx.x; v0 < total; v0 += 4 * (int)blockDim.x) {
      Vec<W, V> r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = v0 + u * (int)blockDim.x;
        if (v >= total) break;
        if (flat) r[u] = load_vec<Vec<W, V>, LOAD_ONCE>(x + v * V);
        else {
          const int row = div(v, by_vectors), col = (v - row * vectors) * V;
          const W* const p = x + row * ld + col;
          if (col + V <= C) r[u] = load_vec<Vec<W, V>, LOAD_ONCE>(p);
          else
#pragma unroll
            for (int i = 0; i < V; ++i) if (col + i < C) r[u].v[i] = p[i];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = v0 + u * (int)blockDim.x;
        if (v >= total) break;
        if (flat && P == C) store_vec(sm + v * V, r[u]);
        else if (flat) {
          int at[V];
          places(v * V, at);
#pragma unroll
          for (int i = 0; i < V; ++i) sm[at[i]] = r[u].v[i];
        } else {
          const int row = div(v, by_vectors), col = (v - row * vectors) * V;
#pragma unroll
          for (int i = 0; i < V; ++i) if (col + i < C) sm[row * P + col + i] = r[u].v[i];
        }
      }
    }
    if (flat)
      for (int f = total * V + threadIdx.x; f < words; f += (int)blockDim.x) { const int row = div(f, by_C); sm[row * P + f - row * C] = x[f]; }
  }
  __device__ __forceinline__ void store(const W* sm, W* y, long long ld, int mode) const {
    if (mode == TILE_FLAT) {
      const int words = rows * C, total = words / V;
      for (int v = threadIdx.x; v < total; v += (int)blockDim.x) {
        Vec<W, V> r;
        if (P == C) r = load_vec<Vec<W, V>>(sm + v * V);
        else {
          int at[V];
          places(v * V, at);
#pragma unroll
          for (int i = 0; i < V; ++i) r.v[i] = sm[at[i]];
        }
        store_vec_once(y + v * V, r);
      }
      for (int f = total * V + threadIdx.x; f < words; f += (int)blockDim.x) { const int row = div(f, by_C); y[f] = sm[row * P + f - row * C]; }
    } else if (mode == TILE_VECTORS) {
      for (int v = threadIdx.x; v < rows * vectors; v += (int)blockDim.x) {
        const int row = div(v, by_vectors), col = (v - row * vectors) * V;
        W* const p = y + row * ld + col;
        if (col + V <= C) {
          Vec<W, V> r;
#pragma unroll
          for (int i = 0; i < V; ++i) r.v[i] = sm[row * P + col + i];
          store_vec_once(p, r);
        } else {
          for (int i = 0; col + i < C; ++i) p[i] = sm[row * P + col + i];
        }
      }
    } else {
      for (int f = threadIdx.x; f < rows * C; f += (int)blockDim.x) { const int row = div(f, by_C), col = f - row * C; y[row * ld + col] = sm[row * P + col]; }
    }
  }
};


// TPR threads to a row, which take its words in turn.  KMAX: places for the top in registers (k <= KMAX; 0: none asked for).
// 16-bit rows are words of two classes in shared memory.  PAIRS: in global memory too.  Otherwise the tile comes by element, or by vectors over rows without gaps, and a row of an odd width is (C - 1) / 2 words,
// from its first even place on, and one lone class: its first or its last.  (400 000 x 171 bf16 with the gradient 93 us, by single elements 121; 57 061 x 701 60 / 77; 851 063 x 47 47 / 55.)
template <class T, bool PAIRS, int MODE, int KMAX, int TPR>
__global__ void __launch_bounds__(ROW_THREADS) rows_kernel(const Args a) {
  extern __shared__ __align__(16) unsigned char logprob_shared[];
  constexpr bool TWO = sizeof(T) == 2, LONE = TWO && !PAIRS;
  using W = typename Word<T, PAIRS>::type;       // what is copied
  using Q = typename Word<T, TWO>::type;         // what is computed with
  constexpr int NW = Word<T, TWO>::n, CN = Word<T, PAIRS>::n, STEP = 8 / NW, ROWS = ROW_THREADS / TPR;      // words of 8 classes; rows of a tile
  W* const sm = reinterpret_cast<W*>(logprob_shared);
  const int C = a.C, all = C / NW, sub = threadIdx.x % TPR, CW = (all - sub + TPR - 1) / TPR;      // CW: words of this thread
  const long long tiles = (a.n + ROWS - 1) / ROWS;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const long long row0 = tile * ROWS, row = row0 + threadIdx.x / TPR;
    const Tile<W> t = {(int)(a.n - row0 < ROWS ? a.n - row0 : ROWS), C / CN, a.pitch, a.vectors, a.by_C, a.by_vectors};
    t.load(sm, reinterpret_cast<const W*>(static_cast<const T*>(a.x) + row0 * a.ld), a.ld / CN, a.mode_in);
    const int label = row < a.n ? label_of(a, row) : -1;
    __syncthreads();
    if (TPR > 1 || row < a.n) {                  // (exchanges take all threads of a warp: rows behind the last are whatever the tile held)
      T* const elements = reinterpret_cast<T*>(sm + threadIdx.x / TPR * a.pitch);
      const int odd = LONE ? threadIdx.x / TPR * a.pitch & 1 : 0;            // the row begins in the middle of a word
      Q* const mine = reinterpret_cast<Q*>(elements + odd) + sub;            // its words are TPR apart
      const bool lone = LONE && C & 1;
      const int lone_class = odd ? 0 : C - 1;
      const float alone = lone ? to_f32<T>(elements[lone_class]) : -INFINITY;
      RowResult r;
      if (MODE != GRAD) {
        // Maxima of G classes of classes: the j-th largest of a thread's has j values at least that are not below it.  With j = k / TPR, rounded up, the least of the threads' j-th has k:
        // what is below it is not among the top k.  (The k-th of one thread's own, in lists of KMAX: 133 333 x 300 fp32 top 16 259 us, top 8 107, top 3 68.)
        // More threads than classes asked for: the largest of some threads' together instead of each one's, as long as there are k of those.
        constexpr int J = (KMAX + TPR - 1) / TPR, G = J <= 4 ? 8 : J <= 8 ? 16 : 32, TOGETHER = KMAX ? (TPR + KMAX - 1) / KMAX : 1;
        float most[G];
        if constexpr (NW == 2) {
          using T2 = std::conditional_t<std::is_same_v<T, __nv_bfloat16>, __nv_bfloat162, __half2>;
          T2 two[G / 2];
          const T least = from_f32<T>(-INFINITY);
          T2 none;
          none.x = none.y = least;
#pragma unroll
          for (int i = 0; i < G / 2; ++i) two[i] = none;
          int j = 0;
          for (; j + G / 2 <= CW; j += G / 2)
#pragma unroll
            for (int i = 0; i < G / 2; ++i) two[i] = __hmax2_nan(two[i], reinterpret_cast<const T2*>(mine)[(j + i) * TPR]);
#pragma unroll
          for (int i = 0; i < G / 2; ++i) if (j + i < CW) two[i] = __hmax2_nan(two[i], reinterpret_cast<const T2*>(mine)[(j + i) * TPR]);
#pragma unroll
          for (int i = 0; i < G / 2; ++i) { most[2 * i] = to_f32<T>(two[i].x); most[2 * i + 1] = to_f32<T>(two[i].y); }
        } else {
#pragma unroll
          for (int i = 0; i < G; ++i) most[i] = -INFINITY;
          int j = 0;
          for (; j + G <= CW; j += G)
#pragma unroll
            for (int i = 0; i < G; ++i) most[i] = max_nan(most[i], to_f32<T>(reinterpret_cast<const T*>(mine)[(j + i) * TPR]));
#pragma unroll
          for (int i = 0; i < G; ++i) if (j + i < CW) most[i] = max_nan(most[i], to_f32<T>(reinterpret_cast<const T*>(mine)[(j + i) * TPR]));
        }
        float m = LONE ? max_nan(most[0], alone) : most[0];
#pragma unroll
        for (int i = 1; i < G; ++i) m = max_nan(m, most[i]);
#pragma unroll
        for (int d = TPR / 2; d; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
        const bool bad = !(m < INFINITY);
        float top[KMAX ? KMAX : 1], floor = -INFINITY;
        int cls[KMAX ? KMAX : 1];
        if (KMAX) {
          float first[J ? J : 1];
#pragma unroll
          for (int i = 0; i < J; ++i) first[i] = -INFINITY;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float v = most[g];
#pragma unroll
            for (int i = 0; i < J; ++i) { const float up = fmaxf(first[i], v); v = fminf(first[i], v); first[i] = up; }
          }
          const int j = (a.k + TPR - 1) / TPR;
#pragma unroll
          for (int i = 0; i < J; ++i) if (i == j - 1) floor = first[i];
#pragma unroll
          for (int d = TPR / 2; d; d >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, floor, d);
            floor = TPR / 2 / d < TOGETHER ? fmaxf(floor, o) : fminf(floor, o);
          }
          if (bad) floor = -INFINITY;                       // a NaN hides its class of classes
#pragma unroll
          for (int i = 0; i < KMAX; ++i) { top[i] = -INFINITY; cls[i] = -1; }
        }
        // The sums, and the top's candidates, 64 classes at a time.
        RowSums sum;
        int behind = 0;
        const float m8 = m * (1.f / CUT);
        if (LONE && lone && sub == 0) { sum.add2(alone, -INFINITY, m8); behind = 1; }
        for (int j0 = 0; j0 < CW; j0 += 64 / NW) {
          uint32_t found[2] = {0, 0};
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll 1
            for (int i0 = 0; i0 < 32 / NW; i0 += STEP) {
              const int j1 = j0 + half * (32 / NW) + i0;
              if (j1 >= CW) break;
              // 8 classes; behind the row's end a class that is masked adds nothing to s and q (and one to others)
              float v[8];
              if (j1 + STEP <= CW) {
#pragma unroll
                for (int i = 0; i < STEP; ++i) {
                  float w[NW];
                  unpack<T>(mine[(j1 + i) * TPR], w);
#pragma unroll
                  for (int e = 0; e < NW; ++e) v[i * NW + e] = w[e];
                }
              } else {
#pragma unroll
                for (int i = 0; i < STEP; ++i) {
                  float w[NW];
#pragma unroll
                  for (int e = 0; e < NW; ++e) w[e] = -INFINITY;
                  if (j1 + i < CW) unpack<T>(mine[(j1 + i) * TPR], w);
#pragma unroll
                  for (int e = 0; e < NW; ++e) v[i * NW + e] = w[e];
                }
                behind += (j1 + STEP - CW) * NW;
              }
              uint32_t bits = 0;
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                sum.add2(v[e], v[e + 1], m8);
                if (KMAX) {
                  if (v[e] >= floor) bits |= 1u << e;
                  if (v[e + 1] >= floor) bits |= 2u << e;
                }
              }
              if (KMAX) found[half] |= bits << (i0 * NW);
            }
          if (KMAX)
            while (found[0] | found[1]) {
              const bool low = found[0] != 0;
              const uint32_t bits = low ? found[0] : found[1];
              const int place = j0 * NW + (low ? 0 : 32) + __ffs(bits) - 1, word = place / NW, at = (word * TPR + sub) * NW + place % NW + odd;
              if (low) found[0] = bits & (bits - 1); else found[1] = bits & (bits - 1);
              const float v = word < CW ? to_f32<T>(reinterpret_cast<const T*>(mine + word * TPR)[place % NW]) : -INFINITY;
              if (v > top[KMAX - 1]) {                     // equal ones keep their places: they have the lower classes
#pragma unroll
                for (int i = KMAX - 1; i > 0; --i) {
                  const bool down = v > top[i - 1], here = !down && v > top[i];
                  cls[i] = down ? cls[i - 1] : here ? at : cls[i];
                  top[i] = down ? top[i - 1] : here ? v : top[i];
                }
                if (v > top[0]) { top[0] = v; cls[0] = at; }
              }
            }
        }
        if (LONE && KMAX && lone && sub == 0 && alone > -INFINITY) {                 // of equal ones the first class comes first, the last one last
          const auto better = [&](float o) { return odd ? alone >= o : alone > o; };
          if (better(top[KMAX - 1])) {
#pragma unroll
            for (int i = KMAX - 1; i > 0; --i) {
              const bool down = better(top[i - 1]), here = !down && better(top[i]);
              cls[i] = down ? cls[i - 1] : here ? lone_class : cls[i];
              top[i] = down ? top[i - 1] : here ? alone : top[i];
            }
            if (better(top[0])) { top[0] = alone; cls[0] = lone_class; }
          }
        }
        float sums = sum.both(sum.s), q = sum.both(sum.q), others = sum.both(sum.others) - (float)behind;
#pragma unroll
        for (int d = TPR / 2; d; d >>= 1) {
          sums += __shfl_xor_sync(0xffffffffu, sums, d);
          q += __shfl_xor_sync(0xffffffffu, q, d);
          others += __shfl_xor_sync(0xffffffffu, others, d);
        }
        r = row_result({m, sums + ((float)(C - 1) - others), -CUT * q}, bad);
        if (sub == 0 && row < a.n) {
          if (a.logprob) a.logprob[row] = label < 0 ? 0.f : log_p(to_f32<T>(elements[label]), r);
          if (a.entropy) a.entropy[row] = r.H;
          if (a.stats) a.stats[row] = make_float2(r.m, r.l);
        }
        if (KMAX) {
          if (TPR == 1) {
#pragma unroll
            for (int i = 0; i < KMAX; ++i)
              if (i < a.k) {
                if (a.top_logprob) a.top_logprob[row * a.k + i] = cls[i] < 0 ? -INFINITY : log_p(top[i], r);
                if (a.top_class) a.top_class[row * a.k + i] = cls[i];
              }
          } else {
            // the threads' first ones, the best of them taken k times
            for (int i = 0; i < a.k; ++i) {
              float best = top[0];
              int where = cls[0] < 0 ? 0x7fffffff : cls[0];
#pragma unroll
              for (int d = TPR / 2; d; d >>= 1) {
                const float o = __shfl_xor_sync(0xffffffffu, best, d);
                const int oc = __shfl_xor_sync(0xffffffffu, where, d);
                if (o > best || (o == best && oc < where)) { best = o; where = oc; }
              }
              if (where == cls[0]) {
#pragma unroll
                for (int t = 0; t + 1 < KMAX; ++t) { top[t] = top[t + 1]; cls[t] = cls[t + 1]; }
                top[KMAX - 1] = -INFINITY; cls[KMAX - 1] = -1;
              }
              const bool none = where == 0x7fffffff;
              if (sub == 0 && row < a.n) {
                if (a.top_logprob) a.top_logprob[row * a.k + i] = none ? -INFINITY : log_p(best, r);
                if (a.top_class) a.top_class[row * a.k + i] = none ? -1 : where;
              }
            }
          }
        }
      } else {
        const long long from = row < a.n ? row : a.n - 1;
        const float2 ml = a.stats_in[from];
        r = {ml.x, ml.y, a.entropy_in ? a.entropy_in[from] : 0.f};
      }
      if (MODE != FORWARD) {
        const GradRow gr = grad_row(a, row < a.n ? row : a.n - 1, label, r);
        const bool special = label >= 0 && (LONE && lone && label == lone_class ? 0 : (label - odd) / NW % TPR) == sub;      // this thread has the label's word
        const float at = special ? to_f32<T>(elements[label]) : 0.f;
        if (TPR > 1) __syncwarp();               // (its logit has been read for the row's log probability too)
        int j = 0;
        for (; j + STEP <= CW; j += STEP) {
          Q w[STEP];
#pragma unroll
          for (int i = 0; i < STEP; ++i) w[i] = mine[(j + i) * TPR];
#pragma unroll
          for (int i = 0; i < STEP; i += 2 / NW) {
            float v[2], y[2];
            if constexpr (NW == 2) unpack<T>(w[i], v);
            else { v[0] = to_f32<T>(w[i]); v[1] = to_f32<T>(w[i + 1]); }
            grad_of2(gr, v[0], v[1], y, y + 1);
            if constexpr (NW == 2) mine[(j + i) * TPR] = pack<T>(y);
            else { mine[(j + i) * TPR] = from_f32<T>(y[0]); mine[(j + i + 1) * TPR] = from_f32<T>(y[1]); }
          }
        }
        for (; j < CW; ++j) {
          float v[NW];
          unpack<T>(mine[j * TPR], v);
#pragma unroll
          for (int e = 0; e < NW; ++e) v[e] = grad_of(gr, v[e]);
          mine[j * TPR] = pack<T>(v);
        }
        if (LONE && lone && sub == 0) elements[lone_class] = from_f32<T>(grad_of(gr, alone));
        if (special) elements[label] = from_f32<T>(grad_of_label(gr, at));
      }
    }
    __syncthreads();
    if (MODE != FORWARD) {
      t.store(sm, reinterpret_cast<W*>(static_cast<T*>(a.dx) + row0 * a.ld_dx), a.ld_dx / CN, a.mode_out);
      __syncthreads();
    }
  }
}

template <class T, bool PAIRS>
void set_tile(Args* a, int tpr) {
  constexpr int NW = PAIRS ? 2 : 1, V = 16 / (NW * (int)sizeof(T));               // elements of a word, words of a vector
  const int C = a->C / NW;
  // A warp reads words j tpr + sub of its 32 / tpr rows at once: how many of them meet in a bank hangs on the pitch.  Up to four cost less than rows set apart, which
  // cannot be copied by vectors.  (More threads to a row instead, up to 8, which meet by fours: 625 000 x 64 fp32 49 -> 91 us, 156 250 x 256 55 -> 58, with its gradient in bf16 61 -> 58.)
  const auto meet = [&](int pitch) {
    int most = 0, count[32] = {};
    for (int t = 0; t < 32; ++t) most = std::max(most, ++count[(t / tpr * pitch + t % tpr) % 32]);
    return most;
  };
  a->pitch = C;
  if (sizeof(T) * NW == 4 && meet(C) > 4)
    while (meet(a->pitch) > 2) ++a->pitch;
  const auto by = [](int d) { return d == 1 ? 0u : (unsigned)(((1ull << 32) + d - 1) / d); };
  a->vectors = (C + V - 1) / V;
  a->by_C = by(C); a->by_vectors = by(a->vectors);
  const auto mode = [&](const void* p, long long ld) {
    if (!rows_aligned(p, 16)) return (int)TILE_ELEMENTS;
    return ld == a->C ? (int)TILE_FLAT : ld % (V * NW) == 0 ? (int)TILE_VECTORS : (int)TILE_ELEMENTS;
  };
  a->mode_in = mode(a->x, a->ld);
  a->mode_out = mode(a->dx, a->ld_dx);
}

// What a kernel may ask for is set to the same figure by every call: calls of several host threads do not take it from one another.  (A tile of one thread to a row has 64 KB and
// what sets its rows apart.)
constexpr int TILE_MOST = 72 * 1024;
template <class T, bool PAIRS, int MODE, int KMAX, int TPR>
void launch_tiles(Launches& enqueue, Args a) {
  constexpr int ROWS = ROW_THREADS / TPR;
  set_tile<T, PAIRS>(&a, TPR);
  const size_t smem = (size_t)a.pitch * sizeof(T) * (PAIRS ? 2 : 1) * ROWS;
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(rows_kernel<T, PAIRS, MODE, KMAX, TPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, TILE_MOST);
    if (e != cudaSuccess) { enqueue.error = e; return; }
  }
  const int64_t tiles = (a.n + ROWS - 1) / ROWS;
  enqueue(rows_kernel<T, PAIRS, MODE, KMAX, TPR>, dim3((unsigned)std::min<int64_t>(tiles, 1 << 30)), ROW_THREADS, smem, a);
}
// Threads to a row: as many as leave each `EACH` bytes of it at most (a tile: 128 times that).  Fewer threads have fewer exchanges, and the top is found by each for itself before it is
// joined: the longer it is, the more classes to a thread; more threads have smaller tiles, more of them on an SM, and fewer of a warp's reads in one bank.  Without a top, 256 / 512: 400 000 x 172
// bf16 with gradient 73 / 76 us, 312 500 x 128 fp32 105 / 125, 57 142 x 700 bf16 59 / 63.  Top 3, 256 / 512: 312 500 x 128 fp32 69 / 87, 130 73 / 66, 80 000 x 500 62 / 83; top 8: 156 250 x 256 82 / 105,
// 133 333 x 300 88 / 80; top 16: 133 333 x 300 182 / 132, 232 558 x 172 177 / 136, 40 000 x 1 000 126 / 114.
template <class T, bool PAIRS, int MODE, int KMAX, int TPR = 1>
void launch_by_width(Launches& enqueue, const Args& a) {
  constexpr int EACH = KMAX == 0 ? 256 : KMAX <= 4 ? 320 : KMAX <= 8 ? 384 : 512, MOST = tile_classes(sizeof(T), MODE != FORWARD, KMAX) * (int)sizeof(T);
  if constexpr (TPR * EACH >= MOST) launch_tiles<T, PAIRS, MODE, KMAX, TPR>(enqueue, a);
  else if (a.C * (int)sizeof(T) <= TPR * EACH) launch_tiles<T, PAIRS, MODE, KMAX, TPR>(enqueue, a);
  else launch_by_width<T, PAIRS, MODE, KMAX, 2 * TPR>(enqueue, a);
}
template <class T, bool PAIRS>
void launch_rows(Launches& enqueue, const Args& a, int mode) {
  if (mode == TRAIN) launch_by_width<T, PAIRS, TRAIN, 0>(enqueue, a);
  else if (mode == GRAD) launch_by_width<T, PAIRS, GRAD, 0>(enqueue, a);
  else if (a.k == 0) launch_by_width<T, PAIRS, FORWARD, 0>(enqueue, a);
  else if (a.k <= 4) launch_by_width<T, PAIRS, FORWARD, 4>(enqueue, a);
  else if (a.k <= 8) launch_by_width<T, PAIRS, FORWARD, 8>(enqueue, a);
  else launch_by_width<T, PAIRS, FORWARD, MAX_TOP>(enqueue, a);
}

}  // namespace

#if LOGPROB_ROWS_TYPE == 0
void logprob_rows_f32(Launches& enqueue, const LogprobArgs& a, int mode) { launch_rows<float, false>(enqueue, a, mode); }
#elif LOGPROB_ROWS_TYPE == 1
void logprob_rows_bf16(Launches& enqueue, const LogprobArgs& a, int mode, bool pairs) {
  if (pairs) launch_rows<__nv_bfloat16, true>(enqueue, a, mode); else launch_rows<__nv_bfloat16, false>(enqueue, a, mode);
}
#else
void logprob_rows_f16(Launches& enqueue, const LogprobArgs& a, int mode, bool pairs) {
  if (pairs) launch_rows<__half, true>(enqueue, a, mode); else launch_rows<__half, false>(enqueue, a, mode);
}
#endif
