// Log probabilities of given classes from rows of logits, with the entropy and the top alternatives, and the gradient of the logits.
//
//   m = max x,  l = log sum e^(x - m),  log p_j = (x_j - m) - l,  H = -sum p log p = l - (sum e^(x - m) (x - m)) / e^l
//   grad x_j = g (delta_j,label - p_j) - h p_j (log p_j + H)           g: weight of log p_label, h: weight of H
//
// The largest term of the sum is 1: it is left out of the sum s of the others, and l = log1p(s), H = l - t / (1 + s).  Both parts of H are positive and nothing
// cancels: a row whose first class has nearly everything keeps all digits of l, H and 1 - p.  Differences are cut off at -200 (e^-200 = 0 in fp32): a
// masked class (-inf, or a type's lowest value) then adds 0 to both sums, and no 0 x inf comes up.  A NaN goes into m, and with it into everything; +inf is treated as NaN.
//
// Bytes bound it: the logits in, once (and their gradient out).
// Few classes: a thread to a row (rows_kernel).  A tile of rows comes into shared memory in 16-byte loads whatever the rows' width, each row on an odd number of words
// (16-bit rows of odd width: of halves), so that the threads of a warp read a column without conflicts.  The top's candidates are few: values not below the k-th largest of some
// maxima that the first pass over the row leaves.
// Many classes: a warp or a block to a row, or to a part of one where there are few rows (stream_kernel), in one pass with a running maximum of the warp; parts are joined in their
// order by join_kernel.  Candidates for the top are few (a value has to be above the k-th best so far): they go to a list of the warp in shared memory, sorted when it is half full.
#include <algorithm>

#include "rows.cuh"

namespace {

constexpr int MAX_TOP = TAURUS_MAX_TOP;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LEAST = -200.f;
constexpr int ROW_THREADS = 128;               // threads and rows of a block of rows_kernel
constexpr int WARPS = 8;                       // warps of a block of stream_kernel
constexpr int LIST = 64;                       // places of a warp's list of candidates
constexpr int MAX_PARTS = 64;                  // parts of a row

typedef unsigned long long u64;

struct Args {
  long long n;
  int C;
  const void* x;
  long long ld;
  const long long* labels;
  float *logprob, *entropy;
  float2* stats;
  int k;
  float* top_logprob;
  long long* top_class;
  // gradient
  const float *grad_logprob, *grad_entropy;
  const float2* stats_in;
  const float* entropy_in;
  void* dx;
  long long ld_dx;
  int32_t* status;
  // parts of a row
  int parts, part_len;
  float4* part;                                // [n x parts] (m, s, t, bad)
  u64* part_top;                               // [n x parts x k]
  // tiles of rows_kernel
  int pitch, mode_in, mode_out;
  unsigned by_C, by_vectors;                   // 2^32 / C, 2^32 / vectors of a row, rounded up
  int vectors;
};

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// Order of candidates: larger value first, of equal ones the lower class.  0: none (-inf, NaN).  -0 counts as 0.
__device__ __forceinline__ u64 key_of(float x, int cls) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
  return ((u64)o << 32) | (0xffffffffu - (uint32_t)cls);
}
__device__ __forceinline__ float key_value(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_class(u64 key) { return (int)(0xffffffffu - (uint32_t)key); }

// Sums of some classes of a row.  m: their largest value, whose own term (1) is in neither sum; -inf: no classes yet.
struct Sums { float m, s, t; };
// Joins b's classes, which come behind a's.
__device__ __forceinline__ void join(Sums& a, const Sums& b) {
  if (!(b.m > -INFINITY)) return;
  if (!(a.m > -INFINITY)) { a = b; return; }
  const bool up = b.m > a.m;
  const float d = fmaxf(up ? a.m - b.m : b.m - a.m, LEAST), f = ex2(d * LOG2E);
  const float ws = up ? b.s : a.s, wt = up ? b.t : a.t, os = up ? a.s : b.s, ot = up ? a.t : b.t;     // the side of the maximum, the other side
  const float o1 = 1.f + os;
  a.s = fmaf(o1, f, ws);
  a.t = wt + f * fmaf(o1, d, ot);
  if (up) a.m = b.m;
}

// What a row's sums say.
struct RowResult { float m, l, H; };
__device__ __forceinline__ RowResult row_result(const Sums& s, bool bad) {
  if (bad) return {NAN, NAN, NAN};
  if (!(s.m > -INFINITY)) return {s.m, 0.f, 0.f};
  const float l = log1pf(s.s);
  return {s.m, l, l - s.t / (1.f + s.s)};
}
__device__ __forceinline__ float log_p(float x, const RowResult& r) { return r.m == -INFINITY ? -INFINITY : (x - r.m) - r.l; }

// -1: no label; one outside the classes is reported.
__device__ __forceinline__ int label_of(const Args& a, long long row) {
  if (!a.labels) return -1;
  const long long v = a.labels[row];
  if (v < -1 || v >= a.C) { rows_status(a.status, TAURUS_ERR_INVALID_ARG); return -1; }
  return (int)v;
}
template <class T>
__device__ __forceinline__ void write_row(const Args& a, long long row, int label, const RowResult& r) {
  if (a.logprob) a.logprob[row] = label < 0 ? 0.f : log_p(to_f32<T>(static_cast<const T*>(a.x)[row * a.ld + label]), r);
  if (a.entropy) a.entropy[row] = r.H;
  if (a.stats) a.stats[row] = make_float2(r.m, r.l);
}
__device__ __forceinline__ void write_top(const Args& a, long long row, int i, u64 key, const RowResult& r) {
  if (a.top_logprob) a.top_logprob[row * a.k + i] = key ? log_p(key_value(key), r) : -INFINITY;
  if (a.top_class) a.top_class[row * a.k + i] = key ? key_class(key) : -1;
}

// What the gradient of a row needs.
struct GradRow {
  float m, l, H, g, h, c;
  int label;
};
__device__ __forceinline__ GradRow grad_row(const Args& a, long long row, int label, const RowResult& r) {
  const float g = label >= 0 && a.grad_logprob ? a.grad_logprob[row] : 0.f, h = a.grad_entropy ? a.grad_entropy[row] : 0.f;
  return {r.m, r.l, r.H, g, h, h == 0.f ? -g : fmaf(-h, r.H, -g), label};
}
__device__ __forceinline__ float grad_of(const GradRow& r, float x) {
  const float lp = fmaxf(x - r.m, LEAST) - r.l, p = ex2(lp * LOG2E);
  return x == -INFINITY ? 0.f : p * fmaf(-r.h, lp, r.c);
}
__device__ __forceinline__ float grad_of_label(const GradRow& r, float x) {
  const float lp = fmaxf(x - r.m, LEAST) - r.l, p = ex2(lp * LOG2E);
  return x == -INFINITY ? 0.f : -r.g * expm1f(lp) - r.h * p * (lp + r.H);
}

// ---- few classes: a thread to a row ------------------------------------------------------------------------------------------------------------------

// How a tile of rows lies in global memory: single elements | 16-byte vectors over rows without gaps | vectors within rows of a pitch.
enum { TILE_ELEMENTS = 0, TILE_FLAT = 1, TILE_VECTORS = 2 };
enum { FORWARD = 0, TRAIN = 1, GRAD = 2 };

// Words of shared memory, one element each, or two where 16-bit rows have an even width.
template <class T, bool PAIRS> struct Word { using type = T; static constexpr int n = 1; };
template <class T> struct Word<T, true> { using type = uint32_t; static constexpr int n = 2; };

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
      for (int f = threadIdx.x; f < rows * C; f += ROW_THREADS) { const int row = div(f, by_C), col = f - row * C; sm[row * P + col] = x[row * ld + col]; }
      return;
    }
    const bool flat = mode == TILE_FLAT;
    const int words = rows * C, total = flat ? words / V : rows * vectors;
    for (int v0 = threadIdx.x; v0 < total; v0 += 4 * ROW_THREADS) {
      Vec<W, V> r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = v0 + u * ROW_THREADS;
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
        const int v = v0 + u * ROW_THREADS;
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
      for (int f = total * V + threadIdx.x; f < words; f += ROW_THREADS) { const int row = div(f, by_C); sm[row * P + f - row * C] = x[f]; }
  }
  __device__ __forceinline__ void store(const W* sm, W* y, long long ld, int mode) const {
    if (mode == TILE_FLAT) {
      const int words = rows * C, total = words / V;
      for (int v = threadIdx.x; v < total; v += ROW_THREADS) {
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
      for (int f = total * V + threadIdx.x; f < words; f += ROW_THREADS) { const int row = div(f, by_C); y[f] = sm[row * P + f - row * C]; }
    } else if (mode == TILE_VECTORS) {
      for (int v = threadIdx.x; v < rows * vectors; v += ROW_THREADS) {
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
      for (int f = threadIdx.x; f < rows * C; f += ROW_THREADS) { const int row = div(f, by_C), col = f - row * C; y[row * ld + col] = sm[row * P + col]; }
    }
  }
};

template <class T>
__device__ __forceinline__ void unpack(T w, float (&x)[1]) { x[0] = to_f32<T>(w); }
template <class T>
__device__ __forceinline__ void unpack(uint32_t w, float (&x)[2]) {
  if constexpr (std::is_same_v<T, __nv_bfloat16>) { x[0] = __uint_as_float(w << 16); x[1] = __uint_as_float(w & 0xffff0000u); }
  else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w)); x[0] = f.x; x[1] = f.y; }
}
template <class T>
__device__ __forceinline__ T pack(const float (&x)[1]) { return from_f32<T>(x[0]); }
template <class T>
__device__ __forceinline__ uint32_t pack(const float (&x)[2]) {
  Vec<T, 2> r;
  r.v[0] = from_f32<T>(x[0]); r.v[1] = from_f32<T>(x[1]);
  return *reinterpret_cast<const uint32_t*>(&r);
}

// KMAX: places for the top in registers (k <= KMAX; 0: none asked for).
template <class T, bool PAIRS, int MODE, int KMAX>
__global__ void __launch_bounds__(ROW_THREADS) rows_kernel(const Args a) {
  extern __shared__ __align__(16) unsigned char logprob_shared[];
  using W = typename Word<T, PAIRS>::type;
  constexpr int NW = Word<T, PAIRS>::n;
  W* const sm = reinterpret_cast<W*>(logprob_shared);
  const int C = a.C, CW = C / NW;
  const long long tiles = (a.n + ROW_THREADS - 1) / ROW_THREADS;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const long long row0 = tile * ROW_THREADS, row = row0 + threadIdx.x;
    const Tile<W> t = {(int)(a.n - row0 < ROW_THREADS ? a.n - row0 : ROW_THREADS), CW, a.pitch, a.vectors, a.by_C, a.by_vectors};
    t.load(sm, reinterpret_cast<const W*>(static_cast<const T*>(a.x) + row0 * a.ld), a.ld / NW, a.mode_in);
    __syncthreads();
    if (row < a.n) {
      W* const mine = sm + threadIdx.x * a.pitch;
      const T* const elements = reinterpret_cast<const T*>(mine);
      const int label = label_of(a, row);
      RowResult r;
      if (MODE != GRAD) {
        // Maxima of G classes of classes: the k-th largest of them has k values at least that are not below it, so what is below it is not among the top k.
        constexpr int G = KMAX == 0 ? 4 : KMAX <= 4 ? 8 : 32;
        float most[G];
#pragma unroll
        for (int i = 0; i < G; ++i) most[i] = -INFINITY;
        int j = 0;
        for (; j + G / NW <= CW; j += G / NW)
#pragma unroll
          for (int i = 0; i < G / NW; ++i) {
            float v[NW];
            unpack<T>(mine[j + i], v);
#pragma unroll
            for (int e = 0; e < NW; ++e) most[i * NW + e] = max_nan(most[i * NW + e], v[e]);
          }
#pragma unroll
        for (int i = 0; i < G / NW; ++i)
          if (j + i < CW) {
            float v[NW];
            unpack<T>(mine[j + i], v);
#pragma unroll
            for (int e = 0; e < NW; ++e) most[i * NW + e] = max_nan(most[i * NW + e], v[e]);
          }
        float m = most[0];
#pragma unroll
        for (int i = 1; i < G; ++i) m = max_nan(m, most[i]);
        const bool bad = !(m < INFINITY);
        float top[KMAX ? KMAX : 1], floor = -INFINITY;
        int cls[KMAX ? KMAX : 1];
        if (KMAX) {
#pragma unroll
          for (int i = 0; i < KMAX; ++i) { top[i] = -INFINITY; cls[i] = -1; }
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float v = most[g];
#pragma unroll
            for (int i = 0; i < KMAX; ++i) { const float up = fmaxf(top[i], v); v = fminf(top[i], v); top[i] = up; }
          }
#pragma unroll
          for (int i = 0; i < KMAX; ++i) if (i == a.k - 1) floor = top[i];
          if (bad) floor = -INFINITY;                       // a NaN hides its class of classes
#pragma unroll
          for (int i = 0; i < KMAX; ++i) top[i] = -INFINITY;
        }
        // The sums, of what is below the maximum; how often that comes up; the top's candidates, 32 classes at a time.
        float s = 0.f, q = 0.f;
        int same = 0;
        constexpr int CHUNK = 32 / NW;
        for (int j0 = 0; j0 < CW; j0 += CHUNK) {
          uint32_t found = 0;
          const auto one = [&](int i) {
            float v[NW];
            unpack<T>(mine[j0 + i], v);
#pragma unroll
            for (int e = 0; e < NW; ++e) {
              const float d = fmaxf(v[e] - m, LEAST), p = ex2(d * LOG2E);
              const bool is = v[e] == m;
              same += is;
              s += is ? 0.f : p;
              q = fmaf(p, d, q);
              if (KMAX && v[e] >= floor) found |= 1u << (i * NW + e);
            }
          };
          if (j0 + CHUNK <= CW) {
#pragma unroll 8
            for (int i = 0; i < CHUNK; ++i) one(i);
          } else {
            for (int i = 0; j0 + i < CW; ++i) one(i);
          }
          if (KMAX)
            while (found) {
              const int b = __ffs(found) - 1, at = j0 * NW + b;
              found &= found - 1;
              const float v = to_f32<T>(elements[at]);
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
        r = row_result({m, s + (float)(same - 1), m == -INFINITY ? 0.f : q}, bad);
        if (a.logprob) a.logprob[row] = label < 0 ? 0.f : log_p(to_f32<T>(elements[label]), r);
        if (a.entropy) a.entropy[row] = r.H;
        if (a.stats) a.stats[row] = make_float2(r.m, r.l);
#pragma unroll
        for (int i = 0; i < KMAX; ++i)
          if (i < a.k) {
            if (a.top_logprob) a.top_logprob[row * a.k + i] = cls[i] < 0 ? -INFINITY : log_p(top[i], r);
            if (a.top_class) a.top_class[row * a.k + i] = cls[i];
          }
      } else {
        const float2 ml = a.stats_in[row];
        r = {ml.x, ml.y, a.entropy_in ? a.entropy_in[row] : 0.f};
      }
      if (MODE != FORWARD) {
        const GradRow gr = grad_row(a, row, label, r);
        const float at = label >= 0 ? to_f32<T>(elements[label]) : 0.f;
#pragma unroll 8
        for (int j = 0; j < CW; ++j) {
          float v[NW];
          unpack<T>(mine[j], v);
#pragma unroll
          for (int e = 0; e < NW; ++e) v[e] = grad_of(gr, v[e]);
          mine[j] = pack<T>(v);
        }
        if (label >= 0) reinterpret_cast<T*>(mine)[label] = from_f32<T>(grad_of_label(gr, at));
      }
    }
    __syncthreads();
    if (MODE != FORWARD) {
      t.store(sm, reinterpret_cast<W*>(static_cast<T*>(a.dx) + row0 * a.ld_dx), a.ld_dx / NW, a.mode_out);
      __syncthreads();
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

// A warp's candidates for the top: `count` keys in shared memory.  After a sort they are the k best so far; limit: the k-th best's key (0: fewer than k yet), above: its value.  Classes that
// come later have to be larger than that.  atleast: the largest such value of the block's warps: what is below it is not among the best k of the row.
struct Candidates {
  u64* list;
  int count;
  u64 limit;
  float above, atleast;
};
// Keeps the best k, in order.
__device__ __noinline__ void sort_candidates(Candidates& c, int k, uint32_t* shared_limit) {
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
  if (c.count == k) {
    c.limit = c.list[k - 1];
    c.above = key_value(c.limit);
    if (lane == 0) atomicMax(shared_limit, (uint32_t)(c.limit >> 32));
  }
}
// Every element of a batch, 32 at a time: for the first batch, and for one that brings more candidates than the list takes.
template <class T>
__device__ __noinline__ void add_all(Candidates& c, const Span<T> span, int v0, int U, float most, int k, uint32_t* shared_limit) {
  constexpr int V = Span<T>::V;
  const int lane = threadIdx.x & 31;
  // At least k of the lanes have a value that is not below the k-th largest of the lanes' maxima: what is below that is not among the best k.
  float kth = most != most ? -INFINITY : most;
  int rank = 0;
#pragma unroll 1
  for (int i = 0; i < 32; ++i) { const float o = __shfl_sync(0xffffffffu, kth, i); rank += o > kth || (o == kth && i < lane); }
  kth = __shfl_sync(0xffffffffu, kth, __ffs(__ballot_sync(0xffffffffu, rank == k - 1)) - 1);
  const float floor = fmaxf(kth, fmaxf(c.above, c.atleast));
#pragma unroll 1
  for (int u = 0; u < U; ++u) {
    const int at = span.column(v0 + u * 32 + lane);
#pragma unroll 1
    for (int i = 0; i < V; ++i) {
      u64 key = 0;
      if (at + i >= span.begin && at + i < span.end) {
        const float x = to_f32<T>(span.row[at + i]);
        if (x >= floor) key = key_of(x, at + i);
      }
      const unsigned yes = __ballot_sync(0xffffffffu, key > c.limit);
      if (yes) {
        if (key > c.limit) c.list[c.count + __popc(yes & ((1u << lane) - 1))] = key;
        c.count += __popc(yes);
        if (c.count > LIST - 32) sort_candidates(c, k, shared_limit);
      }
    }
  }
  sort_candidates(c, k, shared_limit);
}

template <class T, bool TOP, int WPR, bool WITH_GRAD>
__global__ void __launch_bounds__(32 * WARPS) stream_kernel(const Args a) {
  constexpr int V = 16 / (int)sizeof(T), U = 4, STEP = 32 * U;
  __shared__ u64 lists[TOP ? WARPS * LIST : 1];
  __shared__ float4 warp_sums[WARPS];
  __shared__ float4 shared_result;
  __shared__ uint32_t shared_limit[WARPS];
  early_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = WPR == 1 ? 0 : warp;
  const long long units = a.n * a.parts, stride = WPR == 1 ? (long long)gridDim.x * WARPS : gridDim.x;
  for (long long unit = WPR == 1 ? (long long)blockIdx.x * WARPS + warp : blockIdx.x; unit < units; unit += stride) {
    const long long row = a.parts == 1 ? unit : unit / a.parts;
    const int part = a.parts == 1 ? 0 : (int)(unit - row * a.parts);
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    const int begin = part * a.part_len, end = a.C - begin < a.part_len ? a.C : begin + a.part_len;
    const Span<T> span(x, begin, end);
    Sums sums = {-INFINITY, 0.f, 0.f};
    bool bad = false;
    Candidates top = {lists + (TOP ? warp * LIST : 0), 0, 0, -INFINITY, -INFINITY};
    uint32_t* const limit = &shared_limit[WPR == 1 ? warp : 0];
    if (TOP) {
      if (WPR == 1 ? lane == 0 : threadIdx.x == 0) *limit = 0;
      if (WPR == 1) __syncwarp(); else __syncthreads();
    }
    for (int v0 = span.first() + sub * STEP; v0 < span.last(); v0 += WPR * STEP) {
      Vec<T, V> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = v0 + u * 32 + lane;
        if (at < span.last()) raw[u] = span.template load<WITH_GRAD ? LOAD_PLAIN : LOAD_ONCE>(at);
        else
#pragma unroll
          for (int i = 0; i < V; ++i) raw[u].v[i] = from_f32<T>(-INFINITY);
      }
      float most = vector_max(raw[0]);
#pragma unroll
      for (int u = 1; u < U; ++u) most = max_nan(most, vector_max(raw[u]));
      if (TOP) {
        if (WPR > 1) {
          const uint32_t o = *reinterpret_cast<volatile uint32_t*>(limit);
          if (o) top.atleast = key_value((u64)o << 32);
        }
        // (not !(most <= ...): a NaN has its lane looked through)
        if (__any_sync(0xffffffffu, !(most <= top.above) && !(most < top.atleast))) {
          bool all = top.limit == 0;
          if (!all) {
            const int had = top.count;
            int mine = 0;
            if (!(most <= top.above) && !(most < top.atleast)) {
#pragma unroll
              for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) { const float x = to_f32<T>(raw[u].v[i]); mine += x > top.above && x >= top.atleast; }
            }
            int upto = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, upto, d); if (lane >= d) upto += o; }
            const int more = __shfl_sync(0xffffffffu, upto, 31);
            all = had + more > LIST;
            if (!all) {
              if (mine) {
                u64* to = top.list + had + upto - mine;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                  for (int i = 0; i < V; ++i) {
                    const float x = to_f32<T>(raw[u].v[i]);
                    if (x > top.above && x >= top.atleast) *to++ = key_of(x, span.column(v0 + u * 32 + lane) + i);
                  }
              }
              top.count = had + more;
              if (top.count > LIST / 2) sort_candidates(top, a.k, limit);
            }
          }
          if (all) add_all<T>(top, span, v0, U, most, a.k, limit);
        }
      }
      if (__any_sync(0xffffffffu, !(most <= sums.m))) {
        float w = most;
#pragma unroll
        for (int d = 16; d; d >>= 1) w = max_nan(w, __shfl_xor_sync(0xffffffffu, w, d));
        bad |= !(w < INFINITY);
        if (w > sums.m) {
          if (sums.m > -INFINITY) {
            const float d = fmaxf(sums.m - w, LEAST), f = ex2(d * LOG2E), s1 = sums.s + (lane == 0 ? 1.f : 0.f);
            sums.t = f * fmaf(s1, d, sums.t);
            sums.s = f * s1;
          }
          sums.m = w;
          if (lane == __ffs(__ballot_sync(0xffffffffu, most == w)) - 1) {        // this lane has the term that is 1
            bool found = false;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int i = 0; i < V; ++i) if (!found && to_f32<T>(raw[u].v[i]) == w) { raw[u].v[i] = from_f32<T>(-INFINITY); found = true; }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = fmaxf(to_f32<T>(raw[u].v[i]) - sums.m, LEAST), p = ex2(d * LOG2E);
          sums.s += p;
          sums.t = fmaf(p, d, sums.t);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      sums.s += __shfl_xor_sync(0xffffffffu, sums.s, d);
      sums.t += __shfl_xor_sync(0xffffffffu, sums.t, d);
    }
    if (TOP) {
      sort_candidates(top, a.k, limit);
      if (lane >= top.count && lane < a.k) top.list[lane] = 0;
    }
    if (WPR > 1) {
      if (lane == 0) warp_sums[warp] = make_float4(sums.m, sums.s, sums.t, bad ? 1.f : 0.f);
      __syncthreads();
      if (warp == 0) {
        const float4 first = warp_sums[0];
        sums = {first.x, first.y, first.z};
        bad = first.w != 0.f;
        for (int w = 1; w < WARPS; ++w) {
          const float4 o = warp_sums[w];
          join(sums, {o.x, o.y, o.z});
          bad |= o.w != 0.f;
        }
      }
    }
    RowResult r = row_result(sums, bad);
    const int label = a.parts == 1 ? label_of(a, row) : -1;
    if (WPR == 1 || warp == 0) {
      if (lane == 0) {
        if (a.parts == 1) write_row<T>(a, row, label, r);
        else a.part[unit] = make_float4(sums.m, sums.s, sums.t, bad ? 1.f : 0.f);
        if (WPR > 1 && WITH_GRAD) shared_result = make_float4(r.m, r.l, r.H, 0.f);
      }
      if (TOP) {
        if (WPR == 1) {
          __syncwarp();
          if (lane < a.k) write_top(a, row, lane, top.list[lane], r);
        } else {
          // the lists' heads, the best of them taken k times
          int head = 0;
          u64 mine = lane < WARPS ? lists[lane * LIST] : 0, keep = 0;
          for (int i = 0; i < a.k; ++i) {
            const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
            const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32) == hi ? (uint32_t)mine : 0u);
            const u64 best = ((u64)hi << 32) | lo;
            if (lane == i) keep = best;
            if (best && mine == best) { ++head; mine = head < a.k ? lists[lane * LIST + head] : 0; }
          }
          if (lane < a.k) {
            if (a.parts == 1) write_top(a, row, lane, keep, r);
            else a.part_top[unit * a.k + lane] = keep;
          }
        }
      }
    }
    if (WITH_GRAD) {
      __syncwarp();                             // the label's logit has been read before its place is written
      if (WPR > 1) {
        __syncthreads();
        const float4 sr = shared_result;
        r = {sr.x, sr.y, sr.z};
      }
      const GradRow gr = grad_row(a, row, label, r);
      T* const dx = static_cast<T*>(a.dx) + row * a.ld_dx;
      const bool alike = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(x)) & 15) == 0;
      // from the end, which the caches have had last
      for (int v = span.last() - 1 - (WPR == 1 ? lane : (int)threadIdx.x); v >= span.first(); v -= 32 * WPR) {
        const Vec<T, V> in = span.template load<LOAD_PLAIN>(v);
        const int c = span.column(v);
        Vec<T, V> out;
#pragma unroll
        for (int i = 0; i < V; ++i) out.v[i] = from_f32<T>(c + i == label ? grad_of_label(gr, to_f32<T>(in.v[i])) : grad_of(gr, to_f32<T>(in.v[i])));
        if (alike && c >= 0 && c + V <= a.C) store_vec_once(dx + c, out);
        else
#pragma unroll
          for (int i = 0; i < V; ++i) if (c + i >= 0 && c + i < a.C) dx[c + i] = out.v[i];
      }
    }
    if (WPR > 1) __syncthreads();
    else __syncwarp();
  }
}

// The parts of a row, in their order: a warp to a row.
template <class T>
__global__ void __launch_bounds__(128) join_kernel(const Args a) {
  early_start();
  const int lane = threadIdx.x & 31;
  for (long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5); row < a.n; row += (long long)gridDim.x * 4) {
    const float4* const part = a.part + row * a.parts;
    Sums sums = {-INFINITY, 0.f, 0.f};
    bool bad = false;
    for (int i = 0; i < a.parts; ++i) {
      const float4 o = part[i];
      join(sums, {o.x, o.y, o.z});
      bad |= o.w != 0.f;
    }
    const RowResult r = row_result(sums, bad);
    const int label = label_of(a, row);
    if (lane == 0) write_row<T>(a, row, label, r);
    if (a.k) {
      const u64* const top = a.part_top + row * a.parts * a.k;
      int head0 = 0, head1 = 0;
      u64 h0 = lane < a.parts ? top[lane * a.k] : 0, h1 = lane + 32 < a.parts ? top[(lane + 32) * a.k] : 0, keep = 0;
      for (int i = 0; i < a.k; ++i) {
        const u64 mine = h0 > h1 ? h0 : h1;
        const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
        const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32) == hi ? (uint32_t)mine : 0u);
        const u64 best = ((u64)hi << 32) | lo;
        if (lane == i) keep = best;
        if (best && h0 == best) { ++head0; h0 = head0 < a.k ? top[lane * a.k + head0] : 0; }
        else if (best && h1 == best) { ++head1; h1 = head1 < a.k ? top[(lane + 32) * a.k + head1] : 0; }
      }
      if (lane < a.k) write_top(a, row, lane, keep, r);
    }
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
      for (int i = 0; i < V; ++i) out.v[i] = from_f32<T>(c + i == gr.label ? grad_of_label(gr, to_f32<T>(in[u].v[i])) : grad_of(gr, to_f32<T>(in[u].v[i])));
      if (alike && c >= 0 && c + V <= a.C) store_vec_once(dx + c, out);
      else
#pragma unroll
        for (int i = 0; i < V; ++i) if (c + i >= 0 && c + i < a.C) dx[c + i] = out.v[i];
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------------------------

constexpr int ROWS_BYTES = 512;                // widest row, in bytes, that a thread takes
inline bool by_thread(int C, int ts) { return (int64_t)C * ts <= ROWS_BYTES; }

// How a row of many classes is split.  What does for n rows does for fewer: parts x n is largest for the fewest rows of a kind, so workspaces are counted for any n below.
constexpr int ENOUGH_WARPS = 148 * 16, ENOUGH_BLOCKS = 148 * 4, PART_MIN = 8192;
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

template <class T, bool PAIRS>
void set_tile(Args* a) {
  constexpr int NW = PAIRS ? 2 : 1, V = 16 / (NW * (int)sizeof(T));               // elements of a word, words of a vector
  const int C = a->C / NW;
  a->pitch = sizeof(T) * NW == 2 ? C : C | 1;                                     // (PAIRS: even widths; else odd ones of 16 bits, or fp32)
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

template <class T, bool PAIRS, int MODE, int KMAX>
void launch_tiles(Launches& enqueue, Args a) {
  set_tile<T, PAIRS>(&a);
  const size_t smem = (size_t)a.pitch * sizeof(T) * (PAIRS ? 2 : 1) * ROW_THREADS;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(rows_kernel<T, PAIRS, MODE, KMAX>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) { enqueue.error = e; return; }
  }
  const int64_t tiles = (a.n + ROW_THREADS - 1) / ROW_THREADS;
  enqueue(rows_kernel<T, PAIRS, MODE, KMAX>, dim3((unsigned)std::min<int64_t>(tiles, 1 << 30)), ROW_THREADS, smem, a);
}
template <class T, int MODE, int KMAX>
void launch_rows(Launches& enqueue, const Args& a) {
  // Pairs: rows of 16 bits that begin at even elements everywhere.
  if constexpr (sizeof(T) == 2) {
    const auto even = [](const void* p, long long ld) { return rows_aligned(p, 4) && ld % 2 == 0; };
    if (a.C % 2 == 0 && even(a.x, a.ld) && (MODE == FORWARD || even(a.dx, a.ld_dx))) { launch_tiles<T, true, MODE, KMAX>(enqueue, a); return; }
  }
  launch_tiles<T, false, MODE, KMAX>(enqueue, a);
}
template <class T>
void launch_grad(Launches& enqueue, const Args& a, int sms) {
  constexpr int V = 16 / (int)sizeof(T);
  const int chunks = ((a.C + 2 * V - 2) / V + GRAD_VECTORS * 32 - 1) / (GRAD_VECTORS * 32);     // vectors of a row wherever it begins
  enqueue(grad_kernel<T>, dim3((unsigned)std::min<int64_t>((a.n * chunks + 7) / 8, (int64_t)sms * 64)), 256, 0, a, chunks);
}
template <class T, bool TOP, bool WITH_GRAD>
void launch_stream(Launches& enqueue, const Args& a, int sms) {
  if (a.parts == 1 && a.n >= ENOUGH_WARPS)
    enqueue(stream_kernel<T, TOP, 1, WITH_GRAD>, dim3((unsigned)std::min<int64_t>((a.n + WARPS - 1) / WARPS, 1 << 30)), 32 * WARPS, 0, a);
  else
    enqueue(stream_kernel<T, TOP, WARPS, WITH_GRAD>, dim3((unsigned)std::min<int64_t>(a.n * a.parts, 1 << 30)), 32 * WARPS, 0, a);
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
  a.parts = by_thread(a.C, ts) ? 1 : parts_of(n, a.C);
  const int64_t need = what != GIVEN_STATS && a.parts > 1 ? (int64_t)sp.bytes : 0;
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) || !workspace_ok(workspace, workspace_bytes, need, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  a.part_len = a.parts == 1 ? a.C : (int)(((int64_t)a.C + a.parts - 1) / a.parts);
  Launches enqueue = {st};
  with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    if (by_thread(a.C, ts)) {
      if (what == GIVEN_STATS) launch_rows<T, GRAD, 0>(enqueue, a);
      else if (what == GIVEN_WEIGHTS) launch_rows<T, TRAIN, 0>(enqueue, a);
      else if (a.k == 0) launch_rows<T, FORWARD, 0>(enqueue, a);
      else if (a.k <= 4) launch_rows<T, FORWARD, 4>(enqueue, a);
      else launch_rows<T, FORWARD, MAX_TOP>(enqueue, a);
      return 0;
    }
    if (what == GIVEN_STATS) { launch_grad<T>(enqueue, a, sms); return 0; }
    if (a.parts == 1) {
      if (what == GIVEN_WEIGHTS) launch_stream<T, false, true>(enqueue, a, sms);
      else if (a.k) launch_stream<T, true, false>(enqueue, a, sms);
      else launch_stream<T, false, false>(enqueue, a, sms);
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
    if (a.k) launch_stream<T, true, false>(enqueue, a, sms);
    else launch_stream<T, false, false>(enqueue, a, sms);
    enqueue(join_kernel<T>, dim3((unsigned)std::min<int64_t>((n + 3) / 4, 1 << 20)), 128, 0, a);
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
