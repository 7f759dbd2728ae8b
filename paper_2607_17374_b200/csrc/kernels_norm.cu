// Group norm with an activation over the rows of a batch of graphs, channels last, and its gradients.
//
// Per graph s (rows [b, e)) and group g (C / groups neighbouring channels), m = (e - b) C / groups elements:
//   mean = sum x / m,  rstd = (sum (x - mean)^2 / m + eps)^-1/2,  xh = (x - mean) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z),  grad_gamma = sum dz xh,  grad_beta = sum dz (over all rows),
//   dx = rstd (gamma dz - mean_g(gamma dz) - xh mean_g(gamma dz xh))
//
// Bytes bound it: x in, y out (dx: x and dy in, dx out).  Statistics need all of a graph before its first row can be written.  A short graph
// is the work of one block, which reads its rows twice, the second time from the caches where they are few.  The rows of a long graph are spread over
// blocks of R rows (stats), their partial statistics joined in a fixed order (combine), and the rows are read again and written (apply).  How long
// a graph is stands in device memory: the kernel for short graphs leaves a word that says whether there are others.
//
// A thread keeps to one vector of channels and walks the rows.  Moments are taken of a batch of its rows in registers (mean first, then squares of
// deviations) and joined as (count, mean, sum of squared deviations): neither an offset nor a single large value eats the variance, as they would with sums of squares.
// All in fp32, the parts of a long graph in fp64.
//
// 1 M x 256 fp32 in 3 graphs: forward 506 us (three passes over the matrix, 6.1 TB/s), backward 808 (five, 6.3 TB/s).  262 144 x 64 bf16 in 9 001 graphs: 41 to 45 us replayed, 46
// with inputs that are new each pass, for which instructions and latency count (22 M by warps, 1 220 a warp and graph, 0.63 a cycle and scheduler), not the 10 us that its bytes take.
#include <algorithm>

#include "rows.cuh"

namespace {

constexpr int MAX_C = TAURUS_MAX_ROW_WIDTH;

struct NormArgs {
  long long n, graphs;
  const long long* offsets;              // null: one graph of n rows
  long long ld_x, ld_y, ld_dy;           // ld_y: of the rows written
  int C, groups, cg, vpr;                // cg: channels of a group; vpr: vectors of a row
  int lanes, shift;                      // rows that a block walks at once, 1 << shift
  float eps;
  const float *gamma, *beta;             // null: ones, zeros
  float *mean, *rstd;                    // [graphs x groups]
  long long R, blocks;                   // rows of a block of rows; their number
  int short_blocks, row_grid;            // blocks of the kernel for short graphs; blocks that share the blocks of rows
  int* any_long;                         // is there a long graph?
  float2* part;                          // [blocks x 2 x groups]
  float2* chan;                          // [(row_grid + short_blocks) x C] (grad_gamma, grad_beta) of a block
  float2* sums;                          // [graphs x groups] backward: the two means of a long graph
  float *grad_gamma, *grad_beta;
  int32_t* status;
};

// 1 / (1 + e^-z) by the hardware's exponential and reciprocal.  By their documented bounds (2 + 1.173 |z| ulp and 2 ulp) z / (1 + e^-z) is off by at most
// |z| s (1 - s) (2 + 1.173 |z|) 2^-23 < 2^-23 from the exponential, largest near |z| = 2, and 2.5 2^-23 of itself from the sum and the division.  Where e^-z is above
// 2^126 the quotient is 0: below z = -87.3, where the value is above -1.2e-36.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  if (ACT == TAURUS_ACT_RELU) return z < 0.f ? 0.f : z;
  if (ACT == TAURUS_ACT_SILU) return z * sigmoid(z);
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == TAURUS_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == TAURUS_ACT_SILU) { const float s = sigmoid(z); return s * (1.f + z * (1.f - s)); }
  return 1.f;
}

__device__ __forceinline__ void graph_rows(const NormArgs& a, long long s, long long* b, long long* e, int32_t* status = nullptr) {
  if (!a.offsets) { *b = 0; *e = a.n; return; }
  group_rows(a.offsets, s, a.n, b, e, status);
}

// The graph that row r belongs to (-1: none): the last one whose offset is not above r.  By one warp, 32 offsets a step.
__device__ __forceinline__ long long graph_of(const NormArgs& a, long long r) {
  if (!a.offsets) return 0;
  const int lane = threadIdx.x & 31;
  long long lo = 0, hi = a.graphs + 1;      // the number of offsets not above r lies in [lo, hi]
  while (lo < hi) {
    const long long step = (hi - lo + 31) / 32;
    const long long i = lo + step * lane;   // offsets[i] <= r for a first run of lanes
    const unsigned yes = __ballot_sync(0xffffffffu, i < hi && a.offsets[i] <= r);
    const int k = __popc(yes);              // (any count: offsets out of order are refused, but read in bounds)
    if (k == 0) break;
    const long long next = lo + step * k;
    lo += step * (k - 1) + 1;
    if (next < hi) hi = next;
    if (step == 1) break;
  }
  const long long s = lo - 1;
  return s >= 0 && s < a.graphs ? s : -1;
}

// Shared memory: red [lanes x vpr x NG] | stat [groups].
__device__ __forceinline__ float2* shared_red() { extern __shared__ __align__(16) float2 norm_shared[]; return norm_shared; }

// SAME: the V channels of a vector are of one group, and a thread has one mean for them; else one for each (NG of them).
template <int V, bool SAME> constexpr int ng() { return SAME ? 1 : V; }
// Row vectors of a thread in flight: of a long graph's rows, and of a short graph's, whose code is run a few times a block only and has to be short
// (with 4 to 8 of them, twice over, it came from beyond the instruction caches: 15 us for a graph of 40 rows).
template <int V> constexpr int batch() { return V == 8 ? 4 : 8; }
template <int V> constexpr int grad_batch() { return V == 8 ? 2 : 4; }
template <int V> constexpr int short_batch() { return V == 8 ? 2 : 4; }
template <int V> constexpr int short_grad_batch() { return V == 8 ? 2 : 4; }
// Vectors of a short graph of average length to a thread: 32 elements, over which what a graph costs each thread is spread (262 144 x 64 in 9 001 graphs,
// bf16 / fp32, 32 elements 41 / 49 us, 16 47 / 54, 64 44 / 55; with the gradient 150 / 149, 145 / 147, 187 / 190).
template <int V> constexpr int short_vectors() { return 32 / V; }

struct Moments { float n, mean, m2; };
__device__ __forceinline__ void join(Moments& a, float nb, float mb, float m2b) {
  if (nb > 0.f) {
    const float d = mb - a.mean, n = a.n + nb, f = __fdividef(nb, n);
    a.m2 += m2b + d * d * a.n * f;
    a.mean += d * f;
    a.n = n;
  }
}

// What a thread knows for the whole launch.
template <class T, int V, bool SAME>
struct Place {
  int cv, r;
  bool on;
  int g[ng<V, SAME>()];
  __device__ __forceinline__ explicit Place(const NormArgs& a) {
    cv = threadIdx.x % a.vpr; r = threadIdx.x / a.vpr;
    on = r < a.lanes;
#pragma unroll
    for (int k = 0; k < ng<V, SAME>(); ++k) g[k] = (cv * V + k) / a.cg;
  }
  // Rows of [b, e) that are this thread's.
  __device__ __forceinline__ int rows(const NormArgs& a, long long b, long long e) const { return rows(a, (int)(e - b)); }
  __device__ __forceinline__ int rows(const NormArgs& a, int len) const {
    return on && len > r ? (len - r + a.lanes - 1) >> a.shift : 0;
  }
  __device__ __forceinline__ const T* at(const T* x, long long ld, long long b) const { return x + (b + r) * ld + cv * V; }
};

template <class T, int V, int U>
__device__ __forceinline__ void load_batch(Vec<T, V> (&v)[U], const T* p, long long step, int left) {
#pragma unroll
  for (int u = 0; u < U; ++u) if (u < left) v[u] = load_vec<Vec<T, V>>(p + u * step);
}
// Keeps vectors as they were loaded: without it the compiler keeps the fp32 values it made of them, twice as many registers for 16-bit types.
template <class T, int V, int U>
__device__ __forceinline__ void as_loaded(Vec<T, V> (&v)[U]) {
  if constexpr (sizeof(T) == 2 && V > 1) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < V / 2; ++i) asm volatile("" : "+r"(reinterpret_cast<unsigned*>(&v[u])[i]));
  }
}
// Joins the first min(left, U) vectors to m.
template <class T, int V, int U, bool SAME>
__device__ __forceinline__ void add_batch(Moments (&m)[ng<V, SAME>()], Vec<T, V> (&v)[U], int left) {
  const int count = left < U ? left : U;
  if (SAME) {
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < left)
#pragma unroll
        for (int k = 0; k < V; ++k) s += to_f32<T>(v[u].v[k]);
    const float n = (float)(count * V), mean = __fdividef(s, n);
    as_loaded(v);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < left)
#pragma unroll
        for (int k = 0; k < V; ++k) { const float d = to_f32<T>(v[u].v[k]) - mean; q += d * d; }
    // (deviations from a mean that is off by its rounding: the square of that is far below the sum)
    join(m[0], n, mean, q);
  } else {
    const float n = (float)count, inv = __fdividef(1.f, n);
#pragma unroll
    for (int k = 0; k < ng<V, SAME>(); ++k) {
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) if (u < left) s += to_f32<T>(v[u].v[k]);
      const float mean = s * inv;
#pragma unroll
      for (int u = 0; u < U; ++u) if (u < left) { const float d = to_f32<T>(v[u].v[k]) - mean; q += d * d; }
      join(m[k], n, mean, q);
    }
  }
}

// Teams of a power of two of threads share a group's entries in `red`: a.lanes rows of w entries, `row` apart.
template <int V, bool SAME>
struct Team {
  int w, row, entries, size, teams, t, first, r0, j0, dr, dj;
  __device__ __forceinline__ explicit Team(const NormArgs& a) {
    w = SAME ? a.cg / V : a.cg; row = SAME ? a.vpr : a.C; entries = a.lanes * w;
    int log = 0;
    while (log < 5 && (1 << log) < entries && (2 << log) * a.groups <= (int)blockDim.x) ++log;
    size = 1 << log;
    teams = blockDim.x >> log; t = threadIdx.x & (size - 1); first = threadIdx.x >> log;
    r0 = t / w; j0 = t % w; dr = size / w; dj = size % w;
  }
  // f(row, value) for this thread's entries of group g
  template <class F>
  __device__ __forceinline__ void each(const float2* red, int g, F f) const {
    int r = r0, j = j0;
    for (int i = t; i < entries; i += size) {
      f(r, red[r * row + g * w + j]);
      r += dr; j += dj;
      if (j >= w) { j -= w; ++r; }
    }
  }
};

// Moments of every group over a part of `len` rows: red holds (mean, m2) of every thread; out[g] = (mean, m2).
template <int V, bool SAME>
__device__ __forceinline__ void join_block(const NormArgs& a, const Team<V, SAME>& team, const float2* red, int len, float2* out) {
  for (int g0 = 0; g0 < a.groups; g0 += team.teams) {
    const int g = g0 + team.first;
    Moments m = {0.f, 0.f, 0.f};
    if (g < a.groups)
      team.each(red, g, [&](int r, float2 p) { join(m, len > r ? (float)(((len - r + a.lanes - 1) >> a.shift) * (SAME ? V : 1)) : 0.f, p.x, p.y); });
    for (int o = team.size / 2; o > 0; o >>= 1) {
      const float n = __shfl_down_sync(0xffffffffu, m.n, o), mean = __shfl_down_sync(0xffffffffu, m.mean, o), m2 = __shfl_down_sync(0xffffffffu, m.m2, o);
      join(m, n, mean, m2);
    }
    if (g < a.groups && team.t == 0) out[g] = make_float2(m.mean, m.m2);
  }
}

template <class T, int V, bool SAME>
__device__ __forceinline__ void put_moments(const Place<T, V, SAME>& at, const NormArgs& a, const Moments (&m)[ng<V, SAME>()], float2* red) {
  if (!at.on) return;
#pragma unroll
  for (int k = 0; k < ng<V, SAME>(); ++k) red[(at.r * a.vpr + at.cv) * ng<V, SAME>() + k] = make_float2(m[k].mean, m[k].m2);
}

// y = act((x - mean) rstd gamma + beta) of a thread's vectors; stat: (mean, rstd).
template <class T, int V, bool SAME>
struct Apply {
  float mean[ng<V, SAME>()], mul[V], add[V];
  __device__ __forceinline__ void set(const Place<T, V, SAME>& at, const float (&gamma)[V], const float (&beta)[V], const float2* stat) {
    stats(at, stat);
#pragma unroll
    for (int k = 0; k < V; ++k) { mul[k] = rstd[SAME ? 0 : k] * gamma[k]; add[k] = beta[k]; }
  }
  __device__ __forceinline__ void set(const Place<T, V, SAME>& at, const float2* channel, const float2* stat) {
    stats(at, stat);
#pragma unroll
    for (int k = 0; k < V; ++k) { const float2 c = channel[k]; mul[k] = rstd[SAME ? 0 : k] * c.x; add[k] = c.y; }
  }
  float rstd[ng<V, SAME>()];
  __device__ __forceinline__ void stats(const Place<T, V, SAME>& at, const float2* stat) {
#pragma unroll
    for (int k = 0; k < ng<V, SAME>(); ++k) { const float2 s = stat[at.g[k]]; mean[k] = s.x; rstd[k] = s.y; }
  }
  template <int ACT>
  __device__ __forceinline__ void row(const Vec<T, V>& v, T* y) const {
    float o[V];
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = act_f<ACT>((to_f32<T>(v.v[k]) - mean[SAME ? 0 : k]) * mul[k] + add[k]);
    store_f32<T, V>(y, o);
  }
};
template <int V>
__device__ __forceinline__ void affine(const NormArgs& a, int cv, float (&gamma)[V], float (&beta)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) { gamma[k] = a.gamma ? a.gamma[cv * V + k] : 1.f; beta[k] = a.beta ? a.beta[cv * V + k] : 0.f; }
}

// Threads of a block: at most 512, but for rows of up to 1 024 vectors.
constexpr int block_limit(int v) { return MAX_C / v > 512 ? 1024 : 512; }
// Threads of a block of the kernels for long graphs, and blocks to an SM (80 registers a thread).
constexpr int ROW_THREADS = 256;
constexpr int row_limit(int v) { return MAX_C / v > ROW_THREADS ? MAX_C / v : ROW_THREADS; }
constexpr int row_blocks(int v) { return row_limit(v) > 768 ? 1 : 768 / row_limit(v); }

// (64 registers a thread, a few of them in local memory: 2 000 graphs of 250 x 256 fp32, forward and backward, 801 -> 752 us)
template <class T, int V, bool SAME, int ACT>
__global__ void __launch_bounds__(block_limit(V), V > 1 ? 2 : 1) norm_short_kernel(const NormArgs a, const T* x, T* y) {
  early_start();
  float2* const red = shared_red();
  float2* const stat = red + (size_t)a.lanes * a.vpr * ng<V, SAME>();
  const Place<T, V, SAME> at(a);
  const Team<V, SAME> team(a);
  float2* const channel = stat + a.groups;                            // (gamma, beta)
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) channel[c] = make_float2(a.gamma ? a.gamma[c] : 1.f, a.beta ? a.beta[c] : 0.f);
  const long long step = a.lanes * a.ld_x, ystep = a.lanes * a.ld_y;
  const int graphs = (int)a.graphs, longest = (int)(2 * a.R < a.n ? 2 * a.R : a.n);
  int b, len, next_b = 0, next_len = 0;                               // (the next graph's offsets are on their way while this one is at work)
  auto look = [&](int s) {
    long long u, v;
    graph_rows(a, s, &u, &v, threadIdx.x == 0 ? a.status : nullptr);
    next_b = (int)u; next_len = (int)(v - u);
  };
  look(blockIdx.x);
  for (int s = blockIdx.x; s < graphs; s += gridDim.x) {
    b = next_b; len = next_len;
    if (s < graphs - (int)gridDim.x) look(s + gridDim.x);
    if (len > longest) {                                            // long: the other kernels'
      if (threadIdx.x == 0) *a.any_long = 1;
      continue;
    }
    if (len == 0) {
      for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        if (a.mean) a.mean[(long long)s * a.groups + g] = 0.f;
        if (a.rstd) a.rstd[(long long)s * a.groups + g] = 0.f;
      }
      continue;
    }
    const int rows = at.rows(a, len);
    constexpr int U = short_batch<V>();
    {
      Moments m[ng<V, SAME>()] = {};
      const T* p = at.at(x, a.ld_x, b);
#pragma unroll 1
      for (int left = rows; left > 0; left -= U) {
        Vec<T, V> v[U];
        load_batch<T, V, U>(v, p, step, left);
        add_batch<T, V, U, SAME>(m, v, left);
        p += U * step;
      }
      put_moments(at, a, m, red);
    }
    __syncthreads();
    join_block(a, team, red, len, stat);
    __syncthreads();
    const float inv = __fdividef(1.f, (float)len * (float)a.cg);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
      const float2 q = stat[g];
      const float rstd = rsqrtf(q.y * inv + a.eps);
      stat[g] = make_float2(q.x, rstd);
      if (a.mean) a.mean[(long long)s * a.groups + g] = q.x;
      if (a.rstd) a.rstd[(long long)s * a.groups + g] = rstd;
    }
    __syncthreads();
    Apply<T, V, SAME> f;
    if (rows > 0) f.set(at, channel + at.cv * V, stat);
    const T* p = at.at(x, a.ld_x, b);
    T* q = y + ((long long)b + at.r) * a.ld_y + at.cv * V;
#pragma unroll 1
    for (int left = rows; left > 0; left -= U) {
      Vec<T, V> v[U];
      load_batch<T, V, U>(v, p, step, left);
#pragma unroll
      for (int u = 0; u < U; ++u) if (u < left) f.template row<ACT>(v[u], q + u * ystep);
      p += U * step; q += U * ystep;
    }
    __syncthreads();                                                  // red and stat are written again
  }
}

// The parts of long graphs in block of rows `blk`: slot 0 is the graph of its first row, slot 1 that of its last row where another one begins
// in the block.  (A long graph has more than 2 R rows, so no third one can meet the block.)
struct Parts { long long s[2], b[2], e[2]; };                       // graph (-1: none), the part's rows
__device__ __forceinline__ void find_parts(const NormArgs& a, long long blk, Parts* p) {     // p in shared memory; by the whole block
  const long long r0 = blk * a.R, r1 = r0 + a.R < a.n ? r0 + a.R : a.n;
  __syncthreads();                        // the block is through with the parts before
  if (threadIdx.x < 32)                   // (both by one warp: a block may have no second one)
    for (int k = 0; k < 2; ++k) {
      long long s = graph_of(a, k ? r1 - 1 : r0), b = 0, e = 0;
      if (s >= 0) {
        graph_rows(a, s, &b, &e);
        if (e - b <= 2 * a.R || (k && b <= r0)) s = -1;
      }
      if (threadIdx.x == 0) {
        const long long pb = b > r0 ? b : r0, pe = e < r1 ? e : r1;
        if (pb >= pe) s = -1;
        p->s[k] = s; p->b[k] = pb; p->e[k] = pe;
      }
    }
  __syncthreads();
}

template <class T, int V, bool SAME>
__global__ void __launch_bounds__(row_limit(V), row_blocks(V)) norm_stats_kernel(const NormArgs a, const T* x) {
  early_start();
  __shared__ Parts parts;
  if (!*a.any_long) return;
  float2* const red = shared_red();
  const Place<T, V, SAME> at(a);
  const Team<V, SAME> team(a);
  const long long step = a.lanes * a.ld_x;
  for (long long blk = blockIdx.x; blk < a.blocks; blk += gridDim.x) {
    find_parts(a, blk, &parts);
    for (int k = 0; k < 2; ++k) {
      if (parts.s[k] < 0) continue;
      const T* p = at.at(x, a.ld_x, parts.b[k]);
      Moments m[ng<V, SAME>()] = {};
      for (int left = at.rows(a, parts.b[k], parts.e[k]); left > 0; left -= batch<V>()) {
        Vec<T, V> v[batch<V>()];
        load_batch<T, V, batch<V>()>(v, p, step, left);
        add_batch<T, V, batch<V>(), SAME>(m, v, left);
        p += batch<V>() * step;
      }
      put_moments(at, a, m, red);
      __syncthreads();
      join_block(a, team, red, (int)(parts.e[k] - parts.b[k]), a.part + (blk * 2 + k) * a.groups);
      __syncthreads();
    }
  }
}

__device__ __forceinline__ double warp_sum(double v) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The partial results of a long graph lie in slot 0 of the blocks of rows it meets, but for the block it begins in the middle of.
struct Owned { long long s, begin, end, first, last; int first_slot; };
// Long graph number i, if it is one: of the graphs themselves where there are fewer than blocks of rows, else the one that begins in block of rows i.  By every warp for itself.
__device__ __forceinline__ long long owners(const NormArgs& a) { return a.graphs < a.blocks ? a.graphs : a.blocks; }
__device__ __forceinline__ bool owned_graph(const NormArgs& a, long long i, Owned* o) {
  const bool by_graph = a.graphs < a.blocks;
  const long long r0 = i * a.R, r1 = r0 + a.R < a.n ? r0 + a.R : a.n;
  o->s = by_graph ? i : graph_of(a, r1 - 1);           // (a long graph that begins in the block does not end in it)
  if (o->s < 0) return false;
  graph_rows(a, o->s, &o->begin, &o->end);
  if (o->end - o->begin <= 2 * a.R || (!by_graph && (o->begin < r0 || o->begin >= r1))) return false;
  o->first = o->begin / a.R; o->last = (o->end - 1) / a.R; o->first_slot = o->begin > o->first * a.R ? 1 : 0;
  return true;
}
__device__ __forceinline__ double part_rows(const NormArgs& a, const Owned& o, long long blk) {
  const long long b = blk * a.R > o.begin ? blk * a.R : o.begin, e = (blk + 1) * a.R < o.end ? (blk + 1) * a.R : o.end;
  return (double)(e - b);
}
__device__ __forceinline__ float2 part_at(const NormArgs& a, const Owned& o, long long blk, int g) {
  return a.part[(blk * 2 + (blk == o.first ? o.first_slot : 0)) * a.groups + g];
}

// f(group, step, first block of rows, stride): the groups of a long graph over the threads of the blocks of a column of the grid; a warp to a group where the
// graph has many parts, else a thread.
constexpr int COMBINE_WARPS = 8, FEW_PARTS = 16;
template <class F>
__device__ __forceinline__ void each_group(const NormArgs& a, const Owned& o, F f) {
  if (o.last - o.first < FEW_PARTS) {
    for (int g = blockIdx.y * blockDim.x + threadIdx.x; g < a.groups; g += gridDim.y * blockDim.x) f(g, o.first, 1, false);
  } else {
    for (int g = blockIdx.y * COMBINE_WARPS + (threadIdx.x >> 5); g < a.groups; g += gridDim.y * COMBINE_WARPS) f(g, o.first + (threadIdx.x & 31), 32, true);
  }
}
__device__ __forceinline__ double lane_sum(double v, bool warp) { return warp ? warp_sum(v) : v; }

// Grid (blocks of rows by stride, groups): joins the parts of the long graph that begins in a block of rows.
__global__ void __launch_bounds__(32 * COMBINE_WARPS) norm_combine_kernel(const NormArgs a) {
  early_start();
  if (!*a.any_long) return;
  for (long long blk0 = blockIdx.x; blk0 < owners(a); blk0 += gridDim.x) {
    Owned o;
    if (!owned_graph(a, blk0, &o)) continue;
    each_group(a, o, [&](int g, long long from, int stride, bool warp) {
      // moments about the first part's mean
      const double rows = (double)(o.end - o.begin), shift = part_at(a, o, o.first, g).x;
      double s = 0, q = 0;
#pragma unroll 8
      for (long long blk = from; blk <= o.last; blk += stride) {
        const float2 p = part_at(a, o, blk, g);
        const double d = (double)p.x - shift, w = part_rows(a, o, blk) * d;
        s += w;
        q += (double)p.y + w * d * a.cg;
      }
      s = lane_sum(s, warp) / rows;
      q = lane_sum(q, warp) / (rows * a.cg) - s * s;
      if (!warp || (threadIdx.x & 31) == 0) {
        a.mean[o.s * a.groups + g] = (float)(shift + s);
        a.rstd[o.s * a.groups + g] = (float)(1.0 / sqrt((q < 0 ? 0 : q) + (double)a.eps));
      }
    });
  }
}

// From the last block of rows to the first: the last ones read are still in the L2.
template <class T, int V, bool SAME, int ACT>
__global__ void __launch_bounds__(row_limit(V), row_blocks(V)) norm_apply_kernel(const NormArgs a, const T* x, T* y) {
  early_start();
  __shared__ Parts parts;
  if (!*a.any_long) return;
  const Place<T, V, SAME> at(a);
  float gamma[V], beta[V];
  affine<V>(a, at.cv, gamma, beta);
  float2* const stat = shared_red();
  const long long step = a.lanes * a.ld_x, ystep = a.lanes * a.ld_y;
  for (long long blk = a.blocks - 1 - blockIdx.x; blk >= 0; blk -= gridDim.x) {
    find_parts(a, blk, &parts);
    for (int k = 0; k < 2; ++k) {
      const long long s = parts.s[k];
      if (s < 0) continue;
      for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stat[g] = make_float2(a.mean[s * a.groups + g], a.rstd[s * a.groups + g]);
      __syncthreads();
      Apply<T, V, SAME> f;
      f.set(at, gamma, beta, stat);
      const T* p = at.at(x, a.ld_x, parts.b[k]);
      T* q = y + (parts.b[k] + at.r) * a.ld_y + at.cv * V;
      for (int left = at.rows(a, parts.b[k], parts.e[k]); left > 0; left -= batch<V>()) {
        Vec<T, V> v[batch<V>()];
        load_batch<T, V, batch<V>()>(v, p, step, left);
#pragma unroll
        for (int u = 0; u < batch<V>(); ++u) if (u < left) f.template row<ACT>(v[u], q + u * ystep);
        p += batch<V>() * step; q += batch<V>() * ystep;
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradients

template <class T, int V, bool SAME>
struct Grads {
  float mean[ng<V, SAME>()], rstd[ng<V, SAME>()];
  float gamma[V], beta[V];
  __device__ __forceinline__ void set(const NormArgs& a, const Place<T, V, SAME>& at, long long s) {
#pragma unroll
    for (int k = 0; k < ng<V, SAME>(); ++k) { mean[k] = a.mean[s * a.groups + at.g[k]]; rstd[k] = a.rstd[s * a.groups + at.g[k]]; }
  }
  template <int ACT>
  __device__ __forceinline__ void element(int k, T xv, T dyv, float* xh, float* dz) const {
    *xh = (to_f32<T>(xv) - mean[SAME ? 0 : k]) * rstd[SAME ? 0 : k];
    *dz = to_f32<T>(dyv) * act_slope<ACT>(*xh * gamma[k] + beta[k]);
  }
};
// c1, c2: sums of dz xh and dz by channel, of the part at hand.
template <int ACT, class T, int V, int U, bool SAME>
__device__ __forceinline__ void add_grads(const Grads<T, V, SAME>& f, const Vec<T, V> (&v)[U], const Vec<T, V> (&w)[U], int left, float (&c1)[V], float (&c2)[V]) {
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u < left)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float xh, dz;
        f.template element<ACT>(k, v[u].v[k], w[u].v[k], &xh, &dz);
        c1[k] += dz * xh; c2[k] += dz;
      }
}
template <int ACT, class T, int V, bool SAME>
__device__ __forceinline__ void write_grad(const Grads<T, V, SAME>& f, const Vec<T, V>& v, const Vec<T, V>& w, const float (&m1)[ng<V, SAME>()],
                                           const float (&m2)[ng<V, SAME>()], T* dx) {
  float o[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float xh, dz;
    f.template element<ACT>(k, v.v[k], w.v[k], &xh, &dz);
    // (the product rounded as it was in the sums: alone in its group an element's gradient is zero)
    o[k] = f.rstd[SAME ? 0 : k] * (__fmul_rn(f.gamma[k], dz) - m2[SAME ? 0 : k] - xh * m1[SAME ? 0 : k]);
  }
  store_f32<T, V>(dx, o);
}

// out[g] = sums of (g1, g2) over a block's threads, from red.
template <int V, bool SAME>
__device__ __forceinline__ void sum_block(const NormArgs& a, const Team<V, SAME>& team, const float2* red, float2* out) {
  for (int g0 = 0; g0 < a.groups; g0 += team.teams) {
    const int g = g0 + team.first;
    float u = 0.f, v = 0.f;
    if (g < a.groups) team.each(red, g, [&](int, float2 p) { u += p.x; v += p.y; });
    for (int o = team.size / 2; o > 0; o >>= 1) { u += __shfl_down_sync(0xffffffffu, u, o); v += __shfl_down_sync(0xffffffffu, v, o); }
    if (g < a.groups && team.t == 0) out[g] = make_float2(u, v);
  }
}
// A part's sums by channel: weighted by gamma into red, for the groups, and added to the block's.
template <class T, int V, bool SAME>
__device__ __forceinline__ void put_sums(const Place<T, V, SAME>& at, const NormArgs& a, const float (&gamma)[V], const float (&p1)[V], const float (&p2)[V], float (&c1)[V],
                                         float (&c2)[V], float2* red) {
  if (!at.on) return;
  float2 g[ng<V, SAME>()] = {};
#pragma unroll
  for (int k = 0; k < V; ++k) {
    g[SAME ? 0 : k].x += gamma[k] * p1[k]; g[SAME ? 0 : k].y += gamma[k] * p2[k];
    c1[k] += p1[k]; c2[k] += p2[k];
  }
#pragma unroll
  for (int k = 0; k < ng<V, SAME>(); ++k) red[(at.r * a.vpr + at.cv) * ng<V, SAME>() + k] = g[k];
}
// A block's sums by channel, its threads' added in the order of their rows; red has room for lanes x C.
template <class T, int V, bool SAME>
__device__ __forceinline__ void put_channels(const Place<T, V, SAME>& at, const NormArgs& a, const float (&c1)[V], const float (&c2)[V], float2* red, float2* out) {
  __syncthreads();
  if (at.on)
#pragma unroll
    for (int k = 0; k < V; ++k) red[at.r * a.C + at.cv * V + k] = make_float2(c1[k], c2[k]);
  __syncthreads();
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
    float u = 0.f, v = 0.f;
    for (int r = 0; r < a.lanes; ++r) { const float2 p = red[r * a.C + c]; u += p.x; v += p.y; }
    out[c] = make_float2(u, v);
  }
}

template <class T, int V, bool SAME, int ACT>
__global__ void __launch_bounds__(block_limit(V)) norm_grad_short_kernel(const NormArgs a, const T* x, const T* dy, T* dx) {
  early_start();
  float2* const stat = shared_red();
  float2* const red = stat + a.groups;
  const Place<T, V, SAME> at(a);
  const Team<V, SAME> team(a);
  Grads<T, V, SAME> f;
  affine<V>(a, at.cv, f.gamma, f.beta);
  float c1[V] = {}, c2[V] = {};
  const long long step = a.lanes * a.ld_x, dstep = a.lanes * a.ld_dy, ystep = a.lanes * a.ld_y;
  const int graphs = (int)a.graphs, longest = (int)(2 * a.R < a.n ? 2 * a.R : a.n);
  int b, len, next_b = 0, next_len = 0;
  auto look = [&](int s) {
    long long u, v;
    graph_rows(a, s, &u, &v, threadIdx.x == 0 ? a.status : nullptr);
    next_b = (int)u; next_len = (int)(v - u);
  };
  look(blockIdx.x);
  for (int s = blockIdx.x; s < graphs; s += gridDim.x) {
    b = next_b; len = next_len;
    if (s < graphs - (int)gridDim.x) look(s + gridDim.x);
    if (len > longest) {
      if (threadIdx.x == 0) *a.any_long = 1;
      continue;
    }
    if (len == 0) continue;
    const int rows = at.rows(a, len);
    constexpr int U = short_grad_batch<V>();
    if (rows > 0) f.set(a, at, s);
    {
      const T *p = at.at(x, a.ld_x, b), *d = at.at(dy, a.ld_dy, b);
      float p1[V] = {}, p2[V] = {};
#pragma unroll 1
      for (int left = rows; left > 0; left -= U) {
        Vec<T, V> v[U], w[U];
        load_batch<T, V, U>(v, p, step, left);
        load_batch<T, V, U>(w, d, dstep, left);
        add_grads<ACT>(f, v, w, left, p1, p2);
        p += U * step; d += U * dstep;
      }
      put_sums(at, a, f.gamma, p1, p2, c1, c2, red);
    }
    __syncthreads();
    sum_block(a, team, red, stat);
    __syncthreads();
    const float inv = __fdividef(1.f, (float)len * (float)a.cg);
    float m1[ng<V, SAME>()] = {}, m2[ng<V, SAME>()] = {};
    if (rows > 0)
#pragma unroll
      for (int k = 0; k < ng<V, SAME>(); ++k) { const float2 q = stat[at.g[k]]; m1[k] = q.x * inv; m2[k] = q.y * inv; }
    const T *p = at.at(x, a.ld_x, b), *d = at.at(dy, a.ld_dy, b);
    T* q = dx + ((long long)b + at.r) * a.ld_y + at.cv * V;
#pragma unroll 1
    for (int left = rows; left > 0; left -= U) {
      Vec<T, V> v[U], w[U];
      load_batch<T, V, U>(v, p, step, left);
      load_batch<T, V, U>(w, d, dstep, left);
#pragma unroll
      for (int u = 0; u < U; ++u) if (u < left) write_grad<ACT>(f, v[u], w[u], m1, m2, q + u * ystep);
      p += U * step; d += U * dstep; q += U * ystep;
    }
    __syncthreads();
  }
  if (a.chan) put_channels(at, a, c1, c2, red, a.chan + (size_t)(a.row_grid + blockIdx.x) * a.C);
}

// (128 registers: with 80, three blocks to an SM, sums by channel went to local memory: 1 366 us a step of 1 M x 256 fp32, forward and backward, against 1 323)
template <class T, int V, bool SAME, int ACT>
__global__ void __launch_bounds__(row_limit(V), row_limit(V) > 256 ? 1 : 2) norm_grad_stats_kernel(const NormArgs a, const T* x, const T* dy) {
  early_start();
  __shared__ Parts parts;
  float2* const red = shared_red();
  const Place<T, V, SAME> at(a);
  const Team<V, SAME> team(a);
  float c1[V] = {}, c2[V] = {};
  if (!*a.any_long) return;                                           // (its sums by channel are not read either)
  {
    Grads<T, V, SAME> f;
    affine<V>(a, at.cv, f.gamma, f.beta);
    const long long step = a.lanes * a.ld_x, dstep = a.lanes * a.ld_dy;
    for (long long blk = blockIdx.x; blk < a.blocks; blk += gridDim.x) {
      find_parts(a, blk, &parts);
      for (int k = 0; k < 2; ++k) {
        if (parts.s[k] < 0) continue;
        f.set(a, at, parts.s[k]);
        const T *p = at.at(x, a.ld_x, parts.b[k]), *d = at.at(dy, a.ld_dy, parts.b[k]);
        float p1[V] = {}, p2[V] = {};
        for (int left = at.rows(a, parts.b[k], parts.e[k]); left > 0; left -= grad_batch<V>()) {
          Vec<T, V> v[grad_batch<V>()], w[grad_batch<V>()];
          load_batch<T, V, grad_batch<V>()>(v, p, step, left);
          load_batch<T, V, grad_batch<V>()>(w, d, dstep, left);
          add_grads<ACT>(f, v, w, left, p1, p2);
          p += grad_batch<V>() * step; d += grad_batch<V>() * dstep;
        }
        put_sums(at, a, f.gamma, p1, p2, c1, c2, red);
        __syncthreads();
        sum_block(a, team, red, a.part + (blk * 2 + k) * a.groups);
        __syncthreads();
      }
    }
  }
  if (a.chan) put_channels(at, a, c1, c2, red, a.chan + (size_t)blockIdx.x * a.C);
}

// The last blocks of a row of the grid (blockIdx.x from `combine` on; of the first one only) add up the sums by channel, 4 channels a block: 64 groups
// of threads share the blocks' sums, which are added in their order.
__global__ void __launch_bounds__(32 * COMBINE_WARPS) norm_grad_combine_kernel(const NormArgs a, int combine) {
  early_start();
  const bool any_long = a.blocks > 0 && *a.any_long;
  if ((int)blockIdx.x >= combine) {
    constexpr int CHANNELS = 4, SHARES = 32 * COMBINE_WARPS / CHANNELS;
    __shared__ double2 part[SHARES][CHANNELS];
    if (blockIdx.y > 0) return;
    const int ch = threadIdx.x % CHANNELS, share = threadIdx.x / CHANNELS, c = ((int)blockIdx.x - combine) * CHANNELS + ch;
    const int rows = a.row_grid + a.short_blocks;
    double u = 0, v = 0;
    if (c < a.C)
#pragma unroll 16
      for (int i = (any_long ? 0 : a.row_grid) + share; i < rows; i += SHARES) { const float2 p = a.chan[(size_t)i * a.C + c]; u += p.x; v += p.y; }
    part[share][ch] = make_double2(u, v);
    __syncthreads();
    if (share == 0 && c < a.C) {
      for (int w = 1; w < SHARES; ++w) { u += part[w][ch].x; v += part[w][ch].y; }
      if (a.grad_gamma) a.grad_gamma[c] = (float)u;
      if (a.grad_beta) a.grad_beta[c] = (float)v;
    }
    return;
  }
  if (!any_long) return;
  for (long long blk0 = blockIdx.x; blk0 < owners(a); blk0 += combine) {
    Owned o;
    if (!owned_graph(a, blk0, &o)) continue;
    each_group(a, o, [&](int g, long long from, int stride, bool warp) {
      double u = 0, v = 0;
#pragma unroll 8
      for (long long blk = from; blk <= o.last; blk += stride) { const float2 p = part_at(a, o, blk, g); u += p.x; v += p.y; }
      u = lane_sum(u, warp); v = lane_sum(v, warp);
      const double m = (double)(o.end - o.begin) * a.cg;
      if (!warp || (threadIdx.x & 31) == 0) a.sums[o.s * a.groups + g] = make_float2((float)(u / m), (float)(v / m));
    });
  }
}

template <class T, int V, bool SAME, int ACT>
__global__ void __launch_bounds__(row_limit(V), row_blocks(V)) norm_grad_apply_kernel(const NormArgs a, const T* x, const T* dy, T* dx) {
  early_start();
  __shared__ Parts parts;
  if (!*a.any_long) return;
  const Place<T, V, SAME> at(a);
  Grads<T, V, SAME> f;
  affine<V>(a, at.cv, f.gamma, f.beta);
  const long long step = a.lanes * a.ld_x, dstep = a.lanes * a.ld_dy, ystep = a.lanes * a.ld_y;
  for (long long blk = a.blocks - 1 - blockIdx.x; blk >= 0; blk -= gridDim.x) {
    find_parts(a, blk, &parts);
    for (int k = 0; k < 2; ++k) {
      const long long s = parts.s[k];
      if (s < 0) continue;
      f.set(a, at, s);
      float m1[ng<V, SAME>()], m2[ng<V, SAME>()];
#pragma unroll
      for (int j = 0; j < ng<V, SAME>(); ++j) { const float2 q = a.sums[s * a.groups + at.g[j]]; m1[j] = q.x; m2[j] = q.y; }
      const T *p = at.at(x, a.ld_x, parts.b[k]), *d = at.at(dy, a.ld_dy, parts.b[k]);
      T* q = dx + (parts.b[k] + at.r) * a.ld_y + at.cv * V;
      for (int left = at.rows(a, parts.b[k], parts.e[k]); left > 0; left -= grad_batch<V>()) {
        Vec<T, V> v[grad_batch<V>()], w[grad_batch<V>()];
        load_batch<T, V, grad_batch<V>()>(v, p, step, left);
        load_batch<T, V, grad_batch<V>()>(w, d, dstep, left);
#pragma unroll
        for (int u = 0; u < grad_batch<V>(); ++u) if (u < left) write_grad<ACT>(f, v[u], w[u], m1, m2, q + u * ystep);
        p += grad_batch<V>() * step; d += grad_batch<V>() * dstep; q += grad_batch<V>() * ystep;
      }
    }
  }
}

__global__ void norm_no_rows_kernel(const NormArgs a) {
  early_start();
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < a.graphs * a.groups; i += (long long)gridDim.x * blockDim.x) {
    if (a.mean) a.mean[i] = 0.f;
    if (a.rstd) a.rstd[i] = 0.f;
  }
  for (int c = blockIdx.x * blockDim.x + threadIdx.x; c < a.C; c += gridDim.x * blockDim.x) {
    if (a.grad_gamma) a.grad_gamma[c] = 0.f;
    if (a.grad_beta) a.grad_beta[c] = 0.f;
  }
}

// ---------------------------------------------------------------------------------------------------------------- host

constexpr int DEVICE_SMS = 148, ROW_BLOCKS_PER_SM = 8, ROW_GRID_PER_SM = 8;
// Rows of a block of rows: at least 8 192 elements, about eight blocks to an SM; where there are graphs enough to fill the device, four times the average
// graph's: the graphs of an ordinary batch are short ones then.  (By the number of SMs this is built for, so that a workspace's size depends on the sizes alone.)
long long block_rows(int64_t n, int64_t graphs, int C) {
  const long long even = std::max<long long>(std::max(1, 8192 / C), (n + DEVICE_SMS * ROW_BLOCKS_PER_SM - 1) / (DEVICE_SMS * ROW_BLOCKS_PER_SM));
  return graphs >= DEVICE_SMS * ROW_BLOCKS_PER_SM ? std::max<long long>(even, 4 * (n / graphs)) : even;
}

struct NormSpace { long long R, blocks; int short_blocks, row_grid; size_t flag, part, chan, sums, mean, rstd, bytes; };
// most: what no call with as many rows and graphs, or fewer, exceeds (the blocks of rows are longer where there are many graphs).
NormSpace norm_space(int64_t n, int64_t graphs, int C, int groups, bool grad, bool most = false) {
  NormSpace s;
  s.R = block_rows(n, most ? 1 : graphs, C);
  const bool long_ones = n > 2 * s.R;                            // else no graph can be long
  s.blocks = long_ones ? (n + s.R - 1) / s.R : 0;
  if (most && long_ones) s.blocks = std::min<long long>(DEVICE_SMS * ROW_BLOCKS_PER_SM, (n + std::max(1, 8192 / C) - 1) / std::max(1, 8192 / C));
  s.row_grid = (int)std::min<long long>(s.blocks, DEVICE_SMS * ROW_GRID_PER_SM);
  s.short_blocks = (int)std::min<long long>(graphs, DEVICE_SMS * 16);      // (gradients: at most)
  size_t at = 0;
  auto take = [&](size_t b) { const size_t o = at; at += (b + 255) / 256 * 256; return o; };
  s.flag = take(long_ones ? 4 : 0);
  s.part = take((size_t)s.blocks * 2 * groups * 8);
  s.chan = take(grad ? (size_t)(s.row_grid + s.short_blocks) * C * 8 : 0);
  s.sums = take(grad && long_ones ? (size_t)graphs * groups * 8 : 0);
  s.mean = take(!grad && long_ones ? (size_t)graphs * groups * 4 : 0);
  s.rstd = take(!grad && long_ones ? (size_t)graphs * groups * 4 : 0);
  s.bytes = at;
  return s;
}

bool norm_shape_ok(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  return n >= 0 && n < (1ll << 31) && graphs >= 1 && graphs <= (1ll << 30) && width >= 1 && groups >= 1 && width % groups == 0;
}

// Vectors of at most 16 bytes; of at most four elements where they would reach over several groups (each has moments of its own then).
int norm_vector(int size, int width, int cg, const void* a, int64_t lda, const void* b, int64_t ldb, const void* c, int64_t ldc) {
  int v = 16 / size;
  auto bad = [&](const void* p, int64_t ld) { return p && (ld % v != 0 || !rows_aligned(p, v * size)); };
  if (cg % v != 0 && v > 4) v = 4;
  while (v > 1 && (width % v != 0 || bad(a, lda) || bad(b, ldb) || bad(c, ldc))) v >>= 1;
  return v;
}

// Rows that a block of about `threads` threads walks at once, a power of two, and its threads.
void set_block(NormArgs* a, int v, int threads, int* out_threads) {
  a->vpr = a->C / v;
  a->shift = 0;
  while ((2 << a->shift) * a->vpr <= threads) ++a->shift;
  a->lanes = 1 << a->shift;
  *out_threads = (a->lanes * a->vpr + 31) / 32 * 32;
}

// f(tag of the element type, vector length, is a vector of one group, activation) for the kernels that fit; v from norm_vector.
template <class F>
void with_norm_kernels(int32_t type, int v, int cg, int act, F f0) {
  auto f = [&](auto tt, auto vc, auto same) {
    if (act == TAURUS_ACT_RELU) f0(tt, vc, same, std::integral_constant<int, TAURUS_ACT_RELU>());
    else if (act == TAURUS_ACT_SILU) f0(tt, vc, same, std::integral_constant<int, TAURUS_ACT_SILU>());
    else f0(tt, vc, same, std::integral_constant<int, TAURUS_ACT_NONE>());
  };
  with_row_type(type, [&](auto tt) {
    return with_vector(v, [&](auto vc) {
      constexpr int V = decltype(vc)::value;
      using Tag = std::decay_t<decltype(tt)>;
      if constexpr (V * sizeof(typename Tag::type) <= 16) {
        if (cg % V == 0) f(tt, vc, std::true_type());
        else if constexpr (V > 1 && V <= 4) f(tt, vc, std::false_type());
      }
      return 0;
    });
  });
}

// Columns of the grid that joins parts: one for each eight groups where a few graphs have all the parts.
unsigned combine_columns(long long blocks, int64_t graphs, int groups) { return blocks / graphs >= 64 ? (unsigned)((groups + COMBINE_WARPS - 1) / COMBINE_WARPS) : 1u; }

// Threads for a short graph: at most `batch` vectors each for a graph of the average length.
int short_threads(int64_t n, int64_t graphs, int vpr, int batch) {
  const long long vectors = std::min<long long>(n / graphs + 1, 1ll << 20) * vpr;
  int t = 32;
  while (t < 512 && t * batch < vectors) t *= 2;
  return t;
}

}  // namespace

extern "C" int64_t taurus_norm_rows_workspace(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  if (!norm_shape_ok(n, graphs, width, groups)) return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)norm_space(n, graphs, width, groups, false, true).bytes;
}
extern "C" int64_t taurus_norm_rows_grad_workspace(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  if (!norm_shape_ok(n, graphs, width, groups)) return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)norm_space(n, graphs, width, groups, true, true).bytes;
}

extern "C" int taurus_norm_rows(int64_t n, int64_t graphs, const int64_t* offsets, const void* x, int64_t ld_x, int32_t type, int32_t width, int32_t groups,
                                const float* gamma, const float* beta, float eps, int32_t act, void* out_rows, int64_t ld_out, float* mean, float* rstd,
                                void* workspace, int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const int ts = row_type_size(type);
  if (!ts || !norm_shape_ok(n, graphs, width, groups) || ld_x < width || ld_out < width || !rows_fit(n, ld_x, 4) || !rows_fit(n, ld_out, 4) || !(eps >= 0.f) ||
      act < TAURUS_ACT_NONE || act > TAURUS_ACT_SILU || (!offsets && graphs != 1) || !rows_aligned(offsets, 8) || !rows_aligned(gamma, 4) || !rows_aligned(beta, 4) ||
      !rows_aligned(mean, 4) || !rows_aligned(rstd, 4) || !rows_aligned(status, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  if (n > 0 && (!x || !out_rows || !rows_aligned(x, ts) || !rows_aligned(out_rows, ts))) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const NormSpace s = norm_space(n, graphs, width, groups, false);
  const size_t stat_bytes = (size_t)graphs * groups * 4, cb = (size_t)width * 4;
  const Region rows = region_of_rows(x, n, ld_x, width, ts);
  const bool in_place = out_rows == x && ld_out == ld_x;
  const Region outs[] = {region_of_rows(out_rows, n, ld_out, width, ts), region_of(mean, stat_bytes), region_of(rstd, stat_bytes), region_of(status, 4)};
  const Region ins[] = {in_place ? region_of(nullptr, 0) : rows, region_of(offsets, (size_t)(graphs + 1) * 8), region_of(gamma, cb), region_of(beta, cb)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) ||
      !workspace_ok(workspace, workspace_bytes, n > 0 ? (int64_t)s.bytes : 0, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  Launches enqueue = {st};
  char* const ws = static_cast<char*>(workspace);
  NormArgs a = {};
  a.n = n; a.graphs = graphs; a.offsets = reinterpret_cast<const long long*>(offsets); a.ld_x = ld_x; a.ld_y = ld_out; a.C = width; a.groups = groups;
  a.cg = width / groups; a.eps = eps; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd; a.status = status;
  a.R = s.R; a.blocks = s.blocks; a.row_grid = s.row_grid;
  const bool whole = s.blocks > 0 && !offsets;                                              // one graph of n rows: a long one
  a.short_blocks = whole ? 0 : s.short_blocks;
  a.any_long = reinterpret_cast<int*>(ws + s.flag);
  if (s.blocks > 0) {
    const cudaError_t e = cudaMemsetAsync(a.any_long, whole ? 1 : 0, 4, st);
    if (e != cudaSuccess) { taurus_note_cuda_error(e, "norm"); return TAURUS_ERR_CUDA; }
  }
   a.part = reinterpret_cast<float2*>(ws + s.part);
  if (n == 0) {
    if (mean || rstd) enqueue(norm_no_rows_kernel, dim3((unsigned)((int)std::min<long long>((graphs * groups + 255) / 256, 4096))), 256, 0, a);
  } else {
    if (s.blocks > 0) {
      if (!a.mean) a.mean = reinterpret_cast<float*>(ws + s.mean);
      if (!a.rstd) a.rstd = reinterpret_cast<float*>(ws + s.rstd);
    }
    const int v = norm_vector(ts, width, a.cg, x, ld_x, out_rows, ld_out, nullptr, 0);
    with_norm_kernels(type, v, a.cg, act, [&](auto tt, auto vc, auto same, auto ac) {
      using T = typename decltype(tt)::type;
      constexpr int V = decltype(vc)::value;
      constexpr bool SAME = decltype(same)::value;
      constexpr int ACT = decltype(ac)::value;
      const T* const xp = static_cast<const T*>(x);
      T* const yp = static_cast<T*>(out_rows);
      int threads;
      if (a.short_blocks > 0) {
        set_block(&a, V, short_threads(n, graphs, width / V, short_vectors<V>()), &threads);
        const size_t smem = (size_t)a.lanes * a.vpr * ng<V, SAME>() * 8 + (size_t)groups * 8 + (size_t)width * 8;
        enqueue(norm_short_kernel<T, V, SAME, ACT>, dim3((unsigned)((int)std::min<int64_t>(graphs, 1 << 20))), threads, smem, a, xp, yp);
      }
      if (s.blocks > 0) {
        set_block(&a, V, ROW_THREADS, &threads);
        enqueue(norm_stats_kernel<T, V, SAME>, dim3((unsigned)(s.row_grid)), threads, (size_t)a.lanes * a.vpr * ng<V, SAME>() * 8, a, xp);
        enqueue(norm_combine_kernel, dim3((unsigned)std::min<int64_t>(s.row_grid, graphs), combine_columns(s.blocks, graphs, groups)), 32 * COMBINE_WARPS, 0, a);
        enqueue(norm_apply_kernel<T, V, SAME, ACT>, dim3((unsigned)(s.row_grid)), threads, (size_t)groups * 8, a, xp, yp);
      }
    });
  }
  return enqueue.done("norm_rows");
}

extern "C" int taurus_norm_rows_grad(int64_t n, int64_t graphs, const int64_t* offsets, const void* x, int64_t ld_x, int32_t type, int32_t width, int32_t groups,
                                     const float* gamma, const float* beta, int32_t act, const float* mean, const float* rstd, const void* grad_out,
                                     int64_t ld_grad, void* grad_x, int64_t ld_grad_x, float* grad_gamma, float* grad_beta, void* workspace,
                                     int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const int ts = row_type_size(type);
  if (!ts || !norm_shape_ok(n, graphs, width, groups) || ld_x < width || ld_grad < width || ld_grad_x < width || !rows_fit(n, ld_x, 4) || !rows_fit(n, ld_grad, 4) ||
      !rows_fit(n, ld_grad_x, 4) || act < TAURUS_ACT_NONE || act > TAURUS_ACT_SILU || (!offsets && graphs != 1) || !mean || !rstd || !rows_aligned(offsets, 8) ||
      !rows_aligned(gamma, 4) || !rows_aligned(beta, 4) || !rows_aligned(mean, 4) || !rows_aligned(rstd, 4) || !rows_aligned(grad_gamma, 4) || !rows_aligned(grad_beta, 4) ||
      !rows_aligned(status, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  if (n > 0 && (!x || !grad_out || !grad_x || !rows_aligned(x, ts) || !rows_aligned(grad_out, ts) || !rows_aligned(grad_x, ts))) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const NormSpace s = norm_space(n, graphs, width, groups, true);
  const size_t stat_bytes = (size_t)graphs * groups * 4, cb = (size_t)width * 4;
  const bool over_x = grad_x == x && ld_grad_x == ld_x, over_grad = grad_x == grad_out && ld_grad_x == ld_grad;      // in place
  const Region rows = region_of_rows(x, n, ld_x, width, ts), grads = region_of_rows(grad_out, n, ld_grad, width, ts);
  const Region outs[] = {region_of_rows(grad_x, n, ld_grad_x, width, ts), region_of(grad_gamma, cb), region_of(grad_beta, cb), region_of(status, 4)};
  const Region ins[] = {over_x ? region_of(nullptr, 0) : rows, over_grad ? region_of(nullptr, 0) : grads, region_of(offsets, (size_t)(graphs + 1) * 8),
                        region_of(gamma, cb), region_of(beta, cb), region_of(mean, stat_bytes), region_of(rstd, stat_bytes)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) ||
      !workspace_ok(workspace, workspace_bytes, n > 0 ? (int64_t)s.bytes : 0, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  Launches enqueue = {st};
  char* const ws = static_cast<char*>(workspace);
  NormArgs a = {};
  a.n = n; a.graphs = graphs; a.offsets = reinterpret_cast<const long long*>(offsets); a.ld_x = ld_x; a.ld_y = ld_grad_x; a.ld_dy = ld_grad; a.C = width; a.groups = groups;
  a.cg = width / groups; a.gamma = gamma; a.beta = beta; a.status = status; a.grad_gamma = grad_gamma; a.grad_beta = grad_beta;
  a.R = s.R; a.blocks = s.blocks; a.row_grid = s.row_grid;
  const bool whole = s.blocks > 0 && !offsets;                                              // one graph of n rows: a long one
  a.short_blocks = whole ? 0 : s.short_blocks;
  a.any_long = reinterpret_cast<int*>(ws + s.flag);
  if (s.blocks > 0) {
    const cudaError_t e = cudaMemsetAsync(a.any_long, whole ? 1 : 0, 4, st);
    if (e != cudaSuccess) { taurus_note_cuda_error(e, "norm"); return TAURUS_ERR_CUDA; }
  }
   a.part = reinterpret_cast<float2*>(ws + s.part); a.chan = reinterpret_cast<float2*>(ws + s.chan);
  a.sums = reinterpret_cast<float2*>(ws + s.sums);
  if (n == 0) {
    if (grad_gamma || grad_beta) enqueue(norm_no_rows_kernel, dim3((unsigned)(4)), 256, 0, a);
  } else {
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);                 // read only here
    if (!grad_gamma && !grad_beta) a.chan = nullptr;
    const int v = norm_vector(ts, width, a.cg, x, ld_x, grad_out, ld_grad, grad_x, ld_grad_x);
    with_norm_kernels(type, v, a.cg, act, [&](auto tt, auto vc, auto same, auto ac) {
      using T = typename decltype(tt)::type;
      constexpr int V = decltype(vc)::value;
      constexpr bool SAME = decltype(same)::value;
      constexpr int ACT = decltype(ac)::value;
      const T *const xp = static_cast<const T*>(x), *const dyp = static_cast<const T*>(grad_out);
      T* const dxp = static_cast<T*>(grad_x);
      int threads;
      if (a.short_blocks > 0) {
        set_block(&a, V, short_threads(n, graphs, width / V, short_vectors<V>()), &threads);
        enqueue(norm_grad_short_kernel<T, V, SAME, ACT>, dim3((unsigned)(a.short_blocks)), threads, (size_t)a.lanes * width * 8 + (size_t)groups * 8, a, xp, dyp, dxp);
      }
      if (s.blocks > 0) {
        set_block(&a, V, ROW_THREADS, &threads);
        enqueue(norm_grad_stats_kernel<T, V, SAME, ACT>, dim3((unsigned)(s.row_grid)), threads, (size_t)a.lanes * width * 8, a, xp, dyp);
      }
      const int channel_blocks = a.chan ? (width + 3) / 4 : 0;
      const int owner_blocks = (int)std::min<int64_t>(s.row_grid, graphs);
      if (owner_blocks + channel_blocks > 0)
        enqueue(norm_grad_combine_kernel, dim3((unsigned)(owner_blocks + channel_blocks), s.blocks > 0 ? combine_columns(s.blocks, graphs, groups) : 1u), 32 * COMBINE_WARPS, 0, a, owner_blocks);
      if (s.blocks > 0) enqueue(norm_grad_apply_kernel<T, V, SAME, ACT>, dim3((unsigned)(s.row_grid)), threads, 0, a, xp, dyp, dxp);
    });
  }
  return enqueue.done("norm_rows_grad");
}
