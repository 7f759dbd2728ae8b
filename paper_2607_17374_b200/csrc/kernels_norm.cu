// Group norm with an activation over the rows of a batch of graphs, channels last, and its gradients.
//
// Per graph s (rows [b, e)) and group g (C / groups neighbouring channels), m = (e - b) C / groups elements:
//   mean = sum x / m,  rstd = (sum (x - mean)^2 / m + eps)^-1/2,  xh = (x - mean) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z),  grad_gamma = sum dz xh,  grad_beta = sum dz (over all rows),
//   dx = rstd (gamma dz - mean_g(gamma dz) - xh mean_g(gamma dz xh))
//
// Bytes bound it: x in, y out (dx: x and dy in, dx out).  Statistics need all of a graph before its first row can be written.  A short graph
// is the work of one block, which reads its rows a second time from registers or the caches.  The rows of a long graph are spread over blocks
// of R rows (stats), their partial statistics joined in a fixed order (combine), and the rows are read again and written (apply).  How long
// a graph is stands in device memory: every launch decides for itself which graphs are its own.
//
// A thread keeps to one vector of channels and walks the rows.  Sums of x are taken of x - pivot (the channel's value in the part's first
// row), so that an offset does not eat the variance, in fp32 over at most R rows; parts are joined by (count, mean, sum of squared
// deviations) in fp64.
#include <algorithm>

#include "rows.cuh"

namespace {

constexpr int MAX_C = TAURUS_MAX_ROW_WIDTH;
constexpr int BATCH = 4;                 // row vectors of a thread in flight; a short graph's first ones stay in registers

struct NormArgs {
  long long n, graphs;
  const long long* offsets;              // null: one graph of n rows
  long long ld_x, ld_y, ld_dy;           // ld_y: of the rows written
  int C, groups, cg, vpr, lanes;         // cg: channels of a group; vpr: vectors of a row; lanes: rows that a block walks at once
  int act;
  float eps;
  const float *gamma, *beta;             // null: ones, zeros
  float *mean, *rstd;                    // [graphs x groups]
  long long R, blocks, short_blocks;     // rows of a block of rows; their number; blocks of the kernel for short graphs
  float2* part;                          // [blocks x 2 x groups]
  float2* chan;                          // [(blocks + short_blocks) x C] (grad_gamma, grad_beta) of a block
  float2* sums;                          // [graphs x groups] backward: the two means of a long graph
  float *grad_gamma, *grad_beta;
  int32_t* status;
};

__device__ __forceinline__ float act_f(int act, float z) {
  if (act == TAURUS_ACT_RELU) return z < 0.f ? 0.f : z;
  if (act == TAURUS_ACT_SILU) return z / (1.f + expf(-z));
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == TAURUS_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == TAURUS_ACT_SILU) { const float s = 1.f / (1.f + expf(-z)); return s * (1.f + z * (1.f - s)); }
  return 1.f;
}

__device__ __forceinline__ void graph_rows(const NormArgs& a, long long s, long long* b, long long* e) {
  if (!a.offsets) { *b = 0; *e = a.n; return; }
  group_rows(a.offsets, s, a.n, b, e, nullptr);
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
    if (k == 0) { hi = lo; break; }
    const long long first = lo + step * (k - 1);
    const long long next = lo + step * k;
    lo = first + 1;
    if (next < hi) hi = next;
    if (step == 1) break;
  }
  const long long s = lo - 1;
  return s >= 0 && s < a.graphs ? s : -1;
}

// Sums over the row lanes of a block: red[c] holds channel c's afterwards, and the block is in step.
__device__ __forceinline__ void sum_lanes(float2* red, int C, int lanes) {
  __syncthreads();
  while (lanes > 1) {
    const int half = (lanes + 1) / 2;
    for (int i = threadIdx.x; i < (lanes - half) * C; i += blockDim.x) {
      const float2 o = red[i + half * C];
      red[i].x += o.x; red[i].y += o.y;
    }
    __syncthreads();
    lanes = half;
  }
}

// Lanes that share a group: a power of two of them, each with its channels; f(g, first channel of the lane, step) -> value to sum.
__device__ __forceinline__ int team_of(int cg) { int t = 1; while (t < cg && t < 32) t *= 2; return t; }
__device__ __forceinline__ float team_sum(float v, int team) {
  for (int o = team / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// (mean, sum of squared deviations) of every group of a part with `rows` rows from red[c] = sums of (x - pivot) and its square.
__device__ __forceinline__ void group_moments(const NormArgs& a, const float2* red, const float* pivot, long long rows, float2* out) {
  const int team = team_of(a.cg), per_warp = 32 / team, warps = blockDim.x >> 5;
  const int lane = threadIdx.x & 31, t = lane % team;
  const float inv = 1.f / (float)rows;
  for (int g0 = (threadIdx.x >> 5) * per_warp; g0 < a.groups; g0 += warps * per_warp) {
    const int g = g0 + lane / team;
    const bool in = g < a.groups;
    float m = 0.f;
    if (in) for (int c = t; c < a.cg; c += team) m += pivot[g * a.cg + c] + red[g * a.cg + c].x * inv;
    const float mean = team_sum(m, team) / (float)a.cg;
    float q = 0.f;
    if (in)
      for (int c = t; c < a.cg; c += team) {
        const float2 s = red[g * a.cg + c];
        const float d = (pivot[g * a.cg + c] - mean) + s.x * inv, m2 = s.y - s.x * s.x * inv;
        q += (m2 < 0.f ? 0.f : m2) + (float)rows * d * d;
      }
    q = team_sum(q, team);
    if (in && t == 0) out[g] = make_float2(mean, q);
  }
  __syncthreads();
}

// Sums of x - pivot of rows [b, e) into red; the pivots into `pivot`.  KEEP: the thread's first BATCH vectors stay in `keep`.
template <class T, int V>
__device__ __forceinline__ void sum_rows(const NormArgs& a, const T* x, long long b, long long e, float2* red, float* pivot, Vec<T, V> (&keep)[BATCH]) {
  const int cv = threadIdx.x % a.vpr, r = threadIdx.x / a.vpr;
  if (r < a.lanes) {
    const T* const col = x + cv * V;
    float p[V], s1[V] = {}, s2[V] = {};
    load_f32<T, V>(col + b * a.ld_x, p);
    for (long long i = b + r; i < e; i += (long long)a.lanes * BATCH) {
      Vec<T, V> v[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) if (i + (long long)u * a.lanes < e) v[u] = load_vec<Vec<T, V>>(col + (i + (long long)u * a.lanes) * a.ld_x);
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (i + (long long)u * a.lanes < e)
#pragma unroll
          for (int k = 0; k < V; ++k) { const float d = to_f32<T>(v[u].v[k]) - p[k]; s1[k] += d; s2[k] += d * d; }
      if (i == b + r)
#pragma unroll
        for (int u = 0; u < BATCH; ++u) keep[u] = v[u];
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      red[r * a.C + cv * V + k] = make_float2(s1[k], s2[k]);
      if (r == 0) pivot[cv * V + k] = p[k];
    }
  }
  sum_lanes(red, a.C, a.lanes);
}

// y = act((x - mean) rstd gamma + beta) for rows [b, e); stat[g] = (mean, rstd).
template <class T, int V, bool KEPT>
__device__ __forceinline__ void write_rows(const NormArgs& a, const T* x, T* y, long long b, long long e, const float2* stat, const Vec<T, V> (&keep)[BATCH]) {
  const int cv = threadIdx.x % a.vpr, r = threadIdx.x / a.vpr;
  if (r >= a.lanes) return;
  float mean[V], mul[V], add[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int c = cv * V + k;
    const float2 s = stat[c / a.cg];
    mean[k] = s.x;
    mul[k] = s.y * (a.gamma ? a.gamma[c] : 1.f);
    add[k] = a.beta ? a.beta[c] : 0.f;
  }
  for (long long i = b + r; i < e; i += (long long)a.lanes * BATCH) {
    Vec<T, V> v[BATCH];
    if (KEPT && i == b + r) {
#pragma unroll
      for (int u = 0; u < BATCH; ++u) v[u] = keep[u];
    } else {
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (i + (long long)u * a.lanes < e) v[u] = load_vec<Vec<T, V>, KEPT ? LOAD_PLAIN : LOAD_ONCE>(x + (i + (long long)u * a.lanes) * a.ld_x + cv * V);
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const long long row = i + (long long)u * a.lanes;
      if (row >= e) break;
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = act_f(a.act, (to_f32<T>(v[u].v[k]) - mean[k]) * mul[k] + add[k]);
      store_f32<T, V>(y + row * a.ld_y + cv * V, o);
    }
  }
}

// Threads of a block: at most 512, but for rows of up to 1 024 vectors.
constexpr int block_limit(int v) { return MAX_C / v > 512 ? 1024 : 512; }

// Shared memory: red [lanes x C] | pivot [C] | stat [groups], and in the backward pass chan [C].
__device__ __forceinline__ float2* shared_red() { extern __shared__ __align__(16) float2 norm_shared[]; return norm_shared; }

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_short_kernel(const NormArgs a, const T* x, T* y) {
  float2* const red = shared_red();
  float2* const stat = red + (size_t)a.lanes * a.C;
  float* const pivot = reinterpret_cast<float*>(stat + a.groups);
  for (long long s = blockIdx.x; s < a.graphs; s += gridDim.x) {
    long long b, e;
    graph_rows(a, s, &b, &e);
    if (threadIdx.x == 0 && a.offsets) { long long u, v; group_rows(a.offsets, s, a.n, &u, &v, a.status); }
    if (e - b > 2 * a.R) continue;                                    // long: the other kernels'
    if (b == e) {
      for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
        if (a.mean) a.mean[s * a.groups + g] = 0.f;
        if (a.rstd) a.rstd[s * a.groups + g] = 0.f;
      }
      continue;
    }
    Vec<T, V> keep[BATCH];
    sum_rows<T, V>(a, x, b, e, red, pivot, keep);
    group_moments(a, red, pivot, e - b, stat);
    const float inv = 1.f / ((float)(e - b) * (float)a.cg);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
      const float2 m = stat[g];
      const float rstd = 1.f / sqrtf(m.y * inv + a.eps);
      stat[g] = make_float2(m.x, rstd);
      if (a.mean) a.mean[s * a.groups + g] = m.x;
      if (a.rstd) a.rstd[s * a.groups + g] = rstd;
    }
    __syncthreads();
    write_rows<T, V, true>(a, x, y, b, e, stat, keep);
    __syncthreads();                                                  // stat is written again
  }
}

// The parts of long graphs in block of rows `blk`: slot 0 is the graph of its first row, slot 1 that of its last row where another one begins
// in the block.  (A long graph has more than 2 R rows, so no third one can meet the block.)
struct Parts { long long s[2], b[2], e[2], begin[2], end[2]; };     // graph (-1: none), the part's rows, the graph's rows
__device__ __forceinline__ void find_parts(const NormArgs& a, long long blk, Parts* p) {     // p in shared memory; by the whole block
  const long long r0 = blk * a.R, r1 = r0 + a.R < a.n ? r0 + a.R : a.n;
  const int warp = threadIdx.x >> 5;
  if (warp == 0) {                        // (both by one warp: a block may have no second one)
    for (int k = 0; k < 2; ++k) {
      long long s = graph_of(a, k ? r1 - 1 : r0), b = 0, e = 0;
      if (s >= 0) {
        graph_rows(a, s, &b, &e);
        if (e - b <= 2 * a.R || (k && b <= r0)) s = -1;
      }
      if (threadIdx.x == 0) {
        const long long pb = b > r0 ? b : r0, pe = e < r1 ? e : r1;
        if (pb >= pe) s = -1;
        p->s[k] = s; p->begin[k] = b; p->end[k] = e; p->b[k] = pb; p->e[k] = pe;
      }
    }
  }
  __syncthreads();
}

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_stats_kernel(const NormArgs a, const T* x) {
  __shared__ Parts parts;
  float2* const red = shared_red();
  float2* const stat = red + (size_t)a.lanes * a.C;
  float* const pivot = reinterpret_cast<float*>(stat + a.groups);
  const long long blk = blockIdx.x;
  find_parts(a, blk, &parts);
  for (int k = 0; k < 2; ++k) {
    if (parts.s[k] < 0) continue;
    Vec<T, V> keep[BATCH];
    sum_rows<T, V>(a, x, parts.b[k], parts.e[k], red, pivot, keep);
    group_moments(a, red, pivot, parts.e[k] - parts.b[k], stat);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) a.part[(blk * 2 + k) * a.groups + g] = stat[g];
    __syncthreads();
  }
}

__device__ __forceinline__ double warp_sum(double v) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The partial results of a long graph lie in slot 0 of the blocks of rows it meets, but for the block it begins in the middle of.
// Block (x, y): the long graph that begins in block of rows x, groups y * warps + warp.
struct Owned { long long s, begin, end, first, last; int first_slot; };
__device__ __forceinline__ bool owned_graph(const NormArgs& a, long long blk, Owned* o) {    // by every warp for itself
  const long long r0 = blk * a.R, r1 = r0 + a.R < a.n ? r0 + a.R : a.n;
  o->s = graph_of(a, r1 - 1);           // a long graph that begins in the block does not end in it
  if (o->s < 0) return false;
  graph_rows(a, o->s, &o->begin, &o->end);
  if (o->end - o->begin <= 2 * a.R || o->begin < r0 || o->begin >= r1) return false;
  o->first = blk; o->last = (o->end - 1) / a.R; o->first_slot = o->begin > r0 ? 1 : 0;
  return true;
}
__device__ __forceinline__ double part_rows(const NormArgs& a, const Owned& o, long long blk) {
  const long long b = blk * a.R > o.begin ? blk * a.R : o.begin, e = (blk + 1) * a.R < o.end ? (blk + 1) * a.R : o.end;
  return (double)(e - b);
}

__global__ void norm_combine_kernel(const NormArgs a) {
  Owned o;
  if (!owned_graph(a, blockIdx.x, &o)) return;
  const int lane = threadIdx.x & 31, g = blockIdx.y * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (g >= a.groups) return;
  auto at = [&](long long blk) { return a.part[(blk * 2 + (blk == o.first ? o.first_slot : 0)) * a.groups + g]; };
  const double rows = (double)(o.end - o.begin);
  double m = 0;
  for (long long blk = o.first + lane; blk <= o.last; blk += 32) m += part_rows(a, o, blk) * (double)at(blk).x;
  const double mean = warp_sum(m) / rows;
  double q = 0;
  for (long long blk = o.first + lane; blk <= o.last; blk += 32) {
    const float2 p = at(blk);
    const double d = (double)p.x - mean;
    q += (double)p.y + part_rows(a, o, blk) * a.cg * d * d;
  }
  q = warp_sum(q);
  if (lane == 0) {
    a.mean[o.s * a.groups + g] = (float)mean;
    a.rstd[o.s * a.groups + g] = (float)(1.0 / sqrt(q / (rows * a.cg) + (double)a.eps));
  }
}

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_apply_kernel(const NormArgs a, const T* x, T* y) {
  __shared__ Parts parts;
  float2* const stat = shared_red();
  find_parts(a, blockIdx.x, &parts);
  for (int k = 0; k < 2; ++k) {
    const long long s = parts.s[k];
    if (s < 0) continue;
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stat[g] = make_float2(a.mean[s * a.groups + g], a.rstd[s * a.groups + g]);
    __syncthreads();
    Vec<T, V> none[BATCH];
    write_rows<T, V, false>(a, x, y, parts.b[k], parts.e[k], stat, none);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradients

template <int V>
struct ChannelConsts {
  float mean[V], rstd[V], gamma[V], beta[V];
  __device__ __forceinline__ void load(const NormArgs& a, long long s, int cv) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = cv * V + k, g = c / a.cg;
      mean[k] = a.mean[s * a.groups + g]; rstd[k] = a.rstd[s * a.groups + g];
      gamma[k] = a.gamma ? a.gamma[c] : 1.f; beta[k] = a.beta ? a.beta[c] : 0.f;
    }
  }
};

// red[c] = (sum dz xh, sum dz) over rows [b, e).
template <class T, int V>
__device__ __forceinline__ void sum_grads(const NormArgs& a, const T* x, const T* dy, long long s, long long b, long long e, float2* red) {
  const int cv = threadIdx.x % a.vpr, r = threadIdx.x / a.vpr;
  if (r < a.lanes) {
    ChannelConsts<V> c;
    c.load(a, s, cv);
    float s1[V] = {}, s2[V] = {};
    for (long long i = b + r; i < e; i += (long long)a.lanes * BATCH) {
      Vec<T, V> v[BATCH], w[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const long long row = i + (long long)u * a.lanes;
        if (row < e) { v[u] = load_vec<Vec<T, V>>(x + row * a.ld_x + cv * V); w[u] = load_vec<Vec<T, V>>(dy + row * a.ld_dy + cv * V); }
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u)
        if (i + (long long)u * a.lanes < e)
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float xh = (to_f32<T>(v[u].v[k]) - c.mean[k]) * c.rstd[k];
            const float dz = to_f32<T>(w[u].v[k]) * act_slope(a.act, xh * c.gamma[k] + c.beta[k]);
            s1[k] += dz * xh; s2[k] += dz;
          }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) red[r * a.C + cv * V + k] = make_float2(s1[k], s2[k]);
  }
  sum_lanes(red, a.C, a.lanes);
}

// out[g] = (sum gamma dz xh, sum gamma dz) over the group's channels.
__device__ __forceinline__ void group_grads(const NormArgs& a, const float2* red, float2* out) {
  const int team = team_of(a.cg), per_warp = 32 / team, warps = blockDim.x >> 5;
  const int lane = threadIdx.x & 31, t = lane % team;
  for (int g0 = (threadIdx.x >> 5) * per_warp; g0 < a.groups; g0 += warps * per_warp) {
    const int g = g0 + lane / team;
    float u = 0.f, v = 0.f;
    if (g < a.groups)
      for (int c = g * a.cg + t; c < (g + 1) * a.cg; c += team) {
        const float w = a.gamma ? a.gamma[c] : 1.f;
        u += w * red[c].x; v += w * red[c].y;
      }
    u = team_sum(u, team); v = team_sum(v, team);
    if (g < a.groups && t == 0) out[g] = make_float2(u, v);
  }
  __syncthreads();
}

// dx for rows [b, e); mean_g[g] = (mean of gamma dz xh, mean of gamma dz).
template <class T, int V>
__device__ __forceinline__ void write_grads(const NormArgs& a, const T* x, const T* dy, T* dx, long long s, long long b, long long e, const float2* mean_g) {
  const int cv = threadIdx.x % a.vpr, r = threadIdx.x / a.vpr;
  if (r >= a.lanes) return;
  ChannelConsts<V> c;
  c.load(a, s, cv);
  float m1[V], m2[V];
#pragma unroll
  for (int k = 0; k < V; ++k) { const float2 m = mean_g[(cv * V + k) / a.cg]; m1[k] = m.x; m2[k] = m.y; }
  for (long long i = b + r; i < e; i += (long long)a.lanes * BATCH) {
    Vec<T, V> v[BATCH], w[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const long long row = i + (long long)u * a.lanes;
      if (row < e) { v[u] = load_vec<Vec<T, V>, LOAD_ONCE>(x + row * a.ld_x + cv * V); w[u] = load_vec<Vec<T, V>, LOAD_ONCE>(dy + row * a.ld_dy + cv * V); }
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const long long row = i + (long long)u * a.lanes;
      if (row >= e) break;
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float xh = (to_f32<T>(v[u].v[k]) - c.mean[k]) * c.rstd[k];
        const float dz = to_f32<T>(w[u].v[k]) * act_slope(a.act, xh * c.gamma[k] + c.beta[k]);
        o[k] = c.rstd[k] * (c.gamma[k] * dz - m2[k] - xh * m1[k]);
      }
      store_f32<T, V>(dx + row * a.ld_y + cv * V, o);
    }
  }
}

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_grad_short_kernel(const NormArgs a, const T* x, const T* dy, T* dx) {
  float2* const red = shared_red();
  float2* const stat = red + (size_t)a.lanes * a.C;
  float2* const chan = stat + a.groups;
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) chan[c] = make_float2(0.f, 0.f);
  for (long long s = blockIdx.x; s < a.graphs; s += gridDim.x) {
    long long b, e;
    graph_rows(a, s, &b, &e);
    if (threadIdx.x == 0 && a.offsets) { long long u, v; group_rows(a.offsets, s, a.n, &u, &v, a.status); }
    if (e - b > 2 * a.R || b == e) continue;
    sum_grads<T, V>(a, x, dy, s, b, e, red);
    group_grads(a, red, stat);
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) { chan[c].x += red[c].x; chan[c].y += red[c].y; }
    const float inv = 1.f / ((float)(e - b) * (float)a.cg);
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stat[g] = make_float2(stat[g].x * inv, stat[g].y * inv);
    __syncthreads();
    write_grads<T, V>(a, x, dy, dx, s, b, e, stat);
    __syncthreads();
  }
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) a.chan[(size_t)(a.blocks + blockIdx.x) * a.C + c] = chan[c];
}

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_grad_stats_kernel(const NormArgs a, const T* x, const T* dy) {
  __shared__ Parts parts;
  float2* const red = shared_red();
  float2* const stat = red + (size_t)a.lanes * a.C;
  float2* const chan = stat + a.groups;
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) chan[c] = make_float2(0.f, 0.f);
  const long long blk = blockIdx.x;
  find_parts(a, blk, &parts);
  for (int k = 0; k < 2; ++k) {
    if (parts.s[k] < 0) continue;
    sum_grads<T, V>(a, x, dy, parts.s[k], parts.b[k], parts.e[k], red);
    group_grads(a, red, stat);
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) { chan[c].x += red[c].x; chan[c].y += red[c].y; }
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) a.part[(blk * 2 + k) * a.groups + g] = stat[g];
    __syncthreads();
  }
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) a.chan[(size_t)blk * a.C + c] = chan[c];
}

__global__ void norm_grad_combine_kernel(const NormArgs a) {
  Owned o;
  if (!owned_graph(a, blockIdx.x, &o)) return;
  const int lane = threadIdx.x & 31, g = blockIdx.y * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (g >= a.groups) return;
  double u = 0, v = 0;
  for (long long blk = o.first + lane; blk <= o.last; blk += 32) {
    const float2 p = a.part[(blk * 2 + (blk == o.first ? o.first_slot : 0)) * a.groups + g];
    u += p.x; v += p.y;
  }
  u = warp_sum(u); v = warp_sum(v);
  const double m = (double)(o.end - o.begin) * a.cg;
  if (lane == 0) a.sums[o.s * a.groups + g] = make_float2((float)(u / m), (float)(v / m));
}

template <class T, int V>
__global__ void __launch_bounds__(block_limit(V)) norm_grad_apply_kernel(const NormArgs a, const T* x, const T* dy, T* dx) {
  __shared__ Parts parts;
  float2* const stat = shared_red();
  find_parts(a, blockIdx.x, &parts);
  for (int k = 0; k < 2; ++k) {
    const long long s = parts.s[k];
    if (s < 0) continue;
    for (int g = threadIdx.x; g < a.groups; g += blockDim.x) stat[g] = a.sums[s * a.groups + g];
    __syncthreads();
    write_grads<T, V>(a, x, dy, dx, s, parts.b[k], parts.e[k], stat);
    __syncthreads();
  }
}

// grad_gamma, grad_beta: a lane to a channel, the warps share the blocks' sums, added in their order.
constexpr int CHANNEL_WARPS = 32;
__global__ void __launch_bounds__(32 * CHANNEL_WARPS) norm_channels_kernel(const NormArgs a) {
  __shared__ double2 part[CHANNEL_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const long long rows = a.blocks + a.short_blocks;
  double u = 0, v = 0;
  if (c < a.C)
    for (long long i = warp; i < rows; i += CHANNEL_WARPS) { const float2 p = a.chan[(size_t)i * a.C + c]; u += p.x; v += p.y; }
  part[warp][lane] = make_double2(u, v);
  __syncthreads();
  if (warp == 0 && c < a.C) {
    for (int w = 1; w < CHANNEL_WARPS; ++w) { u += part[w][lane].x; v += part[w][lane].y; }
    if (a.grad_gamma) a.grad_gamma[c] = (float)u;
    if (a.grad_beta) a.grad_beta[c] = (float)v;
  }
}

__global__ void norm_no_rows_kernel(const NormArgs a) {
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

constexpr int STAT_BLOCKS_PER_SM = 8, DEVICE_SMS = 148;
// Rows of a block of rows: at least 8 192 elements, and about eight blocks to an SM.  (By the device's number of SMs as built for, so
// that a workspace's size depends on the sizes alone.)
long long block_rows(int64_t n, int C) { return std::max<long long>(std::max(1, 8192 / C), (n + DEVICE_SMS * STAT_BLOCKS_PER_SM - 1) / (DEVICE_SMS * STAT_BLOCKS_PER_SM)); }

struct NormSpace { long long R, blocks, short_blocks; size_t part, chan, sums, mean, rstd, bytes; };
NormSpace norm_space(int64_t n, int64_t graphs, int C, int groups, bool grad) {
  NormSpace s;
  s.R = block_rows(n, C);
  const bool long_ones = n > 2 * s.R;                            // else no graph can be long
  s.blocks = long_ones ? (n + s.R - 1) / s.R : 0;
  s.short_blocks = std::min<long long>(graphs, DEVICE_SMS * 16);
  size_t at = 0;
  auto take = [&](size_t b) { const size_t o = at; at += (b + 255) / 256 * 256; return o; };
  s.part = take((size_t)s.blocks * 2 * groups * 8);
  s.chan = take(grad ? (size_t)(s.blocks + s.short_blocks) * C * 8 : 0);
  s.sums = take(grad && long_ones ? (size_t)graphs * groups * 8 : 0);
  s.mean = take(!grad && long_ones ? (size_t)graphs * groups * 4 : 0);
  s.rstd = take(!grad && long_ones ? (size_t)graphs * groups * 4 : 0);
  s.bytes = at;
  return s;
}

bool norm_shape_ok(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  return n >= 0 && n < (1ll << 31) && graphs >= 1 && graphs < (1ll << 31) && width >= 1 && groups >= 1 && width % groups == 0;
}

int norm_vector(int size, int width, const void* a, int64_t lda, const void* b, int64_t ldb, const void* c, int64_t ldc) {
  int v = 16 / size;
  auto bad = [&](const void* p, int64_t ld) { return p && (ld % v != 0 || !rows_aligned(p, v * size)); };
  while (v > 1 && (width % v != 0 || bad(a, lda) || bad(b, ldb) || bad(c, ldc))) v >>= 1;
  return v;
}

void set_block(NormArgs* a, int v, int threads, int* out_threads) {
  a->vpr = a->C / v;
  threads = std::max(threads, (a->vpr + 31) / 32 * 32);
  a->lanes = threads / a->vpr;
  *out_threads = threads;
}

// Threads for a short graph: about four vectors each for a graph of the average length.
int short_threads(int64_t n, int64_t graphs, int vpr) {
  const long long vectors = std::min<long long>(n / graphs + 1, 1ll << 20) * vpr;
  int t = 32;
  while (t < 512 && t * BATCH < vectors) t *= 2;
  return t;
}

}  // namespace

extern "C" int64_t taurus_norm_rows_workspace(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  if (!norm_shape_ok(n, graphs, width, groups)) return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)norm_space(n, graphs, width, groups, false).bytes;
}
extern "C" int64_t taurus_norm_rows_grad_workspace(int64_t n, int64_t graphs, int32_t width, int32_t groups) {
  if (!norm_shape_ok(n, graphs, width, groups)) return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)norm_space(n, graphs, width, groups, true).bytes;
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
  const size_t stat_bytes = (size_t)graphs * groups * 4;
  for (const void* p : {(const void*)offsets, (const void*)gamma, (const void*)beta, (const void*)mean, (const void*)rstd, (const void*)status})
    if (p && !rows_on_device(p, dev)) return TAURUS_ERR_INVALID_ARG;
  if (n > 0) {
    if (!rows_on_device(x, dev) || !rows_on_device(out_rows, dev)) return TAURUS_ERR_INVALID_ARG;
    const size_t out_bytes = rows_bytes(n, ld_out, width, ts), x_bytes = rows_bytes(n, ld_x, width, ts);
    if (rows_overlap(out_rows, out_bytes, x, x_bytes) && !(out_rows == x && ld_out == ld_x)) return TAURUS_ERR_INVALID_ARG;
    struct { const void* p; size_t n; } in[] = {{offsets, offsets ? (size_t)(graphs + 1) * 8 : 0}, {gamma, gamma ? (size_t)width * 4 : 0}, {beta, beta ? (size_t)width * 4 : 0},
                                                {mean, mean ? stat_bytes : 0}, {rstd, rstd ? stat_bytes : 0}};
    for (auto& i : in) if (rows_overlap(out_rows, out_bytes, i.p, i.n)) return TAURUS_ERR_INVALID_ARG;
    if (s.bytes) {
      if (!workspace || !rows_aligned(workspace, 256) || workspace_bytes < (int64_t)s.bytes || !rows_on_device(workspace, dev)) return TAURUS_ERR_INVALID_ARG;
      if (rows_overlap(workspace, s.bytes, out_rows, out_bytes) || rows_overlap(workspace, s.bytes, x, x_bytes)) return TAURUS_ERR_INVALID_ARG;
      for (auto& i : in) if (rows_overlap(workspace, s.bytes, i.p, i.n)) return TAURUS_ERR_INVALID_ARG;
    }
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  NormArgs a = {};
  a.n = n; a.graphs = graphs; a.offsets = reinterpret_cast<const long long*>(offsets); a.ld_x = ld_x; a.ld_y = ld_out; a.C = width; a.groups = groups;
  a.cg = width / groups; a.act = act; a.eps = eps; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd; a.status = status;
  a.R = s.R; a.blocks = s.blocks; a.short_blocks = s.blocks > 0 && !offsets ? 0 : s.short_blocks;   // (one graph of n rows: a long one)
  a.part = reinterpret_cast<float2*>(ws + s.part);
  if (n == 0) {
    if (mean || rstd) norm_no_rows_kernel<<<(int)std::min<long long>((graphs * groups + 255) / 256, 4096), 256, 0, st>>>(a);
  } else {
    if (s.blocks > 0) {
      if (!a.mean) a.mean = reinterpret_cast<float*>(ws + s.mean);
      if (!a.rstd) a.rstd = reinterpret_cast<float*>(ws + s.rstd);
    }
    const int v = norm_vector(ts, width, x, ld_x, out_rows, ld_out, nullptr, 0);
    with_row_type(type, [&](auto tt) {
      using T = typename decltype(tt)::type;
      return with_vector(v, [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V * sizeof(T) <= 16) {
          const T* const xp = static_cast<const T*>(x);
          T* const yp = static_cast<T*>(out_rows);
          int threads;
          if (a.short_blocks > 0) {
            set_block(&a, V, short_threads(n, graphs, width / V), &threads);
            const size_t smem = (size_t)a.lanes * width * 8 + (size_t)groups * 8 + (size_t)width * 4;
            norm_short_kernel<T, V><<<(int)a.short_blocks, threads, smem, st>>>(a, xp, yp);
          }
          if (s.blocks > 0) {
            set_block(&a, V, 256, &threads);
            const size_t smem = (size_t)a.lanes * width * 8 + (size_t)groups * 8 + (size_t)width * 4;
            norm_stats_kernel<T, V><<<(int)s.blocks, threads, smem, st>>>(a, xp);
            norm_combine_kernel<<<dim3((unsigned)s.blocks, (unsigned)((groups + 7) / 8)), 256, 0, st>>>(a);
            norm_apply_kernel<T, V><<<(int)s.blocks, threads, (size_t)groups * 8, st>>>(a, xp, yp);
          }
        }
        return 0;
      });
    });
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "norm_rows"); return TAURUS_ERR_CUDA; }
  return TAURUS_OK;
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
  for (const void* p : {(const void*)offsets, (const void*)gamma, (const void*)beta, (const void*)mean, (const void*)rstd, (const void*)grad_gamma, (const void*)grad_beta,
                        (const void*)status})
    if (p && !rows_on_device(p, dev)) return TAURUS_ERR_INVALID_ARG;
  if (rows_overlap(grad_gamma, grad_gamma ? cb : 0, grad_beta, grad_beta ? cb : 0)) return TAURUS_ERR_INVALID_ARG;
  struct { const void* p; size_t n; } in[] = {{offsets, offsets ? (size_t)(graphs + 1) * 8 : 0}, {gamma, gamma ? cb : 0}, {beta, beta ? cb : 0}, {mean, stat_bytes}, {rstd, stat_bytes}};
  struct { const void* p; size_t n; } sum[] = {{grad_gamma, grad_gamma ? cb : 0}, {grad_beta, grad_beta ? cb : 0}};
  for (auto& o : sum) for (auto& i : in) if (rows_overlap(o.p, o.n, i.p, i.n)) return TAURUS_ERR_INVALID_ARG;
  if (n > 0) {
    if (!rows_on_device(x, dev) || !rows_on_device(grad_out, dev) || !rows_on_device(grad_x, dev)) return TAURUS_ERR_INVALID_ARG;
    const size_t dx_bytes = rows_bytes(n, ld_grad_x, width, ts), x_bytes = rows_bytes(n, ld_x, width, ts), dy_bytes = rows_bytes(n, ld_grad, width, ts);
    if (rows_overlap(grad_x, dx_bytes, x, x_bytes) && !(grad_x == x && ld_grad_x == ld_x)) return TAURUS_ERR_INVALID_ARG;
    if (rows_overlap(grad_x, dx_bytes, grad_out, dy_bytes) && !(grad_x == grad_out && ld_grad_x == ld_grad)) return TAURUS_ERR_INVALID_ARG;
    for (auto& i : in) if (rows_overlap(grad_x, dx_bytes, i.p, i.n)) return TAURUS_ERR_INVALID_ARG;
    for (auto& o : sum)
      if (rows_overlap(o.p, o.n, grad_x, dx_bytes) || rows_overlap(o.p, o.n, x, x_bytes) || rows_overlap(o.p, o.n, grad_out, dy_bytes)) return TAURUS_ERR_INVALID_ARG;
    if (s.bytes) {
      if (!workspace || !rows_aligned(workspace, 256) || workspace_bytes < (int64_t)s.bytes || !rows_on_device(workspace, dev)) return TAURUS_ERR_INVALID_ARG;
      if (rows_overlap(workspace, s.bytes, grad_x, dx_bytes) || rows_overlap(workspace, s.bytes, x, x_bytes) || rows_overlap(workspace, s.bytes, grad_out, dy_bytes)) return TAURUS_ERR_INVALID_ARG;
      for (auto& i : in) if (rows_overlap(workspace, s.bytes, i.p, i.n)) return TAURUS_ERR_INVALID_ARG;
      for (auto& o : sum) if (rows_overlap(workspace, s.bytes, o.p, o.n)) return TAURUS_ERR_INVALID_ARG;
    }
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  NormArgs a = {};
  a.n = n; a.graphs = graphs; a.offsets = reinterpret_cast<const long long*>(offsets); a.ld_x = ld_x; a.ld_y = ld_grad_x; a.ld_dy = ld_grad; a.C = width; a.groups = groups;
  a.cg = width / groups; a.act = act; a.gamma = gamma; a.beta = beta; a.status = status; a.grad_gamma = grad_gamma; a.grad_beta = grad_beta;
  a.R = s.R; a.blocks = s.blocks; a.short_blocks = s.blocks > 0 && !offsets ? 0 : s.short_blocks;   // (one graph of n rows: a long one)
  a.part = reinterpret_cast<float2*>(ws + s.part); a.chan = reinterpret_cast<float2*>(ws + s.chan);
  a.sums = reinterpret_cast<float2*>(ws + s.sums);
  if (n == 0) {
    if (grad_gamma || grad_beta) norm_no_rows_kernel<<<4, 256, 0, st>>>(a);
  } else {
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);                 // read only here
    const int v = norm_vector(ts, width, x, ld_x, grad_out, ld_grad, grad_x, ld_grad_x);
    with_row_type(type, [&](auto tt) {
      using T = typename decltype(tt)::type;
      return with_vector(v, [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V * sizeof(T) <= 16) {
          const T *const xp = static_cast<const T*>(x), *const dyp = static_cast<const T*>(grad_out);
          T* const dxp = static_cast<T*>(grad_x);
          int threads;
          if (a.short_blocks > 0) {
            set_block(&a, V, short_threads(n, graphs, width / V), &threads);
            const size_t smem = (size_t)a.lanes * width * 8 + (size_t)groups * 8 + (size_t)width * 8;
            norm_grad_short_kernel<T, V><<<(int)a.short_blocks, threads, smem, st>>>(a, xp, dyp, dxp);
          }
          if (s.blocks > 0) {
            set_block(&a, V, 256, &threads);
            const size_t smem = (size_t)a.lanes * width * 8 + (size_t)groups * 8 + (size_t)width * 8;
            norm_grad_stats_kernel<T, V><<<(int)s.blocks, threads, smem, st>>>(a, xp, dyp);
            norm_grad_combine_kernel<<<dim3((unsigned)s.blocks, (unsigned)((groups + 7) / 8)), 256, 0, st>>>(a);
            norm_grad_apply_kernel<T, V><<<(int)s.blocks, threads, (size_t)groups * 8, st>>>(a, xp, dyp, dxp);
          }
        }
        return 0;
      });
    });
    if (grad_gamma || grad_beta) norm_channels_kernel<<<(width + 31) / 32, 32 * CHANNEL_WARPS, 0, st>>>(a);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "norm_rows_grad"); return TAURUS_ERR_CUDA; }
  return TAURUS_OK;
}
