// Norms before and after a block, fused with its gate and its residual scale, and the gradients.
//
//   u = N1(b) post_gamma (or b),  r' = r + alpha gate_g u,  y = N2(r') gamma + beta          N: (x - mean) rstd by row, or x rstd (RMS)
//   D = dr' + N2'(dy gamma),  dr = D,  dgate_g = alpha sum D u,  du = alpha gate_g D,  dpost_gamma = sum du h1,  db = N1'(du post_gamma) (or du)
//   dgamma = sum dy h2,  dbeta = sum dy         h: normalised rows,  N'(d) = rstd (d - mean(d) - h mean(d h)), without the first mean for RMS
//
// Bytes bound it: r and b in, r' and y out; r, b, dr', dy in, dr and db out.  A row is the work of a team of 1 to 128 neighbouring threads with 8 elements each, which
// stay in registers from the load to the store: statistics first the mean, then the squares of deviations.  A team takes neighbouring rows, so that the group of a row (the last one whose
// offset is not above it) is looked for once a group, and reads the next row before it sums up the one that it has.
// Sums by channel of the gradient stay in the threads' registers (a thread keeps its columns), are joined by block in shared memory, then by resnorm_join_kernel in the blocks' order.
// Sums by group: a group inside a team's rows is written at once; one that reaches over leaves a part in each team, "first" where it began before, "last" where it
// begins there and goes on; the join kernel adds them up in the teams' order.
#include <algorithm>

#include "rows.cuh"

namespace {

constexpr int THREADS = 256, N = 8;             // threads of a block, elements of a thread
constexpr int MAX_C = TAURUS_MAX_ROW_WIDTH;
constexpr int GRAD_BLOCKS = 2;                   // blocks of an SM that the gradient is spread over

struct Args {
  long long n;
  int C, team_shift;                             // a team is 1 << team_shift threads
  int layer, post, groups;
  float alpha, eps, inv_C;
  const void *res, *block, *dres, *dy;
  long long ld_res, ld_block, ld_dres, ld_dy;
  void *out_res, *out;                           // backward: gradients of res, block
  long long ld_out_res, ld_out;
  const float *post_gamma, *gate, *gamma, *beta;
  const long long* offsets;
  float4* stats;
  long long rows_a_team, teams;
  int32_t* status;
  // backward
  int blocks;
  float* chan;                                   // [blocks x 3 x C] (gamma, beta, post_gamma) of a block
  float *first, *last;                           // [teams x C]
  int2* span;                                    // [teams] (group, teams behind this one) of a group that goes on
  float *d_post, *d_gate, *d_gamma, *d_beta;
};

// Row r's group and its rows, kept inside [0, groups); -1: none.
struct Group {
  int g;
  long long begin, end;
};
__device__ __forceinline__ void find_group(const Args& a, long long r, Group* at) {
  if (!a.offsets) { *at = {0, 0, a.n}; return; }
  int g = at->g;
  if (g >= 0 && at->end <= r) {                  // most often one of the next ones
#pragma unroll 1
    for (int i = 0; i < 4 && g + 1 < a.groups; ++i) {
      ++g;
      const long long e = a.offsets[g + 1];
      if (e > r) {
        const long long b = a.offsets[g];
        if (b <= r) { *at = {g, b, e}; return; }
        break;
      }
    }
  }
  int lo = 0, hi = a.groups;                     // offsets[lo - 1] <= r < offsets[hi + 1], so to say
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.offsets[mid] <= r) lo = mid; else hi = mid - 1;
  }
  const long long b = a.offsets[lo];
  if (b > r) { *at = {-1, 0, b < a.n ? b : a.n}; return; }             // in front of the first group, up to its rows
  if (lo == a.groups) { *at = {-1, b, a.n}; return; }                   // behind the last
  const long long e = a.offsets[lo + 1];
  *at = {lo, b, e > r ? e : r + 1};
}
__device__ __forceinline__ void check_offsets(const Args& a) {
  if (!a.offsets) return;
  for (long long g = (long long)blockIdx.x * THREADS + threadIdx.x; g < a.groups; g += (long long)gridDim.x * THREADS) {
    const long long b = a.offsets[g], e = a.offsets[g + 1];
    if (b < 0 || e > a.n || e < b) rows_status(a.status, TAURUS_ERR_INVALID_ARG);
  }
}

// A thread's place in its team and the columns that it keeps: vectors lane, lane + size, ... of V elements.
template <int V, bool MULTI>
struct Team {
  static constexpr int NV = N / V;
  int size, lane, warps, id;                     // id: of the block's teams
  int col[NV];
  bool on[NV];
  float2* slot;                                  // shared memory of teams of several warps: [2][warps]
  int flip = 0;
  __device__ __forceinline__ explicit Team(const Args& a) {
    __shared__ float2 slots[2 * THREADS / 32];
    size = 1 << a.team_shift; lane = threadIdx.x & (size - 1); id = threadIdx.x >> a.team_shift; warps = size >> 5;
    slot = slots + id * 2 * warps;
#pragma unroll
    for (int j = 0; j < NV; ++j) { col[j] = (j * size + lane) * V; on[j] = col[j] < a.C; }
  }
  __device__ __forceinline__ float2 sum(float x, float y) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      if (MULTI || d < size) { x += __shfl_xor_sync(0xffffffffu, x, d); y += __shfl_xor_sync(0xffffffffu, y, d); }
    return MULTI ? across(x, y) : make_float2(x, y);
  }
  __device__ __forceinline__ float sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      if (MULTI || d < size) x += __shfl_xor_sync(0xffffffffu, x, d);
    return MULTI ? across(x, 0.f).x : x;
  }
  // The two halves of the slots are used in turn: a warp that is through with one sum may write the next while others still read.
  __device__ __forceinline__ float2 across(float x, float y) {
    float2* const s = slot + flip * warps;
    flip ^= 1;
    if ((threadIdx.x & 31) == 0) s[lane >> 5] = make_float2(x, y);
    asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(size) : "memory");
    float2 t = s[0];
    for (int w = 1; w < warps; ++w) { t.x += s[w].x; t.y += s[w].y; }
    return t;
  }
  template <class T>
  __device__ __forceinline__ void load(const T* row, float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = 0.f;
      if (on[j]) load_f32<T, V, LOAD_ONCE>(row + col[j], v);
#pragma unroll
      for (int i = 0; i < V; ++i) x[j * V + i] = v[i];
    }
  }
  template <class T>
  __device__ __forceinline__ void load_raw(const T* row, Vec<T, V> (&x)[NV]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) if (on[j]) x[j] = load_vec<Vec<T, V>, LOAD_ONCE>(row + col[j]);
  }
  template <class T>
  __device__ __forceinline__ void to_floats(const Vec<T, V> (&r)[NV], float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) x[j * V + i] = on[j] ? to_f32<T>(r[j].v[i]) : 0.f;
  }
  // A row of fp32 parameters, or `otherwise` where there is none.
  __device__ __forceinline__ void load_row(const float* row, float otherwise, float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = otherwise;
      if (row && on[j]) load_f32<float, V>(row + col[j], v);
#pragma unroll
      for (int i = 0; i < V; ++i) x[j * V + i] = v[i];
    }
  }
  template <class T>
  __device__ __forceinline__ void store(T* row, const float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = x[j * V + i];
      if (on[j]) store_f32_once<T, V>(row + col[j], v);
    }
  }
  __device__ __forceinline__ void store_row(float* row, const float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = x[j * V + i];
      if (on[j]) store_f32<float, V>(row + col[j], v);
    }
  }
  __device__ __forceinline__ bool valid(int e) const { return on[e / V]; }
  // (mean, rstd) of a row; RMS: mean 0.
  __device__ __forceinline__ float2 statistics(const Args& a, const float (&x)[N]) {
    float mean = 0.f, q = 0.f;
    if (a.layer) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) s += x[e];
      mean = sum(s) * a.inv_C;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) { const float d = valid(e) ? x[e] - mean : 0.f; q = fmaf(d, d, q); }
    return make_float2(mean, rsqrtf(fmaf(sum(q), a.inv_C, a.eps)));
  }
};

template <class T, class R, int V, bool MULTI>
__global__ void __launch_bounds__(THREADS) resnorm_kernel(const Args a) {
  check_offsets(a);
  Team<V, MULTI> team(a);
  constexpr int NV = Team<V, MULTI>::NV;
  const long long mine = ((long long)blockIdx.x * THREADS + threadIdx.x) >> a.team_shift;
  const long long begin = mine * a.rows_a_team, end = begin + a.rows_a_team < a.n ? begin + a.rows_a_team : a.n;
  // A warp of small teams goes on while one of its teams has rows: the shuffles take all of its threads.
  const long long most = MULTI || a.team_shift >= 5 ? end : __reduce_max_sync(0xffffffffu, begin < end ? (unsigned)(end - begin) : 0u) + begin;
  float ga[N], be[N], pg[N], gt[N];
  team.load_row(a.gamma, 1.f, ga);
  team.load_row(a.beta, 0.f, be);
  team.load_row(a.post_gamma, 1.f, pg);
#pragma unroll
  for (int e = 0; e < N; ++e) gt[e] = a.alpha;
  const R* const res = static_cast<const R*>(a.res);
  const T* const block = static_cast<const T*>(a.block);
  Vec<R, V> raw_r[NV];
  Vec<T, V> raw_b[NV];
  const auto fetch = [&](long long row) {
    if (row >= end) return;
    team.load_raw(res + row * a.ld_res, raw_r);
    if (block) team.load_raw(block + row * a.ld_block, raw_b);
  };
  fetch(begin);
  Group group = {-1, 0, 0};
  for (long long row = begin; row < most; ++row) {
    const bool have = row < end;
    if (have && a.gate && (row == begin || row >= group.end)) {
      find_group(a, row, &group);
      if (group.g >= 0) {
        team.load_row(a.gate + (long long)group.g * a.C, 1.f, gt);
#pragma unroll
        for (int e = 0; e < N; ++e) gt[e] *= a.alpha;
      }
    }
    float r[N], b[N];
    team.to_floats(raw_r, r);
    if (block) team.to_floats(raw_b, b);
    fetch(row + 1);
    float2 s1 = make_float2(0.f, 0.f);
    if (block) {
      if (a.post) {
        s1 = team.statistics(a, b);
#pragma unroll
        for (int e = 0; e < N; ++e) b[e] = (b[e] - s1.x) * s1.y * pg[e];
      }
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = team.valid(e) ? fmaf(gt[e], b[e], r[e]) : 0.f;
    }
    const float2 s2 = team.statistics(a, r);
    if (have && (!a.gate || group.g >= 0)) {
      if (a.out_res) team.store(static_cast<R*>(a.out_res) + row * a.ld_out_res, r);
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = fmaf((r[e] - s2.x) * s2.y, ga[e], be[e]);
      team.store(static_cast<T*>(a.out) + row * a.ld_out, r);
      if (a.stats && team.lane == 0) a.stats[row] = make_float4(s1.x, s1.y, s2.x, s2.y);
    }
  }
}

template <class T, class R, int V, bool MULTI>
__global__ void __launch_bounds__(THREADS, GRAD_BLOCKS) resnorm_grad_kernel(const Args a) {
  extern __shared__ __align__(16) float resnorm_shared[];             // [teams of the block x C]
  check_offsets(a);
  Team<V, MULTI> team(a);
  const long long mine = ((long long)blockIdx.x * THREADS + threadIdx.x) >> a.team_shift;
  const long long begin = mine * a.rows_a_team, end = begin + a.rows_a_team < a.n ? begin + a.rows_a_team : a.n;
  const long long most = MULTI || a.team_shift >= 5 ? end : __reduce_max_sync(0xffffffffu, begin < end ? (unsigned)(end - begin) : 0u) + begin;
  float ga[N], pg[N], gt[N];
  team.load_row(a.gamma, 1.f, ga);
  team.load_row(a.post_gamma, 1.f, pg);
#pragma unroll
  for (int e = 0; e < N; ++e) gt[e] = a.alpha;
  float sum_ga[N] = {}, sum_be[N] = {}, sum_pg[N] = {}, sum_gt[N] = {};
  Group group = {-1, 0, 0};
  const R *const res = static_cast<const R*>(a.res), *const dres = static_cast<const R*>(a.dres);
  const T *const block = static_cast<const T*>(a.block), *const dy = static_cast<const T*>(a.dy);
  int2 goes_on = make_int2(-1, 0);
  // The sums of the group that ends in front of `row`.
  const auto close_group = [&](long long row) {
    if (!a.d_gate || group.g < 0) return;
#pragma unroll
    for (int e = 0; e < N; ++e) sum_gt[e] *= a.alpha;
    const bool before = group.begin < begin, after = row >= end && group.end > end;
    if (!before && !after) team.store_row(a.d_gate + (long long)group.g * a.C, sum_gt);
    else if (before) team.store_row(a.first + mine * a.C, sum_gt);
    else {
      team.store_row(a.last + mine * a.C, sum_gt);
      goes_on = make_int2(group.g, (int)((group.end < a.n ? group.end - 1 : a.n - 1) / a.rows_a_team - mine));
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sum_gt[e] = 0.f;
  };
  for (long long row = begin; row < most; ++row) {
    const bool have = row < end;
    if (have && a.gate && (row == begin || row >= group.end)) {
      if (row > begin) close_group(row);
      find_group(a, row, &group);
      if (group.g >= 0) {
        team.load_row(a.gate + (long long)group.g * a.C, 1.f, gt);
#pragma unroll
        for (int e = 0; e < N; ++e) gt[e] *= a.alpha;
      }
    }
    const bool live = have && (!a.gate || group.g >= 0);
    float x[N], u[N], d[N], g[N];
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) {
      team.load(res + row * a.ld_res, x);
      if (block) team.load(block + row * a.ld_block, u);
      if (dres) team.load(dres + row * a.ld_dres, d);
      if (dy) team.load(dy + row * a.ld_dy, g);
      st = a.stats[row];
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = u[e] = 0.f;
    }
    if (!live || !dres) {
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = 0.f;
    }
    if (!live || !dy) {
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = 0.f;
    }
    if (block) {
      if (a.post) {
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = team.valid(e) ? (u[e] - st.x) * st.y : 0.f;                  // h1
      }
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = fmaf(gt[e], a.post ? u[e] * pg[e] : u[e], x[e]);
    }
    if (dy) {
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[e] = team.valid(e) ? (x[e] - st.z) * st.w : 0.f;                                              // h2
        sum_be[e] += g[e];
        sum_ga[e] = fmaf(g[e], x[e], sum_ga[e]);
        g[e] *= ga[e];
        s += g[e];
        q = fmaf(g[e], x[e], q);
      }
      const float2 t = team.sum(s, q);
      const float m1 = a.layer ? t.x * a.inv_C : 0.f, m2 = t.y * a.inv_C;
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = fmaf(st.w, g[e] - m1 - x[e] * m2, d[e]);
    }
    if (live) team.store(static_cast<R*>(a.out_res) + row * a.ld_out_res, d);
    if (block) {
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float dv = team.valid(e) ? d[e] : 0.f;
        sum_gt[e] = fmaf(dv, a.post ? u[e] * pg[e] : u[e], sum_gt[e]);
        d[e] = dv * gt[e];                                                                              // du
        if (a.post) {
          sum_pg[e] = fmaf(d[e], u[e], sum_pg[e]);
          d[e] *= pg[e];
          s += d[e];
          q = fmaf(d[e], u[e], q);
        }
      }
      if (a.post) {
        const float2 t = team.sum(s, q);
        const float m1 = a.layer ? t.x * a.inv_C : 0.f, m2 = t.y * a.inv_C;
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = st.y * (d[e] - m1 - u[e] * m2);
      }
      if (live && a.out) team.store(static_cast<T*>(a.out) + row * a.ld_out, d);
    }
  }
  if (begin < end) close_group(end);
  if (a.span && team.lane == 0 && mine < a.teams) a.span[mine] = goes_on;
  if (a.chan) {
    const int teams = THREADS >> a.team_shift;
    float* const mine_row = resnorm_shared + team.id * a.C;
    for (int which = 0; which < 3; ++which) {
      __syncthreads();
      if (which == 0) team.store_row(mine_row, sum_ga);
      else if (which == 1) team.store_row(mine_row, sum_be);
      else team.store_row(mine_row, sum_pg);
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += THREADS) {
        float s = 0.f;
        for (int t = 0; t < teams; ++t) s += resnorm_shared[t * a.C + c];
        a.chan[((long long)blockIdx.x * 3 + which) * a.C + c] = s;
      }
    }
  }
}

// Joins what the blocks and teams left: 32 columns a block, 32 parts at a time.
constexpr int JOIN = 32;
__device__ __forceinline__ float join_columns(float mine) {          // over the 32 rows of threads; for the first of them
  __shared__ float part[JOIN][JOIN + 1];
  const int x = threadIdx.x % JOIN, y = threadIdx.x / JOIN;
  __syncthreads();
  part[y][x] = mine;
  __syncthreads();
  float s = part[x][y];                                               // a warp to a column
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;                                                           // of the column with the warp's number
}
__global__ void __launch_bounds__(JOIN * JOIN) resnorm_join_kernel(const Args a, int column_blocks) {
  early_start();
  const int cb = blockIdx.x % column_blocks, tx = threadIdx.x % JOIN, ty = threadIdx.x / JOIN;
  const long long unit0 = blockIdx.x / column_blocks, units = gridDim.x / column_blocks;
  const int c = cb * JOIN + tx, cw = cb * JOIN + ty;
  for (long long unit = unit0; unit < 3; unit += units) {
    float* const out = unit == 0 ? a.d_gamma : unit == 1 ? a.d_beta : a.d_post;
    if (!out) continue;
    float s = 0.f;
    if (c < a.C)
      for (int b = ty; b < a.blocks; b += JOIN) s += a.chan[((long long)b * 3 + unit) * a.C + c];
    s = join_columns(s);
    if (tx == 0 && cw < a.C) out[cw] = s;
  }
  if (!a.d_gate) return;
  for (long long t = unit0; t < a.teams; t += units) {
    const int2 span = a.span[t];
    if (span.x < 0) continue;
    float s = 0.f;
    if (c < a.C) {
      if (ty == 0) s = a.last[t * a.C + c];
      const long long to = t + span.y < a.teams ? t + span.y : a.teams - 1;
      for (long long i = t + 1 + ty; i <= to; i += JOIN) s += a.first[i * a.C + c];
    }
    s = join_columns(s);
    if (tx == 0 && cw < a.C) a.d_gate[(long long)span.x * a.C + cw] = s;
  }
  // groups without rows
  for (long long g = unit0 * JOIN + ty; g < a.groups; g += units * JOIN) {
    long long b = 0, e = a.n;
    if (a.offsets) group_rows(a.offsets, g, a.n, &b, &e, nullptr);
    if (b >= e && c < a.C) a.d_gate[g * a.C + c] = 0.f;
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------------------------

inline int team_shift_of(int C) {
  int s = 0;
  while ((N << s) < C) ++s;
  return s;                                      // up to 7
}

constexpr int SMS = 148;                         // for workspaces, which are counted without a device
constexpr int MIN_ROWS = 2;                      // rows of a team at least

struct Plan { int64_t rows_a_team, teams, blocks; };
Plan plan_of(int64_t n, int C, int64_t rows_a_team) {
  const int64_t a_block = THREADS >> team_shift_of(C), teams = (n + rows_a_team - 1) / rows_a_team;
  return {rows_a_team, teams, (teams + a_block - 1) / a_block};
}
// Forward: up to 16 rows, as long as eight blocks an SM have work.
Plan forward_plan(int64_t n, int C, int sms) {
  const int64_t a_block = THREADS >> team_shift_of(C);
  return plan_of(n, C, std::max<int64_t>(1, std::min<int64_t>(16, n / (a_block * sms * 8))));
}
// Gradient: all rows over the blocks that are resident at once, two rows a team at least.
Plan grad_plan(int64_t n, int C, int sms) {
  const int64_t a_block = THREADS >> team_shift_of(C), teams = a_block * std::min(sms, SMS) * GRAD_BLOCKS;
  return plan_of(n, C, std::max<int64_t>(MIN_ROWS, (n + teams - 1) / teams));
}
struct Space { size_t chan, first, last, span, bytes; };
Space space_of(int64_t n, int C, int groups) {
  Space s = {};
  if (n == 0) return s;
  // (what does for n rows does for fewer: the number of blocks and of teams is bounded by that of the largest plan)
  const int64_t a_block = THREADS >> team_shift_of(C);
  const int64_t blocks = std::min<int64_t>((int64_t)SMS * GRAD_BLOCKS, (n + a_block - 1) / a_block), teams = std::min<int64_t>(blocks * a_block, n);
  size_t at = 0;
  const auto take = [&](size_t b) { const size_t here = at; at += (b + 255) / 256 * 256; return here; };
  s.chan = take((size_t)blocks * 3 * C * 4);
  if (groups > 0) {
    s.first = take((size_t)teams * C * 4);
    s.last = take((size_t)teams * C * 4);
    s.span = take((size_t)teams * sizeof(int2));
  }
  s.bytes = at;
  return s;
}

// Elements of a vector that every row array allows.
struct Rows { const void* p; int64_t ld; int size; };
template <int K>
int vector_of(int C, int full, const Rows (&rows)[K], const void* const* params, int count) {
  for (int v = full; v > 1; v = v == 8 ? 4 : 1) {
    bool ok = C % v == 0;
    for (const Rows& r : rows) if (r.p) { const int b = std::min(16, v * r.size); ok = ok && rows_aligned(r.p, b) && (r.ld * r.size) % b == 0; }
    for (int i = 0; i < count; ++i) if (params[i]) ok = ok && rows_aligned(params[i], 16);
    if (ok) return v;
  }
  return 1;
}
// f(tag of T, tag of R, vector) for the types and the vector.
template <class F>
void with_rows(int32_t type, int32_t res_type, int v, F f) {
  with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    const auto with = [&](auto rt) {
      if constexpr (sizeof(T) == 2) { if (v == 8) { f(tt, rt, std::integral_constant<int, 8>()); return; } }
      if (v >= 4) f(tt, rt, std::integral_constant<int, 4>());
      else f(tt, rt, std::integral_constant<int, 1>());
    };
    if constexpr (sizeof(T) == 2) { if (res_type == type) { with(tt); return 0; } }
    with(RowTag<float>());
    return 0;
  });
}

bool shape_ok(int64_t n, int32_t width, int32_t groups) { return n >= 0 && n < (1ll << 31) && width >= 1 && groups >= 0 && groups <= (1 << 30); }

int resnorm_check(int64_t n, int32_t width, const void* res, int64_t ld_res, int32_t res_type, const void* block, int64_t ld_block, int32_t type, int32_t kind, int32_t post,
                  const float* post_gamma, int32_t groups, const int64_t* offsets, const float* gate, float alpha, const float* gamma, const int32_t* status) {
  const int ts = row_type_size(type), rs = row_type_size(res_type);
  if (!ts || !rs || (res_type != type && res_type != TAURUS_F32) || !shape_ok(n, width, groups) || ld_res < width || !rows_fit(n, ld_res, 4) ||
      (block && (ld_block < width || !rows_fit(n, ld_block, 4))) || (kind != TAURUS_NORM_LAYER && kind != TAURUS_NORM_RMS) || (post != 0 && post != 1) || (post_gamma && !post) ||
      !(alpha - alpha == 0.f) || (gate ? groups < 1 : groups != 0) || (offsets && !gate) || (gate && !offsets && groups != 1) || (!block && n > 0 && (post || gate)) ||
      !rows_aligned(offsets, 8) || !rows_aligned(gate, 4) || !rows_aligned(gamma, 4) || !rows_aligned(post_gamma, 4) || !rows_aligned(status, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  if (n > 0 && (!res || !rows_aligned(res, rs) || !rows_aligned(block, ts))) return TAURUS_ERR_INVALID_ARG;
  return TAURUS_OK;
}

}  // namespace

extern "C" int taurus_residual_norm(int64_t n, int32_t width, const void* res, int64_t ld_res, int32_t res_type, const void* block, int64_t ld_block, int32_t type, int32_t kind,
                                    int32_t post, const float* post_gamma, int32_t groups, const int64_t* offsets, const float* gate, float alpha, const float* gamma,
                                    const float* beta, float eps, void* out_res, int64_t ld_out_res, void* out, int64_t ld_out, float* stats, int32_t* status, void* cuda_stream) {
  const int rc = resnorm_check(n, width, res, ld_res, res_type, block, ld_block, type, kind, post, post_gamma, groups, offsets, gate, alpha, gamma, status);
  if (rc != TAURUS_OK) return rc;
  const int ts = row_type_size(type), rs = row_type_size(res_type);
  if (!(eps >= 0.f) || ld_out < width || !rows_fit(n, ld_out, 4) || (out_res && (ld_out_res < width || !rows_fit(n, ld_out_res, 4))) || !rows_aligned(beta, 4) || !rows_aligned(stats, 16) ||
      !rows_aligned(out_res, rs) || !rows_aligned(out, ts) || (n > 0 && (!out || (block && !out_res) || (!block && out_res))))
    return TAURUS_ERR_INVALID_ARG;
  if (n == 0) return TAURUS_OK;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const size_t cb = (size_t)width * 4;
  const bool over_res = out_res == res && ld_out_res == ld_res, over_block = out == block && ld_out == ld_block;       // in place
  const Region outs[] = {region_of_rows(out_res, n, ld_out_res, width, rs), region_of_rows(out, n, ld_out, width, ts), region_of(stats, (size_t)n * 16), region_of(status, 4)};
  const Region ins[] = {over_res ? region_of(nullptr, 0) : region_of_rows(res, n, ld_res, width, rs), over_block ? region_of(nullptr, 0) : region_of_rows(block, n, ld_block, width, ts),
                        region_of(offsets, (size_t)(groups + 1) * 8), region_of(gate, cb * (size_t)groups), region_of(post_gamma, cb), region_of(gamma, cb), region_of(beta, cb)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins)) return TAURUS_ERR_INVALID_ARG;
  Args a = {};
  a.n = n; a.C = width; a.team_shift = team_shift_of(width); a.layer = kind == TAURUS_NORM_LAYER; a.post = post; a.groups = groups; a.alpha = alpha; a.eps = eps;
  a.inv_C = 1.f / (float)width; a.res = res; a.ld_res = ld_res; a.block = block; a.ld_block = ld_block; a.out_res = out_res; a.ld_out_res = ld_out_res; a.out = out; a.ld_out = ld_out;
  a.post_gamma = post_gamma; a.gate = gate; a.gamma = gamma; a.beta = beta; a.offsets = reinterpret_cast<const long long*>(offsets); a.stats = reinterpret_cast<float4*>(stats);
  a.status = status;
  const Plan p = forward_plan(n, width, sms);
  a.rows_a_team = p.rows_a_team; a.teams = p.teams;
  const Rows rows[] = {{res, ld_res, rs}, {block, ld_block, ts}, {out_res, ld_out_res, rs}, {out, ld_out, ts}};
  const void* const params[] = {post_gamma, gate, gamma, beta};
  Launches enqueue = {static_cast<cudaStream_t>(cuda_stream)};
  with_rows(type, res_type, vector_of(width, ts == 2 ? 8 : 4, rows, params, 4), [&](auto tt, auto rt, auto vc) {
    using T = typename decltype(tt)::type;
    using R = typename decltype(rt)::type;
    constexpr int V = decltype(vc)::value;
    if (a.team_shift > 5) enqueue(resnorm_kernel<T, R, V, true>, dim3((unsigned)p.blocks), THREADS, 0, a);
    else enqueue(resnorm_kernel<T, R, V, false>, dim3((unsigned)p.blocks), THREADS, 0, a);
  });
  return enqueue.done("residual norm");
}

extern "C" int64_t taurus_residual_norm_grad_workspace(int64_t n, int32_t width, int32_t groups) {
  if (!shape_ok(n, width, groups)) return TAURUS_ERR_INVALID_ARG;
  if (width > MAX_C) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)space_of(n, width, groups).bytes;
}

extern "C" int taurus_residual_norm_grad(int64_t n, int32_t width, const void* res, int64_t ld_res, int32_t res_type, const void* block, int64_t ld_block, int32_t type, int32_t kind,
                                         int32_t post, const float* post_gamma, int32_t groups, const int64_t* offsets, const float* gate, float alpha, const float* gamma,
                                         const float* stats, const void* grad_out_res, int64_t ld_grad_out_res, const void* grad_out, int64_t ld_grad_out, void* grad_res,
                                         int64_t ld_grad_res, void* grad_block, int64_t ld_grad_block, float* grad_post_gamma, float* grad_gate, float* grad_gamma, float* grad_beta,
                                         void* workspace, int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const int rc = resnorm_check(n, width, res, ld_res, res_type, block, ld_block, type, kind, post, post_gamma, groups, offsets, gate, alpha, gamma, status);
  if (rc != TAURUS_OK) return rc;
  const int ts = row_type_size(type), rs = row_type_size(res_type);
  const struct { const void* p; int64_t ld; int size; } more[] = {{grad_out_res, ld_grad_out_res, rs}, {grad_out, ld_grad_out, ts}, {grad_res, ld_grad_res, rs}, {grad_block, ld_grad_block, ts}};
  for (const auto& r : more) if (r.p && (r.ld < width || !rows_fit(n, r.ld, 4) || !rows_aligned(r.p, r.size))) return TAURUS_ERR_INVALID_ARG;
  if (!rows_aligned(stats, 16) || !rows_aligned(grad_post_gamma, 4) || !rows_aligned(grad_gate, 4) || !rows_aligned(grad_gamma, 4) || !rows_aligned(grad_beta, 4) ||
      (grad_post_gamma && !post) || (grad_gate && !gate) || (n > 0 && (!stats || !grad_res || (!grad_out_res && !grad_out) || (grad_block && !block))))
    return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const size_t cb = (size_t)width * 4;
  const Region none = region_of(nullptr, 0);
  const auto same = [](const void* p, int64_t ld, const void* q, int64_t l) { return p && p == q && ld == l; };
  const bool res_in_place = same(grad_res, ld_grad_res, res, ld_res), dres_in_place = same(grad_res, ld_grad_res, grad_out_res, ld_grad_out_res);
  const bool block_in_place = same(grad_block, ld_grad_block, block, ld_block), dy_in_place = same(grad_block, ld_grad_block, grad_out, ld_grad_out);
  const Region outs[] = {region_of_rows(grad_res, n, ld_grad_res, width, rs), region_of_rows(grad_block, n, ld_grad_block, width, ts), region_of(grad_post_gamma, cb),
                         region_of(grad_gate, cb * (size_t)groups), region_of(grad_gamma, cb), region_of(grad_beta, cb), region_of(status, 4)};
  const Region ins[] = {res_in_place ? none : region_of_rows(res, n, ld_res, width, rs), block_in_place ? none : region_of_rows(block, n, ld_block, width, ts),
                        dres_in_place ? none : region_of_rows(grad_out_res, n, ld_grad_out_res, width, rs), dy_in_place ? none : region_of_rows(grad_out, n, ld_grad_out, width, ts),
                        region_of(offsets, (size_t)(groups + 1) * 8), region_of(gate, cb * (size_t)groups), region_of(post_gamma, cb), region_of(gamma, cb), region_of(stats, (size_t)n * 16)};
  const Space s = space_of(n, width, groups);
  const bool joins = grad_post_gamma || grad_gate || grad_gamma || grad_beta;
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) || !workspace_ok(workspace, workspace_bytes, joins ? (int64_t)s.bytes : 0, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  if (n == 0 && !joins) return TAURUS_OK;
  char* const ws = static_cast<char*>(workspace);
  Args a = {};
  a.n = n; a.C = width; a.team_shift = team_shift_of(width); a.layer = kind == TAURUS_NORM_LAYER; a.post = post; a.groups = groups; a.alpha = alpha; a.inv_C = 1.f / (float)width;
  a.res = res; a.ld_res = ld_res; a.block = block; a.ld_block = ld_block; a.dres = grad_out_res; a.ld_dres = ld_grad_out_res; a.dy = grad_out; a.ld_dy = ld_grad_out;
  a.out_res = grad_res; a.ld_out_res = ld_grad_res; a.out = grad_block; a.ld_out = ld_grad_block; a.post_gamma = post_gamma; a.gate = gate; a.gamma = gamma;
  a.offsets = reinterpret_cast<const long long*>(offsets); a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats)); a.status = status;      // read only here
  a.d_post = grad_post_gamma; a.d_gate = grad_gate; a.d_gamma = grad_gamma; a.d_beta = grad_beta;
  Launches enqueue = {static_cast<cudaStream_t>(cuda_stream)};
  if (n > 0) {
    const Plan p = grad_plan(n, width, sms);
    a.rows_a_team = p.rows_a_team; a.teams = p.teams; a.blocks = (int)p.blocks;
    if (grad_post_gamma || grad_gamma || grad_beta) a.chan = reinterpret_cast<float*>(ws + s.chan);
    if (grad_gate) { a.first = reinterpret_cast<float*>(ws + s.first); a.last = reinterpret_cast<float*>(ws + s.last); a.span = reinterpret_cast<int2*>(ws + s.span); }
    const Rows rows[] = {{res, ld_res, rs}, {block, ld_block, ts}, {grad_out_res, ld_grad_out_res, rs}, {grad_out, ld_grad_out, ts}, {grad_res, ld_grad_res, rs}, {grad_block, ld_grad_block, ts}};
    const void* const params[] = {post_gamma, gate, gamma, grad_gate};
    with_rows(type, res_type, vector_of(width, ts == 2 ? 8 : 4, rows, params, 4), [&](auto tt, auto rt, auto vc) {
      using T = typename decltype(tt)::type;
      using R = typename decltype(rt)::type;
      constexpr int V = decltype(vc)::value;
      const size_t smem = a.chan ? (size_t)(THREADS >> a.team_shift) * width * 4 : 0;
      if (a.team_shift > 5) enqueue(resnorm_grad_kernel<T, R, V, true>, dim3((unsigned)p.blocks), THREADS, smem, a);
      else enqueue(resnorm_grad_kernel<T, R, V, false>, dim3((unsigned)p.blocks), THREADS, smem, a);
    });
  }
  if (joins) {
    const int column_blocks = (width + JOIN - 1) / JOIN;
    const int64_t units = std::max<int64_t>(3, std::min<int64_t>(grad_gate ? std::max<int64_t>(a.teams, groups / JOIN) : 3, 1184 / column_blocks));
    if (n == 0) a.blocks = 0;
    enqueue.early = n > 0;
    enqueue(resnorm_join_kernel, dim3((unsigned)(units * column_blocks)), JOIN * JOIN, 0, a, column_blocks);
  }
  return enqueue.done("residual norm's gradient");
}
