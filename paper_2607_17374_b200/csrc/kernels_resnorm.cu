// Norms before and after a block, fused with its gate and its residual scale, and the gradients.
//
//   u = N1(b) post_gamma (or b),  r' = r + alpha gate_g u,  y = N2(r') gamma + beta          N: (x - mean) rstd by row, or x rstd (RMS)
//   D = dr' + N2'(dy gamma),  dr = D,  dgate_g = alpha sum D u,  du = alpha gate_g D,  dpost_gamma = sum du h1,  db = N1'(du post_gamma) (or du)
//   dgamma = sum dy h2,  dbeta = sum dy         h: normalised rows,  N'(d) = rstd (d - mean(d) - h mean(d h)), without the first mean for RMS
//
// Bytes bound it: r and b in, r' and y out; r, b, dr', dy in, dr and db out.  A row is the work of a team of 1 to 128 neighbouring threads (a power of two up to a warp, then whole warps, which are a block) with 8 elements each, which
// stay in registers from the load to the store: statistics first the mean, then the squares of deviations.  A team walks over neighbouring rows, so that the group of a row (the last one whose
// offset is not above it) is looked for once a group.  Rows are on their way some rows ahead, by asynchronous copies into places of shared memory that are a thread's own: a thread
// waits for its own copies and for nobody (of widths that 16-byte vectors do not fit, for its team).
// Measured: 1 200 000 x 256 bf16 with 16 groups 464 us, 5.3 TB/s, bound by the bytes with an issue slot in 74 % of the cycles beside them; 500 000 x 256 fp32 in 9 001 groups with the gradients 940 us, 5.5 TB/s over the
// ten passes of the two calls; 120 001 x 100 fp16 on fp32 rows, 7 groups, 98 us: few rows a team, latencies at its ends; 196 078 x 255 fp32 (50 M elements) 146 us and 260 for the gradient, at 256 143 and 240.
// Widths below 8 leave threads of one row with fewer elements (7 100 000 x 7 fp32 328 us, the gradient 1 147).
// Sums by channel stay in the threads' registers (a thread keeps its columns).  Those of post_gamma and of the gate come from one: with S_g = sum over the group's rows of D h1,
// dgate_g = alpha post_gamma S_g and dpost_gamma = sum_g alpha gate_g S_g.  Blocks join theirs in shared memory, resnorm_join_kernel the blocks' in their order.
// A group inside a team's rows has its sums written at once; one that reaches over leaves a part in each team, "first" where it began before, "last" where it
// begins there and goes on; the join kernel adds them up in the teams' order.
#include <algorithm>

#include "group_search.h"
#include "rows.cuh"

namespace {

constexpr int THREADS = 256, N = 8;             // threads of a block (of a team of several warps: that team's), elements of a thread
constexpr int MAX_C = TAURUS_MAX_ROW_WIDTH;
constexpr int GRAD_BLOCKS = 2;                   // blocks of an SM that the gradient is spread over

struct Args {
  long long n;
  int C, team_shift;                             // a team is 1 << team_shift threads (up to a warp)
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
  int edge_rows;                                 // rows that reach less than 15 bytes from an end of a matrix of rows without gaps
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
  const int lo = last_offset_not_above(a.offsets, a.groups, r);
  const long long b = a.offsets[lo];
  if (b > r) { *at = {-1, 0, b < a.n ? b : a.n}; return; }             // in front of the first group, up to its rows
  if (lo == a.groups) { *at = {-1, b, a.n}; return; }                   // behind the last
  const long long e = a.offsets[lo + 1];
  *at = {lo, b, e > r ? e : r + 1};
}
__device__ __forceinline__ void check_offsets(const Args& a) {
  if (!a.offsets) return;
  for (long long g = (long long)blockIdx.x * blockDim.x + threadIdx.x; g < a.groups; g += (long long)gridDim.x * blockDim.x) {
    const long long b = a.offsets[g], e = a.offsets[g + 1];
    if (b < 0 || e > a.n || e < b) rows_status(a.status, TAURUS_ERR_INVALID_ARG);
  }
}

// Teams smaller than a warp, of a warp, of several warps.
enum { PART = 0, WARP = 1, MULTI = 2 };

// A thread's place in its team and the columns that it keeps: vectors lane, lane + size, ... of V elements.
template <int V, int KIND>
struct Team {
  static constexpr int NV = N / V;
  int size, lane, warps, id, threads;            // id: of the block's teams; threads: of the block
  int col[NV];
  bool on[NV];
  float2* slot;                                  // shared memory of teams of several warps: [2][warps]
  int flip = 0;
  __device__ __forceinline__ explicit Team(const Args& a) {
    __shared__ float2 slots[KIND == MULTI ? 2 * 4 : 1];
    size = KIND == MULTI ? blockDim.x : KIND == WARP ? 32 : 1 << a.team_shift;
    lane = KIND == MULTI ? threadIdx.x : threadIdx.x & (size - 1); id = KIND == MULTI ? 0 : KIND == WARP ? threadIdx.x >> 5 : threadIdx.x >> a.team_shift; warps = size >> 5;
    threads = KIND == MULTI ? size : THREADS;    // a team of several warps is a block
    slot = slots;
#pragma unroll
    for (int j = 0; j < NV; ++j) { col[j] = (j * size + lane) * V; on[j] = col[j] < a.C; }
  }
  __device__ __forceinline__ float2 sum(float x, float y) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      if (KIND != PART || d < size) { x += __shfl_xor_sync(0xffffffffu, x, d); y += __shfl_xor_sync(0xffffffffu, y, d); }
    return KIND == MULTI ? across(x, y) : make_float2(x, y);
  }
  __device__ __forceinline__ float sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      if (KIND != PART || d < size) x += __shfl_xor_sync(0xffffffffu, x, d);
    return KIND == MULTI ? across(x, 0.f).x : x;
  }
  // The two halves of the slots are used in turn: a warp that is through with one sum may write the next while others still read.
  __device__ __forceinline__ float2 across(float x, float y) {
    float2* const s = slot + flip * warps;
    flip ^= 1;
    if ((threadIdx.x & 31) == 0) s[lane >> 5] = make_float2(x, y);
    __syncthreads();
    float2 t = s[0];
    for (int w = 1; w < warps; ++w) { t.x += s[w].x; t.y += s[w].y; }
    return t;
  }
  // All threads of the team have come here.
  __device__ __forceinline__ void sync() const {
    if (KIND == MULTI) __syncthreads();
    else __syncwarp();
  }
  // A row of fp32 parameters, or `otherwise` where there is none; zeros behind the row.
  __device__ __forceinline__ void load_row(const float* row, float otherwise, float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = on[j] ? otherwise : 0.f;
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
  // The same for two rows; their means and factors.
  __device__ __forceinline__ void centre(const Args& a, float (&x)[2][N], float2* means, float2* factors) {
    float2 mean = make_float2(0.f, 0.f);
    if (a.layer) {
      float s = 0.f, t = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) { s += x[0][e]; t += x[1][e]; }
      const float2 both = sum(s, t);
      mean = make_float2(both.x * a.inv_C, both.y * a.inv_C);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const float m = on[j] ? mean.x : 0.f, n = on[j] ? mean.y : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) { x[0][j * V + i] -= m; x[1][j * V + i] -= n; }
      }
    }
    float q = 0.f, p = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) { q = fmaf(x[0][e], x[0][e], q); p = fmaf(x[1][e], x[1][e], p); }
    const float2 both = sum(q, p);
    *means = mean;
    *factors = make_float2(rsqrtf(fmaf(both.x, a.inv_C, a.eps)), rsqrtf(fmaf(both.y, a.inv_C, a.eps)));
  }
  // (1 / sqrt(var + eps)) of a row that is left without its mean (RMS: as it is); elements behind the row are 0 before and after.
  __device__ __forceinline__ float2 centre(const Args& a, float (&x)[N]) {
    float mean = 0.f;
    if (a.layer) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) s += x[e];
      mean = sum(s) * a.inv_C;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const float m = on[j] ? mean : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) x[j * V + i] -= m;
      }
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) q = fmaf(x[e], x[e], q);
    return make_float2(mean, rsqrtf(fmaf(sum(q), a.inv_C, a.eps)));
  }
};

template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const uint32_t s = (uint32_t)__cvta_generic_to_shared(to);
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(s), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void end_of_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_for_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// The rows of one array, AHEAD of them on their way into shared memory.  Vectors: a thread's pieces of a row, 16 bytes apart from its neighbours', for itself alone.
template <class T, int V, int AHEAD>
struct Source {
  static constexpr int NV = N / V, VB = V * (int)sizeof(T), PB = VB < 16 ? VB : 16, PIECES = VB / PB;
  static constexpr bool SHARED = false;          // with the team's other threads
  static __host__ __device__ int bytes(int, int, int threads) { return AHEAD * NV * VB * threads; }
  unsigned char* mine;
  int apart;                                     // bytes from a piece to the next
  __device__ __forceinline__ unsigned char* at(int place, int j, int piece) const { return mine + ((place * NV + j) * PIECES + piece) * apart; }
  template <class Place>
  __device__ __forceinline__ void open(unsigned char* smem, const Place& team, int) {
    mine = smem + threadIdx.x * PB;
    apart = team.threads * PB;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (!team.on[j])
        for (int p = 0; p < AHEAD; ++p)
#pragma unroll
          for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int w = 0; w < PB / 4; ++w) reinterpret_cast<uint32_t*>(at(p, j, k))[w] = 0;
  }
  template <class Place>
  __device__ __forceinline__ void fetch(const T* row, int place, const Place& team, int, bool) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (team.on[j])
#pragma unroll
        for (int k = 0; k < PIECES; ++k) copy_async<PB>(at(place, j, k), reinterpret_cast<const unsigned char*>(row + team.col[j]) + k * PB);
  }
  template <class Place>
  __device__ __forceinline__ void get(const T*, int place, const Place&, float (&x)[N]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const auto r = load_vec<Vec<T, PB / (int)sizeof(T)>>(at(place, j, k));
#pragma unroll
        for (int i = 0; i < PB / (int)sizeof(T); ++i) x[j * V + k * (PB / (int)sizeof(T)) + i] = to_f32<T>(r.v[i]);
      }
  }
};
// Rows that vectors do not fit: the team copies the 16-byte words that a row touches, wherever it begins, and its threads take elements from them.  What the first and the last of
// these words hold beside the row are other rows of the matrix; rows less than a word from its ends are brought by element.
template <class T, int AHEAD>
struct Source<T, 1, AHEAD> {
  static constexpr bool SHARED = true;
  static __host__ __device__ int window(int C) { return (C * (int)sizeof(T) + 15 + 15) / 16 * 16; }
  static __host__ __device__ int bytes(int C, int teams, int) { return AHEAD * window(C) * teams; }
  unsigned char* mine;
  int step;
  template <class Place>
  __device__ __forceinline__ void open(unsigned char* smem, const Place& team, int C) {
    step = window(C);
    mine = smem + team.id * AHEAD * step;
  }
  static __device__ __forceinline__ int shift(const T* row) { return (int)(reinterpret_cast<uintptr_t>(row) & 15); }
  template <class Place>
  __device__ __forceinline__ void fetch(const T* row, int place, const Place& team, int C, bool edge) {
    unsigned char* const to = mine + place * step;
    const int s = shift(row);
    if (edge) {
#pragma unroll
      for (int e = 0; e < N; ++e) if (team.on[e]) reinterpret_cast<T*>(to + s)[team.col[e]] = row[team.col[e]];
      return;
    }
    const unsigned char* const from = reinterpret_cast<const unsigned char*>(row) - s;
    const int words = (s + C * (int)sizeof(T) + 15) / 16;
    for (int w = team.lane; w < words; w += team.size) copy_async<16>(to + 16 * w, from + 16 * w);
  }
  template <class Place>
  __device__ __forceinline__ void get(const T* row, int place, const Place& team, float (&x)[N]) const {
    const T* const from = reinterpret_cast<const T*>(mine + place * step + shift(row));
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = team.on[e] ? to_f32<T>(from[team.col[e]]) : 0.f;
  }
};
template <int V> constexpr int ahead(int rows) { return V == 1 ? 2 : rows; }
// (Two ahead instead: 195 312 x 256 bf16 72.8 -> 73.9 us, fp32 141.9 -> 140.5, 1 024 605 -> 587; six 74.0, 144.1, 614; the gradient two ahead 130.9 -> 130.7, 224.7 -> 224.4, 761.6 -> 759.2.
// The first kernel, without rows ahead, took 1 190 for 1 200 000 x 256 bf16.)
constexpr int FORWARD_AHEAD = 4, GRAD_AHEAD = 3;
constexpr int forward_ahead(int V, int kind) { return V == 1 && kind != MULTI ? 2 : FORWARD_AHEAD; }

// Rows that the threads of a warp go through together: as many as the longest of its teams has (the exchanges take all threads).
template <int KIND>
__device__ __forceinline__ int rows_to_walk(long long begin, long long end) {
  const int mine = begin < end ? (int)(end - begin) : 0;
  return KIND == PART ? (int)__reduce_max_sync(0xffffffffu, (unsigned)mine) : mine;
}

template <class T, class R, int V, int KIND>
__global__ void __launch_bounds__(KIND == MULTI ? 128 : THREADS, KIND == MULTI ? 4 : V == 1 ? 2 : 3) resnorm_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) unsigned char resnorm_rows[];
  constexpr int AHEAD = forward_ahead(V, KIND);
  check_offsets(a);
  Team<V, KIND> team(a);
  // A block has neighbouring rows, which its teams take in turn.
  const int teams = KIND == MULTI ? 1 : KIND == WARP ? THREADS / 32 : THREADS >> a.team_shift;
  const long long block_begin = (long long)blockIdx.x * a.rows_a_team * teams, begin = block_begin + team.id;
  const long long left = (block_begin + a.rows_a_team * teams < a.n ? block_begin + a.rows_a_team * teams : a.n) - begin;
  const int rows = left > 0 ? (int)((left + teams - 1) / teams) : 0, walk = KIND == PART ? (int)__reduce_max_sync(0xffffffffu, (unsigned)rows) : rows;
  const long long step_res = teams * a.ld_res, step_block = teams * a.ld_block, step_out_res = teams * a.ld_out_res, step_out = teams * a.ld_out;
  Source<R, V, AHEAD> res;
  Source<T, V, AHEAD> block;
  res.open(resnorm_rows, team, a.C);
  block.open(resnorm_rows + res.bytes(a.C, teams, team.threads), team, a.C);
  const R* next_res = static_cast<const R*>(a.res) + begin * a.ld_res;
  const T* next_block = static_cast<const T*>(a.block) + begin * a.ld_block;
  R* out_res = static_cast<R*>(a.out_res) + begin * a.ld_out_res;
  T* out = static_cast<T*>(a.out) + begin * a.ld_out;
  int place = 0;
  const auto fetch = [&](int i) {
    if (i < rows) {
      const long long r = begin + (long long)i * teams;
      const bool edge = r < a.edge_rows || r >= a.n - a.edge_rows;
      res.fetch(next_res, place, team, a.C, edge);
      if (a.block) block.fetch(next_block, place, team, a.C, edge);
      next_res += step_res;
      next_block += step_block;
    }
    end_of_copies();
    place = place + 1 == AHEAD ? 0 : place + 1;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(i);
  float ga[N], be[N], gt[N];                     // gt: alpha gate post_gamma
  team.load_row(a.gamma, 1.f, ga);
  team.load_row(a.beta, 0.f, be);
  const auto gate = [&](int g) {
    float pg[N];
    team.load_row(a.post_gamma, 1.f, pg);
    team.load_row(g < 0 ? nullptr : a.gate + (long long)g * a.C, 1.f, gt);
#pragma unroll
    for (int e = 0; e < N; ++e) gt[e] = gt[e] * a.alpha * pg[e];
  };
  gate(-1);
  Group group = {-1, 0, 0};
  if constexpr (KIND == MULTI) {
    // Two rows of a group at a time: an exchange between the warps is for both.  (One at a time, 48 828 x 1 024 bf16 132 us, 102 by twos; fp32 158 / 149; 130 208 x 384 bf16 161 / 127; 97 656 x 512 fp32 146 / 154;
    // a mean and its squares of each warp in one exchange instead 144, 148, 189; six blocks on an SM, with registers spilled, 132, 187, 169.)
    for (int i = 0; i < rows;) {
      const long long row = begin + i;
      if (a.gate && (i == 0 || row >= group.end)) {
        find_group(a, row, &group);
        if (group.g >= 0) gate(group.g);
      }
      const bool two = i + 1 < rows && (!a.gate || row + 1 < group.end), write = !a.gate || group.g >= 0;
      wait_for_copies<AHEAD - 2>();
      if (res.SHARED) team.sync();
      const int place1 = place + 1 == AHEAD ? 0 : place + 1;
      float r[2][N], b[2][N];
      res.get(static_cast<const R*>(a.res) + row * a.ld_res, place, team, r[0]);
      if (two) res.get(static_cast<const R*>(a.res) + (row + 1) * a.ld_res, place1, team, r[1]);
      else {
#pragma unroll
        for (int e = 0; e < N; ++e) r[1][e] = b[1][e] = 0.f;
      }
      float2 scale = make_float2(1.f, 1.f), mean = make_float2(0.f, 0.f), s1 = mean, s2 = mean;
      if (a.block) {
        block.get(static_cast<const T*>(a.block) + row * a.ld_block, place, team, b[0]);
        if (two) block.get(static_cast<const T*>(a.block) + (row + 1) * a.ld_block, place1, team, b[1]);
        if (a.post) { team.centre(a, b, &mean, &scale); s1 = scale; }
#pragma unroll
        for (int e = 0; e < N; ++e) { r[0][e] = fmaf(gt[e], b[0][e] * scale.x, r[0][e]); r[1][e] = fmaf(gt[e], b[1][e] * scale.y, r[1][e]); }
      }
      if (write && a.out_res) {
        team.store(out_res, r[0]);
        if (two) team.store(out_res + step_out_res, r[1]);
      }
      float2 mean2;
      team.centre(a, r, &mean2, &s2);
      fetch(i + AHEAD);
      if (two) fetch(i + 1 + AHEAD);
#pragma unroll
      for (int e = 0; e < N; ++e) { r[0][e] = fmaf(r[0][e] * s2.x, ga[e], be[e]); r[1][e] = fmaf(r[1][e] * s2.y, ga[e], be[e]); }
      if (write) {
        team.store(out, r[0]);
        if (two) team.store(out + step_out, r[1]);
        if (a.stats && team.lane == 0) {
          a.stats[row] = make_float4(mean.x, s1.x, mean2.x, s2.x);
          if (two) a.stats[row + 1] = make_float4(mean.y, s1.y, mean2.y, s2.y);
        }
      }
      const int n = two ? 2 : 1;
      out_res += n * step_out_res;
      out += n * step_out;
      i += n;
    }
    return;
  }
  for (int i = 0; i < walk; ++i) {
    const long long row = begin + (long long)i * teams;
    const bool have = i < rows;
    if (a.gate && have && (i == 0 || row >= group.end)) {
      find_group(a, row, &group);
      if (group.g >= 0) gate(group.g);
    }
    wait_for_copies<AHEAD - 1>();
    if (res.SHARED) team.sync();
    float r[N], b[N];
    res.get(static_cast<const R*>(a.res) + row * a.ld_res, place, team, r);
    if (a.block) block.get(static_cast<const T*>(a.block) + row * a.ld_block, place, team, b);
    float2 s1 = make_float2(0.f, 0.f);
    if (a.block) {
      float scale = 1.f;
      if (a.post) {
        s1 = team.centre(a, b);
        scale = s1.y;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = fmaf(gt[e], b[e] * scale, r[e]);
    }
    const bool write = have && (!a.gate || group.g >= 0);
    if (write && a.out_res) team.store(out_res, r);
    const float2 s2 = team.centre(a, r);
    fetch(i + AHEAD);                            // into the place of this row, whose values have gone into the sums (of all of the team's threads)
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = fmaf(r[e] * s2.y, ga[e], be[e]);
    if (write) {
      team.store(out, r);
      if (a.stats && team.lane == 0) a.stats[row] = make_float4(s1.x, s1.y, s2.x, s2.y);
    }
    out_res += step_out_res;
    out += step_out;
  }
}

template <class T, class R, int V, int KIND>
__global__ void __launch_bounds__(KIND == MULTI ? 128 : THREADS, KIND == MULTI ? 2 * GRAD_BLOCKS : GRAD_BLOCKS) resnorm_grad_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) unsigned char resnorm_rows[];                // the rows on their way; at the end [teams of the block x C] sums
  constexpr int AHEAD = ahead<V>(GRAD_AHEAD);
  check_offsets(a);
  Team<V, KIND> team(a);
  const long long mine = KIND == MULTI ? blockIdx.x : KIND == WARP ? (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5) : ((long long)blockIdx.x * THREADS + threadIdx.x) >> a.team_shift;
  const long long begin = mine * a.rows_a_team, end = begin + a.rows_a_team < a.n ? begin + a.rows_a_team : a.n;
  const int rows = begin < end ? (int)(end - begin) : 0, walk = rows_to_walk<KIND>(begin, end);
  Source<R, V, AHEAD> res, dres;
  Source<T, V, AHEAD> block, dy;
  {
    const int teams = KIND == MULTI ? 1 : THREADS >> a.team_shift, rb = res.bytes(a.C, teams, team.threads), tb = block.bytes(a.C, teams, team.threads);
    res.open(resnorm_rows, team, a.C);
    dres.open(resnorm_rows + rb, team, a.C);
    block.open(resnorm_rows + 2 * rb, team, a.C);
    dy.open(resnorm_rows + 2 * rb + tb, team, a.C);
  }
  long long ahead_row = begin;
  int place = 0;
  const auto fetch = [&](int i) {
    if (i < rows) {
      const bool edge = ahead_row < a.edge_rows || ahead_row >= a.n - a.edge_rows;
      res.fetch(static_cast<const R*>(a.res) + ahead_row * a.ld_res, place, team, a.C, edge);
      if (a.block) block.fetch(static_cast<const T*>(a.block) + ahead_row * a.ld_block, place, team, a.C, edge);
      if (a.dres) dres.fetch(static_cast<const R*>(a.dres) + ahead_row * a.ld_dres, place, team, a.C, edge);
      if (a.dy) dy.fetch(static_cast<const T*>(a.dy) + ahead_row * a.ld_dy, place, team, a.C, edge);
    }
    ++ahead_row;
    end_of_copies();
    place = place + 1 == AHEAD ? 0 : place + 1;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(i);
  float4 next_stats = rows > 0 ? a.stats[begin] : make_float4(0.f, 0.f, 0.f, 0.f);
  float ga[N], gt[N];                            // gt: alpha gate post_gamma
  team.load_row(a.gamma, 1.f, ga);
  const auto gate = [&](int g) {
    float pg[N];
    team.load_row(a.post_gamma, 1.f, pg);
    team.load_row(g < 0 ? nullptr : a.gate + (long long)g * a.C, 1.f, gt);
#pragma unroll
    for (int e = 0; e < N; ++e) gt[e] = gt[e] * a.alpha * pg[e];
  };
  gate(-1);
  float sum_ga[N] = {}, sum_be[N] = {}, sum_pg[N] = {}, sum_h[N] = {};         // sum_h: of D h1 over the group's rows
  Group group = {-1, 0, 0};
  int2 goes_on = make_int2(-1, 0);
  // The sums of the group that ends in front of `row`.
  const auto close_group = [&](long long row) {
    if (a.gate && group.g < 0) return;
    float x[N];
    if (a.d_post) {
      team.load_row(a.gate ? a.gate + (long long)group.g * a.C : nullptr, 1.f, x);
#pragma unroll
      for (int e = 0; e < N; ++e) sum_pg[e] = fmaf(x[e] * a.alpha, sum_h[e], sum_pg[e]);
    }
    if (a.d_gate) {
      team.load_row(a.post_gamma, 1.f, x);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] *= a.alpha * sum_h[e];
      const bool before = group.begin < begin, after = row >= end && group.end > end;
      if (!before && !after) team.store_row(a.d_gate + (long long)group.g * a.C, x);
      else if (before) team.store_row(a.first + mine * a.C, x);
      else {
        team.store_row(a.last + mine * a.C, x);
        goes_on = make_int2(group.g, (int)((group.end < a.n ? group.end - 1 : a.n - 1) / a.rows_a_team - mine));
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sum_h[e] = 0.f;
  };
  for (int i = 0; i < walk; ++i) {
    const long long row = begin + i;
    const bool have = i < rows;
    if (a.gate && have && (i == 0 || row >= group.end)) {
      if (i > 0) close_group(row);
      find_group(a, row, &group);
      if (group.g >= 0) gate(group.g);
    }
    const bool live = have && (!a.gate || group.g >= 0);
    float4 st = next_stats;
    if (i + 1 < rows) next_stats = a.stats[row + 1];
    wait_for_copies<AHEAD - 1>();
    if (res.SHARED) team.sync();
    float x[N], u[N], d[N], g[N];
    res.get(static_cast<const R*>(a.res) + row * a.ld_res, place, team, x);
    if (a.block) block.get(static_cast<const T*>(a.block) + row * a.ld_block, place, team, u);
    if (a.dres) dres.get(static_cast<const R*>(a.dres) + row * a.ld_dres, place, team, d);
    if (a.dy) dy.get(static_cast<const T*>(a.dy) + row * a.ld_dy, place, team, g);
    if (res.SHARED) team.sync();                 // every thread has its elements: the place may be filled again
    if (KIND == PART ? !__all_sync(0xffffffffu, live) : !live) {     // whatever stands in a row that does not count, it adds to nothing
      if (!live) {
        st = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = u[e] = d[e] = g[e] = 0.f;
      }
    }
    if (!a.dres) {
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = 0.f;
    }
    if (a.block) {
      if (a.post) {
#pragma unroll
        for (int j = 0; j < N / V; ++j) {
          const float m = team.on[j] ? st.x : 0.f;
#pragma unroll
          for (int k = 0; k < V; ++k) u[j * V + k] = (u[j * V + k] - m) * st.y;        // h1
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = fmaf(gt[e], u[e], x[e]);
    }
    if (a.dy) {
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int j = 0; j < N / V; ++j) {
        const float m = team.on[j] ? st.z : 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int e = j * V + k;
          x[e] = (x[e] - m) * st.w;                                                    // h2
          sum_be[e] += g[e];
          sum_ga[e] = fmaf(g[e], x[e], sum_ga[e]);
          g[e] *= ga[e];
          s += g[e];
          q = fmaf(g[e], x[e], q);
        }
      }
      const float2 t = team.sum(s, q);
      const float m1 = a.layer ? t.x * a.inv_C : 0.f, m2 = t.y * a.inv_C;
#pragma unroll
      for (int j = 0; j < N / V; ++j) {
        const float m = team.on[j] ? m1 : 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) { const int e = j * V + k; d[e] = fmaf(st.w, fmaf(-x[e], m2, g[e] - m), d[e]); }
      }
    }
    if (live) team.store(static_cast<R*>(a.out_res) + row * a.ld_out_res, d);
    if (a.block) {
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        sum_h[e] = fmaf(d[e], u[e], sum_h[e]);
        d[e] *= gt[e];                                                                 // du post_gamma
        s += d[e];
        q = fmaf(d[e], u[e], q);
      }
      if (a.post) {
        const float2 t = team.sum(s, q);
        const float m1 = a.layer ? t.x * a.inv_C : 0.f, m2 = t.y * a.inv_C;
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = st.y * fmaf(-u[e], m2, d[e] - m1);
      }
      if (live && a.out) team.store(static_cast<T*>(a.out) + row * a.ld_out, d);
    }
    fetch(i + AHEAD);                            // into the place of this row, whose values have been used
  }
  if (rows > 0) close_group(end);
  if (a.span && team.lane == 0 && mine < a.teams) a.span[mine] = goes_on;
  if (a.chan) {
    wait_for_copies<0>();
    float* const sums = reinterpret_cast<float*>(resnorm_rows);
    const int teams = KIND == MULTI ? 1 : THREADS >> a.team_shift;
    float* const mine_row = sums + team.id * a.C;
    for (int which = 0; which < 3; ++which) {
      __syncthreads();
      if (which == 0) team.store_row(mine_row, sum_ga);
      else if (which == 1) team.store_row(mine_row, sum_be);
      else team.store_row(mine_row, sum_pg);
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += team.threads) {
        float s = 0.f;
        for (int t = 0; t < teams; ++t) s += sums[t * a.C + c];
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
#pragma unroll 8
      for (int b = ty; b < a.blocks; b += JOIN) s += a.chan[((long long)b * 3 + unit) * a.C + c];
    s = join_columns(s);
    if (tx == 0 && cw < a.C) out[cw] = s;
  }
  if (!a.d_gate) return;
  // Groups over several teams: up to SHORT parts by one warp, a column a thread; more by the block.
  constexpr int SHORT = 4 * JOIN;                                     // (32: gradient of 3 000 x 1 024 in 10 groups 31.0 -> 34.9 us, of 300 000 in 300 1 174 -> 1 300)
  __shared__ int longer[JOIN];
  for (long long t0 = unit0 * JOIN; t0 < a.teams; t0 += units * JOIN) {
    const long long t = t0 + ty;
    const int2 span = t < a.teams ? a.span[t] : make_int2(-1, 0);
    const bool more = span.x >= 0 && span.y > SHORT;
    if (tx == 0) longer[ty] = more;
    if (span.x >= 0 && !more && c < a.C) {
      float s = a.last[t * a.C + c];
      const float* const first = a.first + (t + 1) * a.C + c;
      const int parts = (int)(t + span.y < a.teams ? span.y : a.teams - 1 - t);
#pragma unroll 8
      for (int i = 0; i < parts; ++i) s += first[(long long)i * a.C];
      a.d_gate[(long long)span.x * a.C + c] = s;
    }
    if (!__syncthreads_or(more)) continue;
    for (int k = 0; k < JOIN; ++k) {
      if (!longer[k]) continue;
      const int2 of = a.span[t0 + k];
      float s = 0.f;
      if (c < a.C) {
        if (ty == 0) s = a.last[(t0 + k) * a.C + c];
        const long long to = t0 + k + of.y < a.teams ? t0 + k + of.y : a.teams - 1;
#pragma unroll 8
        for (long long i = t0 + k + 1 + ty; i <= to; i += JOIN) s += a.first[i * a.C + c];
      }
      s = join_columns(s);
      if (tx == 0 && cw < a.C) a.d_gate[(long long)of.x * a.C + cw] = s;
    }
    __syncthreads();
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
// Shared memory that a kernel may ask for: the same figure in every call, so that calls of several host threads do not take it from one another.  (The gradient's four arrays
// three rows ahead, 256 threads of 8 fp32 elements: 96 KB.)
constexpr int SHARED_MOST = 96 * 1024;
constexpr int MIN_ROWS = 2;                      // rows of a team at least (8: gradient of 300 x 256 fp32 11.8 -> 16.9 us, of 3 000 20.5 -> 18.9; 1: 10.3, 20.5, 300 x 1 024 14.4 -> 15.4)

// Threads and teams of a block.
inline int block_threads(int C) { return C > 32 * N ? (C + 32 * N - 1) / (32 * N) * 32 : THREADS; }
inline int64_t block_teams(int C) { return C > 32 * N ? 1 : THREADS >> team_shift_of(C); }
// Blocks of the gradient on an SM: of 256 threads, or as many threads in smaller ones.
inline int64_t grad_blocks(int C) { return (int64_t)GRAD_BLOCKS * (THREADS / block_threads(C)); }
struct Plan { int64_t rows_a_team, teams, blocks; };
Plan plan_of(int64_t n, int C, int64_t rows_a_team) {
  const int64_t a_block = block_teams(C), teams = (n + rows_a_team - 1) / rows_a_team;
  return {rows_a_team, teams, (teams + a_block - 1) / a_block};
}
// All rows over the blocks that are resident at once.
Plan forward_plan(int64_t n, int C, int64_t blocks) {
  const int64_t teams = block_teams(C) * blocks;
  return plan_of(n, C, std::max<int64_t>(1, (n + teams - 1) / teams));
}
// Gradient: all rows over the blocks that are resident at once, two rows a team at least.
Plan grad_plan(int64_t n, int C, int sms) {
  const int64_t teams = block_teams(C) * std::min(sms, SMS) * grad_blocks(C);
  return plan_of(n, C, std::max<int64_t>(MIN_ROWS, (n + teams - 1) / teams));
}
struct Space { size_t chan, first, last, span, bytes; };
Space space_of(int64_t n, int C, int groups) {
  Space s = {};
  if (n == 0) return s;
  // (what does for n rows does for fewer: the number of blocks and of teams is bounded by that of the largest plan)
  const int64_t a_block = block_teams(C);
  const int64_t blocks = std::min<int64_t>((int64_t)SMS * grad_blocks(C), (n + a_block - 1) / a_block), teams = std::min<int64_t>(blocks * a_block, n);
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

template <class F>
void with_kind(int team_shift, F f) {
  if (team_shift > 5) f(std::integral_constant<int, MULTI>());
  else if (team_shift == 5) f(std::integral_constant<int, WARP>());
  else f(std::integral_constant<int, PART>());
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
  a.inv_C = 1.f / (float)width; a.edge_rows = 1 + 15 / (width * std::min(ts, rs)); a.res = res; a.ld_res = ld_res; a.block = block; a.ld_block = ld_block; a.out_res = out_res; a.ld_out_res = ld_out_res; a.out = out; a.ld_out = ld_out;
  a.post_gamma = post_gamma; a.gate = gate; a.gamma = gamma; a.beta = beta; a.offsets = reinterpret_cast<const long long*>(offsets); a.stats = reinterpret_cast<float4*>(stats);
  a.status = status;
  const Rows rows[] = {{res, ld_res, rs}, {block, ld_block, ts}, {out_res, ld_out_res, rs}, {out, ld_out, ts}};
  const void* const params[] = {post_gamma, gate, gamma, beta};
  Launches enqueue = {static_cast<cudaStream_t>(cuda_stream)};
  with_rows(type, res_type, vector_of(width, ts == 2 ? 8 : 4, rows, params, 4), [&](auto tt, auto rt, auto vc) {
    using T = typename decltype(tt)::type;
    using R = typename decltype(rt)::type;
    constexpr int V = decltype(vc)::value;
    const auto go = [&](auto kind) {
      constexpr int KIND = decltype(kind)::value;
      const int teams = (int)block_teams(width), threads = block_threads(width);
      const size_t smem = (size_t)Source<R, V, forward_ahead(V, KIND)>::bytes(width, teams, threads) + (size_t)Source<T, V, forward_ahead(V, KIND)>::bytes(width, teams, threads);
      int resident = 0;
      cudaError_t e = smem > 40 * 1024 ? cudaFuncSetAttribute(resnorm_kernel<T, R, V, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED_MOST) : cudaSuccess;
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, resnorm_kernel<T, R, V, KIND>, threads, smem);
      if (e != cudaSuccess) { enqueue.error = e; return; }
      const Plan p = forward_plan(n, width, (int64_t)sms * std::max(resident, 1));
      a.rows_a_team = p.rows_a_team; a.teams = p.teams;
      enqueue(resnorm_kernel<T, R, V, KIND>, dim3((unsigned)p.blocks), threads, smem, a);
    };
    with_kind(a.team_shift, go);
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
  a.n = n; a.C = width; a.team_shift = team_shift_of(width); a.layer = kind == TAURUS_NORM_LAYER; a.post = post; a.groups = groups; a.alpha = alpha; a.inv_C = 1.f / (float)width; a.edge_rows = 1 + 15 / (width * std::min(ts, rs));
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
      const auto go = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        const int teams = (int)block_teams(width), threads = block_threads(width);
        const size_t rows_bytes = 2 * ((size_t)Source<R, V, ahead<V>(GRAD_AHEAD)>::bytes(width, teams, threads) + (size_t)Source<T, V, ahead<V>(GRAD_AHEAD)>::bytes(width, teams, threads));
        const size_t smem = std::max<size_t>(rows_bytes, (size_t)threads * N * 4);            // (a block's teams x columns are at most its threads x elements)
        const cudaError_t e = smem > 40 * 1024 ? cudaFuncSetAttribute(resnorm_grad_kernel<T, R, V, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED_MOST) : cudaSuccess;
        if (e != cudaSuccess) { enqueue.error = e; return; }
        enqueue(resnorm_grad_kernel<T, R, V, KIND>, dim3((unsigned)p.blocks), threads, smem, a);
      };
      with_kind(a.team_shift, go);
    });
  }
  if (joins) {
    const int column_blocks = (width + JOIN - 1) / JOIN;
    const int64_t units = std::max<int64_t>(3, std::min<int64_t>(grad_gate ? std::max<int64_t>(a.teams, groups) / JOIN + 1 : 3, 2 * SMS / column_blocks));
    if (n == 0) a.blocks = 0;
    enqueue.early = n > 0;
    enqueue(resnorm_join_kernel, dim3((unsigned)(units * column_blocks)), JOIN * JOIN, 0, a, column_blocks);
  }
  return enqueue.done("residual norm's gradient");
}
