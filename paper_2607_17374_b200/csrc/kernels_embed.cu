// Rows of a learned table: lookup by id with scaling, and the gradient of the table.
//
//   out[i]        = scale * table[ids[i]]                       (zeros for id -1)
//   grad_table[v] = scale * sum of grad_rows[i] over ids[i] = v, added in ascending i; zeros for a row that no id names
//
// Both are copies and sums: bytes bound them.  The lookup is one kernel, a vector of elements a thread.  The gradient sorts (id, position)
// pairs, so that the rows of one id stand together and are added in one order whatever the launch looks like: no float atomics, the same bits
// every time.  The sorted positions are cut into pieces of equal length, a warp to a piece; an id whose positions lie in one piece is written
// there, the others leave one partial row per piece, which a second kernel adds up.
// 65 536 x 100 fp32 looked up: 8.4 us (6.3 TB/s); gradient of 400 000 x 128 fp32 from 500 000 ids: 161 us, of which the sort of two digits takes 55 (six launches, each a
// few latencies long), sums and zeros 97 (4.7 TB/s).
#include <algorithm>

#include "rows.cuh"

namespace {

// Two vectors a thread in flight: with four the blocks' rows lie too far apart (1.2 M rows of 512 bf16 to fp32: 656 us, with eight 973; two 586, and
// 548 with 16 bytes of bf16 a vector).  Rows written are not read again here: they leave the L2 to the table.
constexpr int LOOKUP_THREADS = 256, LOOKUP_UNROLL = 2;

// A block takes `rows_per_block` rows of `vpr` vectors; q = i / vpr by a multiplication (i < 2^16, magic = 2^32 / vpr rounded up).
template <class T, class O, int V>
__global__ void __launch_bounds__(LOOKUP_THREADS)
embed_rows_kernel(long long n, const long long* __restrict__ ids, const T* __restrict__ table, long long table_rows, long long ld_table, int vpr,
                  unsigned magic, int rows_per_block, float scale, O* __restrict__ out, long long ld_out, int32_t* status) {
  for (long long row0 = (long long)blockIdx.x * rows_per_block; row0 < n; row0 += (long long)gridDim.x * rows_per_block) {
    const int rows = (int)(n - row0 < rows_per_block ? n - row0 : rows_per_block), items = rows * vpr;
    for (int i0 = threadIdx.x; i0 < items; i0 += LOOKUP_THREADS * LOOKUP_UNROLL) {
      float x[LOOKUP_UNROLL][V];
      int r[LOOKUP_UNROLL], c[LOOKUP_UNROLL];
#pragma unroll
      for (int u = 0; u < LOOKUP_UNROLL; ++u) {
        const int i = i0 + u * LOOKUP_THREADS;
        if (i >= items) break;
        r[u] = vpr == 1 ? i : (int)__umulhi((unsigned)i, magic);
        c[u] = (i - r[u] * vpr) * V;
        const long long id = ids[row0 + r[u]];
        if (id >= 0 && id < table_rows) {
          load_f32<T, V>(table + id * ld_table + c[u], x[u]);
#pragma unroll
          for (int k = 0; k < V; ++k) x[u][k] *= scale;
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k) x[u][k] = 0.f;
          if (id != -1) rows_status(status, TAURUS_ERR_INVALID_ARG);
        }
      }
#pragma unroll
      for (int u = 0; u < LOOKUP_UNROLL; ++u) {
        if (i0 + u * LOOKUP_THREADS >= items) break;
        store_f32_once<O, V>(out + (row0 + r[u]) * ld_out + c[u], x[u]);
      }
    }
  }
}

// Largest vector (in elements, at most `limit`) that base, pitch and width allow; it is read and written 16 bytes at a time.
int vector_of(int limit, int size, const void* p, int64_t ld, int width) {
  int v = limit;
  while (v > 1 && (width % v != 0 || ld % v != 0 || !rows_aligned(p, std::min(16, v * size)))) v >>= 1;
  return v;
}

// ---------------------------------------------------------------------------------------------------------------- sort
// Stable counting sort by digits of the ids, least significant first: per pass the digits of each block's items are counted (count), the counts of
// every digit summed over the blocks in front (scan), and the items moved (move).  Digits of up to 11 bits: a table of up to 2 048 rows takes one pass, of
// 4 M two.  Up to SMALL items one block does it all.
constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32, MAX_DIGIT = 11, MAX_BINS = 1 << MAX_DIGIT, TILE = 1024, MAX_ITEMS = 32 * TILE;
constexpr int SMALL = 2048, SMALL_THREADS = 1024;
constexpr int SORT_BLOCKS = 300;      // beyond which a block takes more items

struct SortPlan { int passes, bits, items, blocks; };   // bits of a digit; items of a block
SortPlan sort_plan(int64_t n, int64_t table_rows) {
  int key = 1;
  while (key < 32 && (table_rows >> key) > 0) ++key;      // of the key table_rows too
  SortPlan p;
  p.passes = (key + MAX_DIGIT - 1) / MAX_DIGIT;
  p.bits = (key + p.passes - 1) / p.passes;
  p.items = TILE;
  while (p.items < MAX_ITEMS && n / p.items > SORT_BLOCKS) p.items *= 2;      // two blocks to an SM
  p.blocks = (int)((n + p.items - 1) / p.items);
  return p;
}

struct SortArgs {
  long long n, table_rows;
  const long long* ids;        // first pass: the ids, else null
  const unsigned* key_in;
  const int* pos_in;
  unsigned* key_out;
  int* pos_out;
  unsigned* hist;              // [blocks x bins]
  int shift, bits, items, blocks;
  int* open_count;             // two words, cleared by the first pass
  int32_t* status;
};

// A missing id or one outside the table sorts behind all others.
__device__ __forceinline__ unsigned key_of(long long id, long long table_rows, int32_t* status) {
  if (id >= 0 && id < table_rows) return (unsigned)id;
  if (id != -1) rows_status(status, TAURUS_ERR_INVALID_ARG);
  return (unsigned)table_rows;
}
__device__ __forceinline__ unsigned sort_key(const SortArgs& a, long long i, int32_t* status) {
  return a.ids ? key_of(a.ids[i], a.table_rows, status) : a.key_in[i];
}

// Lanes of the warp with the same low `bits` bits: a vote a bit (a move of 500 000 items: 19.7 us, with match.any 21.8).
__device__ __forceinline__ unsigned peers(unsigned d, int bits) {
  unsigned same = 0xffffffffu;
  for (int b = 0; b < bits; ++b) {
    const unsigned ones = __ballot_sync(0xffffffffu, (d >> b) & 1u);
    same &= (d >> b) & 1u ? ones : ~ones;
  }
  return same;
}

__global__ void __launch_bounds__(SORT_THREADS) embed_count_kernel(const SortArgs a) {
  __shared__ unsigned h[MAX_BINS];
  const int bins = 1 << a.bits;
  if (a.ids && blockIdx.x == 0 && threadIdx.x < 2) a.open_count[threadIdx.x] = 0;
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) h[i] = 0;
  __syncthreads();
  const long long b = (long long)blockIdx.x * a.items, e = b + a.items < a.n ? b + a.items : a.n;
  for (long long i0 = b; i0 < e; i0 += 4 * SORT_THREADS) {
    unsigned d[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * SORT_THREADS + threadIdx.x;
      d[u] = i < e ? (sort_key(a, i, a.status) >> a.shift) & (bins - 1) : ~0u;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (d[u] != ~0u) atomicAdd(&h[d[u]], 1u);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) a.hist[((size_t)blockIdx.x << a.bits) + i] = h[i];
}

// hist[b][d] -> items of digit d in the blocks in front of b; the digit's total in totals[d].  A lane to a digit, the warps share the blocks.
constexpr int SCAN_WARPS = 32, SCAN_THREADS = 32 * SCAN_WARPS;
__global__ void __launch_bounds__(SCAN_THREADS) embed_scan_kernel(unsigned* hist, unsigned* totals, int bins, int blocks) {
  __shared__ unsigned part[SCAN_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
  const int per = (blocks + SCAN_WARPS - 1) / SCAN_WARPS, from = min(warp * per, blocks), to = min(from + per, blocks);
  unsigned sum = 0;
  if (d < bins)
#pragma unroll 8
    for (int b = from; b < to; ++b) sum += hist[(size_t)b * bins + d];
  part[warp][lane] = sum;
  __syncthreads();
  unsigned before = 0, all = 0;
  for (int w = 0; w < SCAN_WARPS; ++w) { const unsigned p = part[w][lane]; before += w < warp ? p : 0; all += p; }
  if (d >= bins) return;
  if (warp == 0) totals[d] = all;
  for (int b0 = from; b0 < to; b0 += 8) {
    unsigned v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = b0 + u < to ? hist[(size_t)(b0 + u) * bins + d] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (b0 + u < to) { hist[(size_t)(b0 + u) * bins + d] = before; before += v[u]; }
  }
}

// Exclusive sums of v[0 .. count) in place, count <= threads * 8; by a whole block of WARPS warps.
template <int WARPS>
__device__ __forceinline__ void scan_block(unsigned* v, int count, unsigned* warp_sums) {
  const int per = (count + WARPS * 32 - 1) / (WARPS * 32), at = threadIdx.x * per, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned s = 0;
  for (int i = at; i < at + per && i < count; ++i) s += v[i];
  unsigned x = s;
  for (int o = 1; o < 32; o <<= 1) { const unsigned y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  unsigned before = x - s;
  for (int w = 0; w < warp; ++w) before += warp_sums[w];
  for (int i = at; i < at + per && i < count; ++i) { const unsigned c = v[i]; v[i] = before; before += c; }
  __syncthreads();
}

// A warp takes a run of neighbouring items; where an item goes: its digit's base, the block's items of that digit in front of the warp's, and those
// that the warp has moved.
__global__ void __launch_bounds__(SORT_THREADS) embed_move_kernel(const SortArgs a, const unsigned* __restrict__ totals) {
  __shared__ unsigned base[MAX_BINS];
  __shared__ __align__(4) unsigned short mine[SORT_WARPS][MAX_BINS];
  __shared__ unsigned warp_sums[SORT_WARPS];
  const int bins = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) base[i] = totals[i];
  for (int i = threadIdx.x; i < SORT_WARPS * MAX_BINS / 2; i += SORT_THREADS) reinterpret_cast<unsigned*>(&mine[0][0])[i] = 0;
  __syncthreads();
  scan_block<SORT_WARPS>(base, bins, warp_sums);
  const int run = a.items / SORT_WARPS;
  const long long b = (long long)blockIdx.x * a.items + warp * run, e = b + run < a.n ? b + run : a.n;
  for (long long i0 = b; i0 < e; i0 += 128) {
    unsigned d[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) { const long long i = i0 + u * 32 + lane; d[u] = i < e ? (sort_key(a, i, nullptr) >> a.shift) & (bins - 1) : ~0u; }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const unsigned same = peers(d[u], a.bits + 1);
      if (d[u] != ~0u && lane == __ffs(same) - 1) mine[warp][d[u]] += (unsigned short)__popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += SORT_THREADS) {
    base[i] += a.hist[((size_t)blockIdx.x << a.bits) + i];
    unsigned short sum = 0;
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) { const unsigned short c = mine[w][i]; mine[w][i] = sum; sum += c; }
  }
  __syncthreads();
  for (long long i0 = b; i0 < e; i0 += 128) {
    unsigned k[4];
    int p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * 32 + lane;
      k[u] = i < e ? sort_key(a, i, nullptr) : 0;
      p[u] = i < e ? (a.ids ? (int)i : a.pos_in[i]) : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool in = i0 + u * 32 + lane < e;
      const unsigned d = in ? (k[u] >> a.shift) & (bins - 1) : ~0u, same = peers(d, a.bits + 1);
      unsigned to = 0;
      if (in) to = base[d] + mine[warp][d] + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (in && lane == __ffs(same) - 1) mine[warp][d] += (unsigned short)__popc(same);
      __syncwarp();
      if (in) { a.key_out[to] = k[u]; a.pos_out[to] = p[u]; }
    }
  }
}

// Up to SMALL items by one block: every pass in shared memory.
__global__ void __launch_bounds__(SMALL_THREADS) embed_sort_small_kernel(const SortArgs a, int passes) {
  constexpr int WARPS = SMALL_THREADS / 32, RUN = SMALL / WARPS, BITS = 8, BINS = 1 << BITS;     // (digits of 8 bits here: 32 warps count on their own)
  __shared__ unsigned key[SMALL];
  __shared__ unsigned short pos[SMALL], mine[WARPS][BINS];
  __shared__ unsigned base[BINS], warp_sums[WARPS];
  const int n = (int)a.n, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x < 2) a.open_count[threadIdx.x] = 0;
  unsigned k[RUN / 32];
  int p[RUN / 32];
#pragma unroll
  for (int u = 0; u < RUN / 32; ++u) {
    p[u] = warp * RUN + u * 32 + lane;
    k[u] = p[u] < n ? key_of(a.ids[p[u]], a.table_rows, a.status) : ~0u;      // what is missing sorts behind everything
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * BITS;
    for (int i = threadIdx.x; i < WARPS * BINS; i += SMALL_THREADS) (&mine[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < RUN / 32; ++u) {
      const unsigned d = (k[u] >> shift) & (BINS - 1), same = peers(d, BITS);
      if (lane == __ffs(same) - 1) mine[warp][d] += (unsigned short)__popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (threadIdx.x < BINS) {
      unsigned short sum = 0;
      for (int w = 0; w < WARPS; ++w) { const unsigned short c = mine[w][threadIdx.x]; mine[w][threadIdx.x] = sum; sum += c; }
      base[threadIdx.x] = sum;
    }
    __syncthreads();
    scan_block<WARPS>(base, BINS, warp_sums);
#pragma unroll
    for (int u = 0; u < RUN / 32; ++u) {
      const unsigned d = (k[u] >> shift) & (BINS - 1), same = peers(d, BITS);
      const unsigned to = base[d] + mine[warp][d] + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (lane == __ffs(same) - 1) mine[warp][d] += (unsigned short)__popc(same);
      __syncwarp();
      key[to] = k[u];
      pos[to] = (unsigned short)p[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < RUN / 32; ++u) { const int i = warp * RUN + u * 32 + lane; k[u] = key[i]; p[u] = pos[i]; }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < RUN / 32; ++u) {
    const int i = warp * RUN + u * 32 + lane;
    if (i < n) { a.key_out[i] = k[u]; a.pos_out[i] = p[u]; }
  }
}

// ---------------------------------------------------------------------------------------------------------------- sums
struct GradArgs {
  long long n, table_rows, ld_grad, ld_table;
  const unsigned* key;     // sorted
  const int* pos;
  float* head;             // [pieces x width] sum of the id that a piece begins in the middle of
  float* tail;             // [pieces x width] sum of the id that begins in a piece and goes on behind it
  int* open_count;         // pieces whose last id goes on: over up to LONG pieces, over more,
  int *open, *open_long;   // and which
  int width, vpr, piece, pieces, slabs;
  int sum_blocks;          // the first blocks add; the others write zeros
  float scale;
};

constexpr int GRAD_THREADS = 256, GRAD_WARPS = GRAD_THREADS / 32;
constexpr int JOIN_THREADS = 512, JOIN_WARPS = JOIN_THREADS / 32, LONG = 32;

// First sorted position whose key is at least k: by a thread, and by a warp (32 keys a step).
__device__ __forceinline__ long long lower_bound(const unsigned* key, long long n, unsigned k) {
  long long lo = 0, hi = n;
  while (lo < hi) { const long long m = (lo + hi) >> 1; if (key[m] < k) lo = m + 1; else hi = m; }
  return lo;
}
__device__ __forceinline__ long long lower_bound_warp(const unsigned* key, long long lo, long long hi, unsigned k) {
  const int lane = threadIdx.x & 31;
  while (lo < hi) {                        // the position lies in [lo, hi]
    const long long step = (hi - lo + 31) / 32, i = lo + step * lane;
    const int below = __popc(__ballot_sync(0xffffffffu, i < hi && key[i] < k));
    if (below == 0) break;
    const long long next = lo + step * below;
    lo += step * (below - 1) + 1;
    if (next < hi) hi = next;
    if (step == 1) break;
  }
  return lo;
}

// A warp to a piece and NC x 32 vectors of columns.  U rows are on their way at a time.
template <class G, class T, int V, int NC, int U>
__device__ __forceinline__ void sum_piece(const GradArgs& a, const G* __restrict__ grad, T* __restrict__ table, int p, int slab) {
  const int lane = threadIdx.x & 31, c0 = slab * 32 * NC + lane;
  const long long b = (long long)p * a.piece, e = b + a.piece < a.n ? b + a.piece : a.n;
  const unsigned none = (unsigned)a.table_rows;
  float acc[NC][V] = {};
  unsigned cur = a.key[b];
  const unsigned before = b > 0 ? a.key[b - 1] : none, behind = e < a.n ? a.key[e] : none;
  bool began_before = b > 0 && before == cur;
  auto flush = [&](bool goes_on) {
    if (cur != none) {
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = c0 + j * 32;
        if (c >= a.vpr) continue;
        if (began_before) store_f32<float, V>(a.head + (size_t)p * a.width + c * V, acc[j]);
        else if (goes_on) store_f32<float, V>(a.tail + (size_t)p * a.width + c * V, acc[j]);
        else {
          float o[V];
#pragma unroll
          for (int k = 0; k < V; ++k) o[k] = acc[j][k] * a.scale;
          store_f32<T, V>(table + (long long)cur * a.ld_table + c * V, o);
        }
      }
      if (goes_on && !began_before && slab == 0 && lane == 0) {        // (in any order: each is a row of its own)
        const long long far = (long long)(p + 1 + LONG) * a.piece;
        if (far < a.n && a.key[far] == cur) a.open_long[atomicAdd(a.open_count + 1, 1)] = p;
        else a.open[atomicAdd(a.open_count, 1)] = p;
      }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) acc[j][k] = 0.f;
    began_before = false;
  };
  for (long long i = b; i < e; i += 32) {
    const int m = (int)(e - i < 32 ? e - i : 32);
    const unsigned my_key = lane < m ? a.key[i + lane] : none;
    const int my_pos = lane < m ? a.pos[i + lane] : 0;
    for (int j = 0; j < m; j += U) {
      Vec<G, V> x[U][NC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long row = __shfl_sync(0xffffffffu, my_pos, j + u);
        const unsigned k = __shfl_sync(0xffffffffu, my_key, j + u);
        if (k != none)
#pragma unroll
          for (int q = 0; q < NC; ++q) { const int c = c0 + q * 32; if (c < a.vpr) x[u][q] = load_vec<Vec<G, V>, LOAD_ONCE>(grad + row * a.ld_grad + c * V); }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned k = __shfl_sync(0xffffffffu, my_key, j + u);
        if (j + u >= m) break;
        if (k != cur) { flush(false); cur = k; }
        if (k != none)
#pragma unroll
          for (int q = 0; q < NC; ++q)
            if (c0 + q * 32 < a.vpr)
#pragma unroll
              for (int l = 0; l < V; ++l) acc[q][l] += to_f32<G>(x[u][q].v[l]);
      }
    }
  }
  flush(e < a.n && behind == cur);
}

template <class G, class T, int V, int NC>
__global__ void __launch_bounds__(GRAD_THREADS)
embed_sum_kernel(const GradArgs a, const G* __restrict__ grad, T* __restrict__ table) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < a.sum_blocks) {
    const long long unit = (long long)blockIdx.x * GRAD_WARPS + warp;
    const int p = (int)(unit / a.slabs);
    if (p < a.pieces) sum_piece<G, T, V, NC, NC == 1 ? 8 : 4>(a, grad, table, p, (int)(unit % a.slabs));
    return;
  }
  // rows that no id names: a lane finds out for one row, the warp writes
  const long long r0 = ((long long)(blockIdx.x - a.sum_blocks) * GRAD_WARPS + warp) * 32, r = r0 + lane;
  if (r0 >= a.table_rows) return;
  const long long from = lower_bound_warp(a.key, 0, a.n, (unsigned)r0), to = lower_bound_warp(a.key, from, a.n, (unsigned)(r0 + 32 < a.table_rows ? r0 + 32 : a.table_rows));
  bool empty = r < a.table_rows;
  if (empty) {
    const long long p = from + lower_bound(a.key + from, to - from, (unsigned)r);
    empty = p >= to || a.key[p] != (unsigned)r;
  }
  unsigned todo = __ballot_sync(0xffffffffu, empty);
  float zero[V] = {};
  while (todo) {
    const int k = __ffs(todo) - 1;
    todo &= todo - 1;
    for (int c = lane; c < a.vpr; c += 32) store_f32<T, V>(table + (r0 + k) * a.ld_table + c * V, zero);
  }
}

// The ids that go on behind their piece, 32 vectors of columns at a time (blockIdx.y).  A long one is the work of a block, whose warps share the partial rows;
// the others of a warp each.  Partial rows are added in their order.
template <class T, int V>
__global__ void __launch_bounds__(JOIN_THREADS)
embed_join_kernel(const GradArgs a, T* __restrict__ table) {
  __shared__ float part[JOIN_WARPS][32 * V];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.y * 32 + lane;
  const int count = a.open_count[0], long_count = a.open_count[1];
  auto add_heads = [&](float (&acc)[V], int from, int to) {      // partial rows [from, to)
    for (int q = from; q < to; q += 8) {
      float x[8][V];
#pragma unroll
      for (int u = 0; u < 8; ++u) if (q + u < to) load_f32<float, V>(a.head + (size_t)(q + u) * a.width + c * V, x[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (q + u < to)
#pragma unroll
          for (int l = 0; l < V; ++l) acc[l] += x[u][l];
    }
  };
  auto finish = [&](float (&acc)[V], unsigned k) {
#pragma unroll
    for (int l = 0; l < V; ++l) acc[l] *= a.scale;
    store_f32<T, V>(table + (long long)k * a.ld_table + c * V, acc);
  };
  for (int i = blockIdx.x; i < long_count; i += gridDim.x) {
    const int p = a.open_long[i];
    const long long e = (long long)(p + 1) * a.piece;
    const unsigned k = a.key[e];
    const int end = (int)((lower_bound_warp(a.key, e, a.n, k + 1u) - 1) / a.piece) + 1;          // behind the piece that it ends in
    const int per = (end - p - 1 + JOIN_WARPS - 1) / JOIN_WARPS, from = min(p + 1 + warp * per, end);
    float acc[V] = {};
    if (c < a.vpr) {
      if (warp == 0) load_f32<float, V>(a.tail + (size_t)p * a.width + c * V, acc);
      add_heads(acc, from, min(from + per, end));
    }
#pragma unroll
    for (int l = 0; l < V; ++l) part[warp][lane * V + l] = acc[l];
    __syncthreads();
    if (warp == 0 && c < a.vpr) {
      for (int w = 1; w < JOIN_WARPS; ++w)
#pragma unroll
        for (int l = 0; l < V; ++l) acc[l] += part[w][lane * V + l];
      finish(acc, k);
    }
    __syncthreads();
  }
  for (int i = blockIdx.x * JOIN_WARPS + warp; i < count; i += gridDim.x * JOIN_WARPS) {
    const int p = a.open[i];
    const long long at = (long long)(p + 1 + lane) * a.piece;
    const unsigned mine = at < a.n ? a.key[at] : ~0u, k = __shfl_sync(0xffffffffu, mine, 0);
    const int rows = __ffs(~__ballot_sync(0xffffffffu, mine == k)) - 1;                          // pieces that begin in the middle of it (fewer than 32 or all)
    if (c >= a.vpr) continue;
    float acc[V];
    load_f32<float, V>(a.tail + (size_t)p * a.width + c * V, acc);
    add_heads(acc, p + 1, p + 1 + (rows < 0 ? LONG : rows));
    finish(acc, k);
  }
}

// Pieces: short ones give warps enough to fill the device a few times over, long ones keep the partial rows few.
constexpr int GRAD_PIECES = 148 * 64;      // at least, before they get longer
int grad_piece(int64_t n) {
  int piece = 32;
  while (piece < 256 && n / (2 * piece) >= GRAD_PIECES) piece *= 2;
  return piece;
}

struct GradSpace { size_t key[2], pos[2], hist, totals, open, open_long, head, tail, bytes; };
// most: what no call with as many ids, or fewer, exceeds (where pieces and sort blocks get longer there are fewer of them).
GradSpace grad_space(int64_t n, int64_t table_rows, int32_t width, bool most = false) {
  size_t pieces = (size_t)((n + grad_piece(n) - 1) / grad_piece(n));
  SortPlan p = sort_plan(n, table_rows);
  if (most) {
    pieces = std::max(pieces, (size_t)std::min<int64_t>((n + 31) / 32, 2 * GRAD_PIECES));
    p.blocks = std::max(p.blocks, (int)std::min<int64_t>((n + TILE - 1) / TILE, SORT_BLOCKS + 1));
  }
  GradSpace s;
  size_t at = 0;
  auto take = [&](size_t b) { const size_t o = at; at += (b + 255) / 256 * 256; return o; };
  for (int i = 0; i < 2; ++i) { s.key[i] = take((size_t)n * 4); s.pos[i] = take((size_t)n * 4); }
  s.hist = take(n > SMALL ? (size_t)p.blocks << (p.bits + 2) : 0); s.totals = take(MAX_BINS * 4);
  s.open = take((pieces + 2) * 4); s.open_long = take(pieces * 4);
  s.head = take(pieces * (size_t)width * 4); s.tail = take(pieces * (size_t)width * 4);
  s.bytes = n > 0 ? at : 0;
  return s;
}

bool table_shape_ok(int64_t n, int64_t table_rows, int32_t width, int64_t ld_rows, int64_t ld_table) {
  return n >= 0 && n < (1ll << 31) && table_rows >= 1 && table_rows < (1ll << 31) && width >= 1 && ld_rows >= width && ld_table >= width &&
         rows_fit(n, ld_rows, 4) && rows_fit(table_rows, ld_table, 4);
}

}  // namespace

extern "C" int taurus_embed_rows(int64_t n, const int64_t* ids, const void* table, int32_t table_type, int64_t table_rows, int32_t width,
                                 int64_t ld_table, float scale, void* out_rows, int32_t out_type, int64_t ld_out, int32_t* status, void* cuda_stream) {
  const int ts = row_type_size(table_type), os = row_type_size(out_type);
  if (!ts || !os || !table_shape_ok(n, table_rows, width, ld_out, ld_table)) return TAURUS_ERR_INVALID_ARG;
  if (width > TAURUS_MAX_ROW_WIDTH) return TAURUS_ERR_UNSUPPORTED;
  if (n == 0) return TAURUS_OK;
  int dev = 0, sms = 0;
  if (!ids || !table || !out_rows || !rows_aligned(ids, 8) || !rows_aligned(table, ts) || !rows_aligned(out_rows, os) || !rows_aligned(status, 4)) return TAURUS_ERR_INVALID_ARG;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const Region outs[] = {region_of_rows(out_rows, n, ld_out, width, os), region_of(status, 4)};
  const Region ins[] = {region_of_rows(table, table_rows, ld_table, width, ts), region_of(ids, (size_t)n * 8)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins)) return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // vectors of 16 bytes of the table; of a 16-bit table 32 bytes of fp32 output, as two of 16
  const int limit = ts == 2 ? 8 : 4;
  const int v = std::min(vector_of(limit, ts, table, ld_table, width), vector_of(limit, os, out_rows, ld_out, width));
  const int vpr = width / v;
  const int rows_per_block = std::max(1, LOOKUP_THREADS * LOOKUP_UNROLL / vpr);
  const unsigned magic = (unsigned)(((1ull << 32) + vpr - 1) / vpr);
  const long long blocks = (n + rows_per_block - 1) / rows_per_block;
  const int grid = (int)std::min<long long>(blocks, (long long)sms * 64);
  const int rc = with_row_type(table_type, [&](auto tt) {
    return with_row_type(out_type, [&](auto ot) {
      using T = typename decltype(tt)::type;
      using O = typename decltype(ot)::type;
      auto go = [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V == 8 && sizeof(T) == 4) return (int)TAURUS_ERR_INTERNAL;   // not chosen above
        else {
          embed_rows_kernel<T, O, V><<<grid, LOOKUP_THREADS, 0, st>>>(n, reinterpret_cast<const long long*>(ids), static_cast<const T*>(table), table_rows, ld_table,
                                                                      vpr, magic, rows_per_block, scale, static_cast<O*>(out_rows), ld_out, status);
          return (int)TAURUS_OK;
        }
      };
      return with_vector(v, go);
    });
  });
  if (rc) return rc;
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "embed_rows"); return TAURUS_ERR_CUDA; }
  return TAURUS_OK;
}

// Has the launch in front gone through?  A kernel behind one that has not would take what stands in the workspace for places of rows.
static bool launched() {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) taurus_note_cuda_error(e, "embed_grad");
  return e == cudaSuccess;
}

extern "C" int64_t taurus_embed_grad_workspace(int64_t n, int64_t table_rows, int32_t width) {
  if (!table_shape_ok(n, table_rows, width, width, width)) return TAURUS_ERR_INVALID_ARG;
  if (width > TAURUS_MAX_ROW_WIDTH) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)grad_space(n, table_rows, width, true).bytes;
}

extern "C" int taurus_embed_grad(int64_t n, const int64_t* ids, const void* grad_rows, int32_t grad_type, int64_t ld_grad, int32_t width, float scale,
                                 void* grad_table, int32_t table_type, int64_t table_rows, int64_t ld_table, void* workspace, int64_t workspace_bytes,
                                 int32_t* status, void* cuda_stream) {
  const int gs = row_type_size(grad_type), ts = row_type_size(table_type);
  if (!gs || !ts || !table_shape_ok(n, table_rows, width, ld_grad, ld_table)) return TAURUS_ERR_INVALID_ARG;
  if (width > TAURUS_MAX_ROW_WIDTH) return TAURUS_ERR_UNSUPPORTED;
  if (!grad_table || !rows_aligned(grad_table, ts) || !rows_aligned(status, 4)) return TAURUS_ERR_INVALID_ARG;
  if (n > 0 && (!ids || !grad_rows || !workspace || !rows_aligned(ids, 8) || !rows_aligned(grad_rows, gs) || !rows_aligned(workspace, 256))) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const GradSpace s = grad_space(n, table_rows, width);
  const Region outs[] = {region_of_rows(grad_table, table_rows, ld_table, width, ts), region_of(status, 4)};
  const Region ins[] = {region_of_rows(grad_rows, n, ld_grad, width, gs), region_of(ids, (size_t)n * 8)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) || !workspace_ok(workspace, workspace_bytes, (int64_t)s.bytes, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  const int limit = gs == 2 && ts == 2 ? 8 : 4;
  const int v = std::min(vector_of(limit, gs, grad_rows, ld_grad, width), vector_of(limit, ts, grad_table, ld_table, width));
  const SortPlan plan = sort_plan(n, table_rows);
  const bool small = n <= SMALL;
  const int last = small ? 0 : (plan.passes - 1) & 1;             // of the two pairs of arrays: the sorted one
  GradArgs a;
  a.n = n; a.table_rows = table_rows; a.ld_grad = ld_grad; a.ld_table = ld_table;
  a.key = reinterpret_cast<unsigned*>(ws + s.key[last]); a.pos = reinterpret_cast<int*>(ws + s.pos[last]);
  a.head = reinterpret_cast<float*>(ws + s.head); a.tail = reinterpret_cast<float*>(ws + s.tail);
  a.open_count = reinterpret_cast<int*>(ws + s.open); a.open = a.open_count + 2; a.open_long = reinterpret_cast<int*>(ws + s.open_long);
  a.width = width; a.vpr = width / v; a.scale = scale;
  a.piece = grad_piece(n); a.pieces = (int)((n + a.piece - 1) / a.piece);
  const int nc = v > 2 || a.vpr <= 32 ? 1 : a.vpr <= 64 ? 2 : 4;  // vectors of a row that a lane takes: several where they are short
  a.slabs = (a.vpr + 32 * nc - 1) / (32 * nc);
  const long long sum_blocks = ((long long)a.pieces * a.slabs + GRAD_WARPS - 1) / GRAD_WARPS;
  const long long zero_blocks = (table_rows + GRAD_THREADS - 1) / GRAD_THREADS;
  if (sum_blocks + zero_blocks > 0x7fffffff) return TAURUS_ERR_UNSUPPORTED;
  a.sum_blocks = (int)sum_blocks;
  if (n > 0) {
    SortArgs q = {};
    q.n = n; q.table_rows = table_rows; q.ids = reinterpret_cast<const long long*>(ids); q.status = status; q.open_count = a.open_count;
    q.hist = reinterpret_cast<unsigned*>(ws + s.hist); q.bits = plan.bits; q.items = plan.items; q.blocks = plan.blocks;
    unsigned* const totals = reinterpret_cast<unsigned*>(ws + s.totals);
    for (int pass = 0; pass < (small ? 1 : plan.passes); ++pass) {
      const int to = pass & 1;
      q.key_out = reinterpret_cast<unsigned*>(ws + s.key[to]); q.pos_out = reinterpret_cast<int*>(ws + s.pos[to]);
      if (small) {
        int key = 1;
        while (key < 32 && (table_rows >> key) > 0) ++key;
        // (what fills the block up is all ones and starts behind the items: it stays there)
        embed_sort_small_kernel<<<1, SMALL_THREADS, 0, st>>>(q, (key + 7) / 8);
        if (!launched()) return TAURUS_ERR_CUDA;
        break;
      }
      q.shift = pass * plan.bits;
      embed_count_kernel<<<plan.blocks, SORT_THREADS, 0, st>>>(q);
      if (!launched()) return TAURUS_ERR_CUDA;
      embed_scan_kernel<<<((1 << plan.bits) + 31) / 32, SCAN_THREADS, 0, st>>>(q.hist, totals, 1 << plan.bits, plan.blocks);
      if (!launched()) return TAURUS_ERR_CUDA;
      embed_move_kernel<<<plan.blocks, SORT_THREADS, 0, st>>>(q, totals);
      if (!launched()) return TAURUS_ERR_CUDA;
      q.ids = nullptr;
      q.key_in = q.key_out; q.pos_in = q.pos_out;
    }
  }
  const int rc = with_row_type(grad_type, [&](auto gt) {
    return with_row_type(table_type, [&](auto tt) {
      using G = typename decltype(gt)::type;
      using T = typename decltype(tt)::type;
      return with_vector(v, [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V == 8 && (sizeof(T) == 4 || sizeof(G) == 4)) return (int)TAURUS_ERR_INTERNAL;   // not chosen above
        else {
          const int grid = (int)(sum_blocks + zero_blocks);
          const G* const g = static_cast<const G*>(grad_rows);
          T* const t = static_cast<T*>(grad_table);
          if constexpr (V <= 2) {
            if (nc == 4) embed_sum_kernel<G, T, V, 4><<<grid, GRAD_THREADS, 0, st>>>(a, g, t);
            if (nc == 2) embed_sum_kernel<G, T, V, 2><<<grid, GRAD_THREADS, 0, st>>>(a, g, t);
          }
          if (nc == 1) embed_sum_kernel<G, T, V, 1><<<grid, GRAD_THREADS, 0, st>>>(a, g, t);
          if (!launched()) return (int)TAURUS_ERR_CUDA;
          if (a.pieces > 1) embed_join_kernel<T, V><<<dim3((unsigned)std::min((a.pieces - 1 + JOIN_WARPS - 1) / JOIN_WARPS, sms * 4), (unsigned)((a.vpr + 31) / 32)), JOIN_THREADS, 0, st>>>(a, t);
          return (int)TAURUS_OK;
        }
      });
    });
  });
  if (rc) return rc;
  return launched() ? TAURUS_OK : TAURUS_ERR_CUDA;
}
