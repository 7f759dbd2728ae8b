// Rows of a learned table: lookup by id with scaling, and the gradient of the table.
//
//   out[i]        = scale * table[ids[i]]                       (zeros for id -1)
//   grad_table[v] = scale * sum of grad_rows[i] over ids[i] = v, added in ascending i; zeros for a row that no id names
//
// Both are copies and sums: bytes bound them.  The lookup is one kernel, a vector of elements a thread.  The gradient sorts (id, position)
// pairs, so that the rows of one id stand together and are added in one order whatever the launch looks like: no atomics, the same bits
// every time.  The sorted positions are cut into pieces of equal length, a warp to a piece and to 32 vectors of columns; an id whose
// positions lie in one piece is written there, the others leave one partial row per piece, which a second kernel adds up.
#include <cub/cub.cuh>

#include <algorithm>

#include "rows.cuh"

namespace {

constexpr int LOOKUP_THREADS = 256, LOOKUP_UNROLL = 4;

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
        store_f32<O, V>(out + (row0 + r[u]) * ld_out + c[u], x[u]);
      }
    }
  }
}

// Largest vector (in elements) that base, pitch and width allow, of at most 16 bytes.
int vector_of(int limit, int size, const void* p, int64_t ld, int width) {
  int v = limit;
  while (v > 1 && (v * size > 16 || width % v != 0 || ld % v != 0 || !rows_aligned(p, v * size))) v >>= 1;
  return v;
}

// ---------------------------------------------------------------------------------------------------------------- gradient

__global__ void embed_keys_kernel(long long n, const long long* __restrict__ ids, long long table_rows, unsigned* __restrict__ key, int* __restrict__ pos,
                                  int32_t* status) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    const long long id = ids[i];
    const bool in = id >= 0 && id < table_rows;
    if (!in && id != -1) rows_status(status, TAURUS_ERR_INVALID_ARG);
    key[i] = in ? (unsigned)id : (unsigned)table_rows;      // without a row: behind all others
    pos[i] = (int)i;
  }
}

struct GradArgs {
  long long n, table_rows, ld_grad, ld_table;
  const unsigned* key;     // sorted
  const int* pos;
  float* head;             // [pieces x width] sum of the id that a piece begins in the middle of
  float* tail;             // [pieces x width] sum of the id that begins in a piece and goes on behind it
  int width, vpr, piece, pieces, slabs;
  int sum_blocks;          // the first blocks add; the others write zeros
  float scale;
};

constexpr int GRAD_THREADS = 256, GRAD_WARPS = GRAD_THREADS / 32, GRAD_UNROLL = 8;

// First sorted position whose key is at least k.
__device__ __forceinline__ long long lower_bound(const unsigned* key, long long n, unsigned k) {
  long long lo = 0, hi = n;
  while (lo < hi) { const long long m = (lo + hi) >> 1; if (key[m] < k) lo = m + 1; else hi = m; }
  return lo;
}

template <class G, class T, int V>
__global__ void __launch_bounds__(GRAD_THREADS)
embed_sum_kernel(const GradArgs a, const G* __restrict__ grad, T* __restrict__ table) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x >= a.sum_blocks) {
    // rows that no id names: a lane finds out for one row, the warp writes
    const long long warps = (long long)(gridDim.x - a.sum_blocks) * GRAD_WARPS;
    for (long long r0 = ((long long)(blockIdx.x - a.sum_blocks) * GRAD_WARPS + warp) * 32; r0 < a.table_rows; r0 += warps * 32) {
      const long long r = r0 + lane;
      bool empty = false;
      if (r < a.table_rows) {
        const long long p = lower_bound(a.key, a.n, (unsigned)r);
        empty = p >= a.n || a.key[p] != (unsigned)r;
      }
      unsigned todo = __ballot_sync(0xffffffffu, empty);
      float zero[V] = {};
      while (todo) {
        const int k = __ffs(todo) - 1;
        todo &= todo - 1;
        for (int c = lane; c < a.vpr; c += 32) store_f32<T, V>(table + (r0 + k) * a.ld_table + c * V, zero);
      }
    }
    return;
  }
  const long long unit = (long long)blockIdx.x * GRAD_WARPS + warp;
  const int p = (int)(unit / a.slabs), c = (int)(unit % a.slabs) * 32 + lane;
  if (p >= a.pieces) return;
  const long long b = (long long)p * a.piece, e = b + a.piece < a.n ? b + a.piece : a.n;
  const bool col = c < a.vpr;
  float acc[V] = {};
  unsigned cur = a.key[b];
  bool began_before = b > 0 && a.key[b - 1] == cur;
  auto flush = [&](bool goes_on) {
    if (col && cur != (unsigned)a.table_rows) {
      if (began_before) store_f32<float, V>(a.head + (size_t)p * a.width + c * V, acc);
      else if (goes_on) store_f32<float, V>(a.tail + (size_t)p * a.width + c * V, acc);
      else {
        float o[V];
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = acc[k] * a.scale;
        store_f32<T, V>(table + (long long)cur * a.ld_table + c * V, o);
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] = 0.f;
    began_before = false;
  };
  for (long long i = b; i < e; i += 32) {
    const int m = (int)(e - i < 32 ? e - i : 32);
    const unsigned my_key = lane < m ? a.key[i + lane] : 0u;
    const int my_pos = lane < m ? a.pos[i + lane] : 0;
    for (int j = 0; j < m; j += GRAD_UNROLL) {
      float x[GRAD_UNROLL][V];
#pragma unroll
      for (int u = 0; u < GRAD_UNROLL; ++u) {
        const long long row = __shfl_sync(0xffffffffu, my_pos, (j + u) & 31);
        const unsigned k = __shfl_sync(0xffffffffu, my_key, (j + u) & 31);
        if (j + u < m && col && k != (unsigned)a.table_rows) load_f32<G, V, LOAD_ONCE>(grad + row * a.ld_grad + c * V, x[u]);
      }
#pragma unroll
      for (int u = 0; u < GRAD_UNROLL; ++u) {
        const unsigned k = __shfl_sync(0xffffffffu, my_key, (j + u) & 31);
        if (j + u >= m) continue;
        if (k != cur) { flush(false); cur = k; }
        if (col && k != (unsigned)a.table_rows)
#pragma unroll
          for (int q = 0; q < V; ++q) acc[q] += x[u][q];
      }
    }
  }
  flush(e < a.n && a.key[e] == cur);
}

// The ids that go on behind their piece: a block to a piece and slab, its warps share the partial rows, added in their order.
template <class T, int V>
__global__ void __launch_bounds__(GRAD_THREADS)
embed_join_kernel(const GradArgs a, T* __restrict__ table) {
  const int p = (int)(blockIdx.x / a.slabs), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = (int)(blockIdx.x % a.slabs) * 32 + lane;
  const long long e = (long long)(p + 1) * a.piece;      // of a piece with another behind it
  const unsigned k = a.key[e - 1];
  if (k == (unsigned)a.table_rows || a.key[e] != k) return;                                    // nothing goes on
  const long long b = e - a.piece;
  if (a.key[b] == k && b > 0 && a.key[b - 1] == k) return;                                     // it began in an earlier piece
  const int last = (int)((lower_bound(a.key, a.n, k + 1u) - 1) / a.piece);                      // piece that it ends in
  const int rows = last - p, per = (rows + GRAD_WARPS - 1) / GRAD_WARPS;
  const int from = p + 1 + warp * per, to = from + per - 1 < last ? from + per - 1 : last;
  __shared__ float part[GRAD_WARPS][32 * V];
  float acc[V] = {};
  if (c < a.vpr) {
    if (warp == 0) load_f32<float, V>(a.tail + (size_t)p * a.width + c * V, acc);
    for (int q = from; q <= to; q += 4) {
      float x[4][V];
#pragma unroll
      for (int u = 0; u < 4; ++u) if (q + u <= to) load_f32<float, V>(a.head + (size_t)(q + u) * a.width + c * V, x[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (q + u <= to)
#pragma unroll
          for (int i = 0; i < V; ++i) acc[i] += x[u][i];
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) part[warp][lane * V + i] = acc[i];
  __syncthreads();
  if (warp == 0 && c < a.vpr) {
    for (int w = 1; w < GRAD_WARPS; ++w)
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += part[w][lane * V + i];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] *= a.scale;
    store_f32<T, V>(table + (long long)k * a.ld_table + c * V, acc);
  }
}

// Pieces: short ones fill the device where there are few positions, long ones keep the partial rows few.
int grad_piece(int64_t n) {
  int piece = 16;
  while (piece < 256 && n / piece > 148 * 32) piece *= 2;
  return piece;
}
int key_bits(int64_t table_rows) { int b = 1; while (b < 32 && (table_rows >> b) > 0) ++b; return b; }   // of the key table_rows too

struct GradSpace { size_t key_in, key, pos_in, pos, head, tail, sort, bytes, sort_bytes; };
int grad_space(int64_t n, int64_t table_rows, int32_t width, GradSpace* s) {
  size_t sort = 0;
  unsigned* const k = nullptr;
  int* const v = nullptr;
  const cudaError_t e = cub::DeviceRadixSort::SortPairs(nullptr, sort, k, k, v, v, (int)n, 0, key_bits(table_rows));
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "workspace of the sort"); return TAURUS_ERR_CUDA; }
  const size_t pieces = (size_t)((n + grad_piece(n) - 1) / grad_piece(n));
  size_t at = 0;
  auto take = [&](size_t b) { const size_t o = at; at += (b + 255) / 256 * 256; return o; };
  s->key_in = take((size_t)n * 4); s->key = take((size_t)n * 4); s->pos_in = take((size_t)n * 4); s->pos = take((size_t)n * 4);
  s->head = take(pieces * (size_t)width * 4); s->tail = take(pieces * (size_t)width * 4);
  s->sort = take(sort); s->sort_bytes = sort; s->bytes = at;
  return TAURUS_OK;
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
  if (!rows_on_device(ids, dev) || !rows_on_device(table, dev) || !rows_on_device(out_rows, dev) || (status && !rows_on_device(status, dev))) return TAURUS_ERR_INVALID_ARG;
  const size_t out_bytes = rows_bytes(n, ld_out, width, os);
  if (rows_overlap(out_rows, out_bytes, table, rows_bytes(table_rows, ld_table, width, ts)) || rows_overlap(out_rows, out_bytes, ids, (size_t)n * 8)) return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // vectors of 16 bytes on the wider side
  const int limit = ts == 2 && os == 2 ? 8 : 4;
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
        if constexpr (V == 8 && (sizeof(T) == 4 || sizeof(O) == 4)) return (int)TAURUS_ERR_INTERNAL;   // not chosen above
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

extern "C" int64_t taurus_embed_grad_workspace(int64_t n, int64_t table_rows, int32_t width) {
  if (!table_shape_ok(n, table_rows, width, width, width)) return TAURUS_ERR_INVALID_ARG;
  if (width > TAURUS_MAX_ROW_WIDTH) return TAURUS_ERR_UNSUPPORTED;
  GradSpace s;
  const int rc = grad_space(n, table_rows, width, &s);
  return rc ? rc : (int64_t)s.bytes;
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
  if (!rows_on_device(grad_table, dev) || (status && !rows_on_device(status, dev))) return TAURUS_ERR_INVALID_ARG;
  GradSpace s;
  if (const int rc = grad_space(n, table_rows, width, &s)) return rc;
  const size_t table_bytes = rows_bytes(table_rows, ld_table, width, ts);
  if (n > 0) {
    if (!rows_on_device(ids, dev) || !rows_on_device(grad_rows, dev) || !rows_on_device(workspace, dev)) return TAURUS_ERR_INVALID_ARG;
    if (workspace_bytes < (int64_t)s.bytes) return TAURUS_ERR_INVALID_ARG;
    const size_t grad_bytes = rows_bytes(n, ld_grad, width, gs), id_bytes = (size_t)n * 8;
    if (rows_overlap(grad_table, table_bytes, grad_rows, grad_bytes) || rows_overlap(grad_table, table_bytes, ids, id_bytes) ||
        rows_overlap(workspace, s.bytes, grad_table, table_bytes) || rows_overlap(workspace, s.bytes, grad_rows, grad_bytes) ||
        rows_overlap(workspace, s.bytes, ids, id_bytes))
      return TAURUS_ERR_INVALID_ARG;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  unsigned *key_in = reinterpret_cast<unsigned*>(ws + s.key_in), *key = reinterpret_cast<unsigned*>(ws + s.key);
  int *pos_in = reinterpret_cast<int*>(ws + s.pos_in), *pos = reinterpret_cast<int*>(ws + s.pos);
  const int limit = gs == 2 && ts == 2 ? 8 : 4;
  const int v = std::min(vector_of(limit, gs, grad_rows, ld_grad, width), vector_of(limit, ts, grad_table, ld_table, width));
  GradArgs a;
  a.n = n; a.table_rows = table_rows; a.ld_grad = ld_grad; a.ld_table = ld_table; a.key = key; a.pos = pos;
  a.head = reinterpret_cast<float*>(ws + s.head); a.tail = reinterpret_cast<float*>(ws + s.tail);
  a.width = width; a.vpr = width / v; a.slabs = (a.vpr + 31) / 32; a.scale = scale;
  a.piece = grad_piece(n); a.pieces = (int)((n + a.piece - 1) / a.piece);
  const long long sum_blocks = ((long long)a.pieces * a.slabs + GRAD_WARPS - 1) / GRAD_WARPS;
  const long long joins = (long long)(a.pieces - 1) * a.slabs;
  if (sum_blocks > (1 << 30) || joins > (1 << 30)) return TAURUS_ERR_UNSUPPORTED;
  a.sum_blocks = (int)sum_blocks;
  const int zero_blocks = (int)std::min<long long>((table_rows + GRAD_THREADS - 1) / GRAD_THREADS, (long long)sms * 8);
  if (n > 0) {
    embed_keys_kernel<<<(int)std::min<long long>((n + 255) / 256, (long long)sms * 8), 256, 0, st>>>(n, reinterpret_cast<const long long*>(ids), table_rows, key_in, pos_in, status);
    size_t tb = s.sort_bytes;
    const cudaError_t e = cub::DeviceRadixSort::SortPairs(ws + s.sort, tb, key_in, key, pos_in, pos, (int)n, 0, key_bits(table_rows), st);
    if (e != cudaSuccess) { taurus_note_cuda_error(e, "sort of the ids"); return TAURUS_ERR_CUDA; }
  }
  const int rc = with_row_type(grad_type, [&](auto gt) {
    return with_row_type(table_type, [&](auto tt) {
      using G = typename decltype(gt)::type;
      using T = typename decltype(tt)::type;
      auto go = [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V == 8 && (sizeof(T) == 4 || sizeof(G) == 4)) return (int)TAURUS_ERR_INTERNAL;   // not chosen above
        else {
          embed_sum_kernel<G, T, V><<<(int)sum_blocks + zero_blocks, GRAD_THREADS, 0, st>>>(a, static_cast<const G*>(grad_rows), static_cast<T*>(grad_table));
          if (joins > 0) embed_join_kernel<T, V><<<(int)joins, GRAD_THREADS, 0, st>>>(a, static_cast<T*>(grad_table));
          return (int)TAURUS_OK;
        }
      };
      return with_vector(v, go);
    });
  });
  if (rc) return rc;
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "embed_grad"); return TAURUS_ERR_CUDA; }
  return TAURUS_OK;
}
