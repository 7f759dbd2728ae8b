// Projection by vertex type: rows grouped by type, a weight matrix to each type, and the gradients.
//
//   out[r] = x[r] W[g] + bias[g],  grad_x[r] = grad_out[r] W[g]^T,  grad_W[g] = sum_r x[r]^T grad_out[r],  grad_bias[g] = sum_r grad_out[r]
//
// over the rows r in [offsets[g], offsets[g + 1]), offsets in device memory.  This file: arguments, and the kernels for few rows, which read
// every weight once per row and add in fp32 FMAs (bytes and latency bound them; measured at FEW_ROWS); kernels_typed_tc.cu: the others.
#include <algorithm>

#include "typed.cuh"

namespace {

// Rows up to which the kernels for few rows are taken, whatever the widths.  Both sides at 64 rows of one type, us (these kernels / the tensor cores):
//                   64 -> 64       256 -> 256     1 024 -> 1 024
//   fp32  forward   2.9 / 7.7      4.2 / 16.9     23 / 44
//         grad_x    2.7 / 7.6      3.9 / 15.7     21 / 40
//         grad_W    7.9 / 7.4      8.3 / 8.9      17 / 9.2
//   bf16  forward   3.0 / 4.3      4.3 / 6.7      18 / 11
//         grad_x    2.8 / 4.2      3.4 / 6.3      17 / 9.7
//         grad_W    18 / 5.1       19 / 6.8       31 / 6.9
// They win at 8 to 32 rows too, but for 16-bit rows of 1 024 columns and for grad_W of types of more than some 16 rows (16 bits) or 32 (fp32), which a thread
// walks one after another.
constexpr int FEW_ROWS = 64;
constexpr int FEW_THREADS = 256, COL_VECTORS = 8, K_LANES = FEW_THREADS / COL_VECTORS;

// The type of row r (-1: none), by a warp: the offsets not above r are counted.
__device__ __forceinline__ int type_of(const long long* offsets, int types, long long r) {
  int k = 0;
  for (int i = threadIdx.x & 31; i <= types; i += 32) k += offsets[i] <= r;
  k = __reduce_add_sync(0xffffffffu, k) - 1;
  return k < types ? k : -1;
}
// By one block of a launch: are the offsets what they have to be?
__device__ __forceinline__ void check_offsets(const long long* offsets, int types, long long n, int32_t* status) {
  for (int g = threadIdx.x; g < types; g += blockDim.x) { long long b, e; group_rows(offsets, g, n, &b, &e, status); }
}

// A block to a row and 8 vectors of columns; 32 lanes share the sum over d_in.
template <class T, class O, int V>
__global__ void __launch_bounds__(FEW_THREADS)
typed_few_kernel(long long n, int types, const long long* __restrict__ offsets, const T* __restrict__ x, long long ld_x, const T* __restrict__ W,
                 const float* __restrict__ bias, int K, int N, int tiles, O* __restrict__ out, long long ld_out, int32_t* status) {
  __shared__ float part[K_LANES][COL_VECTORS * V];
  const int cv = threadIdx.x % COL_VECTORS, kl = threadIdx.x / COL_VECTORS;
  if (blockIdx.x == 0) check_offsets(offsets, types, n, status);
  for (long long unit = blockIdx.x; unit < n * tiles; unit += gridDim.x) {
    const long long r = unit / tiles;
    const int c = ((int)(unit % tiles) * COL_VECTORS + cv) * V, g = type_of(offsets, types, r);
    if (g < 0) continue;
    float acc[V] = {};
    if (c < N) {
      const T* const w = W + (long long)g * K * N + c;
#pragma unroll 8
      for (int k = kl; k < K; k += K_LANES) {
        const float a = to_f32<T>(x[r * ld_x + k]);
        float b[V];
        load_f32<T, V>(w + (long long)k * N, b);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += a * b[j];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) part[kl][cv * V + j] = acc[j];
    __syncthreads();
    for (int j = threadIdx.x; j < COL_VECTORS * V; j += FEW_THREADS) {
      const int col = (int)(unit % tiles) * COL_VECTORS * V + j;
      if (col >= N) continue;
      float s = 0.f;
#pragma unroll 8
      for (int l = 0; l < K_LANES; ++l) s += part[l][j];
      out[r * ld_out + col] = from_f32<O>(s + (bias ? bias[(long long)g * N + col] : 0.f));
    }
    __syncthreads();
  }
}

// A block to a row and 32 columns of grad_x, a warp to four of them: sums along the rows of W.
template <class T, int V>
__global__ void __launch_bounds__(FEW_THREADS)
typed_few_dx_kernel(long long n, int types, const long long* __restrict__ offsets, const T* __restrict__ dy, long long ld_dy, const T* __restrict__ W,
                    int K, int N, int tiles, T* __restrict__ dx, long long ld_dx, int32_t* status) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x == 0) check_offsets(offsets, types, n, status);
  for (long long unit = blockIdx.x; unit < n * tiles; unit += gridDim.x) {
    const long long r = unit / tiles;
    const int k0 = (int)(unit % tiles) * 32 + warp * 4, g = type_of(offsets, types, r);
    if (g < 0) continue;
    float acc[4] = {};
    for (int c = lane * V; c < N; c += 32 * V) {
      float a[V];
      load_f32<T, V>(dy + r * ld_dy + c, a);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (k0 + q >= K) break;
        float b[V];
        load_f32<T, V>(W + ((long long)g * K + k0 + q) * N + c, b);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[q] += a[j] * b[j];
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      for (int o = 16; o > 0; o >>= 1) acc[q] += __shfl_xor_sync(0xffffffffu, acc[q], o);
      if (lane == 0 && k0 + q < K) dx[r * ld_dx + k0 + q] = from_f32<T>(acc[q]);
    }
  }
}

// A thread to V neighbouring elements of a row of grad_W (row K of it stands for the bias), which walks the rows of its type.
template <class T, class O, int V>
__global__ void __launch_bounds__(FEW_THREADS)
typed_few_dw_kernel(long long n, int types, const long long* __restrict__ offsets, const T* __restrict__ x, long long ld_x, const T* __restrict__ dy,
                    long long ld_dy, int K, int N, O* __restrict__ dW, float* __restrict__ db, int32_t* status) {
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(offsets, types, n, status);
  const int vpr = N / V, vectors = (K + 1) * vpr;
  for (int g = blockIdx.y; g < types; g += gridDim.y) {
    long long b, e;
    group_rows(offsets, g, n, &b, &e, nullptr);
    for (int i = blockIdx.x * FEW_THREADS + threadIdx.x; i < vectors; i += gridDim.x * FEW_THREADS) {
      const int k = i / vpr, c = (i - k * vpr) * V;
      if (k == K ? !db : !dW) continue;
      float acc[V] = {};
#pragma unroll 4
      for (long long r = b; r < e; ++r) {
        const float a = k == K ? 1.f : to_f32<T>(x[r * ld_x + k]);
        float d[V];
        load_f32<T, V>(dy + r * ld_dy + c, d);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += a * d[j];
      }
      if (k == K)
#pragma unroll
        for (int j = 0; j < V; ++j) db[(long long)g * N + c + j] = acc[j];
      else store_f32<O, V>(dW + ((long long)g * K + k) * N + c, acc);
    }
  }
}

bool typed_shape_ok(int64_t n, int32_t types, int32_t d_in, int32_t d_out, int32_t type) {
  return n >= 0 && n < (1ll << 31) && types >= 1 && d_in >= 1 && d_out >= 1 && row_type_size(type) != 0;
}
bool typed_supported(int32_t types, int32_t d_in, int32_t d_out) { return types <= TAURUS_MAX_TYPES && d_in <= TAURUS_MAX_ROW_WIDTH && d_out <= TAURUS_MAX_ROW_WIDTH; }

int vector_of(int size, const void* p, int64_t ld) {
  int v = 16 / size;
  while (v > 1 && (ld % v != 0 || !rows_aligned(p, v * size))) v >>= 1;
  return v;
}

// A call's workspace: W laid out anew (where it is: packs), partial results of grad_W, rows of grad_out and of x at other pitches.  The workspace functions
// answer for weights at any address and for as many rows or fewer (most), a call asks for what it uses.
struct Space {
  size_t part = 0, dy = 0, x = 0, bytes = 0;
  Space(int64_t n, int32_t types, int32_t d_in, int32_t d_out, int32_t type, bool packs, bool grad, bool most = false) {
    if (n <= FEW_ROWS) return;
    auto take = [&](size_t b) { const size_t o = bytes; bytes += (b + 255) / 256 * 256; return o; };
    if (packs) take(typed_tc_pack_bytes(types, d_in, d_out, type));
    if (grad) { part = take(typed_tc_part_bytes(n, types, d_in, d_out, type, most)); dy = take(typed_tc_row_bytes(n, d_out, type)); }
    x = take(typed_tc_row_bytes(n, d_in, type));
  }
  TypedSpaces at(void* workspace) const {
    char* const p = static_cast<char*>(workspace);
    return {p, p + part, p + dy, p + x};
  }
};

}  // namespace

extern "C" int64_t taurus_typed_project_workspace(int64_t n, int32_t types, int32_t d_in, int32_t d_out, int32_t type) {
  if (!typed_shape_ok(n, types, d_in, d_out, type)) return TAURUS_ERR_INVALID_ARG;
  if (!typed_supported(types, d_in, d_out)) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)Space(n, types, d_in, d_out, type, true, false, true).bytes;
}
extern "C" int64_t taurus_typed_project_grad_workspace(int64_t n, int32_t types, int32_t d_in, int32_t d_out, int32_t type) {
  if (!typed_shape_ok(n, types, d_in, d_out, type)) return TAURUS_ERR_INVALID_ARG;
  if (!typed_supported(types, d_in, d_out)) return TAURUS_ERR_UNSUPPORTED;
  return (int64_t)Space(n, types, d_in, d_out, type, true, true, true).bytes;
}

extern "C" int taurus_typed_project(int64_t n, int32_t types, const int64_t* offsets, const void* x, int64_t ld_x, int32_t type, const void* W,
                                    const float* bias, int32_t d_in, int32_t d_out, void* out, int32_t out_type, int64_t ld_out, void* workspace,
                                    int64_t workspace_bytes, int32_t* status, void* cuda_stream) {
  const int ts = row_type_size(type), os = row_type_size(out_type);
  if (!typed_shape_ok(n, types, d_in, d_out, type) || (out_type != type && out_type != TAURUS_F32) || ld_x < d_in || ld_out < d_out || !rows_fit(n, ld_x, ts) ||
      !rows_fit(n, ld_out, os))
    return TAURUS_ERR_INVALID_ARG;
  if (!typed_supported(types, d_in, d_out)) return TAURUS_ERR_UNSUPPORTED;
  if (n == 0) return TAURUS_OK;
  if (!offsets || !x || !W || !out || !rows_aligned(offsets, 8) || !rows_aligned(x, ts) || !rows_aligned(W, ts) || !rows_aligned(bias, 4) || !rows_aligned(out, os) ||
      !rows_aligned(status, 4))
    return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const Region outs[] = {region_of_rows(out, n, ld_out, d_out, os), region_of(status, 4)};
  const Region ins[] = {region_of(offsets, (size_t)(types + 1) * 8), region_of_rows(x, n, ld_x, d_in, ts), region_of(W, (size_t)types * d_in * d_out * ts),
                        region_of(bias, (size_t)types * d_out * 4)};
  const bool packs = typed_tc_packs(W, type, d_out);
  const Space space(n, types, d_in, d_out, type, packs, false);
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) ||
      !workspace_ok(workspace, workspace_bytes, (int64_t)space.bytes, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const long long* const off = reinterpret_cast<const long long*>(offsets);
  int rc = TAURUS_OK;
  if (n > FEW_ROWS) {
    rc = typed_tc_project(n, types, off, x, ld_x, type, W, bias, d_in, d_out, out, out_type, ld_out, space.at(workspace), status, sms, st);
  } else with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    return with_vector(vector_of(ts, W, d_out), [&](auto vc) {
      constexpr int V = decltype(vc)::value;
      if constexpr (V * sizeof(T) <= 16) {
        const int tiles = (d_out + COL_VECTORS * V - 1) / (COL_VECTORS * V);
        const int grid = (int)std::min<long long>(n * tiles, (long long)sms * 64);
        const T *const xp = static_cast<const T*>(x), *const wp = static_cast<const T*>(W);
        if (out_type == type)
          typed_few_kernel<T, T, V><<<grid, FEW_THREADS, 0, st>>>(n, types, off, xp, ld_x, wp, bias, d_in, d_out, tiles, static_cast<T*>(out), ld_out, status);
        else
          typed_few_kernel<T, float, V><<<grid, FEW_THREADS, 0, st>>>(n, types, off, xp, ld_x, wp, bias, d_in, d_out, tiles, static_cast<float*>(out), ld_out, status);
      }
      return 0;
    });
  });
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "typed_project"); return TAURUS_ERR_CUDA; }
  return rc;
}

extern "C" int taurus_typed_project_grad(int64_t n, int32_t types, const int64_t* offsets, const void* x, int64_t ld_x, int32_t type, const void* W,
                                         const void* grad_out, int64_t ld_grad, int32_t d_in, int32_t d_out, void* grad_x, int64_t ld_grad_x, void* grad_W,
                                         int32_t grad_W_type, float* grad_bias, void* workspace, int64_t workspace_bytes, int32_t* status,
                                         void* cuda_stream) {
  if (!grad_W) grad_W_type = type;
  const int ts = row_type_size(type), ws = row_type_size(grad_W_type);
  if (!typed_shape_ok(n, types, d_in, d_out, type) || (grad_W && grad_W_type != type && grad_W_type != TAURUS_F32) || (x && ld_x < d_in) || ld_grad < d_out || (grad_x && ld_grad_x < d_in) ||
      (x && !rows_fit(n, ld_x, ts)) || !rows_fit(n, ld_grad, ts) || (grad_x && !rows_fit(n, ld_grad_x, ts)))
    return TAURUS_ERR_INVALID_ARG;
  if (!typed_supported(types, d_in, d_out)) return TAURUS_ERR_UNSUPPORTED;
  if (!grad_x && !grad_W && !grad_bias) return TAURUS_OK;
  if (!offsets || !rows_aligned(offsets, 8) || !rows_aligned(x, ts) || !rows_aligned(W, ts) || !rows_aligned(grad_out, ts) || !rows_aligned(grad_x, ts) ||
      !rows_aligned(grad_W, ws) || !rows_aligned(grad_bias, 4) || !rows_aligned(status, 4))
    return TAURUS_ERR_INVALID_ARG;
  if (n > 0 && (!grad_out || (grad_x && !W) || (grad_W && !x))) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  const size_t w_count = (size_t)types * d_in * d_out;
  const Region outs[] = {region_of_rows(grad_x, n, ld_grad_x, d_in, ts), region_of(grad_W, w_count * ws), region_of(grad_bias, (size_t)types * d_out * 4), region_of(status, 4)};
  const Region ins[] = {region_of(offsets, (size_t)(types + 1) * 8), region_of_rows(x, n, ld_x, d_in, ts), region_of(W, w_count * ts), region_of_rows(grad_out, n, ld_grad, d_out, ts)};
  const bool packs = grad_x && typed_tc_packs(W, type, d_out);
  const Space space(n, types, d_in, d_out, type, packs, true);
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins) ||
      !workspace_ok(workspace, workspace_bytes, (int64_t)space.bytes, dev, outs, ins))
    return TAURUS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const long long* const off = reinterpret_cast<const long long*>(offsets);
  int rc = TAURUS_OK;
  if (n > FEW_ROWS) {
    rc = typed_tc_project_grad(n, types, off, x, ld_x, type, W, grad_out, ld_grad, d_in, d_out, grad_x, ld_grad_x, grad_W, grad_W_type, grad_bias, space.at(workspace), status, sms, st);
  } else with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    const T *const xp = static_cast<const T*>(x), *const wp = static_cast<const T*>(W), *const dyp = static_cast<const T*>(grad_out);
    if (grad_x && n > 0)
      with_vector(std::min(vector_of(ts, W, d_out), vector_of(ts, grad_out, ld_grad)), [&](auto vc) {
        constexpr int V = decltype(vc)::value;
        if constexpr (V * sizeof(T) <= 16) {
          const int tiles = (d_in + 31) / 32;
          const int grid = (int)std::min<long long>(n * tiles, (long long)sms * 64);
          typed_few_dx_kernel<T, V><<<grid, FEW_THREADS, 0, st>>>(n, types, off, dyp, ld_grad, wp, d_in, d_out, tiles, static_cast<T*>(grad_x), ld_grad_x, status);
        }
        return 0;
      });
    if (grad_W || grad_bias) {
      const bool four = vector_of(ts, grad_out, ld_grad) >= 4 && d_out % 4 == 0 && rows_aligned(grad_W, 16);
      auto go = [&](auto vc, auto* dw) {
        constexpr int V = decltype(vc)::value;
        using O = std::remove_pointer_t<decltype(dw)>;
        const dim3 grid((unsigned)std::min((((d_in + 1) * (d_out / V)) + FEW_THREADS - 1) / FEW_THREADS, 1024), (unsigned)types);
        typed_few_dw_kernel<T, O, V><<<grid, FEW_THREADS, 0, st>>>(n, types, off, xp, ld_x, dyp, ld_grad, d_in, d_out, dw, grad_bias, status);
      };
      auto with_output = [&](auto vc) {
        if (grad_W_type == type) go(vc, static_cast<T*>(grad_W));
        else go(vc, static_cast<float*>(grad_W));
      };
      if (four) with_output(std::integral_constant<int, 4>());
      else with_output(std::integral_constant<int, 1>());
    }
    return 0;
  });
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "typed_project_grad"); return TAURUS_ERR_CUDA; }
  return rc;
}
