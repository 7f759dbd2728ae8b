// What the operators on typed rows share (embedding lookup, products by vertex type, norm): element types, vectors of elements, the
// status word, and the host's checks of their arguments.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "taurus_internal.h"

static inline int row_type_size(int32_t t) { return t == TAURUS_F32 ? 4 : t == TAURUS_BF16 || t == TAURUS_F16 ? 2 : 0; }   // 0: no such type

// The device that is current; every operator's arguments have to live there.  (The number of SMs is asked for once per device: it does not change.)
static inline bool rows_current_device(int* dev, int* sms) {
  static std::atomic<int> known[64];
  cudaError_t e = cudaGetDevice(dev);
  if (e == cudaSuccess) {
    std::atomic<int>* const k = *dev >= 0 && *dev < 64 ? &known[*dev] : nullptr;
    *sms = k ? k->load(std::memory_order_relaxed) : 0;
    if (*sms == 0) {
      e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
      if (e == cudaSuccess && k) k->store(*sms, std::memory_order_relaxed);
    }
  }
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "current device"); return false; }
  return true;
}
static inline bool rows_on_device(const void* p, int dev) {
  cudaPointerAttributes at;
  if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return false; }
  return (at.type == cudaMemoryTypeDevice && at.device == dev) || at.type == cudaMemoryTypeManaged;
}
static inline bool rows_aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
// An array of a call: `rows` rows of `width` bytes, `pitch` bytes apart; no rows where there is none.
struct Region {
  const void* p;
  size_t rows, width, pitch;
  size_t bytes() const { return rows > 0 ? (rows - 1) * pitch + width : 0; }
};
static inline Region region_of(const void* p, size_t bytes) { return {p, p && bytes ? (size_t)1 : (size_t)0, bytes, bytes}; }
static inline Region region_of_rows(const void* p, int64_t n, int64_t ld, int64_t width, int size) {
  return {p, p ? (size_t)n : (size_t)0, (size_t)width * (size_t)size, (size_t)ld * (size_t)size};
}
// Do two arrays share a byte?  Columns of one matrix do not share any with others of it: rows of one pitch are compared by where they lie in it.
static inline bool regions_share(const Region& a, const Region& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  if (a.rows == 0 || b.rows == 0 || x >= y + b.bytes() || y >= x + a.bytes()) return false;
  if ((a.rows == 1 && b.rows == 1) || (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch)) return true;
  const size_t pitch = a.rows > 1 ? a.pitch : b.pitch, d = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;
  return d < a.width || d + b.width > pitch;
}
// No array of `out` shares a byte with one of `in`, nor with another of `out`.
template <int A, int B>
static inline bool regions_apart(const Region (&out)[A], const Region (&in)[B]) {
  for (int i = 0; i < A; ++i) {
    for (int j = 0; j < B; ++j) if (regions_share(out[i], in[j])) return false;
    for (int j = 0; j < i; ++j) if (regions_share(out[i], out[j])) return false;
  }
  return true;
}
template <int A>
static inline bool regions_on_device(const Region (&r)[A], int dev) {
  for (const Region& i : r) if (i.rows > 0 && !rows_on_device(i.p, dev)) return false;
  return true;
}
// Is the workspace of the call, `need` bytes, there and apart from its arrays?
template <int A, int B>
static inline bool workspace_ok(const void* p, int64_t bytes, int64_t need, int dev, const Region (&out)[A], const Region (&in)[B]) {
  if (need == 0) return true;
  if (!p || !rows_aligned(p, 256) || bytes < need || !rows_on_device(p, dev)) return false;
  const Region mine[] = {region_of(p, (size_t)need)};
  return regions_apart(mine, out) && regions_apart(mine, in);
}
// n rows of ld elements of `size` bytes stay below 2^62 bytes, so that no product of sizes overflows.
static inline bool rows_fit(int64_t n, int64_t ld, int size) { return n == 0 || ld <= (int64_t)((1ll << 62) / size) / n; }

// The launches of a call: each but the first may come up while the one before it ends (early_start at the start of every kernel waits for what that
// wrote).  Data of an earlier kernel of the call is not read through __restrict__ pointers: such loads may be moved ahead of the wait.  For the norm, most of whose
// launches find nothing to do in a batch of short graphs: 262 144 x 64 bf16 in 9 001 graphs 43.1 -> 41.3 us.  The sort of the ids lost by it (161 -> 184 us for 500 000:
// blocks that wait take the places of blocks that work), the products by type did not change.
struct Launches {
  cudaStream_t st;
  bool early = false;
  template <class... P, class... A>
  void operator()(void (*kernel)(P...), dim3 grid, int threads, size_t smem, A... args) {
    if (error != cudaSuccess) return;            // a kernel behind one that did not run would take what stands in the workspace for indexes
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = &at; cfg.numAttrs = early ? 1 : 0;
    error = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    early = true;
  }
  cudaError_t error = cudaSuccess;
  // The call's result: what a launch said, with its text kept.
  int done(const char* what) {
    const cudaError_t last = cudaGetLastError();
    const cudaError_t e = error != cudaSuccess ? error : last;
    if (e == cudaSuccess) return TAURUS_OK;
    taurus_note_cuda_error(e, what);
    return TAURUS_ERR_CUDA;
  }
};

// A status word keeps the first error of the calls it was given to.
static __device__ __forceinline__ void rows_status(int32_t* status, int code) { if (status) atomicCAS(status, 0, code); }

template <class T> static __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <class T> static __device__ __forceinline__ T from_f32(float v);     // rounded to nearest, once
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N elements that start at a multiple of their own size.
template <class T, int N> struct __align__(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Vec { T v[N]; };

enum { LOAD_PLAIN = 0, LOAD_ONCE = 1 };   // LOAD_ONCE: not expected to be read again soon

template <class V, int HOW = LOAD_PLAIN>
static __device__ __forceinline__ V load_vec(const void* p) {
  V r;
  if constexpr (sizeof(V) % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 16; ++i)
      reinterpret_cast<uint4*>(&r)[i] = HOW == LOAD_ONCE ? __ldcs(reinterpret_cast<const uint4*>(p) + i) : reinterpret_cast<const uint4*>(p)[i];
  } else if constexpr (sizeof(V) == 8) {
    *reinterpret_cast<uint2*>(&r) = HOW == LOAD_ONCE ? __ldcs(reinterpret_cast<const uint2*>(p)) : *reinterpret_cast<const uint2*>(p);
  } else if constexpr (sizeof(V) == 4) {
    *reinterpret_cast<uint32_t*>(&r) = HOW == LOAD_ONCE ? __ldcs(reinterpret_cast<const uint32_t*>(p)) : *reinterpret_cast<const uint32_t*>(p);
  } else {
    *reinterpret_cast<uint16_t*>(&r) = *reinterpret_cast<const uint16_t*>(p);
  }
  return r;
}
template <class V>
static __device__ __forceinline__ void store_vec(void* p, const V& r) {
  if constexpr (sizeof(V) % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(&r)[i];
  } else if constexpr (sizeof(V) == 8) {
    *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(&r);
  } else if constexpr (sizeof(V) == 4) {
    *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(&r);
  } else {
    *reinterpret_cast<uint16_t*>(p) = *reinterpret_cast<const uint16_t*>(&r);
  }
}
// Written past the caches' lines that are read again.
template <class V>
static __device__ __forceinline__ void store_vec_once(void* p, const V& r) {
  if constexpr (sizeof(V) % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 16; ++i) __stcs(reinterpret_cast<uint4*>(p) + i, reinterpret_cast<const uint4*>(&r)[i]);
  } else if constexpr (sizeof(V) == 8) {
    __stcs(reinterpret_cast<uint2*>(p), *reinterpret_cast<const uint2*>(&r));
  } else if constexpr (sizeof(V) == 4) {
    __stcs(reinterpret_cast<uint32_t*>(p), *reinterpret_cast<const uint32_t*>(&r));
  } else {
    __stcs(reinterpret_cast<uint16_t*>(p), *reinterpret_cast<const uint16_t*>(&r));
  }
}
template <class T, int N>
static __device__ __forceinline__ void store_f32_once(T* p, const float (&x)[N]) {
  Vec<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(x[i]);
  store_vec_once(p, r);
}
template <class T, int N>
static __device__ __forceinline__ void store_f32(T* p, const float (&x)[N]) {
  Vec<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(x[i]);
  store_vec(p, r);
}
template <class T, int N, int HOW = LOAD_PLAIN>
static __device__ __forceinline__ void load_f32(const T* p, float (&x)[N]) {
  const Vec<T, N> r = load_vec<Vec<T, N>, HOW>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = to_f32<T>(r.v[i]);
}

// Group g's rows by its two offsets, kept inside [0, n] whatever the offsets hold; a group that runs backwards or leaves [0, n] is reported.
static __device__ __forceinline__ void group_rows(const long long* offsets, long long g, long long n, long long* begin, long long* end, int32_t* status) {
  const long long a = offsets[g], b = offsets[g + 1];
  if (a < 0 || b > n || b < a) rows_status(status, TAURUS_ERR_INVALID_ARG);
  *begin = a < 0 ? 0 : a > n ? n : a;
  *end = b < *begin ? *begin : b > n ? n : b;
}

// f(tag of T) for the element type `t`.
template <class T> struct RowTag { using type = T; };
template <class F> static inline int with_row_type(int32_t t, F f) {
  if (t == TAURUS_F32) return f(RowTag<float>());
  if (t == TAURUS_BF16) return f(RowTag<__nv_bfloat16>());
  return f(RowTag<__half>());
}
// f(integral_constant of the vector length v).
template <class F> static inline int with_vector(int v, F f) {
  return v == 8 ? f(std::integral_constant<int, 8>()) : v == 4 ? f(std::integral_constant<int, 4>())
         : v == 2 ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, 1>());
}
