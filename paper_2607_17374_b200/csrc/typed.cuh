// What the two forms of the products by vertex type share: the kernels for few rows (kernels_typed.cu) and those on the tensor cores
// (kernels_typed_tc.cu).
#pragma once

#include "rows.cuh"

// An fp32 value as three bf16 values: hi + mid + lo = x exactly while lo is above bf16's smallest.  hi is cut off, not rounded, so that it stays finite.
// What is not finite is hi alone.
struct Split3 { float hi, mid, lo; };
static __device__ __forceinline__ Split3 split3(float x) {
  Split3 s;
  s.hi = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
  const float r = x - s.hi;                                         // 16 bits
  s.mid = __bfloat162float(__float2bfloat16_rn(r));
  s.lo = r - s.mid;                                                 // at most 8 bits
  if ((__float_as_uint(x) & 0x7F800000u) == 0x7F800000u) {
    s.hi = x != x ? __uint_as_float(0x7FC00000u) : x;
    s.mid = s.lo = 0.f;
  }
  return s;
}

// ---- kernels_typed_tc.cu
bool typed_tc_usable();
bool typed_tc_packs(int32_t type, int d_out);
size_t typed_tc_pack_bytes(int32_t types, int d_in, int d_out, int32_t type);
size_t typed_tc_part_bytes(int64_t n, int32_t types, int d_in, int d_out, int32_t type);
int typed_tc_pack(int32_t type, const void* W, int32_t types, int d_in, int d_out, void* packed, int sms, cudaStream_t st);
int typed_tc_rows(bool transposed, int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* w, const float* bias, int d_in, int d_out,
                  void* out, int32_t out_type, int64_t ld_out, int32_t* status, int sms, cudaStream_t st);
int typed_tc_weights(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* dy, int64_t ld_dy, int d_in, int d_out, void* dW,
                     int32_t dW_type, float* db, float* part, int32_t* status, int sms, cudaStream_t st);
