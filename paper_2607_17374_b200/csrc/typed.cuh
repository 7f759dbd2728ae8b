// What the two forms of the products by vertex type share: the kernels for few rows (kernels_typed.cu) and those on the tensor cores
// (kernels_typed_tc.cu).
#pragma once

#include <math.h>
#include <string.h>

#include "rows.cuh"

// Two fp32 values as three pairs of bf16 values, hi + mid + lo = x exactly from 2^-110 on (below that lo is cut off at bf16's smallest value, 2^-133).  hi and mid are rounded to
// nearest, so that mid is at most 2^-8 and lo 2^-17 of x, and what mid lo, lo mid and lo lo add up to is below 2^-24 of a product; lo has 7 bits left and is the upper half of its
// fp32 word.  (With hi cut off it is 2^-22.)  By the conversion instruction, which is no slower than an addition to the bits: grad_W of 400 000 rows,
// 100 -> 256: 243 us, mid by an addition 249, both 256.  rest: not finite where a value is not, or where hi is not (values above 2^128 (1 - 2^-8)): split_special.
struct Split2 { unsigned hi, mid, lo; float rest; };
static __host__ __device__ __forceinline__ unsigned bits_of(float x) {
#ifdef __CUDA_ARCH__
  return __float_as_uint(x);
#else
  unsigned u;
  memcpy(&u, &x, 4);
  return u;
#endif
}
static __host__ __device__ __forceinline__ float float_of(unsigned u) {
#ifdef __CUDA_ARCH__
  return __uint_as_float(u);
#else
  float x;
  memcpy(&x, &u, 4);
  return x;
#endif
}
static __host__ __device__ __forceinline__ unsigned bf16_pair(float a, float b) {      // a in the lower half
  union { __nv_bfloat162 h; unsigned u; } x;
  x.h = __floats2bfloat162_rn(a, b);
  return x.u;
}
static __host__ __device__ __forceinline__ unsigned upper_halves(unsigned a, unsigned b) {
#ifdef __CUDA_ARCH__
  return __byte_perm(a, b, 0x7632);
#else
  return a >> 16 | (b & 0xFFFF0000u);
#endif
}
static __host__ __device__ __forceinline__ bool all_finite(float x) { return fabsf(x) <= 3.402823466e38f; }
static __host__ __device__ __forceinline__ Split2 split2(float a, float b) {
  Split2 s;
  s.hi = bf16_pair(a, b);
  const float ra = a - float_of(s.hi << 16), rb = b - float_of(s.hi & 0xFFFF0000u);     // at most 16 bits
  s.mid = bf16_pair(ra, rb);
  const float la = ra - float_of(s.mid << 16), lb = rb - float_of(s.mid & 0xFFFF0000u);
  s.lo = upper_halves(bits_of(la), bits_of(lb));
  s.rest = ra + rb;
  return s;
}
// A value that is not finite is hi alone, and a NaN stays one; of a finite one whose hi would not be, hi is cut off instead.
static __host__ __device__ __forceinline__ void split_one(float x, unsigned* hi, unsigned* mid, unsigned* lo) {
  const unsigned u = bits_of(x);
  if (!all_finite(x)) { *hi = x != x ? 0x7FC0u : u >> 16; *mid = *lo = 0; return; }
  const unsigned up = u + 0x8000u, h = (up & 0x7F800000u) == 0x7F800000u ? u : up;
  const float r = x - float_of(h & 0xFFFF0000u);
  const unsigned m = bits_of(r) + 0x8000u;
  *hi = h >> 16; *mid = m >> 16; *lo = bits_of(r - float_of(m & 0xFFFF0000u)) >> 16;
}
static __host__ __device__ __noinline__ Split2 split_special(float a, float b) {
  unsigned ha, ma, la, hb, mb, lb;
  split_one(a, &ha, &ma, &la);
  split_one(b, &hb, &mb, &lb);
  return {ha | hb << 16, ma | mb << 16, la | lb << 16, 0.f};
}
// Four values into their three planes of 8 bytes.
struct Split4 { uint2 hi, mid, lo; };
static __host__ __device__ __forceinline__ Split4 split4(float a, float b, float c, float d) {
  Split2 p = split2(a, b), q = split2(c, d);
  const float rest = p.rest + q.rest;
  if (!all_finite(rest)) { p = split_special(a, b); q = split_special(c, d); }
  return {make_uint2(p.hi, q.hi), make_uint2(p.mid, q.mid), make_uint2(p.lo, q.lo)};
}

// Can TMA read rows of 16-bit elements?  (A tensor map holds pitches below 2^40 bytes.)
static inline bool tma_rows(const void* p, long long ld) { return ld % 8 == 0 && ld < (1ll << 39) && rows_aligned(p, 16); }

// ---- kernels_typed_tc.cu
// Parts of a call's workspace: W laid out anew, partial results of grad_W, rows of grad_out and of x at other pitches.
struct TypedSpaces { void *W, *part, *dy, *x; };
bool typed_tc_packs(const void* W, int32_t type, int d_out);
size_t typed_tc_pack_bytes(int32_t types, int d_in, int d_out, int32_t type);
size_t typed_tc_row_bytes(int64_t n, int width, int32_t type);
size_t typed_tc_part_bytes(int64_t n, int32_t types, int d_in, int d_out, int32_t type, bool most);
// (arguments as checked by the entry points; TAURUS_ERR_CUDA with nothing enqueued where a tensor map cannot be made)
int typed_tc_project(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const float* bias, int d_in, int d_out, void* out,
                     int32_t out_type, int64_t ld_out, const TypedSpaces& spaces, int32_t* status, int sms, cudaStream_t st);
int typed_tc_project_grad(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const void* grad_out, int64_t ld_grad, int d_in,
                          int d_out, void* grad_x, int64_t ld_grad_x, void* grad_W, int32_t grad_W_type, float* grad_bias, const TypedSpaces& spaces, int32_t* status, int sms,
                          cudaStream_t st);
