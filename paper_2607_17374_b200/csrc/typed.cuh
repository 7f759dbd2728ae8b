// What the two forms of the products by vertex type share: the kernels for few rows (kernels_typed.cu) and those on the tensor cores
// (kernels_typed_tc.cu).
#pragma once

#include "rows.cuh"

// Two fp32 values as three pairs of bf16 values: hi + mid + lo = x exactly while lo is above bf16's smallest.  hi is cut off, not rounded, so that it
// stays finite; mid is rounded to nearest, by an addition to its bits (the conversion instruction has a fraction of the rate); lo has 8 bits left and is the upper
// half of its fp32 word.  rest: NaN where a value is not finite (its mid and lo then have to be zeros: split_special).
struct Split2 { unsigned hi, mid, lo; float rest; };
static __device__ __forceinline__ Split2 split2(float a, float b) {
  const unsigned ua = __float_as_uint(a), ub = __float_as_uint(b);
  const float ra = a - __uint_as_float(ua & 0xFFFF0000u), rb = b - __uint_as_float(ub & 0xFFFF0000u);     // 16 bits
  const unsigned ma = __float_as_uint(ra) + 0x8000u, mb = __float_as_uint(rb) + 0x8000u;
  const float la = ra - __uint_as_float(ma & 0xFFFF0000u), lb = rb - __uint_as_float(mb & 0xFFFF0000u);   // at most 8 bits
  Split2 s;
  s.hi = __byte_perm(ua, ub, 0x7632);
  s.mid = __byte_perm(ma, mb, 0x7632);
  s.lo = __byte_perm(__float_as_uint(la), __float_as_uint(lb), 0x7632);
  s.rest = ra + rb;
  return s;
}
// The same for values of which one may be infinite or NaN: that is hi alone, and a NaN stays one.
static __device__ __noinline__ Split2 split_special(float a, float b) {
  const bool fa = fabsf(a) <= 3.402823466e38f, fb = fabsf(b) <= 3.402823466e38f;
  Split2 s = split2(fa ? a : 0.f, fb ? b : 0.f);
  if (!fa) s.hi = (s.hi & 0xFFFF0000u) | (a != a ? 0x7FC0u : __float_as_uint(a) >> 16);
  if (!fb) s.hi = (s.hi & 0xFFFFu) | (b != b ? 0x7FC00000u : __float_as_uint(b) & 0xFFFF0000u);
  return s;
}
// Four values into their three planes of 8 bytes.
struct Split4 { uint2 hi, mid, lo; };
static __device__ __forceinline__ Split4 split4(float a, float b, float c, float d) {
  Split2 p = split2(a, b), q = split2(c, d);
  const float rest = p.rest + q.rest;
  if (rest != rest) { p = split_special(a, b); q = split_special(c, d); }
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
size_t typed_tc_part_bytes(int64_t n, int32_t types, int d_in, int d_out, int32_t type);
// (arguments as checked by the entry points; TAURUS_ERR_CUDA with nothing enqueued where a tensor map cannot be made)
int typed_tc_project(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const float* bias, int d_in, int d_out, void* out,
                     int32_t out_type, int64_t ld_out, const TypedSpaces& spaces, int32_t* status, int sms, cudaStream_t st);
int typed_tc_project_grad(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const void* grad_out, int64_t ld_grad, int d_in,
                          int d_out, void* grad_x, int64_t ld_grad_x, void* grad_W, int32_t grad_W_type, float* grad_bias, const TypedSpaces& spaces, int32_t* status, int sms,
                          cudaStream_t st);
