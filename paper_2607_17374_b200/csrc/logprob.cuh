// Log probabilities of given classes from rows of logits, with the entropy and the top alternatives, and the gradient of the logits.
//
//   m = max x,  l = log sum e^(x - m),  log p_j = (x_j - m) - l,  H = -sum p log p = l - (sum e^(x - m) (x - m)) / e^l
//   grad x_j = g (delta_j,label - p_j) - h p_j (log p_j + H)           g: weight of log p_label, h: weight of H
//
// The largest term of the sum is 1: it is left out of the sum s of the others, and l = log1p(s), H = l - t / (1 + s).  Both parts of H are positive and nothing
// cancels: a row whose first class has nearly everything keeps all digits of l, H and 1 - p.  Differences are cut off at -200 or -256 (e^-200 = 0 in fp32): a
// masked class (-inf, or a type's lowest value) then adds 0 to both sums, and no 0 x inf comes up.  A NaN goes into m, and with it into everything; +inf is treated as NaN.
//
// Bytes are the floor: the logits in, once (and their gradient out).  Instructions bound it: 28 to 34 an element of a tile, 11 of a long row.
// Many rows of up to 1 024 classes come by tiles into shared memory, where 1 to 16 threads have a row (rows_kernel: 1 200 000 x 47 fp32 with the top 3 in 76 us, 3.9 TB/s; 400 000 x 172 bf16 with the gradient
// in 73, 3.9 TB/s; every scheduler issues in three cycles of four).  Fewer are read once and stay in the registers of 8 or 32 lanes, for the gradient too, and so do long fp32 rows (team_kernel: 100 000 x 1 000 with
// the gradient 133 us, 6.0 TB/s).  Wider ones are the work of 1 to 8 warps, or of several
// blocks where there are few rows (stream_kernel, join_kernel: 2 000 x 120 001 bf16 with the top 10 in 131 us, 3.7 TB/s; 50 000 x 3 000 fp32 95 us, 6.3 TB/s): every thread keeps a maximum and sums of its own over its vectors, without a branch, and they are joined at the end.
// The term that is 1 stands in one thread's sum and has eaten that thread's small terms: its vectors are read again without it, by all threads.  The top needs no work in
// the pass either: with the k-th largest of the threads' maxima known, the top k are in the vectors of the k threads whose maxima are not below it, and only those are looked
// through again.
#pragma once

#include <algorithm>

#include "rows.cuh"

struct LogprobArgs {
  long long n;
  int C;
  const void* x;
  long long ld;
  const long long* labels;
  float *logprob, *entropy;
  float2* stats;
  int k;
  float* top_logprob;
  long long* top_class;
  // gradient
  const float *grad_logprob, *grad_entropy;
  const float2* stats_in;
  const float* entropy_in;
  void* dx;
  long long ld_dx;
  int32_t* status;
  // parts of a row
  int parts, part_len;
  float4* part;                                // [n x parts] (m, s, t, bad)
  unsigned long long* part_top;                               // [n x parts x k]
  // tiles of rows_kernel
  int pitch, mode_in, mode_out;
  unsigned by_C, by_vectors;                   // 2^32 / C, 2^32 / vectors of a row, rounded up
  int vectors;
};

namespace {

constexpr int MAX_TOP = TAURUS_MAX_TOP;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LEAST = -200.f;
constexpr int ROW_THREADS = 128;               // threads of a block of rows_kernel
constexpr int WARPS = 8;                       // warps of a block of the others
constexpr int LIST = 64;                       // places of a warp's list of candidates
constexpr int MAX_PARTS = 64;                  // parts of a row
constexpr int TEAM_CLASSES = 1024;             // rows that fit the registers of a warp: 32 elements a lane
// Classes of a row in a tile at most.  fp32 rows of some length are better in registers, read once, than three times from a tile: 100 000 x 1 000 with the gradient 133 / 182 us (256: 69 / 67), without
// it and without a top 91 / 110 (600: 79 / 68).  With a top they are better in tiles (40 000 x 1 000, top 16: 124 / 114), and so are 16-bit rows (400 bf16: 85 / 49).
constexpr int tile_classes(int size, bool grad, int k) { return size == 2 ? TEAM_CLASSES : grad ? 384 : k == 0 ? 768 : TEAM_CLASSES; }

typedef unsigned long long u64;

using Args = LogprobArgs;


__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

__device__ __forceinline__ float fma_sat(float a, float b, float c) { float r; asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ float mul_sat(float a, float b) { float r; asm("mul.rn.sat.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
// (m - x) / 256, at most 1, for m8 = m / 256: the cut that keeps infinities out, in the same instruction as the difference (minima, comparisons and selections go at half
// the rate of multiplications).  Scaling by 2^-8 is exact.  Of two infinities: 0.
constexpr float CUT = 256.f;
__device__ __forceinline__ float below(float x, float m8) { return fma_sat(x, -1.f / CUT, m8); }
__device__ __forceinline__ float exp_below(float z) { return ex2(z * (-CUT * LOG2E)); }
// Pairs of fp32 values and their arithmetic in one instruction.
struct F2 { u64 v; };
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split(F2 x, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(x.v)); }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// Sums over classes with the maximum known, two at a time: s without the terms that equal it (weight 0; else 1), q of z e^-256z, others: how many are below.
struct RowSums {
  F2 s = {0}, q = {0}, others = {0};
  __device__ __forceinline__ void add2(float x, float y, float m8) {
    const float zx = below(x, m8), zy = below(y, m8);
    const F2 z = f2(zx, zy), w = f2(mul_sat(zx, 0x1p126f), mul_sat(zy, 0x1p126f));
    float a, b;
    split(mul(z, f2(-CUT * LOG2E, -CUT * LOG2E)), &a, &b);
    const F2 e = f2(ex2(a), ex2(b));
    s = fma(e, w, s);
    q = fma(e, z, q);
    others = add(others, w);
  }
  __device__ __forceinline__ static float both(F2 x) { float a, b; split(x, &a, &b); return a + b; }
};

// Order of candidates: larger value first, of equal ones the lower class.  0: none (-inf, NaN).  -0 counts as 0.
__device__ __forceinline__ u64 key_of(float x, int cls) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
  return ((u64)o << 32) | (0xffffffffu - (uint32_t)cls);
}
__device__ __forceinline__ float key_value(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_class(u64 key) { return (int)(0xffffffffu - (uint32_t)key); }

// Sums of some classes of a row.  m: their largest value, whose own term (1) is in neither sum; -inf: no classes yet.
struct Sums { float m, s, t; };
// Joins b's classes, which come behind a's.
__device__ __forceinline__ void join(Sums& a, const Sums& b) {
  if (!(b.m > -INFINITY)) return;
  if (!(a.m > -INFINITY)) { a = b; return; }
  const bool up = b.m > a.m;
  const float d = fmaxf(up ? a.m - b.m : b.m - a.m, LEAST), f = ex2(d * LOG2E);
  const float ws = up ? b.s : a.s, wt = up ? b.t : a.t, os = up ? a.s : b.s, ot = up ? a.t : b.t;     // the side of the maximum, the other side
  const float o1 = 1.f + os;
  a.s = fmaf(o1, f, ws);
  a.t = wt + f * fmaf(o1, d, ot);
  if (up) a.m = b.m;
}

// What a row's sums say.
struct RowResult { float m, l, H; };
__device__ __forceinline__ RowResult row_result(const Sums& s, bool bad) {
  if (bad) return {NAN, NAN, NAN};
  if (!(s.m > -INFINITY)) return {s.m, 0.f, 0.f};
  const float l = log1pf(s.s);
  return {s.m, l, l - __fdividef(s.t, 1.f + s.s)};
}
__device__ __forceinline__ float log_p(float x, const RowResult& r) { return r.m == -INFINITY ? -INFINITY : (x - r.m) - r.l; }

// -1: no label; one outside the classes is reported.
__device__ __forceinline__ int label_of(const Args& a, long long row) {
  if (!a.labels) return -1;
  const long long v = a.labels[row];
  if (v < -1 || v >= a.C) { rows_status(a.status, TAURUS_ERR_INVALID_ARG); return -1; }
  return (int)v;
}
template <class T>
__device__ __forceinline__ void write_row(const Args& a, long long row, int label, const RowResult& r) {
  if (a.logprob) a.logprob[row] = label < 0 ? 0.f : log_p(to_f32<T>(static_cast<const T*>(a.x)[row * a.ld + label]), r);
  if (a.entropy) a.entropy[row] = r.H;
  if (a.stats) a.stats[row] = make_float2(r.m, r.l);
}
__device__ __forceinline__ void write_top(const Args& a, long long row, int i, u64 key, const RowResult& r) {
  if (a.top_logprob) a.top_logprob[row * a.k + i] = key ? log_p(key_value(key), r) : -INFINITY;
  if (a.top_class) a.top_class[row * a.k + i] = key ? key_class(key) : -1;
}

// What the gradient of a row needs.
struct GradRow {
  float m8, l, H, g, h, c;                       // m8: the maximum / 256
  int label;
};
__device__ __forceinline__ GradRow grad_row(float g, float h, int label, const RowResult& r) {
  if (r.m == -INFINITY) return {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, label};                        // all masked
  return {r.m * (1.f / CUT), r.l, r.H, g, h, h == 0.f ? -g : fmaf(-h, r.H, -g), label};
}
__device__ __forceinline__ GradRow grad_row(const Args& a, long long row, int label, const RowResult& r) {
  return grad_row(label >= 0 && a.grad_logprob ? a.grad_logprob[row] : 0.f, a.grad_entropy ? a.grad_entropy[row] : 0.f, label, r);
}
__device__ __forceinline__ float grad_of(const GradRow& r, float x) {
  const float lp = fmaf(below(x, r.m8), -CUT, -r.l), p = ex2(lp * LOG2E);
  return p * fmaf(-r.h, lp, r.c);                // (masked: p = 0)
}
__device__ __forceinline__ void grad_of2(const GradRow& r, float x, float y, float* dx, float* dy) {
  const F2 lp = fma(f2(below(x, r.m8), below(y, r.m8)), f2(-CUT, -CUT), f2(-r.l, -r.l));
  float a, b;
  split(mul(lp, f2(LOG2E, LOG2E)), &a, &b);
  split(mul(f2(ex2(a), ex2(b)), fma(f2(-r.h, -r.h), lp, f2(r.c, r.c))), dx, dy);
}
__device__ __forceinline__ float grad_of_label(const GradRow& r, float x) {
  const float lp = fmaf(below(x, r.m8), -CUT, -r.l), p = ex2(lp * LOG2E);
  return x == -INFINITY ? 0.f : -r.g * expm1f(lp) - r.h * p * (lp + r.H);
}

enum { FORWARD = 0, TRAIN = 1, GRAD = 2 };

// What a lane loads at once: an element, or two where 16-bit rows have an even width.
template <class T, bool PAIRS> struct Word { using type = T; static constexpr int n = 1; };
template <class T> struct Word<T, true> { using type = uint32_t; static constexpr int n = 2; };
template <class T>
__device__ __forceinline__ void unpack(T w, float (&x)[1]) { x[0] = to_f32<T>(w); }
template <class T>
__device__ __forceinline__ void unpack(uint32_t w, float (&x)[2]) {
  if constexpr (std::is_same_v<T, __nv_bfloat16>) { x[0] = __uint_as_float(w << 16); x[1] = __uint_as_float(w & 0xffff0000u); }
  else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w)); x[0] = f.x; x[1] = f.y; }
}
template <class T>
__device__ __forceinline__ T pack(const float (&x)[1]) { return from_f32<T>(x[0]); }
template <class T>
__device__ __forceinline__ uint32_t pack(const float (&x)[2]) {
  if constexpr (std::is_same_v<T, __nv_bfloat16>) { const __nv_bfloat162 r = __floats2bfloat162_rn(x[0], x[1]); return *reinterpret_cast<const uint32_t*>(&r); }
  else { const __half2 r = __floats2half2_rn(x[0], x[1]); return *reinterpret_cast<const uint32_t*>(&r); }
}

}  // namespace

// Short rows of a call, many of them (logprob_rows.cuh, a file for each type).  mode: FORWARD, TRAIN or GRAD; pairs: rows of 16-bit elements by twos.  A launch that fails is kept in `enqueue`.
void logprob_rows_f32(Launches& enqueue, const LogprobArgs& a, int mode);
void logprob_rows_bf16(Launches& enqueue, const LogprobArgs& a, int mode, bool pairs);
void logprob_rows_f16(Launches& enqueue, const LogprobArgs& a, int mode, bool pairs);
