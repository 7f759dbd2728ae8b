// One AdamW step over many tensors at once, with states in 32 bits or in 8.
//
//   g = s grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - lr wd p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bytes are the floor: 28 an element with everything in fp32, 10.06 with parameters and gradients in 16 bits and states in 8.  They bound the first (60 M elements in 269 us, 6.2 TB/s); the second is
// bound by instructions, 68 an element of which 26 go at half rate (200 M elements in 516 us, 3.9 TB/s, issue slots 72 % used; the next tile's bytes on their way ahead 566 against 512, pairs in one instruction spilled).  All tensors are cut into tiles of 2 048
// elements, which the blocks of one launch (for each combination of types) take in turn: a tensor costs no launch, and its description and a tile's tensor are read from device memory.
//
// States in 8 bits: m and r = sqrt(v), rounded to nearest in fp32, as e4m3 codes times a power of two for each 256 elements, one warp's.  With the scale the largest code is in [2^7, 2^8), the
// smallest step 2^-16 of the largest value; multiplying by the scale is exact.  Rounded to nearest a state would stand still: a step of e4m3 is 6 to 12 % of the
// value, and v moves by 0.1 % in a step.  So a value is rounded up with the probability of what is cut off, in 65 536ths, by a hash of (seed, step, tensor, element): the same call gives the same
// bits.  An r that is not 0 is not rounded to 0: m beside it would be divided by eps.  The update itself is formed from m and v before they are rounded.
// m and v are formed in separately rounded products and sums, no fused ones: whether a block's largest value reaches the next power of two does not hang on the compiler.
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "rows.cuh"
#include "upload.h"

namespace {

constexpr int THREADS = 256, E = 8, TILE = THREADS * E, BLOCK = TAURUS_STATE_BLOCK;
static_assert(32 * E == BLOCK, "a block of states is a warp's");

struct Tensor {
  void* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale, *master;
  long long count;
  long long first_tile;
  float decay;
  int32_t p_type, g_type;
  int32_t vectors;                               // every array begins at a multiple of 16 bytes (codes: of 8)
  uint32_t index;                                // in the caller's list
};

struct Args {
  const Tensor* tensors;
  const int32_t* tile_tensor;
  long long tiles;
  const long long* step;
  const float *lr, *grad_scale;
  float beta1, rest1, beta2, rest2, eps;
  float up;                                      // eps and what it is added to come multiplied by it, and what they divide: beside an eps below 2^-100 2^24, so that neither is a subnormal number; else 1
  int small_eps;                                 // beside a larger one the root of a subnormal number, 1e-19, is nothing
  double log_beta1, log_beta2;
  unsigned long long seed;
  int32_t* status;
};

// The finaliser of the published generator splitmix64 (Steele, Lea, Flood; constants of Stafford's variant 13), with its increment in absorb().
__device__ __forceinline__ unsigned long long mix64(unsigned long long z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
__device__ __forceinline__ unsigned long long absorb(unsigned long long h, unsigned long long x) { return mix64(h ^ (0x9E3779B97F4A7C15ull * (x + 1))); }
// 32 bits for element i of a tensor: the published finaliser lowbias32 (Wellons) of (i ^ key) + (key >> 32) + (i >> 32) 0x85EBCA6B.
__device__ __forceinline__ uint32_t finish_bits(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

// The root of a subnormal number is 0 with the one, its own with the other, which takes four instructions.
__device__ __forceinline__ float root_of(float x) { float r; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float any_root_of(float x) { float r; asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// (of a subnormal number infinite: a divisor is none)
__device__ __forceinline__ float reciprocal(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max_nan(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

template <class T>
__device__ __forceinline__ void to_floats(const Vec<T, E>& r, float (&x)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = to_f32<T>(r.v[e]);
}
__device__ __forceinline__ void codes_to_floats(uint2 c, float scale, float (&x)[E]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[e / 4] >> (8 * (e & 2))), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    x[e] = f.x * scale; x[e + 1] = f.y * scale;
  }
}
constexpr uint32_t NOT_FINITE = 0x7f800000u, CODE_NAN = 0x7f;

// The root of a v as a code: bits 24 to 30, with 16 random bits added below them (the kernel says how).  least: code 1 where v is not 0.
__device__ __forceinline__ uint32_t code_of_root(float root, float part_v, float least, uint32_t bits) {
  return (__float_as_uint(fmaxf(__fmul_rz(root * part_v, 0x1p-100f), least)) << 4) + __byte_perm(bits, 0, 0x4324);
}
// The hardware's root is off by 2^-23 of itself at most: from the one rounded to nearest by two and a half units in its last place, three where they are cut off, of 16 each here.  It makes another
// code only where the sum is that near to a border between two codes, on either side; 64 with a margin.  Such elements, one in 131 072, are done again with the root rounded to nearest, so that a
// code is what its definition says and not what an instruction makes of it (without it 20 codes of 200 M are a neighbour's, and they take 496 us instead of 516; borders looked for by 16-bit halves 525,
// codes done again where they are found 549, from the state read again 536).
__device__ __forceinline__ uint32_t from_border(uint32_t code) { return code * 256u + 0x4000u; }
constexpr uint32_t AT_BORDER = 0x8000u;
// The root of v rounded to nearest, from one that is a few units off: the middle between two neighbours has 25 bits, its square 50, which fp64 holds.
__device__ __forceinline__ float exact_root_of(float v) {
  uint32_t r = __float_as_uint(any_root_of(v));
  const auto middle_below = [&](uint32_t low) { const double mid = 0.5 * ((double)__uint_as_float(low) + (double)__uint_as_float(low + 1)); return mid * mid < (double)v; };
#pragma unroll 1
  for (int i = 0; i < 4; ++i) if (middle_below(r)) ++r; else if (r && !middle_below(r - 1)) --r; else break;
  return __uint_as_float(r);
}

// What a step multiplies with, besides the arguments: the gradients' scale, 1 / sqrt(1 - b2^t) and -lr / (1 - b1^t) (both times `up`), 1 - lr wd.
struct Factors { float gs, c2, rate, keep; };

// Which elements of a warp's 256 a lane has: 8 in a row where they are 16 bytes at most; else four and four, so that the warp's loads of 16 bytes touch every sector once (8 fp32
// values in a row would be two loads of half of each).
template <bool WIDE>
struct Places {
  static constexpr int GROUP = WIDE ? 4 : 8;
  static __device__ __forceinline__ constexpr int element(int e) { return WIDE ? e / 4 * 128 + e % 4 : e; }
  static __device__ __forceinline__ int lane_place(int lane) { return lane * GROUP; }
  template <class T>
  static __device__ __forceinline__ Vec<T, E> load(const T* p, int lane) {
    if (!WIDE) return load_vec<Vec<T, E>, LOAD_ONCE>(p + lane * E);
    Vec<T, E> r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto q = load_vec<Vec<T, 4>, LOAD_ONCE>(p + h * 128 + lane * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[h * 4 + i] = q.v[i];
    }
    return r;
  }
  template <class T>
  static __device__ __forceinline__ void store(T* p, int lane, const float (&v)[E]) {
    if (!WIDE) { store_f32_once<T, E>(p + lane * E, v); return; }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float q[4] = {v[h * 4], v[h * 4 + 1], v[h * 4 + 2], v[h * 4 + 3]};
      store_f32_once<T, 4>(p + h * 128 + lane * 4, q);
    }
  }
  static __device__ __forceinline__ uint2 load_codes(const uint8_t* p, int lane) {
    if (!WIDE) return __ldcs(reinterpret_cast<const uint2*>(p + lane * E));
    return make_uint2(__ldcs(reinterpret_cast<const uint32_t*>(p + lane * 4)), __ldcs(reinterpret_cast<const uint32_t*>(p + 128 + lane * 4)));
  }
  static __device__ __forceinline__ void store_codes(uint8_t* p, int lane, uint2 c) {
    if (!WIDE) { __stcs(reinterpret_cast<uint2*>(p + lane * E), c); return; }
    __stcs(reinterpret_cast<uint32_t*>(p + lane * 4), c.x);
    __stcs(reinterpret_cast<uint32_t*>(p + 128 + lane * 4), c.y);
  }
};

// A warp's 256 elements of a tensor, from b on.  whole: all 256 are there, in arrays that allow vectors.
template <class PT, class GT, bool EIGHT, bool MASTER, bool whole>
__device__ __forceinline__ void step_block(const Args& a, const Tensor& t, const Factors f, unsigned long long key, long long b) {
  using P = Places<!EIGHT || sizeof(PT) == 4 || sizeof(GT) == 4>;
  const int lane = threadIdx.x & 31, first = P::lane_place(lane);
  const int left = (int)(t.count - b < BLOCK ? t.count - b : BLOCK);    // 1 at least
  const auto in = [&](int e) { return first + P::element(e) < left; };
  PT* const pp = static_cast<PT*>(t.p) + b;
  const GT* const gp = static_cast<const GT*>(t.g) + b;
  uint8_t *const mc = static_cast<uint8_t*>(t.m) + b, *const vc = static_cast<uint8_t*>(t.v) + b;
  float *const mf = static_cast<float*>(t.m) + b, *const vf = static_cast<float*>(t.v) + b;
  float p[E], g[E], m[E], v[E];
  if (whole) {
    // all on their way before the first is used
    const auto rg = P::template load<GT>(gp, lane);
    uint2 cm, cv;
    Vec<float, E> rm, rv, rw;
    Vec<PT, E> rp;
    float ms, vs;
    if (EIGHT) {
      cm = P::load_codes(mc, lane); cv = P::load_codes(vc, lane);
      ms = t.m_scale[b / BLOCK]; vs = t.v_scale[b / BLOCK];
    } else {
      rm = P::template load<float>(mf, lane); rv = P::template load<float>(vf, lane);
    }
    if (MASTER) rw = P::template load<float>(t.master + b, lane);
    else rp = P::template load<PT>(pp, lane);
    if (EIGHT) {
      codes_to_floats(cm, ms, m);
      codes_to_floats(cv, vs, v);
    } else {
      to_floats<float>(rm, m);
      to_floats<float>(rv, v);
    }
    if (MASTER) to_floats<float>(rw, p);
    else to_floats<PT>(rp, p);
    to_floats<GT>(rg, g);
  } else {
    uint2 cm = make_uint2(0, 0), cv = make_uint2(0, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      p[e] = g[e] = m[e] = v[e] = 0.f;
      if (in(e)) {
        const int at = first + P::element(e);
        p[e] = MASTER ? t.master[b + at] : to_f32<PT>(pp[at]);
        g[e] = to_f32<GT>(gp[at]);
        if (EIGHT) {
          (e < 4 ? cm.x : cm.y) |= (uint32_t)mc[at] << (8 * (e & 3));
          (e < 4 ? cv.x : cv.y) |= (uint32_t)vc[at] << (8 * (e & 3));
        } else { m[e] = mf[at]; v[e] = vf[at]; }
      }
    }
    if (EIGHT) {
      codes_to_floats(cm, t.m_scale[b / BLOCK], m);
      codes_to_floats(cv, t.v_scale[b / BLOCK], v);
    }
  }
  float root[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float ge = g[e] * f.gs;
    m[e] = __fadd_rn(__fmul_rn(a.beta1, m[e]), __fmul_rn(a.rest1, ge));
    if (EIGHT) v[e] = __fmul_rn(v[e], v[e]);
    v[e] = __fadd_rn(__fmul_rn(a.beta2, v[e]), __fmul_rn(__fmul_rn(a.rest2, ge), ge));
    root[e] = a.small_eps ? any_root_of(v[e]) : root_of(v[e]);
    p[e] = fmaf(m[e] * f.rate, reciprocal(fmaf(root[e], f.c2, a.eps)), p[e] * f.keep);
  }
  if (whole) {
    P::template store<PT>(pp, lane, p);
    if (MASTER) P::template store<float>(t.master + b, lane, p);
    if (!EIGHT) {
      P::template store<float>(mf, lane, m);
      P::template store<float>(vf, lane, v);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (in(e)) {
        const int at = first + P::element(e);
        pp[at] = from_f32<PT>(p[e]);
        if (MASTER) t.master[b + at] = p[e];
        if (!EIGHT) { mf[at] = m[e]; vf[at] = v[e]; }
      }
  }
  if (EIGHT) {
    float mm = 0.f, mv = 0.f;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      mm = max_nan(mm, fabsf(m[e]), fabsf(m[e + 1]));
      mv = max_nan(mv, v[e], v[e + 1]);
    }
    uint32_t most_m = __reduce_max_sync(0xffffffffu, __float_as_uint(mm) & 0x7fffffffu), most_v = __reduce_max_sync(0xffffffffu, __float_as_uint(mv) & 0x7fffffffu);
    const bool odd = most_m >= NOT_FINITE || most_v >= NOT_FINITE;      // somewhere in the block: scales by what is finite
    if (odd) {
      uint32_t am = 0, av = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t bm = __float_as_uint(m[e]) & 0x7fffffffu, bv = __float_as_uint(v[e]) & 0x7fffffffu;
        if (bm < NOT_FINITE) am = max(am, bm);
        if (bv < NOT_FINITE) av = max(av, bv);
      }
      most_m = __reduce_max_sync(0xffffffffu, am);
      most_v = __reduce_max_sync(0xffffffffu, av);
    }
    // The whole part of the largest one's logarithm, down by 7; of sqrt(v) half of v's.
    const int em = (int)max(most_m >> 23, 8u) - 7, ev = (((int)max(most_v >> 23, 1u) - 127) >> 1) + 120;
    // Codes.  x / scale 2^-120 has e4m3's exponent, 7 above its own, where fp32 has its exponent's last four bits, and below e4m3's smallest exponent it is a subnormal
    // number of fp32 (rounded down at 2^-149, 20 places below the last that stays): its bits 20 to 26 are the code, whatever its size, once the 16 random bits are added below
    // them.  Four places further up a code is a byte, and the sign is gone.  The factor is applied in two parts: one may be too small for fp32.
    if (most_v < (35u << 23) && !a.small_eps) {                       // all below 2^-92: roots of subnormal numbers count too (in other blocks they are below code 1)
#pragma unroll
      for (int e = 0; e < E; ++e) root[e] = any_root_of(v[e]);
    }
    const float part_m = __int_as_float(em < 234 ? (234 - em) << 23 : 1 << (256 - em)), part_v = __int_as_float((234 - ev) << 23);      // 2^(107 - e)
    const uint32_t base = (uint32_t)b ^ (uint32_t)key ^ (uint32_t)P::lane_place(lane), more = (uint32_t)(key >> 32) + (uint32_t)(b >> 32) * 0x85EBCA6Bu;     // (places differ in bits of their own)
    const auto least = [&](int e) { return fminf(v[e] * 0x1p100f, __uint_as_float(1u << 20)); };     // code 1 where v is not 0
    const auto bits_of = [&](int e) { return finish_bits((base ^ (uint32_t)P::element(e)) + more); };
    uint32_t cm[E / 4], cv[E / 4], near = 0xffffffffu;
#pragma unroll
    for (int h = 0; h < E / 4; ++h) {
      uint32_t wm[4], wv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 4 * h + i;
        const float zm = __fmul_rz(m[e] * part_m, 0x1p-100f);
        const uint32_t bits = bits_of(e);
        wm[i] = ((__float_as_uint(zm) << 4) + __byte_perm(bits, 0, 0x4104)) | (__float_as_uint(m[e]) & 0x80000000u);
        wv[i] = code_of_root(root[e], part_v, least(e), bits);
        near = min(near, from_border(wv[i]));
      }
      const auto four = [](const uint32_t* c) { return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410); };
      cm[h] = four(wm);
      cv[h] = four(wv);
      if (odd)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t byte = 0xffu << (8 * i), nan = CODE_NAN << (8 * i);
          if (!(fabsf(m[4 * h + i]) < INFINITY)) cm[h] = (cm[h] & ~byte) | nan;
          if (!(v[4 * h + i] < INFINITY)) cv[h] = (cv[h] & ~byte) | nan;
        }
    }
    if (lane == 0) {
      t.m_scale[b / BLOCK] = __uint_as_float((uint32_t)em << 23);
      t.v_scale[b / BLOCK] = __uint_as_float((uint32_t)ev << 23);
    }
    if (whole) {
      P::store_codes(mc, lane, make_uint2(cm[0], cm[1]));
      P::store_codes(vc, lane, make_uint2(cv[0], cv[1]));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (in(e)) { mc[first + P::element(e)] = (uint8_t)(cm[e / 4] >> (8 * (e % 4))); vc[first + P::element(e)] = (uint8_t)(cv[e / 4] >> (8 * (e % 4))); }
    }
    if (near < AT_BORDER)                        // the lane's codes of the root again
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((whole || in(e)) && v[e] < INFINITY) vc[first + P::element(e)] = (uint8_t)(code_of_root(exact_root_of(v[e]), part_v, least(e), bits_of(e)) >> 24);
  }
}

template <class PT, class GT, bool EIGHT, bool MASTER>
__device__ __noinline__ void step_block_by_element(const Args& a, const Tensor& t, const Factors f, unsigned long long key, long long b) { step_block<PT, GT, EIGHT, MASTER, false>(a, t, f, key, b); }

template <class PT, class GT, bool EIGHT, bool MASTER>
__global__ void __launch_bounds__(THREADS, EIGHT && !MASTER ? 4 : 3) adamw_kernel(const __grid_constant__ Args a) {
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const long long step = *a.step;
  if (step < 1) {
    if (blockIdx.x == 0 && threadIdx.x == 0) rows_status(a.status, TAURUS_ERR_INVALID_ARG);
    return;
  }
  if (!(fabsf(gs) < INFINITY)) return;           // the gradients were not finite: a step that is left out
  const float lr = *a.lr;
  // 1 - b^t = -(e^(t ln b) - 1)
  const float c1 = -1.f / expm1f((float)((double)step * a.log_beta1)), c2 = rsqrtf(-expm1f((float)((double)step * a.log_beta2)));
  Factors f = {gs, c2 * a.up, -lr * c1 * a.up, 1.f};
  unsigned long long seed_key = 0, key = 0;
  if (EIGHT) seed_key = absorb(absorb(0x243F6A8885A308D3ull, a.seed), (unsigned long long)step);
  int known = -1;
  __shared__ Tensor t;                           // (in registers it would take the place of 22 of them)
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int which = a.tile_tensor[tile];
    if (which != known) {
      __syncthreads();
      if (threadIdx.x < sizeof(Tensor) / 4) reinterpret_cast<uint32_t*>(&t)[threadIdx.x] = reinterpret_cast<const uint32_t*>(a.tensors + which)[threadIdx.x];
      __syncthreads();
      known = which;
      f.keep = fmaf(-lr, t.decay, 1.f);
      if (EIGHT) key = absorb(seed_key, t.index);
    }
    const long long b = (tile - t.first_tile) * TILE + (threadIdx.x >> 5) * BLOCK;
    if (b < t.count) {
      if (t.vectors && b + BLOCK <= t.count) step_block<PT, GT, EIGHT, MASTER, true>(a, t, f, key, b);
      else step_block_by_element<PT, GT, EIGHT, MASTER>(a, t, f, key, b);
    }
  }
}

// f(tags of the parameters' and the gradients' type, of the states' kind): tensors are stepped by kind, a launch each.
constexpr int KINDS = 36;
inline int kind_of(int32_t p, int32_t g, bool eight, bool master) { return ((master * 2 + eight) * 3 + p) * 3 + g; }
template <class F>
void with_kind(int kind, F f) {
  with_row_type(kind / 3 % 3, [&](auto pt) {
    return with_row_type(kind % 3, [&](auto gt) {
      const auto with = [&](auto master) { if (kind / 9 % 2) f(pt, gt, std::true_type(), master); else f(pt, gt, std::false_type(), master); };
      if constexpr (sizeof(typename decltype(pt)::type) == 2) { if (kind >= 18) { with(std::true_type()); return 0; } }
      with(std::false_type());
      return 0;
    });
  });
}

struct Interval { uintptr_t begin, end; };

}  // namespace

struct taurus_adamw {
  int device = 0, sms = 0;
  Tensor* tensors = nullptr;                     // device memory, with the tiles' tensors behind them
  int32_t* tile_tensor[KINDS] = {};
  long long tiles[KINDS] = {};
  int resident[KINDS] = {};                      // blocks of an SM
  std::vector<Interval> written;                 // sorted
};

namespace {

bool touches(const std::vector<Interval>& v, const void* p, size_t bytes) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  if (!p || !bytes) return false;
  const auto at = std::lower_bound(v.begin(), v.end(), b, [](const Interval& i, uintptr_t x) { return i.end <= x; });
  return at != v.end() && at->begin < b + bytes;
}

int adamw_create(taurus_adamw** out, const taurus_adamw_tensor* list, int64_t count) {
  std::vector<Tensor> tensors;
  std::vector<int32_t> tiles[KINDS];
  long long all = 0;
  std::vector<Interval> written, read;
  tensors.reserve((size_t)count);
  for (int64_t k = 0; k < count; ++k) {
    const taurus_adamw_tensor& c = list[k];
    const int ps = row_type_size(c.param_type), gsz = row_type_size(c.grad_type);
    const bool eight = c.state_type == TAURUS_E4M3;
    if (!ps || !gsz || (!eight && c.state_type != TAURUS_F32) || c.count < 0 || c.count > (1ll << 40) || !(std::fabs(c.weight_decay) < INFINITY) || (c.master && c.param_type == TAURUS_F32))
      return TAURUS_ERR_INVALID_ARG;
    if (c.count == 0 || !c.grad) continue;       // left alone
    if (!c.param || !c.m || !c.v || (eight && (!c.m_scale || !c.v_scale))) return TAURUS_ERR_INVALID_ARG;
    const size_t n = (size_t)c.count, blocks = (n + BLOCK - 1) / BLOCK, ss = eight ? 1 : 4;
    const struct { const void* p; size_t bytes; int align; bool out; } arrays[] = {
        {c.param, n * ps, ps, true}, {c.m, n * ss, (int)ss, true}, {c.v, n * ss, (int)ss, true}, {eight ? c.m_scale : nullptr, blocks * 4, 4, true},
        {eight ? c.v_scale : nullptr, blocks * 4, 4, true}, {c.master, n * 4, 4, true}, {c.grad, n * gsz, gsz, false}};
    for (const auto& x : arrays) {
      if (!x.p) continue;
      if (!rows_aligned(x.p, x.align)) return TAURUS_ERR_INVALID_ARG;
      (x.out ? written : read).push_back({reinterpret_cast<uintptr_t>(x.p), reinterpret_cast<uintptr_t>(x.p) + x.bytes});
    }
    Tensor t = {};
    t.p = c.param; t.g = c.grad; t.m = c.m; t.v = c.v; t.m_scale = c.m_scale; t.v_scale = c.v_scale; t.master = c.master; t.count = c.count;
    t.decay = c.weight_decay; t.p_type = c.param_type; t.g_type = c.grad_type; t.index = (uint32_t)k;
    t.vectors = rows_aligned(c.param, 16) && rows_aligned(c.grad, 16) && rows_aligned(c.m, eight ? 8 : 16) && rows_aligned(c.v, eight ? 8 : 16) && (!c.master || rows_aligned(c.master, 16));
    std::vector<int32_t>& mine = tiles[kind_of(c.param_type, c.grad_type, eight, c.master != nullptr)];
    t.first_tile = (long long)mine.size();
    const long long more = (c.count + TILE - 1) / TILE;
    all += more;
    if (all > (1ll << 30)) return TAURUS_ERR_UNSUPPORTED;
    mine.insert(mine.end(), (size_t)more, (int32_t)tensors.size());
    tensors.push_back(t);
  }
  // What is written shares no byte with anything else.
  std::sort(written.begin(), written.end(), [](const Interval& x, const Interval& y) { return x.begin < y.begin; });
  for (size_t i = 1; i < written.size(); ++i) if (written[i].begin < written[i - 1].end) return TAURUS_ERR_INVALID_ARG;
  for (const Interval& r : read) if (touches(written, reinterpret_cast<const void*>(r.begin), r.end - r.begin)) return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  for (const std::vector<Interval>* all : {&written, &read})
    for (const Interval& i : *all) if (!rows_on_device(reinterpret_cast<const void*>(i.begin), dev)) return TAURUS_ERR_INVALID_ARG;

  taurus_adamw* h = new taurus_adamw;
  h->device = dev; h->sms = sms;
  h->written.swap(written);
  const size_t tb = (tensors.size() * sizeof(Tensor) + 255) / 256 * 256;
  UploadPart parts[1 + KINDS];
  int count_parts = 0;
  cudaError_t e = cudaSuccess;
  if (!tensors.empty()) {
    char* mem = nullptr;
    e = cudaMalloc(reinterpret_cast<void**>(&mem), tb + (size_t)all * 4);
    if (e == cudaSuccess) {
      h->tensors = reinterpret_cast<Tensor*>(mem);
      parts[count_parts++] = {h->tensors, tensors.data(), tensors.size() * sizeof(Tensor)};
    }
    int32_t* at = reinterpret_cast<int32_t*>(mem + tb);
    for (int k = 0; k < KINDS && e == cudaSuccess; ++k) {
      h->tiles[k] = (long long)tiles[k].size();
      if (!h->tiles[k]) continue;
      h->tile_tensor[k] = at;
      at += h->tiles[k];
      parts[count_parts++] = {h->tile_tensor[k], tiles[k].data(), tiles[k].size() * 4};
      with_kind(k, [&](auto pt, auto gt, auto eight, auto master) {
        using PT = typename decltype(pt)::type;
        using GT = typename decltype(gt)::type;
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&h->resident[k], adamw_kernel<PT, GT, decltype(eight)::value, decltype(master)::value>, THREADS, 0);
      });
    }
    if (e == cudaSuccess)
      e = upload(parts, count_parts, [](const UploadPart& p) { return cudaMemcpyAsync(p.to, p.from, p.bytes, cudaMemcpyHostToDevice, cudaStreamLegacy); },
                 [] { return cudaStreamSynchronize(cudaStreamLegacy); });
  }
  if (e != cudaSuccess) {
    taurus_note_cuda_error(e, "taurus_adamw_create");
    if (h->tensors) cudaFree(h->tensors);
    delete h;
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? TAURUS_ERR_NOMEM : TAURUS_ERR_CUDA;
  }
  *out = h;
  return TAURUS_OK;
}

}  // namespace

extern "C" int taurus_adamw_create(taurus_adamw** out, const taurus_adamw_tensor* tensors, int64_t count) {
  if (!out || count < 0 || count >= (1ll << 31) || (count > 0 && !tensors)) return TAURUS_ERR_INVALID_ARG;
  try {
    return adamw_create(out, tensors, count);
  } catch (const std::bad_alloc&) {
    return TAURUS_ERR_NOMEM;
  } catch (...) {
    return TAURUS_ERR_INTERNAL;
  }
}

extern "C" int taurus_adamw_step(taurus_adamw* h, const int64_t* step, const float* lr, double beta1, double beta2, double eps, const float* grad_scale, uint64_t seed,
                                 int32_t* status, void* cuda_stream) {
  if (!h || !step || !lr || !rows_aligned(step, 8) || !rows_aligned(lr, 4) || !rows_aligned(grad_scale, 4) || !rows_aligned(status, 4) || !(beta1 >= 0.0 && beta1 < 1.0) ||
      !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.f && (float)eps < INFINITY))
    return TAURUS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  if (!rows_current_device(&dev, &sms)) return TAURUS_ERR_CUDA;
  if (dev != h->device) return TAURUS_ERR_INVALID_ARG;
  const Region outs[] = {region_of(status, 4)};
  const Region ins[] = {region_of(step, 8), region_of(lr, 4), region_of(grad_scale, 4)};
  if (!regions_on_device(outs, dev) || !regions_on_device(ins, dev) || !regions_apart(outs, ins)) return TAURUS_ERR_INVALID_ARG;
  if (touches(h->written, status, 4) || touches(h->written, step, 8) || touches(h->written, lr, 4) || touches(h->written, grad_scale, 4)) return TAURUS_ERR_INVALID_ARG;
  Launches enqueue = {static_cast<cudaStream_t>(cuda_stream)};
  Args a = {};
  a.tensors = h->tensors; a.step = reinterpret_cast<const long long*>(step); a.lr = lr; a.grad_scale = grad_scale;
  a.beta1 = (float)beta1; a.rest1 = (float)(1.0 - beta1); a.beta2 = (float)beta2; a.rest2 = (float)(1.0 - beta2); a.up = (float)eps < 0x1p-100f ? 0x1p24f : 1.f; a.eps = (float)eps * a.up; a.small_eps = eps < 1e-11;
  a.log_beta1 = std::log(beta1); a.log_beta2 = std::log(beta2); a.seed = seed; a.status = status;
  for (int k = 0; k < KINDS; ++k) {
    if (!h->tiles[k]) continue;
    a.tile_tensor = h->tile_tensor[k]; a.tiles = h->tiles[k];
    const dim3 grid((unsigned)std::min<long long>(a.tiles, (long long)h->sms * std::max(h->resident[k], 1)));
    enqueue.early = false;                       // the kernels do not wait for one another: they touch different tensors, in stream order
    with_kind(k, [&](auto pt, auto gt, auto eight, auto master) {
      using PT = typename decltype(pt)::type;
      using GT = typename decltype(gt)::type;
      enqueue(adamw_kernel<PT, GT, decltype(eight)::value, decltype(master)::value>, grid, THREADS, 0, a);
    });
  }
  return enqueue.done("taurus_adamw_step");
}

extern "C" void taurus_adamw_destroy(taurus_adamw* h) {
  if (!h) return;
  if (h->tensors) {
    // A list may go at any time, in a program with a garbage collector also while a stream is being captured, in this thread or another: memory may be freed then by a thread that says so, and
    // the capture stays valid.
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    cudaThreadExchangeStreamCaptureMode(&mode);
    if (cudaFree(h->tensors) != cudaSuccess) cudaGetLastError();
    cudaThreadExchangeStreamCaptureMode(&mode);
  }
  delete h;
}
