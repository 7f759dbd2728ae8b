// One AdamW step over many tensors at once, with states in 32 bits or in 8.
//
//   g = s grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p - lr wd p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bytes bound it: 28 an element with everything in fp32, 10.06 with parameters and gradients in 16 bits and states in 8.  All tensors are cut into tiles of 2 048
// elements, which the blocks of one launch take in turn: a tensor costs no launch, and its description and a tile's tensor are read from device memory.
//
// States in 8 bits: m and r = sqrt(v) as e4m3 codes times a power of two for each 256 elements, one warp's.  With the scale the largest code is in [2^7, 2^8), the
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
  double log_beta1, log_beta2;
  unsigned long long seed;
  int32_t* status;
};

__device__ __forceinline__ unsigned long long mix64(unsigned long long z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
__device__ __forceinline__ unsigned long long absorb(unsigned long long h, unsigned long long x) { return mix64(h ^ (0x9E3779B97F4A7C15ull * (x + 1))); }
// 32 bits for element i: the published finaliser lowbias32 (Wellons).
__device__ __forceinline__ uint32_t element_bits(unsigned long long key, long long i) {
  uint32_t x = ((uint32_t)i ^ (uint32_t)key) + (uint32_t)(key >> 32) + (uint32_t)(i >> 32) * 0x85EBCA6Bu;
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

// 8 elements as they lie in memory.
struct Raw { uint4 a, b; };
__device__ __forceinline__ Raw load_raw(const void* p, long long i, int type) {
  Raw r;
  const char* const at = static_cast<const char*>(p) + i * (type == TAURUS_F32 ? 4 : 2);
  r.a = __ldcs(reinterpret_cast<const uint4*>(at));
  r.b = type == TAURUS_F32 ? __ldcs(reinterpret_cast<const uint4*>(at) + 1) : make_uint4(0, 0, 0, 0);
  return r;
}
__device__ __forceinline__ float load_one(const void* p, long long i, int type) {
  if (type == TAURUS_F32) return static_cast<const float*>(p)[i];
  if (type == TAURUS_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
  return to_f32(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_one(void* p, long long i, int type, float x) {
  if (type == TAURUS_F32) static_cast<float*>(p)[i] = x;
  else if (type == TAURUS_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(x);
  else static_cast<__half*>(p)[i] = from_f32<__half>(x);
}
__device__ __forceinline__ void raw_to_f32(const Raw& r, int type, float (&x)[E]) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  if (type == TAURUS_F32) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = __uint_as_float(w[e]);
  } else if (type == TAURUS_BF16) {
#pragma unroll
    for (int e = 0; e < E; e += 2) { x[e] = __uint_as_float(w[e / 2] << 16); x[e + 1] = __uint_as_float(w[e / 2] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[e / 2]));
      x[e] = f.x; x[e + 1] = f.y;
    }
  }
}
__device__ __forceinline__ void store_vector(void* p, long long i, int type, const float (&x)[E]) {
  if (type == TAURUS_F32) store_f32_once<float, E>(static_cast<float*>(p) + i, x);
  else if (type == TAURUS_BF16) store_f32_once<__nv_bfloat16, E>(static_cast<__nv_bfloat16*>(p) + i, x);
  else store_f32_once<__half, E>(static_cast<__half*>(p) + i, x);
}

__device__ __forceinline__ void codes_to_f32(uint2 c, float scale, float (&x)[E]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[e / 4] >> (8 * (e & 2))), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    x[e] = f.x * scale; x[e + 1] = f.y * scale;
  }
}
// |x| below 2^8 as an e4m3 code, up with the probability of what is cut off: bits are added below the three that stay.  Below 2^-6 the step is 2^-9: with
// 2^-6 added (rounded down, as is everything behind the last place of the sum) those values have the same three bits.
__device__ __forceinline__ uint32_t code_of(float q, uint32_t bits16) {
  const bool low = q < 0x1p-6f;
  const float y = low ? __fadd_rz(q, 0x1p-6f) : q;
  return ((__float_as_uint(y) + (bits16 << 4)) >> 20) - (low ? 121u * 8 : 120u * 8);
}
constexpr uint32_t NOT_FINITE = 0x7f800000u, CODE_NAN = 0x7f;

template <bool EIGHT>
__global__ void __launch_bounds__(THREADS) adamw_kernel(const Args a) {
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
  const int lane = threadIdx.x & 31;
  unsigned long long seed_key = 0, key = 0;
  if (EIGHT) seed_key = absorb(absorb(0x243F6A8885A308D3ull, a.seed), (unsigned long long)step);
  int known = -1;
  Tensor t;
  for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int which = a.tile_tensor[tile];
    if (which != known) {
      t = a.tensors[which];
      known = which;
      if (EIGHT) key = absorb(seed_key, t.index);
    }
    const long long i = (tile - t.first_tile) * TILE + threadIdx.x * E;
    const int left = (int)(t.count - i < E ? t.count - i : E);          // (0 or less: none)
    const bool whole = t.vectors && left == E;
    float p[E], g[E], m[E], v[E];
    float ms = 0.f, vs = 0.f;
    if (EIGHT && left > 0) { ms = t.m_scale[i / BLOCK]; vs = t.v_scale[i / BLOCK]; }
    if (whole) {
      const Raw rg = load_raw(t.g, i, t.g_type), rp = t.master ? load_raw(t.master, i, TAURUS_F32) : load_raw(t.p, i, t.p_type);
      if (EIGHT) {
        const uint2 cm = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + i)), cv = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + i));
        codes_to_f32(cm, ms, m);
        codes_to_f32(cv, vs, v);
      } else {
        const Raw rm = load_raw(t.m, i, TAURUS_F32), rv = load_raw(t.v, i, TAURUS_F32);
        raw_to_f32(rm, TAURUS_F32, m);
        raw_to_f32(rv, TAURUS_F32, v);
      }
      raw_to_f32(rg, t.g_type, g);
      raw_to_f32(rp, t.master ? TAURUS_F32 : t.p_type, p);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        p[e] = g[e] = m[e] = v[e] = 0.f;
        if (e < left) {
          g[e] = load_one(t.g, i + e, t.g_type);
          p[e] = t.master ? t.master[i + e] : load_one(t.p, i + e, t.p_type);
          if (EIGHT) {
            __nv_fp8_e4m3 c;
            c.__x = static_cast<const uint8_t*>(t.m)[i + e]; m[e] = (float)c * ms;
            c.__x = static_cast<const uint8_t*>(t.v)[i + e]; v[e] = (float)c * vs;
          } else {
            m[e] = static_cast<const float*>(t.m)[i + e];
            v[e] = static_cast<const float*>(t.v)[i + e];
          }
        }
      }
    }
    float root[E];
    const float keep = fmaf(-lr, t.decay, 1.f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float ge = a.grad_scale ? g[e] * gs : g[e];
      m[e] = __fadd_rn(__fmul_rn(a.beta1, m[e]), __fmul_rn(a.rest1, ge));
      if (EIGHT) v[e] = __fmul_rn(v[e], v[e]);
      v[e] = __fadd_rn(__fmul_rn(a.beta2, v[e]), __fmul_rn(__fmul_rn(a.rest2, ge), ge));
      asm("sqrt.approx.f32 %0, %1;" : "=f"(root[e]) : "f"(v[e]));
      p[e] = fmaf(-lr, __fdividef(m[e] * c1, fmaf(root[e], c2, a.eps)), p[e] * keep);
    }
    if (whole) {
      store_vector(t.p, i, t.p_type, p);
      if (t.master) store_vector(t.master, i, TAURUS_F32, p);
      if (!EIGHT) {
        store_vector(t.m, i, TAURUS_F32, m);
        store_vector(t.v, i, TAURUS_F32, v);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < left) {
          store_one(t.p, i + e, t.p_type, p[e]);
          if (t.master) t.master[i + e] = p[e];
          if (!EIGHT) { static_cast<float*>(t.m)[i + e] = m[e]; static_cast<float*>(t.v)[i + e] = v[e]; }
        }
    }
    if (EIGHT) {
      uint32_t most_m = 0, most_v = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t bm = __float_as_uint(m[e]) & 0x7fffffffu, bv = __float_as_uint(v[e]);
        if (bm < NOT_FINITE) most_m = max(most_m, bm);
        if (bv < NOT_FINITE) most_v = max(most_v, bv);                 // (v is never negative)
      }
      most_m = __reduce_max_sync(0xffffffffu, most_m);
      most_v = __reduce_max_sync(0xffffffffu, most_v);
      // The whole part of the largest one's logarithm, down by 7; of sqrt(v) half of v's.
      const int em = (int)max(most_m >> 23, 8u) - 7, ev = (((int)max(most_v >> 23, 1u) - 127) >> 1) + 120;
      const float inv_m = __uint_as_float((uint32_t)(254 - em) << 23), inv_v = __uint_as_float((uint32_t)(254 - ev) << 23);
      uint32_t cm[E], cv[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t bits = element_bits(key, i + e), bm = __float_as_uint(m[e]);
        const uint32_t c = code_of(fabsf(m[e]) * inv_m, bits & 0xffff) | ((bm >> 24) & 0x80u), d = code_of(root[e] * inv_v, bits >> 16);
        cm[e] = (bm & 0x7fffffffu) < NOT_FINITE ? c : CODE_NAN;
        cv[e] = __float_as_uint(v[e]) < NOT_FINITE ? (v[e] > 0.f ? max(d, 1u) : 0u) : CODE_NAN;
      }
      if (left > 0 && lane == 0) {
        t.m_scale[i / BLOCK] = __uint_as_float((uint32_t)em << 23);
        t.v_scale[i / BLOCK] = __uint_as_float((uint32_t)ev << 23);
      }
      if (whole) {
        const auto four = [](const uint32_t* c) { return c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24); };
        __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + i), make_uint2(four(cm), four(cm + 4)));
        __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + i), make_uint2(four(cv), four(cv + 4)));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e < left) { static_cast<uint8_t*>(t.m)[i + e] = (uint8_t)cm[e]; static_cast<uint8_t*>(t.v)[i + e] = (uint8_t)cv[e]; }
      }
    }
  }
}

struct Interval { uintptr_t begin, end; };

}  // namespace

struct taurus_adamw {
  int device = 0, sms = 0;
  Tensor* tensors = nullptr;                     // device memory, with the tiles' tensors behind them
  int32_t* tile_tensor[2] = {nullptr, nullptr};  // by state: fp32, 8 bits
  long long tiles[2] = {0, 0};
  int resident[2] = {1, 1};                      // blocks of an SM
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
  std::vector<int32_t> tiles[2];
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
    std::vector<int32_t>& mine = tiles[eight];
    t.first_tile = (long long)mine.size();
    const long long more = (c.count + TILE - 1) / TILE;
    if ((long long)tiles[0].size() + (long long)tiles[1].size() + more > (1ll << 30)) return TAURUS_ERR_UNSUPPORTED;
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
  const size_t tb = (tensors.size() * sizeof(Tensor) + 255) / 256 * 256, b0 = (tiles[0].size() * 4 + 255) / 256 * 256, b1 = tiles[1].size() * 4;
  cudaError_t e = cudaSuccess;
  if (!tensors.empty()) {
    char* mem = nullptr;
    e = cudaMalloc(reinterpret_cast<void**>(&mem), tb + b0 + b1);
    if (e == cudaSuccess) {
      h->tensors = reinterpret_cast<Tensor*>(mem);
      h->tile_tensor[0] = reinterpret_cast<int32_t*>(mem + tb);
      h->tile_tensor[1] = reinterpret_cast<int32_t*>(mem + tb + b0);
      e = cudaMemcpy(h->tensors, tensors.data(), tensors.size() * sizeof(Tensor), cudaMemcpyHostToDevice);
    }
    for (int k = 0; k < 2; ++k) {
      h->tiles[k] = (long long)tiles[k].size();
      if (e == cudaSuccess && h->tiles[k]) e = cudaMemcpy(h->tile_tensor[k], tiles[k].data(), tiles[k].size() * 4, cudaMemcpyHostToDevice);
    }
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&h->resident[0], adamw_kernel<false>, THREADS, 0);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&h->resident[1], adamw_kernel<true>, THREADS, 0);
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
  a.beta1 = (float)beta1; a.rest1 = (float)(1.0 - beta1); a.beta2 = (float)beta2; a.rest2 = (float)(1.0 - beta2); a.eps = (float)eps;
  a.log_beta1 = std::log(beta1); a.log_beta2 = std::log(beta2); a.seed = seed; a.status = status;
  for (int k = 0; k < 2; ++k) {
    if (!h->tiles[k]) continue;
    a.tile_tensor = h->tile_tensor[k]; a.tiles = h->tiles[k];
    const dim3 grid((unsigned)std::min<long long>(a.tiles, (long long)h->sms * std::max(h->resident[k], 1)));
    enqueue.early = false;                       // the kernels do not wait for one another: they touch different tensors, in stream order
    if (k == 0) enqueue(adamw_kernel<false>, grid, THREADS, 0, a);
    else enqueue(adamw_kernel<true>, grid, THREADS, 0, a);
  }
  return enqueue.done("taurus_adamw_step");
}

extern "C" void taurus_adamw_destroy(taurus_adamw* h) {
  if (!h) return;
  if (h->tensors) cudaFree(h->tensors);
  delete h;
}
