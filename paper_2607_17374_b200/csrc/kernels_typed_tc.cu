// Products by vertex type on the 5th-generation tensor cores.  One kernel, three products:
//   PROJECT   out[r]    = x[r] W[g] + bias[g]        rows of x are K-major A tiles, W is an MN-major B tile
//   GRAD_X    grad_x[r] = grad_out[r] W[g]^T         rows of grad_out are K-major A tiles, W is a K-major B tile
//   GRAD_W    grad_W[g] = x_g^T grad_out_g           both are MN-major: the rows are what is summed over
//
// Persistent: one CTA per SM walks units, a unit is a 128-row tile of the output of one type and a block of up to BN columns (GRAD_W: 128 rows of
// grad_W[g] and a block of columns, over one chunk of the type's rows; a type of several chunks leaves one partial product a chunk, which
// typed_join_kernel adds up in their order).  Which units there are follows from the offsets in device memory: every CTA works it out for itself.
// Roles:  warp 0       TMA: operands that stand in memory as the tensor core takes them
//         warp 1       tcgen05.mma, accumulators in TMEM, two slots of 256 columns: the epilogue of a unit runs beside the products of the next.  (Where two sums
//                      of more than 128 columns are kept, fp32 rows and 16-bit grad_W, there is one slot, and they take turns.)
//         warps 2..9   epilogue, two to a quadrant of TMEM lanes: TMEM -> registers -> transposed through shared memory -> rows
//         warps 10..17 loaders (LOADED): operands that have to be split, or whose rows TMA cannot address; without loaders, in GRAD_W, they add up the
//                      columns of grad_out for the bias, which the loaders do on the way
//
// fp32 operands: x = hi + mid + lo, three bf16 values that hold its 24 bits (typed.cuh), and six of the nine products: hi hi into one accumulator,
// hi mid + mid hi + mid mid + hi lo + lo hi into another.  What is left out is below 2^-24 of a product, what rounding it to fp32 would cost.
// Each element keeps an exponent of its own, whatever stands beside it; one below 2^-110 is off by up to 2^-133, one below 2^-134 counts as zero (also times an infinity).
// Two accumulators: where hi hi is not finite the sum is what it says (an infinity times a mid or lo of zero would make it NaN).  hi may be larger than x, by 2^-8: where
// products' magnitudes add up to more than (1 - 2^-7) times the largest fp32 value the sum may be infinite.  W is split by a kernel in front (it is read once per tile), rows by the loaders.
//
// What bounds it (1.2 M rows, 512 -> 256 bf16: 359 us replayed on the same inputs, 433 with new ones each pass, 5.1 and 4.3 TB/s of rows): the L2, which gives every 128 rows
// the whole of W's block again, 3 KB a row, 10 TB/s; DRAM at 60 %, the tensor core at 44 %.  fp32 (400 000 rows, 256 -> 256): 299 us forward and 288 for grad_x, 196 of them the six
// products; the output of a block of 256 columns waits for its accumulators and they for it.  grad_W 468 to 514: the loaders' split of both operands.
//
// Every wait is bounded, as in the projection of the layers: a CTA that gives up records TAURUS_ERR_INTERNAL, waits (bounded) for its copies and
// products in flight, frees its TMEM and returns.  Every TMA load is a plain load of the issuing CTA alone.
#include <cuda.h>

#include <algorithm>

#include "stage_waits.h"
#include "typed.cuh"

namespace {

enum { PROJECT = 0, GRAD_X = 1, GRAD_W = 2 };

constexpr int BM = 128, MAX_STAGES = 4, MAX_G = TAURUS_MAX_TYPES;
constexpr unsigned WAIT_LIMIT = 1u << 24;

// Shapes of the kernel.  BK: columns (rows, in GRAD_W) of a stage; BN: columns of a block at most.  fp32: part of the operands' shared memory is a ring of rows as
// they were read, which the loaders fill ahead of the tensor core.  GRAD_W splits both operands, and 16 warps share that (8: 651 us for 400 000 rows of 256 and
// 256, 16: 555); with rows, where one block of 256 columns splits each row once, four warps fewer at the output cost more than eight more loaders bring.
template <class T, int KIND, bool LOADED>
struct Shape {
  static constexpr bool SPLIT = sizeof(T) == 4;
  static constexpr int NP = SPLIT ? 3 : 1, BK = SPLIT ? 32 : 64, BN = SPLIT ? (KIND == GRAD_W ? 128 : 256) : LOADED ? 128 : 256;
  static constexpr int EPI_WARPS = SPLIT && KIND == GRAD_W ? 4 : 8, LOAD_WARPS = SPLIT && KIND == GRAD_W ? 16 : 8;
  static constexpr int PLANE_A = BM * BK * 2, PLANE_B = BN * BK * 2, STAGE_BYTES = NP * (PLANE_A + PLANE_B);
  static constexpr int STAGES = SPLIT ? 2 : 4;
  static constexpr int EPI_ROW = SPLIT && KIND != GRAD_W ? 128 : 64;       // bytes of a row that a warp of the epilogue transposes at a time
  static constexpr int RAW_BYTES = SPLIT ? (KIND == GRAD_W ? 2 : 1) * BM * BK * 4 : 0, RAW_DEPTH = SPLIT ? (KIND == GRAD_W ? 3 : 2) : 0;
  // Loaders, or in GRAD_W those who add up the columns of grad_out.
  static constexpr int THREADS = 32 * (2 + EPI_WARPS + (LOADED || KIND == GRAD_W ? LOAD_WARPS : 0));
  static constexpr int OPERAND_BYTES = STAGES * STAGE_BYTES + RAW_DEPTH * RAW_BYTES;
  static constexpr int SHARED_BYTES = OPERAND_BYTES + EPI_WARPS * 32 * EPI_ROW + LOAD_WARPS * 128 * 4;      // + Shared
};

struct __align__(16) Shared {
  unsigned long long full[MAX_STAGES], empty[MAX_STAGES], acc_full[2], acc_empty[2], sums;
  unsigned tmem_base;
  int abort_flag, loads, mmas;
  int begin[MAX_G + 1];       // rows of type g: [begin[g], begin[g + 1]) (the types' rows follow one another)
  int prefix[MAX_G + 1];      // units (row tiles, chunks) in front of type g
  int slot[MAX_G + 1];        // GRAD_W: partial products in front of type g
};
struct TcArgs {
  long long n;
  const long long* offsets;
  int types;
  int M, N, Kc;               // GRAD_W: rows of grad_W (M), columns (N); else columns of the output (N), length of the sums (Kc)
  int bn, n_blocks, m_blocks; // columns of a block; blocks of columns; GRAD_W: blocks of rows
  int chunk;                  // GRAD_W: rows of a chunk
  const void *a, *b;          // LOADED: rows of A; GRAD_W: rows of B too
  long long lda, ldb;
  int a_vec, b_vec;           // elements, at most four, that the rows are aligned to (fp32: four or not)
  void* out;
  long long ld_out;           // PROJECT, GRAD_X
  int out_f32;                // the output is fp32, else of the operands' type
  int out_vec;                // 16 bytes of columns at a time
  const float* bias;
  float* db;                  // GRAD_W: gradient of the bias
  float* part;                // GRAD_W: [slots x (M + 1) x N]
  int32_t* status;
};

// ---------------------------------------------------------------------------------------------------------------- PTX
__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(unsigned long long* bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned long long* bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(unsigned long long* bar, unsigned parity) {
  unsigned ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait(unsigned long long* bar, unsigned parity, volatile int* abort_flag) {
  for (unsigned i = 0; i < WAIT_LIMIT; ++i) {
    if (mbar_try(bar, parity)) return true;
    if ((i & 63u) == 63u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool mbar_wait_warp(unsigned long long* bar, unsigned parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ void tma_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
// K-major operand: rows of ROW bytes (128- or 64-byte swizzle), groups of 8 rows behind one another.
template <int ROW>
__device__ __forceinline__ unsigned long long desc_k(unsigned addr) {
  static_assert(ROW == 128 || ROW == 64, "operand rows of 128 or 64 bytes");
  return (unsigned long long)((addr & 0x3FFFFu) >> 4) | 1ull << 16 | (unsigned long long)((8 * ROW) >> 4) << 32 | 1ull << 46 | (ROW == 128 ? 2ull : 4ull) << 61;
}
// MN-major operand: rows of 64 elements (128 bytes, 128-byte swizzle), one for each index that is summed over, in groups of 8; the next 64
// elements of the other index `block` bytes on.
__device__ __forceinline__ unsigned long long desc_mn(unsigned addr, unsigned block) {
  return (unsigned long long)((addr & 0x3FFFFu) >> 4) | (unsigned long long)(block >> 4) << 16 | (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ void umma(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// One lane of the (converged) warp, known as such to the compiler: MMA operands stay in uniform registers.
__device__ __forceinline__ bool elected() {
  unsigned p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
// 16 columns of an accumulator, one row per lane.
__device__ __forceinline__ void tmem_ld16(unsigned (&v)[16], unsigned taddr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16, 8 or 4 bytes from global to shared memory, of which the first `bytes` are read and the others zeros.
__device__ __forceinline__ void copy16(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(unsigned dst, const void* src, unsigned bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------------------------- units
// Fills begin, prefix and slot; false (for every thread of every CTA) when the offsets are not what they have to be.
template <int KIND>
__device__ __forceinline__ bool plan(const TcArgs& a, Shared* s) {
  bool bad = false;
  for (int g = threadIdx.x; g <= a.types; g += blockDim.x) {
    const long long b = a.offsets[g], e = g < a.types ? a.offsets[g + 1] : a.n;
    bad |= b < 0 || b > a.n || e > a.n || e < b;
    s->begin[g] = (int)b;
  }
  if (__syncthreads_or(bad)) return false;
  if (threadIdx.x < 32) {
    int units = 0, slots = 0;
    for (int g0 = 0; g0 <= a.types; g0 += 32) {
      const int g = g0 + threadIdx.x, len = g < a.types ? s->begin[g + 1] - s->begin[g] : 0;
      int u = 0, p = 0;
      if (g < a.types) {
        if (KIND == GRAD_W) { u = len > 0 ? (int)(((unsigned)len + a.chunk - 1) / a.chunk) : 1; p = u > 1 ? u : 0; }
        else u = (int)(((unsigned)len + BM - 1) / BM);                             // (unsigned: a type may have 2^31 - 1 rows)
      }
      int iu = u, ip = p;
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, iu, o), y = __shfl_up_sync(0xffffffffu, ip, o);
        if ((int)threadIdx.x >= o) { iu += x; ip += y; }
      }
      if (g <= a.types) { s->prefix[g] = units + iu - u; s->slot[g] = slots + ip - p; }
      units += __shfl_sync(0xffffffffu, iu, 31);
      slots += __shfl_sync(0xffffffffu, ip, 31);
    }
  }
  __syncthreads();
  return true;
}

struct Unit {
  int g, row0, rows;     // type; first row of the tile (of the chunk), rows
  int m0, n0, bw;        // GRAD_W: first row of grad_W; first column of the block, columns (a multiple of 16)
  int steps;             // stages
  int slot;              // GRAD_W: partial product, -1: the result itself
};
template <int KIND, int BK>
__device__ __forceinline__ Unit unit_at(const TcArgs& a, const Shared* s, int w) {
  Unit u;
  const int per = KIND == GRAD_W ? a.m_blocks * a.n_blocks : a.n_blocks;
  const int t = w / per, b = (w + t) % per;       // (turned by one from chunk to chunk, for a CTA to meet every kind of tile: the first ones also sum up columns)
  int lo = 0, hi = a.types;                       // the type g with prefix[g] <= t < prefix[g + 1]
  while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (s->prefix[m] <= t) lo = m; else hi = m; }
  u.g = lo;
  const int nth = t - s->prefix[lo], height = KIND == GRAD_W ? a.chunk : BM;
  u.row0 = s->begin[lo] + nth * height;
  u.rows = min(height, s->begin[lo + 1] - u.row0);
  u.m0 = KIND == GRAD_W ? b / a.n_blocks * BM : 0;
  u.n0 = (KIND == GRAD_W ? b % a.n_blocks : b) * a.bn;
  u.bw = min(a.bn, (a.N - u.n0 + 15) / 16 * 16);
  u.steps = KIND == GRAD_W ? (u.rows + BK - 1) / BK : (a.Kc + BK - 1) / BK;
  u.slot = KIND == GRAD_W && s->prefix[lo + 1] - s->prefix[lo] > 1 ? s->slot[lo] + nth : -1;
  return u;
}

// ---------------------------------------------------------------------------------------------------------------- loaders
// Four neighbouring elements of a row as bf16 planes (fp32) or as they are (16 bits), 8 bytes a plane.
template <class T> struct __align__(sizeof(T) * 4) Quad { T v[4]; };

template <class T>
__device__ __forceinline__ Quad<T> load_quad(const T* row, int c, int limit, bool vec) {     // row null: zeros
  Quad<T> q;
  if (row && vec && c + 4 <= limit) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(&q) = __ldg(reinterpret_cast<const float4*>(row + c));
    else *reinterpret_cast<uint2*>(&q) = __ldg(reinterpret_cast<const uint2*>(row + c));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = row && c + i < limit ? row[c + i] : from_f32<T>(0.f);
  }
  return q;
}
// The places of a CTA's stages, in order: unit after unit, step after step.
template <int KIND, int BK>
struct Walk {
  int w, k;
  Unit u;
  __device__ __forceinline__ Walk(const TcArgs& a, const Shared* s, int units) : w(blockIdx.x), k(0) { find(a, s, units); }
  __device__ __forceinline__ void find(const TcArgs& a, const Shared* s, int units) {
    for (; w < units; w += gridDim.x) { u = unit_at<KIND, BK>(a, s, w); if (u.steps > 0) return; }
  }
  __device__ __forceinline__ bool last() const { return k + 1 == u.steps; }
  // true where another unit begins
  __device__ __forceinline__ bool next(const TcArgs& a, const Shared* s, int units) {
    if (++k < u.steps) return false;
    k = 0; w += gridDim.x;
    find(a, s, units);
    return true;
  }
};

// What a loader thread brings of a stage: quads of A, and in GRAD_W as many of B, in the same column of every DR-th row of the tile.
template <class T, int KIND>
struct Loader {
  static constexpr int LOADERS = 32 * Shape<T, KIND, true>::LOAD_WARPS, BK = Shape<T, KIND, true>::BK, QUADS = BM * BK / 4 / LOADERS;               // of an operand
  static constexpr int ROW_QUADS = KIND == GRAD_W ? 32 : BK / 4, DR = LOADERS / ROW_QUADS;
  static constexpr int ALL = KIND == GRAD_W ? 2 * QUADS : QUADS;
  static constexpr unsigned PLANE = BM * BK * 2;                                       // bytes of a plane of either operand (blocks of 128 columns)

  int r0, q;               // row of the first quad in the tile, column
  const T *pa, *pb;        // where they come from
  long long da, db;        // from a quad to the next
  int rows, cols_a, cols_b;  // rows of the tile from r0 on that there are; columns from the tile's first on

  __device__ __forceinline__ explicit Loader(int t) : r0(t / ROW_QUADS), q(t % ROW_QUADS * 4) {}
  __device__ __forceinline__ void begin(const TcArgs& a, const Unit& u) {
    const long long row = u.row0 + (long long)r0;
    rows = u.rows - r0;
    if (KIND != GRAD_W) {
      pa = static_cast<const T*>(a.a) + row * a.lda + q; da = DR * a.lda; cols_a = a.Kc;
    } else {
      pa = static_cast<const T*>(a.a) + (a.a ? row * a.lda + u.m0 + q : 0); da = DR * a.lda; cols_a = a.a ? a.M - u.m0 : 0;
      pb = static_cast<const T*>(a.b) + row * a.ldb + u.n0 + q; db = DR * a.ldb; cols_b = min(u.bw, a.N - u.n0);
    }
  }
  __device__ __forceinline__ void step(const TcArgs& a) {
    if (KIND != GRAD_W) { pa += BK; cols_a -= BK; }
    else { pa += BK * a.lda; pb += BK * a.ldb; rows -= BK; }
  }
  // f(quad, its address, elements of it that there are: 4 or fewer, perhaps none; of A?)
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
      const bool in = i * DR < rows;
      f(i, pa + i * da, in ? cols_a - q : 0, true);
      if constexpr (KIND == GRAD_W) f(QUADS + i, pb + i * db, in ? cols_b - q : 0, false);
    }
  }
  // The same elements by the warp as a whole, neighbouring lanes neighbouring elements, W at a time, for rows that are not aligned to quads:
  // f(quad group, element of the warp's 128 in it, row and column in the tile, address, elements that there are, of A?)
  template <int W, class F>
  __device__ __forceinline__ void wide(const TcArgs& a, F f) const {
    const int lane = threadIdx.x & 31, dr = lane / ROW_QUADS;
    auto operand = [&](int group, const T* p, long long ld, int cols, bool is_a) {
      p -= dr * ld + q;                                            // the warp's first row, the tile's first column
#pragma unroll
      for (int i = 0; i < QUADS; ++i)
#pragma unroll
        for (int j = 0; j < 4 / W; ++j) {
          const int e = (j * 32 + lane) * W, r = e / (4 * ROW_QUADS) + i * DR, c = e % (4 * ROW_QUADS);
          f(group + i, e, r0 - dr + r, c, p + r * ld + c, r < rows + dr ? min(max(cols - c, 0), W) : 0, is_a);
        }
    };
    operand(0, pa, a.lda, cols_a, true);
    if constexpr (KIND == GRAD_W) operand(QUADS, pb, a.ldb, cols_b, false);
  }
  // Bytes of element (r, c) of the tile behind its operand's A stage.
  static __device__ __forceinline__ unsigned place_of(int r, int c, bool is_a) {
    if constexpr (KIND != GRAD_W) return r * (BK * 2) + (((c >> 3) ^ (BK == 64 ? r & 7 : (r >> 1) & 3)) << 4) + (c & 7) * 2;
    return (is_a ? 0u : Shape<T, KIND, true>::NP * PLANE) + (c >> 6) * (BK * 128) + r * 128 + ((((c & 63) >> 3) ^ (r & 7)) << 4) + (c & 7) * 2;
  }
  // Bytes of quad i in its operand's plane.
  __device__ __forceinline__ unsigned place(int i) const {
    const int r = r0 + i % QUADS * DR, c = q >> 2;
    if constexpr (KIND != GRAD_W) return r * (BK * 2) + (((c >> 1) ^ (BK == 64 ? r & 7 : (r >> 1) & 3)) << 4) + (c & 1) * 8;
    // quad c lies in the block of 64 columns c / 16
    return (i < QUADS ? 0u : Shape<T, KIND, true>::NP * PLANE) + (c >> 4) * (BK * 128) + r * 128 + ((((c & 15) >> 1) ^ (r & 7)) << 4) + (c & 1) * 8;
  }
};

// All loader warps meet (a bounded wait, as every other): false when the CTA is aborting.
__device__ __forceinline__ bool meet(Shared* s, unsigned* phase) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(&s->sums);
  const bool ok = mbar_wait_warp(&s->sums, *phase, &s->abort_flag);
  *phase ^= 1;
  return ok;
}
// Where the sums of grad_out's columns of a unit go.
__device__ __forceinline__ float* bias_place(const TcArgs& a, const Unit& u) {
  return u.slot >= 0 ? a.part + ((long long)u.slot * (a.M + 1) + a.M) * a.N + u.n0 : a.db + (long long)u.g * a.N + u.n0;
}

// ---------------------------------------------------------------------------------------------------------------- epilogue
// PASS columns (ROW bytes of the output) of 32 rows: transposed through the warp's tile, 16-byte chunks of a row in an order of its own, and written
// in pieces of ROW bytes, several rows at a time; out: row 0, column 0 of them; rows <= 32.
template <class O, int ROW>
__device__ __forceinline__ unsigned tile_at(int r, int c) { return r * ROW + ((c ^ (ROW == 128 ? r & 7 : (r >> 1) & 3)) << 4); }
template <class O, int ROW>
__device__ __forceinline__ void put_rows(unsigned char* tile, const float* v, O* out, long long ld, int rows, int columns, bool vec) {
  constexpr int PASS = ROW / sizeof(O), PER = 16 / sizeof(O), CHUNKS = ROW / 16, AT_ONCE = 32 / CHUNKS;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    Vec<O, PER> x;
#pragma unroll
    for (int j = 0; j < PER; ++j) x.v[j] = from_f32<O>(v[c * PER + j]);
    store_vec(tile + tile_at<O, ROW>(lane, c), x);
  }
  __syncwarp();
  if (vec && columns >= PASS) {
    const int c = lane % CHUNKS, r0 = lane / CHUNKS;
    Vec<O, PER> x[CHUNKS];                              // all read before the first is written: the compiler cannot tell the two memories apart
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) x[i] = load_vec<Vec<O, PER>>(tile + tile_at<O, ROW>(i * AT_ONCE + r0, c));
    O* p = out + r0 * ld + c * PER;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      if (i * AT_ONCE + r0 < rows) store_vec(p, x[i]);
      p += AT_ONCE * ld;
    }
  } else {
    static_assert(PASS <= 32, "a lane to a column");
    constexpr int FEW = 32 / PASS, BATCH = 8;            // rows at once; of them on their way
    const int c = lane % PASS, r0 = lane / PASS;
    O* p = out + r0 * ld + c;
#pragma unroll 1
    for (int r = r0; r < rows; r += FEW * BATCH) {
      O x[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) x[i] = *reinterpret_cast<const O*>(tile + tile_at<O, ROW>((r + i * FEW) & 31, c / PER) + c % PER * sizeof(O));
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (r + i * FEW < rows && c < columns) *p = x[i];
        p += FEW * ld;
      }
    }
  }
  __syncwarp();
}

// ---------------------------------------------------------------------------------------------------------------- kernel
template <class T, int KIND, bool LOADED>
__global__ void __launch_bounds__(Shape<T, KIND, LOADED>::THREADS, 1)
typed_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ TcArgs a) {
  static_assert(LOADED || sizeof(T) == 2, "fp32 operands are split by the loaders");
  using S = Shape<T, KIND, LOADED>;
  constexpr int NP = S::NP, BK = S::BK, ROW = BK * 2, STAGES = S::STAGES, EPI_WARPS = S::EPI_WARPS, LOAD_WARPS = S::LOAD_WARPS;
  constexpr unsigned PLANE_A = S::PLANE_A, PLANE_B = S::PLANE_B, STAGE_BYTES = S::STAGE_BYTES;
  constexpr bool SUMS = KIND == GRAD_W && !LOADED;       // the last warps read the stages too
  static_assert(S::SHARED_BYTES + (int)sizeof(Shared) <= 227 * 1024, "shared memory of a block");
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* const staging = smem + S::OPERAND_BYTES;
  float* const bias_smem = reinterpret_cast<float*>(staging + EPI_WARPS * 32 * S::EPI_ROW);     // GRAD_W: sums of grad_out's columns, of each loader warp or of the second half of those who add
  Shared* const sh = reinterpret_cast<Shared*>(bias_smem + LOAD_WARPS * 128);
  volatile int* const abort_flag = &sh->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((smem_u32(smem) & 1023u) != 0) {                     // the swizzled tiles want it
    if (threadIdx.x == 0) rows_status(a.status, TAURUS_ERR_INTERNAL);
    return;
  }
  if (!plan<KIND>(a, sh)) {
    if (threadIdx.x == 0) rows_status(a.status, TAURUS_ERR_INVALID_ARG);
    return;
  }
  const int units = sh->prefix[a.types] * (KIND == GRAD_W ? a.m_blocks * a.n_blocks : a.n_blocks);
  if ((int)blockIdx.x >= units) return;
  constexpr bool TMA_A = !LOADED, TMA_B = !LOADED || KIND != GRAD_W;
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&sh->full[s], (TMA_A || TMA_B ? 1 : 0) + (LOADED ? LOAD_WARPS : 0)); mbar_init(&sh->empty[s], 1 + (SUMS ? LOAD_WARPS : 0)); }
    for (int b = 0; b < 2; ++b) { mbar_init(&sh->acc_full[b], 1); mbar_init(&sh->acc_empty[b], EPI_WARPS); }
    mbar_init(&sh->sums, LOAD_WARPS);
    sh->abort_flag = 0; sh->loads = 0; sh->mmas = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const unsigned tmem_base = sh->tmem_base;
  // accumulators: two slots of 256 columns, or with two sums of more than 128 columns one slot.  PAIR: the stages' products go into the two in turn; the tensor core's
  // sums are cut off, and half as long they lose half as much (16-bit rows, fp32 grad_W: 3.1e-6 of the result in chunks of 4 096 rows, fp32 sums 3e-7).
  constexpr bool PAIR = NP == 1 && KIND == GRAD_W;
  const int slots = (NP == 3 || PAIR) && a.bn > 128 ? 1 : 2, second = slots == 1 ? 256 : 128;
  const unsigned operands = smem_u32(smem);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA
    if ((TMA_A || TMA_B) && lane == 0) {
      int it = 0;
      for (int w = blockIdx.x; w < units && !*abort_flag; w += gridDim.x) {
        const Unit u = unit_at<KIND, BK>(a, sh, w);
        const int boxes_n = (u.bw + 63) / 64;
        bool ok = true;
        for (int k = 0; k < u.steps; ++k, ++it) {
          const int s = it % STAGES;
          if (it >= STAGES && !mbar_wait(&sh->empty[s], (it / STAGES & 1) ^ 1, abort_flag)) { ok = false; break; }
          const unsigned st = operands + s * STAGE_BYTES, sb = st + NP * PLANE_A;
          unsigned long long* const bar = &sh->full[s];
          const unsigned bytes_a = TMA_A && (KIND != GRAD_W || a.out) ? PLANE_A : 0;      // (no grad_W: only the columns of grad_out count)
          const unsigned bytes_b = KIND == GRAD_X ? NP * a.bn * ROW : NP * boxes_n * (BK * 128);
          mbar_expect_tx(bar, bytes_a + bytes_b);
          if (bytes_a) {
            if (KIND == GRAD_W) {
              tma_2d(st, &map_a, u.m0, u.row0 + k * BK, bar);
              tma_2d(st + BK * 128, &map_a, u.m0 + 64, u.row0 + k * BK, bar);      // (behind the last column: zeros)
            } else {
              tma_2d(st, &map_a, k * BK, u.row0, bar);
            }
          }
          if (KIND == GRAD_W) {
            for (int j = 0; j < boxes_n; ++j) tma_2d(sb + j * (BK * 128), &map_b, u.n0 + j * 64, u.row0 + k * BK, bar);
          } else if (KIND == PROJECT) {
            for (int p = 0; p < NP; ++p)
              for (int j = 0; j < boxes_n; ++j) tma_3d(sb + p * PLANE_B + j * (BK * 128), &map_b, u.n0 + j * 64, k * BK, u.g * NP + p, bar);
          } else {
            for (int p = 0; p < NP; ++p) tma_3d(sb + p * PLANE_B, &map_b, k * BK, u.n0, u.g * NP + p, bar);
          }
        }
        if (!ok) break;
      }
      sh->loads = it;
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    int it = 0, nth = 0;
    for (int w = blockIdx.x; w < units; w += gridDim.x) {
      const Unit u = unit_at<KIND, BK>(a, sh, w);
      if (u.steps == 0) continue;
      const int buf = slots == 2 ? nth & 1 : 0;
      if (nth >= slots && !mbar_wait_warp(&sh->acc_empty[buf], ((slots == 2 ? nth >> 1 : nth) & 1) ^ 1, abort_flag)) break;
      ++nth;
      tc_fence_after();
      const unsigned d1 = tmem_base + buf * 256, d2 = d1 + second;
      constexpr bool A_MN = KIND == GRAD_W, B_MN = KIND != GRAD_X;
      constexpr unsigned FORMAT = std::is_same<T, __half>::value ? 0u : 1u;
      const unsigned idesc = 1u << 4 | FORMAT << 7 | FORMAT << 10 | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | (unsigned)(u.bw >> 3) << 17 | (unsigned)(BM >> 4) << 24;
      bool ok = true;
      for (int k = 0; k < u.steps; ++k, ++it) {
        const int s = it % STAGES;
        if (!mbar_wait_warp(&sh->full[s], it / STAGES & 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const unsigned st = operands + s * STAGE_BYTES, sb = st + NP * PLANE_A;
        if (KIND == GRAD_W && !LOADED && u.rows - k * BK < BK) {
          // the rows behind the chunk are another type's, or no one's: zeros in both operands, whatever they hold
          const int first = u.rows - k * BK, count = (BK - first) * 8;
          const int blocks = 2 + (u.bw + 63) / 64;
          for (int i = lane; i < count * blocks; i += 32) {
            const int j = i / count, c = i % count;
            const unsigned at = (j < 2 ? st + j * (BK * 128) : sb + (j - 2) * (BK * 128)) + first * 128 + c * 16;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
          }
          async_fence();
          __syncwarp();
        }
        // The stage's number written out: with addresses that the compiler cannot tell to be the same in every lane each MMA took 110 cycles to issue.
        const int left = KIND != GRAD_W ? a.Kc - k * BK : a.out ? u.rows - k * BK : 0;       // (no grad_W: nothing is multiplied)
        auto issue = [&](auto stage) {
          constexpr unsigned AT = decltype(stage)::value * STAGE_BYTES;
          const unsigned long long da0 = A_MN ? desc_mn(operands + AT, BK * 128) : desc_k<ROW>(operands + AT);
          const unsigned long long db0 = B_MN ? desc_mn(operands + AT + NP * PLANE_A, BK * 128) : desc_k<ROW>(operands + AT + NP * PLANE_A);
          if (elected()) {
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
              if (kk * 16 >= left) break;                // both operands are zeros from there on (400 000 rows, 100 -> 256 fp32: 193 -> 186 us)
              unsigned long long da[NP], db[NP];
#pragma unroll
              for (int p = 0; p < NP; ++p) {             // (addresses are in units of 16 bytes)
                da[p] = da0 + ((p * PLANE_A + kk * (A_MN ? 2048 : 32)) >> 4);
                db[p] = db0 + ((p * PLANE_B + kk * (B_MN ? 2048 : 32)) >> 4);
              }
              const unsigned more = (k | kk) != 0;
              if constexpr (NP == 1) {
                umma(PAIR && (k & 1) ? d2 : d1, da[0], db[0], idesc, PAIR ? k > 1 || kk > 0 : more);
              } else {
                umma(d2, da[2], db[0], idesc, more);
                umma(d2, da[0], db[2], idesc, 1u);
                umma(d2, da[1], db[1], idesc, 1u);
                umma(d2, da[1], db[0], idesc, 1u);
                umma(d2, da[0], db[1], idesc, 1u);
                umma(d1, da[0], db[0], idesc, more);
              }
            }
            umma_commit(&sh->empty[decltype(stage)::value]);
          }
        };
        if (s == 0) issue(std::integral_constant<int, 0>());
        else if (s == 1) issue(std::integral_constant<int, 1>());
        else if constexpr (STAGES > 2) {
          if (s == 2) issue(std::integral_constant<int, 2>());
          else issue(std::integral_constant<int, 3>());
        }
        __syncwarp();
      }
      if (!ok) break;
      if (elected()) umma_commit(&sh->acc_full[buf]);
      __syncwarp();
    }
    if (lane == 0) sh->mmas = it;
  } else if (warp < 2 + EPI_WARPS) {
    // ------------------------------------------------------------ epilogue: TMEM lanes 32 (warp % 4) .., the two warps of a quadrant take turns
    const int q = warp & 3, half = (warp - 2) >> 2;
    unsigned char* const tile = staging + (warp - 2) * 32 * S::EPI_ROW;
    float* const my_bias = bias_smem + (warp - 2) * 128;    // PROJECT: of the warp's columns, at most four times 32 (as many warps write as load)
    int nth = 0;
    for (int w = blockIdx.x; w < units; w += gridDim.x) {
      const Unit u = unit_at<KIND, BK>(a, sh, w);
      const int buf = slots == 2 ? nth & 1 : 0;
      const bool part = KIND == GRAD_W && u.slot >= 0;
      const bool f32 = part || a.out_f32;
      const long long ld = KIND == GRAD_W ? a.N : a.ld_out;
      const int rows = min(32, (KIND == GRAD_W ? a.M - u.m0 : u.rows) - q * 32), columns = min(u.bw, a.N - u.n0);
      const long long first = (KIND == GRAD_W ? ((long long)(part ? u.slot : u.g) * (part ? a.M + 1 : a.M) + u.m0 + q * 32) * ld : (u.row0 + q * 32ll) * ld) + u.n0;
      if (KIND == PROJECT && a.bias) {                  // of this warp's columns; on their way while the products are formed
        const float* const b = a.bias + (long long)u.g * a.N + u.n0;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) { const int c = half * 32 + i * 8 * EPI_WARPS + lane; my_bias[i * 32 + lane] = c < columns ? __ldg(b + c) : 0.f; }
        __syncwarp();
      }
      if (u.steps > 0) {
        if (!mbar_wait_warp(&sh->acc_full[buf], (slots == 2 ? nth >> 1 : nth) & 1, abort_flag)) break;
        ++nth;
        tc_fence_after();
      }
      if (KIND == GRAD_W && u.steps == 0 && a.db && u.m0 == 0 && warp == 2)                  // no rows: no loader passes here
        for (int c = lane; c < columns; c += 32) bias_place(a, u)[c] = 0.f;
      if (rows > 0 && (KIND != GRAD_W || a.out)) {
#pragma unroll 1
        for (int c0 = half * 32; c0 < columns; c0 += 8 * EPI_WARPS) {
          float o[32];
          if (u.steps > 0) {
            const unsigned at = tmem_base + ((unsigned)(q * 32) << 16) + buf * 256 + c0;
            unsigned v[2][16], v2[2][16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              tmem_ld16(v[h], at + h * 16);
              if constexpr (NP == 3 || PAIR) tmem_ld16(v2[h], at + second + h * 16);
            }
            tmem_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              o[j] = __uint_as_float(v[j >> 4][j & 15]);
              if constexpr (NP == 3) {
                const float y = o[j] + __uint_as_float(v2[j >> 4][j & 15]);
                o[j] = (v[j >> 4][j & 15] & 0x7F800000u) == 0x7F800000u ? o[j] : y;
              } else if constexpr (PAIR) {
                if (u.steps > 1) o[j] += __uint_as_float(v2[j >> 4][j & 15]);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0.f;
          }
          if (KIND == PROJECT && a.bias) {
            const float* const b = my_bias + c0 / (8 * EPI_WARPS) * 32;
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 x = *reinterpret_cast<const float4*>(b + j);
              o[j] += x.x; o[j + 1] += x.y; o[j + 2] += x.z; o[j + 3] += x.w;
            }
          }
          if (f32) {
            float* const p = (part ? a.part : static_cast<float*>(a.out)) + first + c0;
            if constexpr (S::EPI_ROW == 128) {
              put_rows<float, 128>(tile, o, p, ld, rows, columns - c0, a.out_vec);
            } else {
              put_rows<float, 64>(tile, o, p, ld, rows, columns - c0, a.out_vec);
              if (columns - c0 > 16) put_rows<float, 64>(tile, o + 16, p + 16, ld, rows, columns - c0 - 16, a.out_vec);
            }
          } else {
            if constexpr (NP == 1) put_rows<T, 64>(tile, o, static_cast<T*>(a.out) + first + c0, ld, rows, columns - c0, a.out_vec);
          }
        }
      }
      if (u.steps > 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->acc_empty[buf]);
      }
    }
  } else if constexpr (LOADED) {
    // ------------------------------------------------------------ loaders
    const int t = threadIdx.x - 32 * (2 + EPI_WARPS);
    using L = Loader<T, KIND>;
    L ld(t);
    float sum[4] = {};                                  // GRAD_W: of this thread's four columns of grad_out
    int it = 0;
    Walk<KIND, BK> at(a, sh, units), ahead = at;
    if (at.w < units) ld.begin(a, at.u);
    auto go_on = [&] { if (ahead.next(a, sh, units)) { if (ahead.w < units) ld.begin(a, ahead.u); } else ld.step(a); };
    auto add = [&](float x, float y, float z, float w) { sum[0] += x; sum[1] += y; sum[2] += z; sum[3] += w; };
    auto arrive = [&](int s) {
      async_fence();                                    // for the tensor core to see
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->full[s]);
    };
    auto free_stage = [&](int i) { return i < STAGES || mbar_wait_warp(&sh->empty[i % STAGES], (i / STAGES & 1) ^ 1, abort_flag); };
    // The unit's sums: those of the eight warps' rows, added in the warps' order.
    unsigned phase = 0;
    auto bias_sums = [&]() -> bool {
      if (KIND != GRAD_W || !a.db || at.u.m0 != 0 || !at.last()) return true;
      const int me = warp - 2 - EPI_WARPS, c = ld.q, columns = min(at.u.bw, a.N - at.u.n0);
      *reinterpret_cast<float4*>(bias_smem + me * 128 + c) = make_float4(sum[0], sum[1], sum[2], sum[3]);
      if (!meet(sh, &phase)) return false;
      if (me == 0) {
        float* const place = bias_place(a, at.u);
        for (int w = 1; w < LOAD_WARPS; ++w) {
          const float4 o = *reinterpret_cast<const float4*>(bias_smem + w * 128 + c);
          add(o.x, o.y, o.z, o.w);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) if (c + j < columns) place[c + j] = sum[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] = 0.f;
      return meet(sh, &phase);
    };
    // An address for a copy that reads nothing, aligned as the rows are: copies want that of a source that they do not read, too.  (offsets need be aligned to 8 bytes
    // only; of grad_W's operands a may be null.)
    const void* const nothing = KIND == GRAD_W ? a.b : a.a;
    if constexpr (NP == 3) {
      // a ring of rows as they were read, filled DEPTH stages ahead; quad i of thread t lies at (i LOADERS + t) 16: a warp reads only what it copied itself
      constexpr int DEPTH = S::RAW_DEPTH;
      unsigned char* const ring = smem + STAGES * STAGE_BYTES;
      auto copy = [&](int i) {
        if (ahead.w < units) {
          const unsigned slot = smem_u32(ring) + i % DEPTH * S::RAW_BYTES + t * 16;
          if (a.a_vec && (KIND != GRAD_W || a.b_vec) && ld.rows > (L::QUADS - 1) * L::DR) {      // every row is there
            const unsigned na = min(max(ld.cols_a - ld.q, 0), 4) * 4, nb = KIND == GRAD_W ? min(max(ld.cols_b - ld.q, 0), 4) * 4 : 0;
            ld.each([&](int i, const T* p, int, bool is_a) { copy16(slot + i * (L::LOADERS * 16), (is_a ? na : nb) ? static_cast<const void*>(p) : nothing, is_a ? na : nb); });
          } else if (a.a_vec && (KIND != GRAD_W || a.b_vec)) {
            ld.each([&](int i, const T* p, int left, bool) {
              left = min(max(left, 0), 4);
              copy16(slot + i * (L::LOADERS * 16), left > 0 ? static_cast<const void*>(p) : nothing, left * 4);
            });
          } else {
            // (a quad's elements are copied by lanes of its warp)
            const unsigned warp_slot = slot - (t & 31) * 16;
            ld.template wide<1>(a, [&](int i, int e, int, int, const T* p, int left, bool) { copy4(warp_slot + i * (L::LOADERS * 16) + e * 4, left > 0 ? static_cast<const void*>(p) : nothing, left * 4); });
          }
          go_on();
        }
        copy_commit();
      };
      for (int d = 0; d < DEPTH; ++d) copy(d);
      for (; at.w < units; ++it) {
        const int s = it % STAGES;
        copy_wait<DEPTH - 1>();
        __syncwarp();
        const float4* const mine = reinterpret_cast<const float4*>(ring + it % DEPTH * S::RAW_BYTES) + t;
        float4 v[L::ALL];
#pragma unroll
        for (int i = 0; i < L::ALL; ++i) v[i] = mine[i * L::LOADERS];
        if (KIND == GRAD_W && a.db && at.u.m0 == 0)
#pragma unroll
          for (int i = L::QUADS; i < L::ALL; ++i) add(v[i].x, v[i].y, v[i].z, v[i].w);
        __syncwarp();
        copy(it + DEPTH);                               // (into the slot just read)
        if (!free_stage(it)) break;
        unsigned char* const stage = smem + s * STAGE_BYTES;
#pragma unroll
        for (int i = 0; i < L::ALL; ++i) {
          if (KIND == GRAD_W && !a.out) break;          // (grad_bias alone: 400 000 rows of 256 columns 242 -> 152 us)
          const Split4 p = split4(v[i].x, v[i].y, v[i].z, v[i].w);
          unsigned char* const to = stage + ld.place(i);
          *reinterpret_cast<uint2*>(to) = p.hi;
          *reinterpret_cast<uint2*>(to + L::PLANE) = p.mid;
          *reinterpret_cast<uint2*>(to + 2 * L::PLANE) = p.lo;
        }
        arrive(s);
        if (!bias_sums()) break;
        at.next(a, sh, units);
      }
      copy_wait<0>();
    } else {
      // copied to their places, AHEAD stages in flight: quads of 8 bytes, or pairs of elements, by the rows' alignment; odd rows go through registers
      constexpr int AHEAD = 2;
      const bool quads = a.a_vec == 4 && (KIND != GRAD_W || a.b_vec == 4), pairs = a.a_vec >= 2 && (KIND != GRAD_W || a.b_vec >= 2);
      auto copy = [&](int i) -> bool {
        if (ahead.w < units) {
          if (!free_stage(i)) return false;
          const unsigned stage = i % STAGES * STAGE_BYTES;
          if (quads) {
            ld.each([&](int i, const T* p, int left, bool) {
              copy8(operands + stage + ld.place(i), left > 0 ? static_cast<const void*>(p) : nothing, min(max(left, 0), 4) * 2);
            });
          } else if (pairs) {
            ld.template wide<2>(a, [&](int, int, int r, int c, const T* p, int left, bool is_a) {
              copy4(operands + stage + L::place_of(r, c, is_a), left > 0 ? static_cast<const void*>(p) : nothing, left * 2);
            });
          } else {
            ld.template wide<1>(a, [&](int, int, int r, int c, const T* p, int left, bool is_a) {
              *reinterpret_cast<T*>(smem + stage + L::place_of(r, c, is_a)) = left > 0 ? __ldg(p) : from_f32<T>(0.f);
            });
          }
          go_on();
        }
        copy_commit();
        return true;
      };
      bool ok = true;
      for (int d = 0; d < AHEAD; ++d) ok = ok && copy(d);
      for (; ok && at.w < units; ++it) {
        if (!copy(it + AHEAD)) break;
        copy_wait<AHEAD>();
        __syncwarp();
        if (KIND == GRAD_W && a.db && at.u.m0 == 0)
#pragma unroll
          for (int i = L::QUADS; i < L::ALL; ++i) {
            const Vec<T, 4> x = load_vec<Vec<T, 4>>(smem + it % STAGES * STAGE_BYTES + ld.place(i));
            add(to_f32<T>(x.v[0]), to_f32<T>(x.v[1]), to_f32<T>(x.v[2]), to_f32<T>(x.v[3]));
          }
        arrive(it % STAGES);
        if (!bias_sums()) break;
        at.next(a, sh, units);
      }
      copy_wait<0>();
    }
    if (t == 0 && !TMA_B) sh->loads = it;
  } else if constexpr (SUMS) {
    // ------------------------------------------------------------ columns of grad_out: a thread to two columns of a quarter of the rows (half, where the
    // block has more than 128 columns)
    static_assert(LOAD_WARPS * 32 == 256, "two columns and a share of the rows to a thread");
    const int t = threadIdx.x - 32 * (2 + EPI_WARPS);
    const int shares = a.bn > 128 ? 2 : 4, share = a.bn > 128 ? t >> 7 : t >> 6, c = (a.bn > 128 ? t & 127 : t & 63) * 2;
    float s0 = 0.f, s1 = 0.f;
    unsigned phase = 0;
    int it = 0;
    for (Walk<KIND, BK> at(a, sh, units); at.w < units; ++it) {
      const int s = it % STAGES;
      if (!mbar_wait_warp(&sh->full[s], it / STAGES & 1, abort_flag)) break;
      const bool mine = a.db && at.u.m0 == 0;
      if (mine && c < at.u.bw) {
        const unsigned byte = (c & 63) * 2, column = s * STAGE_BYTES + NP * PLANE_A + (c >> 6) * (BK * 128) + (byte & 15);
        const int rows = min(BK, at.u.rows - at.k * BK);
        float x0 = 0.f, x1 = 0.f;
        auto add = [&](int r) {
          const Vec<T, 2> p = load_vec<Vec<T, 2>>(smem + column + r * 128 + (((byte >> 4) ^ (r & 7)) << 4));
          if (r & 8) { x0 += to_f32<T>(p.v[0]); x1 += to_f32<T>(p.v[1]); }
          else { s0 += to_f32<T>(p.v[0]); s1 += to_f32<T>(p.v[1]); }
        };
        if (rows == BK && shares == 4) {
#pragma unroll
          for (int r = 0; r < BK / 4; ++r) add(share * (BK / 4) + r);
        } else if (rows == BK) {
#pragma unroll
          for (int r = 0; r < BK / 2; ++r) add(share * (BK / 2) + r);
        } else {
          for (int r = share * (BK / shares); r < min(rows, (share + 1) * (BK / shares)); ++r) add(r);
        }
        s0 += x0; s1 += x1;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->empty[s]);
      if (mine && at.last()) {
        float2* const red = reinterpret_cast<float2*>(bias_smem) + (c >> 1);       // [shares - 1][columns / 2]
        const int pitch = a.bn > 128 ? 128 : 64;
        if (share > 0) red[(share - 1) * pitch] = make_float2(s0, s1);
        if (!meet(sh, &phase)) break;
        if (share == 0) {
          float* const place = bias_place(a, at.u);
          const int columns = min(at.u.bw, a.N - at.u.n0);
          for (int i = 1; i < shares; ++i) { const float2 o = red[(i - 1) * pitch]; s0 += o.x; s1 += o.y; }
          if (c < columns) place[c] = s0;
          if (c + 1 < columns) place[c + 1] = s1;
        }
        if (!meet(sh, &phase)) break;
        s0 = s1 = 0.f;
      }
      at.next(a, sh, units);
    }
  }

  // -------------------------------------------------------------- teardown
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) {
      rows_status(a.status, TAURUS_ERR_INTERNAL);
      wait_last_phases(sh->loads, STAGES, 1u << 16, [&](int s, unsigned parity) { return mbar_try(&sh->full[s], parity); });
      wait_last_phases(sh->mmas, STAGES, 1u << 16, [&](int s, unsigned parity) { return mbar_try(&sh->empty[s], parity); });
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// W as planes of bf16 (fp32) or with rows that TMA can address (16 bits): [types * planes x K x pitch].
template <class T>
__global__ void __launch_bounds__(256) typed_pack_kernel(const T* __restrict__ W, long long types, int K, int N, int pitch, void* __restrict__ out) {
  const long long rows = types * K;
  const int quads = (N + 3) / 4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * quads; i += (long long)gridDim.x * 256) {
    const long long r = i / quads, g = r / K, k = r % K;
    const int c = (int)(i % quads) * 4;                // (the pitch is a multiple of 8: a quad stays inside its row)
    const Quad<T> q = load_quad(W + r * N, c, N, false);
    if constexpr (sizeof(T) == 2) {
      reinterpret_cast<uint2*>(static_cast<T*>(out) + r * pitch + c)[0] = *reinterpret_cast<const uint2*>(&q);
    } else {
      __nv_bfloat16* const o = static_cast<__nv_bfloat16*>(out) + (g * 3 * K + k) * pitch + c;
      const long long plane = (long long)K * pitch;
      const Split4 p = split4(q.v[0], q.v[1], q.v[2], q.v[3]);
      *reinterpret_cast<uint2*>(o) = p.hi;
      *reinterpret_cast<uint2*>(o + plane) = p.mid;
      *reinterpret_cast<uint2*>(o + 2 * plane) = p.lo;
    }
  }
}

// Rows of 16-bit elements whose pitch TMA cannot take, to a pitch that it can: 16 bytes a thread, from words of 4 bytes shifted where a row begins in the middle of one.
__global__ void __launch_bounds__(256) typed_pack_rows_kernel(const unsigned short* __restrict__ rows, long long ld, long long n, int width, int pitch, uint4* __restrict__ out) {
  const int chunks = pitch / 8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n * chunks; i += (long long)gridDim.x * 256) {
    const long long r = i / chunks;
    const int c = (int)(i - r * chunks) * 8;
    const unsigned short* const p = rows + r * ld + c;
    union { unsigned w[4]; unsigned short h[8]; uint4 v; } x;
    if (c + 8 <= width) {
      const unsigned odd = (unsigned)(reinterpret_cast<uintptr_t>(p) >> 1) & 1u;
      if (odd) {                                           // h[0] | four words, the last of which ends the chunk with its first half
        const unsigned* const q = reinterpret_cast<const unsigned*>(p + 1);
        unsigned before = (unsigned)__ldg(p) << 16;
#pragma unroll
        for (int j = 0; j < 3; ++j) { const unsigned w = __ldg(q + j); x.w[j] = __funnelshift_l(before, w, 16); before = w; }
        x.w[3] = before >> 16 | (unsigned)__ldg(p + 7) << 16;
      } else {
        const unsigned* const q = reinterpret_cast<const unsigned*>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.w[j] = __ldg(q + j);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x.h[j] = c + j < width ? __ldg(p + j) : (unsigned short)0;
    }
    out[i] = x.v;
  }
}

// ---------------------------------------------------------------------------------------------------------------- joins
struct JoinArgs {
  long long n;
  const long long* offsets;
  int types, K, N, chunk, out_f32;
  const float* part;
  void* dW;
  float* db;
};
// Chunks of type g and its first partial result (by a block).
__device__ __forceinline__ int chunks_of(const JoinArgs& a, int g, int* first) {
  int mine = 0;
  for (int j = threadIdx.x; j < g; j += blockDim.x) {
    const int c = (int)((a.offsets[j + 1] - a.offsets[j] + a.chunk - 1) / a.chunk);
    mine += c > 1 ? c : 0;
  }
  __shared__ int sum;
  if (threadIdx.x == 0) sum = 0;
  __syncthreads();
  mine = __reduce_add_sync(0xffffffffu, mine);
  if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&sum, mine);      // (whole numbers: any order)
  __syncthreads();
  *first = sum;
  return (int)((a.offsets[g + 1] - a.offsets[g] + a.chunk - 1) / a.chunk);
}
__device__ __forceinline__ bool offsets_bad(const long long* offsets, int types, long long n) {      // by a block
  bool bad = false;
  for (int g = threadIdx.x; g < types; g += blockDim.x) { const long long b = offsets[g], e = offsets[g + 1]; bad |= b < 0 || e > n || e < b; }
  return __syncthreads_or(bad);
}

// The partial results of the types of several chunks, added in the chunks' order.  Grid (elements by stride, types).
template <class O>
__global__ void __launch_bounds__(256) typed_join_kernel(const JoinArgs a) {
  const int g = blockIdx.y;
  if (a.offsets[g + 1] - a.offsets[g] <= a.chunk || offsets_bad(a.offsets, a.types, a.n)) return;
  int first;
  const int chunks = chunks_of(a, g, &first);
  const long long size = (long long)(a.K + 1) * a.N;
  const long long from = a.dW ? 0 : (long long)a.K * a.N, to = a.db ? size : (long long)a.K * a.N;
  for (long long i = from + (long long)blockIdx.x * 256 + threadIdx.x; i < to; i += (long long)gridDim.x * 256) {
    float s = 0.f;
#pragma unroll 16
    for (int c = 0; c < chunks; ++c) s += a.part[(long long)(first + c) * size + i];
    if (i < (long long)a.K * a.N) static_cast<O*>(a.dW)[(long long)g * a.K * a.N + i] = from_f32<O>(s);
    else a.db[(long long)g * a.N + (i - (long long)a.K * a.N)] = s;
  }
}

// ---------------------------------------------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) { cudaGetLastError(); p = nullptr; }
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}
// Elements of 16 bits, box inner x rows (x 1), swizzle of the box's inner bytes (128 or 64).
bool make_map(CUtensorMap* m, int32_t type, const void* base, long long cols, long long rows, long long depth, long long ld, int box_cols, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)rows};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
  const EncodeTiledFn encode = encode_fn();
  const CUresult r = !encode ? CUDA_ERROR_NOT_FOUND
                             : encode(m, type == TAURUS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, depth > 0 ? 3 : 2, const_cast<void*>(base), dims, strides,
                                      box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) taurus_note_cuda_error(static_cast<cudaError_t>(r), "cuTensorMapEncodeTiled");      // (the two enumerations share their numbers)
  return r == CUDA_SUCCESS;
}
// TcArgs::a_vec
int vec_of(const void* p, long long ld, int size) {
  int v = 4;
  while (v > 1 && (ld % v != 0 || !rows_aligned(p, v * size))) v >>= 1;
  return size == 4 && v < 4 ? 0 : v;
}

// Blocks of nearly equal width, a multiple of 16, as wide as they can be: each splits or reads the rows anew.  Against blocks of 64, forward: 400 000 x 100 -> 256 fp32 185 / 324 us, bf16
// 102 / 144, 65 536 x 128 -> 128 fp32 27 / 35; narrower ones would pay only where there are fewer of them than SMs (300 rows of 1 024 -> 1 024 fp32 47 / 33, bf16 12.6 / 10.4).
int block_columns(int N, int most) {
  const int np = taurus_round_up(N, 16), blocks = (np + most - 1) / most;
  return taurus_round_up((np + blocks - 1) / blocks, 16);
}

// A product ready to be launched.  All of a call's are made ready before its first launch: a call that fails has enqueued nothing.
struct Product {
  CUtensorMap ma = {}, mb = {};
  TcArgs a = {};
  long long units = 0;        // at most
  bool loaded = false;
};

template <class T, int KIND, bool LOADED>
int launch(const Product& p, int sms, cudaStream_t st) {
  constexpr int shared = Shape<T, KIND, LOADED>::SHARED_BYTES + (int)sizeof(Shared);
  const cudaError_t e = cudaFuncSetAttribute(typed_tc_kernel<T, KIND, LOADED>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
  if (e != cudaSuccess) { taurus_note_cuda_error(e, "typed_project"); return TAURUS_ERR_CUDA; }
  constexpr int threads = Shape<T, KIND, LOADED>::THREADS;
  typed_tc_kernel<T, KIND, LOADED><<<(int)std::max<long long>(1, std::min<long long>(p.units, sms)), threads, shared, st>>>(p.ma, p.mb, p.a);
  return TAURUS_OK;
}
template <int KIND>
int launch_type(int32_t type, const Product& p, int sms, cudaStream_t st) {
  if (type == TAURUS_F32) return launch<float, KIND, true>(p, sms, st);
  if (type == TAURUS_BF16) return p.loaded ? launch<__nv_bfloat16, KIND, true>(p, sms, st) : launch<__nv_bfloat16, KIND, false>(p, sms, st);
  return p.loaded ? launch<__half, KIND, true>(p, sms, st) : launch<__half, KIND, false>(p, sms, st);
}

int weight_pitch(int d_out) { return taurus_round_up(d_out, 8); }
int bn_most(int32_t type, bool grad_w, bool loaded) { return type == TAURUS_F32 ? (grad_w ? 128 : 256) : loaded ? 128 : 256; }     // Shape::BN

// Rows of a width that keeps TMA off, fp32 aside, are laid out at another pitch (rows of such a width whose own pitch suits TMA are not).
int64_t row_pitch(int width) { return taurus_round_up(width, 8); }
bool packs_rows(const void* p, int64_t ld, int width, int32_t type) { return typed_tc_row_bytes(1, width, type) > 0 && !tma_rows(p, ld); }
// Rows of a chunk of grad_W: about two units to an SM, 1 024 rows at least, 2 048 at most.  fp32: 1 024 (2 700, as 400 000 rows in 5 types would have: 2.9e-6 of the result
// off, where fp32 sums are 1.1e-6).  Chunks of 1 024, 512 or 256 rows at least, grad_W and grad_bias, us: 400 000 x 100 -> 256 fp32 244, 273, 355 (the join of their partial results);
// 65 536 x 128 -> 128 in 5 types fp32 49, 33, 43, bf16 23, 21, 31, in 200 types fp16 35, 34, 43; 5 000 x 256 -> 256 fp32 45, 29, 23, where there are fewer chunks than SMs.
constexpr int CHUNK_LEAST = 1024;
long long weight_tiles(int d_in, int d_out) { return (long long)((d_in + BM - 1) / BM) * ((d_out + 255) / 256); }
int rows_of_chunk(int64_t n, int d_in, int d_out, int32_t type) {
  if (type == TAURUS_F32) return CHUNK_LEAST;
  return (int)std::min<long long>(2048, std::max<long long>(CHUNK_LEAST, taurus_round_up((int)std::min<long long>(n * weight_tiles(d_in, d_out) / (2 * 148), 1 << 20), 64)));
}

}  // namespace

// Does W have to be laid out anew?  Room for it (whatever its address, which a workspace's size does not depend on).
bool typed_tc_packs(const void* W, int32_t type, int d_out) { return type == TAURUS_F32 || d_out % 8 != 0 || !rows_aligned(W, 16); }
size_t typed_tc_pack_bytes(int32_t types, int d_in, int d_out, int32_t type) { return (size_t)types * (type == TAURUS_F32 ? 3 : 1) * d_in * weight_pitch(d_out) * 2; }
// Room for rows at another pitch.
size_t typed_tc_row_bytes(int64_t n, int width, int32_t type) { return type == TAURUS_F32 || width % 8 == 0 ? 0 : (size_t)n * (size_t)row_pitch(width) * 2; }
// A type of more than one chunk has more than `chunk` rows and at most rows / chunk + 1 chunks.
// most: what no call with as many rows, or fewer, exceeds.  (Between the shortest and the longest chunk n / chunk is about two units to an SM, y / (y - 1) of it at most for
// y = n tiles / 296 >= 1 024: less than one more.)
size_t typed_tc_part_bytes(int64_t n, int32_t types, int d_in, int d_out, int32_t type, bool most) {
  int64_t chunks = n / rows_of_chunk(n, d_in, d_out, type);
  if (most) chunks = std::max(chunks, std::min<int64_t>(n / CHUNK_LEAST, 2 * 148 / weight_tiles(d_in, d_out) + 1));
  return (size_t)(chunks + std::min<int64_t>(types, chunks)) * (size_t)(d_in + 1) * d_out * 4;
}

namespace {

void pack_rows(const void* rows, int64_t ld, int64_t n, int width, void* packed, int sms, cudaStream_t st) {
  const int pitch = (int)row_pitch(width);
  const int grid = (int)std::min<long long>((n * (pitch / 8) + 255) / 256, (long long)sms * 32);
  typed_pack_rows_kernel<<<grid, 256, 0, st>>>(static_cast<const unsigned short*>(rows), ld, n, width, pitch, static_cast<uint4*>(packed));
}
void pack_weights(int32_t type, const void* W, int32_t types, int d_in, int d_out, void* packed, int sms, cudaStream_t st) {
  const long long quads = (long long)types * d_in * ((d_out + 3) / 4);
  const int grid = (int)std::min<long long>((quads + 255) / 256, (long long)sms * 16);
  with_row_type(type, [&](auto tt) {
    using T = typename decltype(tt)::type;
    typed_pack_kernel<T><<<grid, 256, 0, st>>>(static_cast<const T*>(W), types, d_in, d_out, weight_pitch(d_out), packed);
    return 0;
  });
}

// out = x W + bias, or grad_x = grad_out W^T (transposed).  w: W itself, or what pack_weights makes of it.
bool ready_rows(Product* p, bool transposed, int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* w, const float* bias, int d_in,
                int d_out, void* out, int32_t out_type, int64_t ld_out, int32_t* status) {
  const int Kc = transposed ? d_out : d_in, N = transposed ? d_in : d_out, planes = type == TAURUS_F32 ? 3 : 1;
  p->loaded = type == TAURUS_F32 || !tma_rows(x, ld_x);
  const int bk = type == TAURUS_F32 ? 32 : 64;
  TcArgs& a = p->a;
  a.n = n; a.offsets = offsets; a.types = types; a.N = N; a.Kc = Kc;
  a.bn = block_columns(N, bn_most(type, false, p->loaded)); a.n_blocks = (N + a.bn - 1) / a.bn;
  a.a = x; a.lda = ld_x; a.a_vec = vec_of(x, ld_x, row_type_size(type));
  a.out = out; a.ld_out = ld_out; a.out_f32 = out_type == TAURUS_F32; a.out_vec = ld_out * row_type_size(out_type) % 16 == 0 && rows_aligned(out, 16);
  a.bias = bias; a.status = status;
  p->units = (n / BM + std::min<long long>(types, n)) * a.n_blocks;
  return (p->loaded || make_map(&p->ma, type, x, Kc, n, 0, ld_x, bk, BM)) &&
         make_map(&p->mb, type, w, d_out, d_in, (long long)types * planes, weight_pitch(d_out), transposed ? bk : 64, transposed ? a.bn : bk);
}

// grad_W and grad_bias (either may be null); part: typed_tc_part_bytes.
bool ready_weights(Product* p, int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* dy, int64_t ld_dy, int d_in, int d_out, void* dW,
                   int32_t dW_type, float* db, float* part, int32_t* status) {
  const int chunk = rows_of_chunk(n, d_in, d_out, type);
  // (by x's rows too where only grad_bias is asked for: its sums are then formed as they are beside grad_W's)
  p->loaded = type == TAURUS_F32 || (x && !tma_rows(x, ld_x)) || !tma_rows(dy, ld_dy);
  const int bk = type == TAURUS_F32 ? 32 : 64, size = row_type_size(type), out_size = row_type_size(dW_type);
  TcArgs& a = p->a;
  a.n = n; a.offsets = offsets; a.types = types; a.M = d_in; a.N = d_out; a.chunk = chunk;
  a.bn = block_columns(d_out, bn_most(type, true, p->loaded)); a.n_blocks = (d_out + a.bn - 1) / a.bn; a.m_blocks = dW ? (d_in + BM - 1) / BM : 1;
  a.a = dW ? x : nullptr; a.lda = ld_x; a.a_vec = vec_of(x, ld_x, size);
  a.b = dy; a.ldb = ld_dy; a.b_vec = vec_of(dy, ld_dy, size);
  a.out = dW; a.out_f32 = dW_type == TAURUS_F32; a.out_vec = d_out * out_size % 16 == 0 && d_out % 4 == 0 && rows_aligned(dW, 16);
  a.db = db; a.part = part; a.status = status;
  p->units = (n / chunk + types) * a.m_blocks * a.n_blocks;
  return p->loaded || ((!dW || make_map(&p->ma, type, x, d_in, n, 0, ld_x, 64, bk)) && make_map(&p->mb, type, dy, d_out, n, 0, ld_dy, 64, bk));
}
int launch_weights(const Product& p, int32_t type, int32_t dW_type, int sms, cudaStream_t st) {
  const TcArgs& a = p.a;
  const int rc = launch_type<GRAD_W>(type, p, sms, st);
  if (rc) return rc;
  JoinArgs j = {};
  j.n = a.n; j.offsets = a.offsets; j.types = a.types; j.K = a.M; j.N = a.N; j.chunk = a.chunk; j.part = a.part; j.dW = a.out; j.db = a.db;
  if (a.n > a.chunk)
    with_row_type(a.out ? dW_type : TAURUS_F32, [&](auto tt) {
      using O = typename decltype(tt)::type;
      const long long size = (long long)(a.M + 1) * a.N;
      typed_join_kernel<O><<<dim3((unsigned)std::min<long long>((size + 255) / 256, std::max(8, 16 * sms / a.types)), (unsigned)a.types), 256, 0, st>>>(j);
      return 0;
    });
  return TAURUS_OK;
}

// Rows as the products take them: where they are, or at `space` at another pitch (laid out there once everything is ready).
struct Rows {
  const void* from;
  int64_t ld_from;
  int width;
  void* space;
  bool packs;
  Rows(const void* rows, int64_t ld, int width, int32_t type, void* space) : from(rows), ld_from(ld), width(width), space(space), packs(rows && packs_rows(rows, ld, width, type)) {}
  const void* at() const { return packs ? space : from; }
  int64_t ld() const { return packs ? row_pitch(width) : ld_from; }
  void lay_out(int64_t n, int sms, cudaStream_t st) const { if (packs) pack_rows(from, ld_from, n, width, space, sms, st); }
};

}  // namespace

int typed_tc_project(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const float* bias, int d_in, int d_out, void* out,
                     int32_t out_type, int64_t ld_out, const TypedSpaces& spaces, int32_t* status, int sms, cudaStream_t st) {
  const bool packs = typed_tc_packs(W, type, d_out);
  const Rows rows(x, ld_x, d_in, type, spaces.x);
  Product p;
  if (!ready_rows(&p, false, n, types, offsets, rows.at(), rows.ld(), type, packs ? spaces.W : W, bias, d_in, d_out, out, out_type, ld_out, status)) return TAURUS_ERR_CUDA;
  if (packs) pack_weights(type, W, types, d_in, d_out, spaces.W, sms, st);
  rows.lay_out(n, sms, st);
  return launch_type<PROJECT>(type, p, sms, st);
}

int typed_tc_project_grad(int64_t n, int32_t types, const long long* offsets, const void* x, int64_t ld_x, int32_t type, const void* W, const void* grad_out, int64_t ld_grad, int d_in,
                          int d_out, void* grad_x, int64_t ld_grad_x, void* grad_W, int32_t grad_W_type, float* grad_bias, const TypedSpaces& spaces, int32_t* status, int sms,
                          cudaStream_t st) {
  const bool packs = grad_x && typed_tc_packs(W, type, d_out), weights = grad_W || grad_bias;
  const Rows dy(grad_out, ld_grad, d_out, type, spaces.dy);
  Rows rows(x, ld_x, d_in, type, spaces.x);
  if (!grad_W && rows.packs) rows = Rows(nullptr, ld_x, d_in, type, nullptr);      // (grad_bias as beside grad_W, whose rows would be laid out for TMA)
  Product p, q;
  if (grad_x && !ready_rows(&p, true, n, types, offsets, dy.at(), dy.ld(), type, packs ? spaces.W : W, nullptr, d_in, d_out, grad_x, type, ld_grad_x, status)) return TAURUS_ERR_CUDA;
  if (weights && !ready_weights(&q, n, types, offsets, rows.at(), rows.ld(), type, dy.at(), dy.ld(), d_in, d_out, grad_W, grad_W_type, grad_bias, static_cast<float*>(spaces.part), status))
    return TAURUS_ERR_CUDA;
  if (packs) pack_weights(type, W, types, d_in, d_out, spaces.W, sms, st);
  dy.lay_out(n, sms, st);
  rows.lay_out(n, sms, st);
  int rc = grad_x ? launch_type<GRAD_X>(type, p, sms, st) : TAURUS_OK;
  if (!rc && weights) rc = launch_weights(q, type, grad_W_type, sms, st);
  return rc;
}
