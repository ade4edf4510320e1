// gemm.cuh -- the matrix product of the dense operators on the tcgen05 tensor
// cores: C[m, n] = sum_k A[m, k] B[n, k], fp32 accumulators in TMEM, one of the
// epilogues of dense.cuh.
//
// One CTA (CG = 1) computes tiles of 128 x BN; a pair of CTAs (CG = 2) one of
// 256 x BN, each holding its 128 rows of A and half of the columns of B, so
// that a byte of B staged in shared memory feeds twice the MMAs. At 128 x 256
// per CTA and step of 64 the operands are 48 KB per 512 tensor clocks, more
// than an SM's share of the L2; the pair takes 32 KB.
//
// Persistent CTAs, roles by warp: 0 issues the TMA loads of a ring of stages,
// 1 the MMAs, 2 owns the TMEM allocation, 4 to 19 run the epilogue of one
// accumulator while the MMAs fill another (four warps per scheduler: the
// epilogue is chains of latencies, and with two the GELU of a 16384 x 832 x
// 3328 product took longer than its MMAs). A stage holds 64 elements of k
// of both operands in the 128-byte swizzled layouts of umma.cuh, rows along m or
// n (K-major) or along k (MN-major), as the operand lies in memory: no operand is
// transposed by a pass of its own.
//
// fp32 operands come as three bf16 pieces each (value = p0 + p1 + p2 to 24
// bits); the six products with the largest terms are accumulated, smallest
// first, and after every 64 elements of k the epilogue warps add the accumulator
// to fp32 registers: the tensor core's own accumulation truncates, and over a
// long k that error would grow with k. A stage holds one piece of both operands,
// three stages make a step of k. (With all pieces of 32 elements in a stage, in
// rows of 64 bytes, the TMA unit was the limit: about a row per clock.)
//
// kEpiJoin splits a long k over a cluster: each of its CTAs sums a range of k of
// the same tile, leaves its accumulators in shared memory, and ends a share of
// the tile's elements from all of them through distributed shared memory, in
// the order of the ranges. One launch instead of two and no way through memory
// (32 x 3328 x 832 called alone 12.0 us with a second launch, 9.3 so).
//
// Every wait has a poll limit. A role that gives up sets the wait flag and
// leaves its loop; the producer then waits for its copies in flight, and TMEM
// is freed.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "debug.cuh"
#include "dense.cuh"
#include "device.cuh"
#include "params.h"
#include "ssd_common.cuh"
#include "umma.cuh"

namespace bds {
namespace {

constexpr int kEpiWarps = 16;
constexpr int kGemmThreads = 128 + 32 * kEpiWarps;

// The i-th piece of a step of k to be loaded: 1, 2, 0, so that the products can
// begin with the smallest terms.
template <int NP>
constexpr int kPiece(int i) {
  return NP == 3 ? (i + 1) % 3 : 0;
}

template <int CG, int BN, int NP, int EPI = kEpiOut>
struct GemmSmem {
  static constexpr int kBk = kGemmBk;                                  // elements of k per stage
  static constexpr uint32_t kRow = kBk * 2u;                           // bytes of a K-major row
  static constexpr uint32_t kA = 128u * kRow;                          // one piece of A
  static constexpr uint32_t kB = (uint32_t)(BN / CG) * kRow;           // one piece of B
  static constexpr uint32_t kCol = kBk * 128u;                         // 64 columns of an MN-major operand
  static constexpr uint32_t kStage = kA + kB;
  // bytes of an epilogue warp: a unit of its output, a gated layer's gradient two
  static constexpr uint32_t kUnit = EPI == kEpiGateDz || EPI == kEpiGateDzRows ? 4096u : 2048u;
  static constexpr uint32_t kEpi = kEpiWarps * kUnit;
  static constexpr int kStages = (int)((232448u - 1024u - 512u - kEpi) / kStage) > 8
                                     ? 8
                                     : (int)((232448u - 1024u - 512u - kEpi) / kStage);
  static constexpr uint32_t kBytes = kStages * kStage + kEpi + 1024u;
  static_assert(kStages > NP, "the stages of a step of k and one more");
};

// ---- cluster and two-CTA forms of the pieces of umma.cuh ----
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ int cluster_size() {
  int n;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;\n" : "=r"(n));
  return n;
}
__device__ __forceinline__ float4 load_cluster4(uint32_t saddr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(saddr)
               : "memory");
  return v;
}
__device__ __forceinline__ uint32_t map_cta(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
// One lane of a warp that executes this together.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// A wait by every lane of a warp, which leaves together.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xffffffffu, umma::bar_wait(bar, parity));
}
// A barrier of the epilogue warps, which tells all of them whether one has given
// up: nobody waits there for a warp that has left its loop.
__device__ __forceinline__ bool epilogue_sync(bool gave_up) {
  uint32_t any;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n bar.red.or.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"(gave_up ? 1u : 0u), "n"(32 * kEpiWarps)
      : "memory");
  return any != 0;
}
// One arrival at the barrier at this offset in the tile's first CTA. What it
// orders is this thread's TMEM loads, which have completed (wait::ld and the
// tcgen05 fence before it); a release at cluster scope would also wait for the
// global stores of the chunks before, which nobody in the cluster reads
// (16384 x 832 x 3328: 80 us with it).
template <int CG>
__device__ __forceinline__ void leader_arrive(uint64_t* bar) {
  if constexpr (CG == 1)
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(umma::smem_u32(bar)) : "memory");
  else
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" ::"r"(map_cta(umma::smem_u32(bar), 0)) : "memory");
}
template <int CG>
__device__ __forceinline__ void gtma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  if constexpr (CG == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];\n" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, "
        "{%2, %3, %4}], [%5];\n" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
template <int CG>
__device__ __forceinline__ void gmma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  if constexpr (CG == 1)
    umma::mma_bf16(d, a, b, idesc, acc);
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u)
        : "memory");
}
// The barrier at this offset in every CTA of the tile completes a phase when
// the MMAs issued so far have finished.
template <int CG>
__device__ __forceinline__ void gcommit(uint64_t* bar) {
  if constexpr (CG == 1)
    umma::mma_commit(bar);
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(
            umma::smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void gtmem_alloc(uint32_t* slot, uint32_t cols) {
  if constexpr (CG == 1)
    asm volatile(
        "tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n"
        "tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::"r"(umma::smem_u32(slot)),
        "r"(cols)
        : "memory");
  else
    asm volatile(
        "tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n"
        "tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::"r"(umma::smem_u32(slot)),
        "r"(cols)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void gtmem_dealloc(uint32_t tm, uint32_t cols) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tm), "r"(cols));
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tm), "r"(cols));
}

// ---- activations ----
// GELU is its tanh form, z (1 + tanh u) / 2 = z sigmoid(2 u): one exponential
// and one reciprocal on the MUFU unit instead of a polynomial per element. An
// overflow of the cube or of the exponential ends in the right limit, sigmoid
// 0 or 1.
constexpr int kActNone = 0, kActSilu = 1, kActGelu = 2;
constexpr float kGeluA = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;
__device__ __forceinline__ float rcp_f(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// exp(-x) of the sigmoid's argument x, as the base-2 exponent that ex2 takes.
__device__ __forceinline__ float silu_arg(float z) { return -kLog2e * z; }
__device__ __forceinline__ float gelu_arg(float z) {
  constexpr float c1 = -2.f * kGeluA * kLog2e, c2 = c1 * kGeluB;
  return z * fmaf(c2, z * z, c1);
}
__device__ __forceinline__ float silu_f(float z) { return z * rcp_f(1.f + ex2(silu_arg(z))); }
__device__ __forceinline__ float gelu_f(float z) { return z * rcp_f(1.f + ex2(gelu_arg(z))); }
// Two at a time with one reciprocal, 1/a = b (1/ab): the MUFU unit gives half
// as many reciprocals per clock as exponentials. Exponentials above 2^60 enter
// the product as that, so that it stays finite. Their own sigmoid has to be
// zero, since z may be large enough to make something of 2^-60: a little more
// than that is taken off every sigmoid, in the product's own instruction, which
// also holds the result in [0, 1] (a select instead: 16384 x 832 x 3328 with
// GELU 67.5 us against 66.0). A NaN stays its own element's through the last
// product, and minus infinity becomes one there.
__device__ __forceinline__ float fma_sat(float a, float b, float c) {
  float y;
  asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
template <float (*ARG)(float)>
__device__ __forceinline__ void sigmoid_mul2(float& z0, float& z1) {
  const float a = 1.f + fminf(ex2(ARG(z0)), 0x1p60f), b = 1.f + fminf(ex2(ARG(z1)), 0x1p60f);
  const float r = rcp_f(a * b);
  constexpr float off = -0x1.00001p-60f;  // the margin covers the roundings of r and of the products, 2^-22
  z0 *= fma_sat(r, b, off);
  z1 *= fma_sat(r, a, off);
}
__device__ __forceinline__ float act_fwd(int act, float z) {
  return act == kActNone ? z : act == kActSilu ? silu_f(z) : gelu_f(z);
}
// The derivative; the argument is clamped to where the sigmoid is 0 or 1 in
// fp32, so that no infinity meets a zero. The clamp would also hide an argument
// that is not finite (fmaxf of a NaN is the other operand): 0 z, added at the
// end, is zero for every finite z and NaN for the others.
__device__ __forceinline__ float act_grad(int act, float z) {
  if (act == kActNone) return 1.f;
  if (act == kActSilu) {
    const float c = fminf(fmaxf(z, -100.f), 100.f);
    const float s = rcp_f(1.f + ex2(-kLog2e * c));
    return fmaf(0.f, z, s * (1.f + c * (1.f - s)));
  }
  const float c = fminf(fmaxf(z, -16.f), 16.f);
  constexpr float c1 = -2.f * kGeluA * kLog2e, c2 = c1 * kGeluB;
  const float s = rcp_f(1.f + ex2(c * fmaf(c2, c * c, c1)));
  return fmaf(0.f, z, s * (1.f + c * (1.f - s) * fmaf(6.f * kGeluA * kGeluB, c * c, 2.f * kGeluA)));
}

// fp32 as three bf16 pieces (8 + 8 + 8 bits). The first is cut towards zero
// where rounding would overflow; a value that is not finite is its own first
// piece.
__device__ __forceinline__ void split3(float v, bf16& a, bf16& b, bf16& c) {
  a = __float2bfloat16_rn(v);
  const float f = __bfloat162float(a);
  if (!isfinite(f)) {
    if (isfinite(v)) a = __float2bfloat16_rz(v);
    else {
      b = c = __float2bfloat16_rn(0.f);
      return;
    }
  }
  const float r = v - __bfloat162float(a);
  b = __float2bfloat16_rn(r);
  c = __float2bfloat16_rn(r - __bfloat162float(b));
}

// What split3 takes of a value: the nearest bf16, towards zero where that
// would overflow, the value itself where it is not finite (the rest is then
// NaN: nothing finite can be made of it).
__device__ __forceinline__ float bf16_part(float v) {
  const float f = __bfloat162float(__float2bfloat16_rn(v));
  return isinf(f) && isfinite(v) ? __bfloat162float(__float2bfloat16_rz(v)) : f;
}

__device__ __forceinline__ float4 load4(const void* p, int f32, int64_t at) {
  if (f32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
  const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const bf16*>(p) + at);
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  return make_float4(a.x, a.y, b.x, b.y);
}
// e += the eight bf16 of u.
__device__ __forceinline__ void add8(float (&e)[8], const uint4& u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e[2 * i] += __uint_as_float(w[i] << 16);
    e[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float load1(const void* p, int f32, int64_t at) {
  return f32 ? static_cast<const float*>(p)[at] : __bfloat162float(static_cast<const bf16*>(p)[at]);
}
__device__ __forceinline__ void store4(void* p, int f32, int64_t at, float4 v) {
  if (f32)
    *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = v;
  else
    *reinterpret_cast<uint2*>(static_cast<bf16*>(p) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}
__device__ __forceinline__ void store1(void* p, int f32, int64_t at, float v) {
  if (f32) static_cast<float*>(p)[at] = v;
  else static_cast<bf16*>(p)[at] = __float2bfloat16_rn(v);
}

// ---- output ----
// A warp's chunk is 32 rows x 32 columns, a thread holding one row (as TMEM
// gives it). Where rows start on 16-byte boundaries it leaves by TMA (kEpiOut,
// kEpiDz), in units of 32 rows x 64 bytes (32 bf16 or 16 fp32 columns): the warp
// writes a unit to its 2 KB of shared memory in the swizzle of the map's box and
// one lane issues the store, which also cuts off what lies outside the matrix.
// A residual comes through the same 2 KB: it is loaded with whole 64-byte rows
// (four lanes each) a unit ahead. Other rows (kEpiRows: unaligned strides,
// mapped rows) go through shared memory to plain stores with 16 lanes per row.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int c0, int c1, int c2, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(c0), "r"(c1), "r"(c2), "r"(src)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
}
// This thread's stores have read shared memory.
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory"); }

// Columns H * 16 .. + 15 (fp32) or all 32 (bf16) of the chunk v to (col, row, z)
// of `map`, plus the residual unit `raw` where `res`. `next` runs once raw has
// been put away: it loads what the next unit needs.
template <bool F32, int H, typename NEXT>
__device__ __forceinline__ void unit_store(const CUtensorMap* map, int col, int row, int z, const float (&v)[32],
                                           bool res, const uint4 (&raw)[4], unsigned char* stg, NEXT next) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) tma_store_wait_read();
  __syncwarp();
  if (res) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 8 * j + (lane >> 2);
      *reinterpret_cast<uint4*>(stg + r * 64 + 16 * ((lane & 3) ^ ((r >> 1) & 3))) = raw[j];
    }
    __syncwarp();
  }
  next();
  unsigned char* mine = stg + lane * 64;
  const int sw = (lane >> 1) & 3;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4* slot = reinterpret_cast<uint4*>(mine + 16 * (j ^ sw));
    if constexpr (F32) {
      float4 e = make_float4(v[16 * H + 4 * j], v[16 * H + 4 * j + 1], v[16 * H + 4 * j + 2], v[16 * H + 4 * j + 3]);
      if (res) {
        const uint4 u = *slot;
        e.x += __uint_as_float(u.x), e.y += __uint_as_float(u.y), e.z += __uint_as_float(u.z), e.w += __uint_as_float(u.w);
      }
      *reinterpret_cast<float4*>(slot) = e;
    } else {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = v[8 * j + i];
      if (res) add8(e, *slot);
      *slot = make_uint4(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]), pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7]));
    }
  }
  umma::fence_async_smem();
  __syncwarp();
  if (lane == 0) tma_store_3d(map, col, row, z, umma::smem_u32(stg));
}
// The residual of a unit at (row0, col): lane l holds 16 bytes of rows l / 4 + 8 j.
// A piece may reach past column n (never read, and inside the row's stride) but
// not past the last row's end.
template <bool F32>
__device__ __forceinline__ void load_res(uint4 (&raw)[4], const GemmParams& p, int64_t row0, int col) {
  constexpr int PE = F32 ? 4 : 8;
  const int lane = threadIdx.x & 31, c = col + PE * (lane & 3);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = row0 + 8 * j + (lane >> 2);
    raw[j] = make_uint4(0, 0, 0, 0);
    if (r >= p.m || c >= p.n) continue;
    const int64_t at = r * p.ld_res + c;
    if (c + PE <= p.n || r + 1 < p.m) {
      raw[j] = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(p.res) + at * (F32 ? 4 : 2));
    } else if constexpr (F32) {
      const uint32_t* q = static_cast<const uint32_t*>(p.res) + at;
      raw[j] = make_uint4(q[0], c + 1 < p.n ? q[1] : 0u, c + 2 < p.n ? q[2] : 0u, 0u);
    } else {
      const unsigned short* q = static_cast<const unsigned short*>(p.res) + at;
      auto two = [&](int i) {
        return (c + i < p.n ? (uint32_t)q[i] : 0u) | (c + i + 1 < p.n ? (uint32_t)q[i + 1] << 16 : 0u);
      };
      raw[j] = make_uint4(two(0), two(2), two(4), two(6));
    }
  }
}
// bf16 bias of 32 columns, the same for every lane, in two steps.
__device__ __forceinline__ void load_bias(uint4 (&r)[4], const GemmParams& p, int col) {
  const uint4* q = reinterpret_cast<const uint4*>(static_cast<const bf16*>(p.bias) + col);
#pragma unroll
  for (int j = 0; j < 4; ++j)  // whole pieces; the last one of an odd width is added from memory
    r[j] = col + 8 * j + 8 <= p.n ? q[j] : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void add_bias(float (&v)[32], const uint4 (&r)[4], const GemmParams& p, int col) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = v[8 * j + i];
    add8(e, r[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[8 * j + i] = e[i];
  }
  if (col + 32 > p.n && (p.n & 7) != 0) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (col + i >= (p.n & ~7) && col + i < p.n) v[i] += load1(p.bias, 0, col + i);
  }
}

// What a chunk's output by plain stores needs besides its accumulators, loaded
// ahead: columns col0 + lane % 16 and 16 further, rows row0 + lane / 16 + 2 i.
// Bits as they lie in memory, so that nothing waits for them yet.
struct RowsAhead {
  uint32_t res[2][16];
  float bias[2];
};
template <bool IN32>
__device__ __forceinline__ void load_rows_ahead(RowsAhead& a, const GemmParams& p, int64_t row0, int col0) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = col0 + 16 * h + (lane & 15);
    if (p.bias != nullptr) a.bias[h] = col < p.n ? load1(p.bias, IN32, col) : 0.f;
    if (p.res == nullptr) continue;
    const int64_t row = row0 + (lane >> 4);
    const int left = col < p.n ? (int)min((int64_t)32, p.m - row) : 0;
    const unsigned char* at = static_cast<const unsigned char*>(p.res) + ((row * p.ld_res + col) << (p.res_f32 ? 2 : 1));
    const int64_t step = p.ld_res << (p.res_f32 ? 3 : 2);
    if (p.res_f32) {
#pragma unroll
      for (int i = 0; i < 16; ++i, at += step)
        if (2 * i < left) a.res[h][i] = *reinterpret_cast<const uint32_t*>(at);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i, at += step)
        if (2 * i < left) a.res[h][i] = *reinterpret_cast<const unsigned short*>(at);
    }
  }
}
// Every second row of one column from `at` on, those below `left`: addresses by
// addition (with a 64-bit product each the rows took 36 instructions per element).
template <bool F32>
__device__ __forceinline__ void store_rows(void* p, int64_t row, int64_t ld, int col, int left, const float (&x)[16]) {
  unsigned char* at = static_cast<unsigned char*>(p) + (row * ld + col) * (F32 ? 4 : 2);
  const int64_t step = 2 * ld * (F32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < 16; ++i, at += step)
    if (2 * i < left) {
      if constexpr (F32) *reinterpret_cast<float*>(at) = x[i];
      else *reinterpret_cast<bf16*>(at) = __float2bfloat16_rn(x[i]);
    }
}
// The output step of rows row, row + 2, ... (those below row + left) of one
// column, by plain stores. IN32: bias and pre are fp32; OF32: the output is;
// PLAIN: there is neither bias, pre, activation nor residual.
template <bool IN32, bool OF32, bool PLAIN>
__device__ __forceinline__ void out_rows(const GemmParams& p, int64_t row, int left, int col, float (&x)[16],
                                         const uint32_t (&res)[16], float bias) {
  if (!PLAIN && p.bias != nullptr) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] += bias;
  }
  if (!PLAIN && p.pre != nullptr) {
    store_rows<IN32>(p.pre, row, p.ld_pre, col, left, x);
  }
  if (!PLAIN && p.act == kActSilu) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) sigmoid_mul2<silu_arg>(x[i], x[i + 1]);
  } else if (!PLAIN && p.act == kActGelu) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) sigmoid_mul2<gelu_arg>(x[i], x[i + 1]);
  }
  if (!PLAIN && p.res != nullptr) {
    const int sh = p.res_f32 ? 0 : 16;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] += 2 * i < left ? __uint_as_float(res[i] << sh) : 0.f;
  }
  if (p.row_map != nullptr) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (2 * i < left)
        store1(p.out, OF32, p.row_map[row + 2 * i] * p.ld_out + col, x[i] * p.row_scale[row + 2 * i]);
    return;
  }
  store_rows<OF32>(p.out, row, p.ld_out, col, left, x);
}
// The same for one element (the last step of a split product).
__device__ __forceinline__ void out1(const GemmParams& p, int64_t row, int col, float v, float bias) {
  v += bias;
  if (p.pre != nullptr) store1(p.pre, p.pre_f32, row * p.ld_pre + col, v);
  v = act_fwd(p.act, v);
  if (p.res != nullptr) v += load1(p.res, p.res_f32, row * p.ld_res + col);
  int64_t orow = row;
  if (p.row_map != nullptr) {
    orow = p.row_map[row];
    v *= p.row_scale[row];
  }
  store1(p.out, p.out_f32, orow * p.ld_out + col, v);
}
// Four columns of a row whose sums are complete (a split product), where rows
// lie on 16-byte boundaries and all four are inside: with bias and residual
// loaded before, or by itself and for the other rows too.
__device__ __forceinline__ void finish4(const GemmParams& p, int64_t row, int c, float4 s, float4 b, float4 r) {
  float e[4] = {s.x + b.x, s.y + b.y, s.z + b.z, s.w + b.w};
  if (p.pre != nullptr) store4(p.pre, p.pre_f32, row * p.ld_pre + c, make_float4(e[0], e[1], e[2], e[3]));
#pragma unroll
  for (int j = 0; j < 4; ++j) e[j] = act_fwd(p.act, e[j]);
  store4(p.out, p.out_f32, row * p.ld_out + c, make_float4(e[0] + r.x, e[1] + r.y, e[2] + r.z, e[3] + r.w));
}
__device__ __forceinline__ void out4(const GemmParams& p, int64_t row, int c, float4 s) {
  if (p.vec && c + 3 < p.n) {
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 b = p.bias != nullptr ? load4(p.bias, p.bias_f32, c) : zero;
    const float4 r = p.res != nullptr ? load4(p.res, p.res_f32, row * p.ld_res + c) : zero;
    finish4(p, row, c, s, b, r);
    return;
  }
  const float e[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < p.n) out1(p, row, c + j, e[j], p.bias != nullptr ? load1(p.bias, p.bias_f32, c + j) : 0.f);
}

// Joins two partial (maximum, sum of exponentials) of a row, base 2. A part
// without a maximum (every entry excluded) adds its sum, 0 or NaN.
__device__ __forceinline__ void stats_join(float& m, float& s, float2 q) {
  const float nm = fmaxf(m, q.x);
  if (nm == -INFINITY) {
    s += q.y;
    return;
  }
  s = s * ex2(m - nm) + q.y * ex2(q.x - nm);
  m = nm;
}

// Loss and log sum of up to 32 rows that count, from row i0 on, by a CTA of
// WARPS warps: the partials in strides over the warps with eight loads in
// flight, then the warps in order.
template <int WARPS>
__device__ __forceinline__ void join_rows(const float2* part, int parts, int64_t rows_ld, const float* at_target,
                                          int n, int i0, const int* idx, const float* weight, float* loss, float* lse,
                                          float2 (*red)[WARPS + 1]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float m = -INFINITY, s = 0.f;
  if (i0 + lane < n) {
    const float2* q = part + i0 + lane;
    for (int k = w; k < parts; k += 8 * WARPS) {
      float2 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = k + WARPS * j < parts ? __ldcg(q + (int64_t)(k + WARPS * j) * rows_ld) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) stats_join(m, s, v[j]);
    }
  }
  red[lane][w] = make_float2(m, s);
  __syncthreads();
  // a warp joins the parts of a row: a butterfly (each step joins the same two on both sides)
  for (int r = w; r < 32 && i0 + r < n; r += WARPS) {
    const float2 mine = lane < WARPS ? red[r][lane] : make_float2(-INFINITY, 0.f);
    m = mine.x, s = mine.y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float2 q = make_float2(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
      stats_join(m, s, q);
    }
    if (lane == 0) {
      const int i = i0 + r, row = idx[i];
      const float l = (m + log2f(s)) * kLn2;
      const float zt = __ldcg(at_target + i);
      // The loss from the target's logit and the maximum in base 2, with the product exact: the logits' own size
      // cancels before anything is rounded (l - zt, with l rounded at that size, was off by |zt| 2^-23, and below zero
      // for targets that are nearly certain). No probability is above one; a NaN stays.
      float d = fmaf(-zt, kLog2e, m) + log2f(s);
      d = d < 0.f ? 0.f : d * kLn2;
      // a target that is the excluded entry has probability zero, also where no entry is left
      if (zt == -INFINITY) d = INFINITY;
      lse[row] = l;
      loss[row] = weight != nullptr ? weight[row] * d : d;
    }
  }
}

// a / b for 0 <= a, 0 < b: by a float reciprocal where that is off by one at
// most (every role divides several times per tile).
__device__ __forceinline__ int fast_div(int a, int b) {
  if (a >= (1 << 20)) return a / b;
  int q = (int)((float)a * rcp_f((float)b));
  const int r = a - q * b;
  if (r < 0) --q;
  else if (r >= b) ++q;
  return q;
}
// Extents of one call with the device's row count applied, and its tiles.
struct Tile {
  int tm, tn, k0, k1, sp, q;  // q: problem of a paired launch
};
template <int CG>
struct Tiles {
  int m, k, mt, nt, nk, total;
  __device__ __forceinline__ Tiles(const GemmParams& p, int bk) {
    m = p.m;
    k = p.k;
    if (p.rows_axis == 1) m = min(m, *p.rows_dev);
    if (p.rows_axis == 2) k = min(k, *p.rows_dev);
    mt = (m + 128 * CG - 1) / (128 * CG);
    nt = (p.n + p.bn - 1) / p.bn;
    nk = (k + bk - 1) / bk;
    total = mt * nt * p.splits;
  }
  // Tile t: groups of group_m row tiles, all column tiles of a group before the
  // next. Its range of k: the split's, or in a cluster that joins, part `part`.
  __device__ __forceinline__ Tile at(const GemmParams& p, int t, int part, int parts) const {
    Tile x;
    x.q = 0;
    x.sp = p.splits == 1 ? 0 : fast_div(t, mt * nt);
    const int r = t - x.sp * (mt * nt), per = p.group_m * nt, g = fast_div(r, per), q = r - g * per;
    const int rows = min(p.group_m, mt - g * p.group_m);
    x.tn = fast_div(q, rows);
    x.tm = g * p.group_m + q - x.tn * rows;
    const int of = p.splits == 1 ? parts : p.splits, at = p.splits == 1 ? part : x.sp;
    x.k0 = of == 1 ? 0 : (int)((int64_t)nk * at / of);
    x.k1 = of == 1 ? nk : (int)((int64_t)nk * (at + 1) / of);
    return x;
  }
};

// Which tiles a unit (a CTA or a pair) works on: every units-th; one in a cluster
// that joins. A paired launch has two products: problem 0, whose tiles take
// longer, is dealt first; where that leaves units with a tile less, those get
// `pair_extra` tiles of problem 1 more (as many as fit beside one of problem 0)
// before the rest is dealt to all.
template <int CG, bool PAIR, bool JOIN>
struct Sched {
  Tiles<CG> T0, T1;
  int unit, units, part, parts;
  int own0, extra, rest, step;  // pair: tiles of problem 0, extra ones of 1, where the rest of 1 begins
  __device__ __forceinline__ Sched(const GemmParams& p0, const GemmParams& p1, int bk, int unit_, int units_, int part_,
                                   int parts_)
      : T0(p0, bk), T1(PAIR ? Tiles<CG>(p1, bk) : T0), unit(unit_), units(units_), part(part_), parts(parts_) {
    if constexpr (PAIR) {
      const int n0 = T0.total, n1 = T1.total, full = n0 / units, r = n0 - full * units;
      own0 = full + (unit < r ? 1 : 0);
      step = units - r;
      rest = r == 0 ? 0 : min(n1, p0.pair_extra * step);
      extra = unit >= r && rest > unit - r ? (rest - (unit - r) + step - 1) / step : 0;
    }
  }
  __device__ __forceinline__ const Tiles<CG>& of(const Tile& x) const { return PAIR && x.q ? T1 : T0; }
  // The unit's i-th tile.
  __device__ __forceinline__ bool get(const GemmParams& p0, const GemmParams& p1, int i, Tile& x) const {
    if constexpr (!PAIR) {
      if (JOIN && i > 0) return false;
      const int t = unit + i * units;
      if (t >= T0.total) return false;
      x = T0.at(p0, t, part, parts);
      return true;
    } else {
      if (i < own0) {
        x = T0.at(p0, unit + i * units, 0, 1);
        return true;
      }
      i -= own0;
      const int t = i < extra ? unit - (units - step) + i * step : rest + unit + (i - extra) * units;
      if (t >= T1.total) return false;
      x = T1.at(p1, t, 0, 1);
      x.q = 1;
      return true;
    }
  }
};

}  // namespace
}  // namespace bds

#include "gemm_gate.cuh"  // the epilogue of a gated layer

namespace bds {
namespace {

template <int CG, int BN, int NP, bool A_MN, bool B_MN, int EPI, bool OF32>
__global__ void __launch_bounds__(kGemmThreads, 1) k_gemm(const __grid_constant__ GemmCall<EPI == kEpiPair ? 2 : 1> call) {
  constexpr bool PAIR = EPI == kEpiPair;
  const GemmParams &p = call.p[0], &p1 = call.p[PAIR ? 1 : 0];
  using S = GemmSmem<CG, BN, NP, EPI>;
  constexpr int ST = S::kStages, BK = S::kBk;
  constexpr bool GATE = epi_gate(EPI);
  constexpr bool FLUSH = NP == 3;
  // accumulators in turn (fp32 loss training 1000 x 448 x 8191: with two 172 us, with four 167)
  constexpr int NA = BN <= 128 ? 4 : 2;
  constexpr uint32_t kCols = NA * BN;
  // debug build: the last output element of the launch (uniform over the grid)
  if (!dguard(kSiteGemm, p.out_last, p.out_extent)) return;
  if (PAIR && !dguard(kSiteGemm, p1.out_last, p1.out_extent)) return;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[8], empty[8], accfull[NA], accempty[NA];
  __shared__ uint32_t tslot;
  unsigned char* sm = align1024(smem_raw);
  const int t = threadIdx.x, lane = t & 31;
  const int w = __shfl_sync(0xffffffffu, t >> 5, 0);  // uniform over the warp, also to the compiler
  const uint32_t rank = CG == 2 ? cta_rank() : 0u;
  constexpr bool JOIN = EPI == kEpiJoin;
  const int parts = JOIN ? cluster_size() : 1, part = JOIN ? (int)cta_rank() : 0;  // ranges of k of a tile
  const int unit = (int)blockIdx.x / (JOIN ? parts : CG);
  const int units = (int)gridDim.x / (JOIN ? parts : CG);
  if (t == 96) {  // the maps are on their way while the barriers and TMEM are set up
#pragma unroll
    for (int q = 0; q < (PAIR ? 2 : 1); ++q) {
      prefetch_map(&call.m[q].a);
      prefetch_map(&call.m[q].b);
    }
    if (EPI == kEpiOut || EPI == kEpiDz || EPI == kEpiGate || EPI == kEpiGateDz) prefetch_map(&call.m[0].out);
    if (EPI == kEpiGateDz) prefetch_map(&call.m[0].pre);
  }
  if (t == 0) {
    for (int i = 0; i < ST; ++i) {
      umma::bar_init(&full[i], 1);
      umma::bar_init(&empty[i], 1);
    }
    for (int i = 0; i < NA; ++i) {
      umma::bar_init(&accfull[i], 1);
      umma::bar_init(&accempty[i], kEpiWarps * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  // The producer starts as soon as the barriers are there; the others also wait
  // for TMEM.
  if constexpr (CG == 2) {
    __syncthreads();
    cluster_sync_all();
  } else {
    __syncthreads();
  }
  uint32_t tm = 0;
  if (w != 0) {
    if (w == 2) gtmem_alloc<CG>(&tslot, kCols);
    umma::fence_before_sync();
    asm volatile("bar.sync 2, %0;\n" ::"n"(kGemmThreads - 32) : "memory");
    umma::fence_after_sync();
    tm = tslot;
  }
  pdl_sync();
  const Sched<CG, PAIR, JOIN> sched(p, p1, BK, unit, units, part, parts);
  const Tiles<CG>& T = sched.T0;
  if (w == 0) {
    // ---------------- producer ----------------
    // Producer and issuer run their loops as whole warps, one elected lane
    // issuing: addresses and descriptors then stay in uniform registers, where
    // the instructions want them. (As loops of lane 0 alone: 722 clocks per 64
    // of k instead of 512, 4864 x 16384 x 1024.)
    const bool leader = elect_one();
    const uint32_t base = umma::smem_u32(sm);
    const uint32_t full0 = CG == 2 ? map_cta(umma::smem_u32(&full[0]), 0) : umma::smem_u32(&full[0]);
    bool ok = true;
    int it = 0, s = 0;
    uint32_t ph = 0;  // stage and its phase
    Tile x;
    for (int i = 0; ok && sched.get(p, p1, i, x); ++i) {
      const GemmParams& pq = PAIR && x.q ? p1 : p;
      const CUtensorMap *amap = &call.m[PAIR ? x.q : 0].a, *bmap = &call.m[PAIR ? x.q : 0].b;
      const bool a_mn = PAIR ? pq.a_mn != 0 : A_MN;
      // columns of B that a CTA loads: its share of the tile, MN-major in whole groups of 64
      const int bcols = B_MN ? (pq.bn / CG + 63) / 64 : pq.bn / CG;
      const uint32_t stage_tx =
          CG * ((a_mn ? S::kA : (uint32_t)pq.a_rows * S::kRow) + (uint32_t)bcols * (B_MN ? S::kCol : S::kRow));
      const int m0 = x.tm * 128 * CG + (int)rank * 128;
      // a gated layer's pair of CTAs loads a projection each, a single CTA both
      const int n0 = GATE ? x.tn * (pq.bn / 2) + (CG == 2 ? (int)rank * (pq.n / 2) : 0)
                          : x.tn * pq.bn + (CG == 2 ? (int)rank * (pq.bn / 2) : 0);
      for (int kb = x.k0; kb < x.k1 && ok; ++kb) {
#pragma unroll
        for (int i = 0; i < NP; ++i, ++it) {
          if (!(ok = warp_wait(&empty[s], ph ^ 1))) break;
          if (leader) {
            const int q = kPiece<NP>(i);
            if (rank == 0) bar_expect_tx(&full[s], stage_tx);
            const uint32_t bar = full0 + 8u * (uint32_t)s;
            const uint32_t a = base + (uint32_t)s * S::kStage, b = a + S::kA;
            if (a_mn) {
#pragma unroll
              for (int j = 0; j < 2; ++j) gtma_load<CG>(a + j * S::kCol, amap, m0 + 64 * j, kb * BK, q, bar);
            } else {
              gtma_load<CG>(a, amap, kb * BK, m0, q, bar);
            }
            if constexpr (B_MN) {
#pragma unroll
              for (int j = 0; j < (BN / CG + 63) / 64; ++j)
                if (j < bcols) gtma_load<CG>(b + j * S::kCol, bmap, n0 + 64 * j, kb * BK, q, bar);
            } else {
              gtma_load<CG>(b, bmap, kb * BK, n0, q, bar);
              if constexpr (GATE && CG == 1)
                gtma_load<CG>(b + (uint32_t)(pq.bn / 2) * S::kRow, bmap, kb * BK, pq.n / 2 + n0, q, bar);
            }
          }
          if (++s == ST) s = 0, ph ^= 1;
        }
      }
    }
    // the stages in flight: consumed (their release has arrived in this CTA), or after a give-up at least landed
    for (int i = max(0, it - ST); i < it; ++i) {
      if (ok) ok = warp_wait(&empty[i % ST], (i / ST) & 1);
      if (!ok && rank == 0) warp_wait(&full[i % ST], (i / ST) & 1);
    }
    if (!ok && leader) atomicExch(p.flag, 1);
  } else if (w == 1) {
    // ---------------- MMA issue ----------------
    if (rank == 0) {
      const bool leader = elect_one();
      const uint32_t base = umma::smem_u32(sm);
      auto desc = [](uint32_t at, bool mn) {
        return umma::sdesc(at, mn ? S::kCol : 16u, 1024u);
      };
      const uint64_t db0 = desc(base + S::kA, B_MN);
      bool ok = true;
      uint32_t job = 0;
      int s = 0;
      uint32_t ph = 0;
      Tile x;
      for (int i = 0; ok && sched.get(p, p1, i, x); ++i) {
        const GemmParams& pq = PAIR && x.q ? p1 : p;
        const bool a_mn = PAIR ? pq.a_mn != 0 : A_MN;
        const uint32_t idesc = umma::idesc_bf16(128 * CG, (uint32_t)pq.bn, a_mn, B_MN);
        const uint32_t astep = a_mn ? 2048u : 32u, bstep = B_MN ? 2048u : 32u;  // bytes per 16 elements of k
        const uint64_t da0 = desc(base, a_mn);
        const int k0 = x.k0, k1 = x.k1;
        for (int kb = k0; kb < k1; ++kb) {
          const bool first = FLUSH || kb == k0, last = FLUSH || kb + 1 == k1;
          if (first) {
            if (!(ok = warp_wait(&accempty[job % NA], ((job / NA) & 1) ^ 1))) break;
            umma::fence_after_sync();
          }
          const uint32_t d = tm + job % NA * BN;
          // the four MMAs of 64 k from the A of stage sa and the B of stage sb
          auto four = [&](int sa, int sb, bool fresh) {
            const uint64_t da = umma::sdesc_adv(da0, (uint32_t)sa * S::kStage);
            const uint64_t db = umma::sdesc_adv(db0, (uint32_t)sb * S::kStage);
            if (leader) {
#pragma unroll
              for (int q = 0; q < BK / 16; ++q)
                gmma<CG>(d, umma::sdesc_adv(da, q * astep), umma::sdesc_adv(db, q * bstep), idesc, !fresh || q > 0);
            }
          };
          if constexpr (NP == 1) {
            if (!(ok = warp_wait(&full[s], ph))) break;
            four(s, s, first);
            if (leader) gcommit<CG>(&empty[s]);
            if (++s == ST) s = 0, ph ^= 1;
          } else {
            auto step = [&]() {  // the next stage once it is full
              const int at = s;
              ok = warp_wait(&full[s], ph);
              if (++s == ST) s = 0, ph ^= 1;
              return at;
            };
            const int s1 = step();
            if (!ok) break;
            four(s1, s1, true);
            const int s2 = step();
            if (!ok) break;
            const int s0 = step();
            if (!ok) break;
            four(s2, s0, false);
            four(s0, s2, false);
            if (leader) gcommit<CG>(&empty[s2]);
            four(s1, s0, false);
            four(s0, s1, false);
            if (leader) gcommit<CG>(&empty[s1]);
            four(s0, s0, false);
            if (leader) gcommit<CG>(&empty[s0]);
          }
          if (last) {
            if (leader) gcommit<CG>(&accfull[job % NA]);
            ++job;
          }
        }
      }
      if (!ok && leader) atomicExch(p.flag, 1);
    }
  } else if (w == 3) {
    // ---------------- column sums on the side ----------------
    if (p.sum_part != nullptr) {
      for (int64_t c = (int64_t)blockIdx.x * 32 + lane; c < p.sum_cols; c += (int64_t)gridDim.x * 32) {
        float sum = 0.f;
#pragma unroll 8
        for (int r = 0; r < p.sum_ranges; ++r) sum += p.sum_part[(int64_t)r * p.sum_cols + c];
        store1(p.sum_out, p.sum_f32, c, sum);
      }
    }
  } else if (GATE && w >= 4) {
    if constexpr (GATE) {
      const bool ok = gate_epilogue<CG, BN, NP, EPI, NA>(p, call.m[0], sched, tm, sm + ST * S::kStage, accfull, accempty,
                                                         (int)rank);
      if (!ok && lane == 0) atomicExch(p.flag, 1);
    }
  } else if (w >= 4) {
    // ---------------- epilogue ----------------
    const int ew = w - 4, quarter = ew >> 2;  // TMEM lanes 32 (w % 4) .. + 31, every fourth chunk of 32 columns
    const uint32_t lanes = tm + ((uint32_t)(32 * (w & 3)) << 16);
    unsigned char* stg = sm + ST * S::kStage + ew * 2048;
    uint32_t turn = 0;
    constexpr int NC = BN < 128 ? 1 : BN / 128;  // chunks of this warp at most
    constexpr bool IN32 = NP == 3;               // type of bias and pre
    const bool has_bias = EPI == kEpiOut && p.bias != nullptr, has_res = EPI == kEpiOut && p.res != nullptr;
    // what a unit needs besides its accumulators is loaded while the unit before is worked on, across tiles too
    uint4 braw[4], rraw[4];
    RowsAhead rahead;
    auto ahead_of = [&](int64_t row0, int col) {
      if constexpr (EPI == kEpiOut) {
        if (!IN32 && has_bias) load_bias(braw, p, col);
        if (has_res) load_res<OF32>(rraw, p, row0, col);
      }
      if constexpr (EPI == kEpiRows) load_rows_ahead<IN32>(rahead, p, row0, col);
    };
    auto first_row = [&](const Tile& x) { return (int64_t)x.tm * 128 * CG + rank * 128 + 32 * (w & 3); };
    bool ok = true;
    uint32_t job = 0;
    Tile x, nx;
    bool another = sched.get(p, p1, 0, nx);
    if (another) ahead_of(first_row(nx), nx.tn * p.bn + 32 * quarter);
    for (int i = 0; another;) {
      x = nx;
      another = sched.get(p, p1, ++i, nx);
      const GemmParams& pq = PAIR && x.q ? p1 : p;
      const int rows_m = sched.of(x).m;
      const int jobs = FLUSH ? x.k1 - x.k0 : (x.k1 > x.k0 ? 1 : 0);
      const int nend = min(pq.n, (x.tn + 1) * pq.bn);
      float acc[FLUSH ? NC * 32 : 1];
      if constexpr (FLUSH) {
#pragma unroll
        for (int i = 0; i < NC * 32; ++i) acc[i] = 0.f;
        if (EPI == kEpiOut && has_bias) {  // the sums start from the bias
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const int col = x.tn * p.bn + 32 * (4 * c + quarter);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float* b = static_cast<const float*>(p.bias) + col + i;
              if (col + i + 4 <= p.n) {
                const float4 u = *reinterpret_cast<const float4*>(b);
                acc[c * 32 + i] = u.x, acc[c * 32 + i + 1] = u.y, acc[c * 32 + i + 2] = u.z, acc[c * 32 + i + 3] = u.w;
              } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                  if (col + i + j < p.n) acc[c * 32 + i + j] = b[j];
              }
            }
          }
        }
        for (int j = 0; j < jobs; ++j, ++job) {
          if (!(ok = warp_wait(&accfull[job % NA], (job / NA) & 1))) break;
          umma::fence_after_sync();
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            float v[32];
            umma::tmem_ld32(lanes + job % NA * BN + 32u * (uint32_t)(4 * c + quarter), v);
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c * 32 + i] += v[i];
          }
          umma::fence_before_sync();
          __syncwarp();
          if (lane == 0) leader_arrive<CG>(&accempty[job % NA]);
        }
      }
      const int64_t row0 = first_row(x), row = row0 + lane;
      // per-row state of the loss epilogues
      float rm = -INFINITY, rs = 0.f, rlse = 0.f, ra = 1.f;
      int rt = -1;
      if constexpr (EPI == kEpiStats || EPI == kEpiDz) {
        if (row < T.m) {
          rt = p.target[row];
          if constexpr (EPI == kEpiDz) {
            rlse = p.lse[row];
            if (p.dz_scale != nullptr) ra = p.dz_scale[row];
          }
        }
      }
      if constexpr (!FLUSH) {
        if (jobs > 0) {
          ok = warp_wait(&accfull[job % NA], (job / NA) & 1);
          umma::fence_after_sync();
        }
      }
      if (!ok) {
        if constexpr (EPI == kEpiStats) epilogue_sync(true);  // this tile's barrier
        break;
      }
      const uint32_t tacc = lanes + job % NA * BN;
#pragma unroll(FLUSH ? NC : 1)
      for (int c = 0; c < NC; ++c) {
        const int ch = 4 * c + quarter;
        const int col0 = x.tn * pq.bn + 32 * ch;
        const bool live = 32 * ch < pq.bn && col0 < nend;  // uniform over the warp
        float v[32];
        if constexpr (FLUSH) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = acc[c * 32 + i];
        } else {
          if (jobs > 0 && live) {
            umma::tmem_ld32(tacc + 32u * (uint32_t)ch, v);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          if (c == NC - 1 && jobs > 0) {  // the accumulator may be overwritten
            umma::fence_before_sync();
            __syncwarp();
            if (lane == 0) leader_arrive<CG>(&accempty[job % NA]);
          }
        }
        // the unit after this chunk's last: the next chunk if that is live, else the next tile's first
        const bool more = c + 1 < NC && 32 * (ch + 4) < p.bn && col0 + 128 < nend;
        auto next = [&]() {
          if (more) ahead_of(row0, col0 + 128);
          else if (another) ahead_of(first_row(nx), nx.tn * p.bn + 32 * quarter);
        };
        if (!live) {
          if (c == 0) next();
          continue;
        }
        if constexpr (EPI == kEpiStats) {
          const int vcol = p.v0 + col0;
          const bool edge = col0 + 32 > nend || (unsigned)(p.excluded - vcol) < 32u;
          if (edge) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col0 + i >= nend || vcol + i == p.excluded) v[i] = -INFINITY;
          }
          if ((unsigned)(rt - vcol) < 32u && rt - vcol < nend - col0) {
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) z = rt - vcol == i ? v[i] : z;
            p.at_target[row] = z;
          }
          float mx = v[0];
#pragma unroll
          for (int i = 1; i < 32; ++i) mx = fmaxf(mx, v[i]);
          const float c = kLog2e * p.scale, nm = fmaxf(rm, mx * c);
          float add = 0.f;
#pragma unroll
          for (int i = 0; i < 32; ++i) add += ex2(fmaf(v[i], c, -nm));
          // a row with nothing so far (every entry excluded or past the end) stays at sum 0
          // (or at NaN, which the maximum passes over)
          if (nm != -INFINITY) {
            rs = rs * ex2(rm - nm) + add;
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) rs = isnan(v[i]) ? v[i] : rs;
          }
          rm = nm;
        } else if constexpr (EPI == kEpiDz) {
          const int vcol = p.v0 + col0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float d = ex2(fmaf(v[i], p.scale, -rlse) * kLog2e);
            d = vcol + i == rt ? d - 1.f : d;
            v[i] = vcol + i == p.excluded ? 0.f : d * ra;
          }
          if (row >= T.m) {  // rows up to the next tile edge are read by the product over rows: exact zeros
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          auto none = [] {};
          // the product over rows reads them in steps of 64; rows behind those are read, by the product for dh, for
          // rows that nobody keeps
          if (row0 >= ((T.m + 63) & ~63)) continue;
          if constexpr (NP == 1) {
            unit_store<false, 0>(&call.m[0].out, col0, (int)row0, 0, v, false, rraw, stg, none);
          } else {
#pragma unroll
            for (int k = 0; k < 3; ++k) {  // the largest piece of what is left of the value
              float q[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                q[i] = bf16_part(v[i]);
                v[i] -= q[i];
              }
              unit_store<false, 0>(&call.m[0].out, col0, (int)row0, k, q, false, rraw, stg, none);
            }
          }
        } else if constexpr (EPI == kEpiOut) {
          auto none = [] {};
          if (!IN32 && has_bias) add_bias(v, braw, p, col0);
          if (p.pre != nullptr) {
            unit_store<IN32, 0>(&call.m[0].pre, col0, (int)row0, 0, v, false, rraw, stg, none);
            if (IN32 && col0 + 16 < p.n) unit_store<IN32, 1>(&call.m[0].pre, col0 + 16, (int)row0, 0, v, false, rraw, stg, none);
          }
          if (p.act == kActSilu) {
#pragma unroll
            for (int i = 0; i < 32; i += 2) sigmoid_mul2<silu_arg>(v[i], v[i + 1]);
          } else if (p.act == kActGelu) {
#pragma unroll
            for (int i = 0; i < 32; i += 2) sigmoid_mul2<gelu_arg>(v[i], v[i + 1]);
          }
          if constexpr (OF32) {
            const bool two = col0 + 16 < p.n;
            unit_store<true, 0>(&call.m[0].out, col0, (int)row0, x.sp, v, has_res, rraw, stg, [&]() {
              if (!two) next();
              else if (has_res) load_res<true>(rraw, p, row0, col0 + 16);
            });
            if (two) unit_store<true, 1>(&call.m[0].out, col0 + 16, (int)row0, x.sp, v, has_res, rraw, stg, next);
          } else {
            unit_store<false, 0>(&call.m[0].out, col0, (int)row0, x.sp, v, has_res, rraw, stg, next);
          }
        } else if constexpr (JOIN) {
          float* mine = reinterpret_cast<float*>(sm) + (32 * (w & 3) + lane) * p.bn;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4*>(mine + 4 * ((8 * ch + j) ^ (lane & 7))) =
                make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        } else if (PAIR && pq.epi == kEpiOut) {
          const CUtensorMap* om = &call.m[PAIR ? x.q : 0].out;
          auto none = [] {};
          unit_store<OF32, 0>(om, col0, (int)row0, 0, v, false, rraw, stg, none);
          if (OF32 && col0 + 16 < pq.n) unit_store<OF32, OF32 ? 1 : 0>(om, col0 + 16, (int)row0, 0, v, false, rraw, stg, none);
        } else {
          // through shared memory, 16 columns at a time: 16 lanes per row, a row per half warp
          if (PAIR) {
            if (lane == 0) tma_store_wait_read();
            __syncwarp();
          }
          float* f = reinterpret_cast<float*>(stg);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              *reinterpret_cast<float4*>(f + lane * 16 + 4 * (j ^ ((lane >> 1) & 3))) =
                  make_float4(v[16 * h + 4 * j], v[16 * h + 4 * j + 1], v[16 * h + 4 * j + 2], v[16 * h + 4 * j + 3]);
            __syncwarp();
            const int cl = lane & 15, col = col0 + 16 * h + cl;
            if (col < nend) {
              float y[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int r = 2 * i + (lane >> 4);
                y[i] = f[r * 16 + 4 * ((cl >> 2) ^ ((r >> 1) & 3)) + (cl & 3)];
              }
              out_rows<IN32, OF32, PAIR>(pq, row0 + (lane >> 4), (int)min((int64_t)32, rows_m - row0) - (lane >> 4),
                                         col, y, rahead.res[h], rahead.bias[h]);
            }
            __syncwarp();
          }
          next();
        }
      }
      if constexpr (EPI == kEpiStats) {
        // the row's four quarters meet in shared memory (two buffers in turn:
        // a warp is at most one tile ahead of the one that joins)
        float2* q = reinterpret_cast<float2*>(sm + ST * S::kStage) + 512 * (turn++ & 1);
        q[128 * quarter + 32 * (w & 3) + lane] = make_float2(rm, rs);
        if (!(ok = !epilogue_sync(false))) break;
        if (quarter == 0 && row < T.m) {
#pragma unroll
          for (int k = 1; k < 4; ++k) stats_join(rm, rs, q[128 * k + 32 * w + lane - 128]);
          p.part[(int64_t)x.tn * p.rows_ld + row] = make_float2(rm, rs);
        }
      }
      if constexpr (!FLUSH) job += jobs;
    }
    // shared memory has been read; the stores themselves end with the grid
    if ((EPI == kEpiOut || EPI == kEpiDz || PAIR) && lane == 0) tma_store_wait_read();
    if (!ok && lane == 0) atomicExch(p.flag, 1);
  }
  umma::fence_before_sync();
  __syncthreads();
  if constexpr (JOIN) {
    // this thread's share of the tile; what its first four columns need besides the sums is loaded before the
    // barrier
    const bool any = unit < T.total;
    const Tile x = any ? T.at(p, unit, 0, 1) : Tile{0, 0, 0, 0, 0, 0};
    const int row0 = x.tm * 128, rows = any ? min(128, T.m - row0) : 0, groups = p.bn / 4;
    const uint32_t base = umma::smem_u32(sm);
    const int first = part * kGemmThreads + t;
    float4 b0 = make_float4(0.f, 0.f, 0.f, 0.f), r0 = b0;
    const int fr = fast_div(first, groups), fcol = x.tn * p.bn + 4 * (first - fr * groups);
    const bool early = p.vec && first < rows * groups && fcol + 3 < p.n;
    if (early) {
      if (p.bias != nullptr) b0 = load4(p.bias, p.bias_f32, fcol);
      if (p.res != nullptr) r0 = load4(p.res, p.res_f32, (row0 + fr) * p.ld_res + fcol);
    }
    cluster_sync_all();
    for (int i = first; i < rows * groups; i += parts * kGemmThreads) {
      const int r = fast_div(i, groups), g = i - r * groups;
      const int col = x.tn * p.bn + 4 * g;
      if (col >= p.n) continue;
      const uint32_t at = base + 16u * (uint32_t)(r * groups + (g ^ (r & 7)));
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k >= parts) break;
        const float4 q = load_cluster4(map_cta(at, k));
        sum.x += q.x, sum.y += q.y, sum.z += q.z, sum.w += q.w;
      }
      if (i == first && early) finish4(p, row0 + r, col, sum, b0, r0);
      else out4(p, row0 + r, col, sum);
    }
    cluster_sync_all();  // nobody leaves while its shared memory is read
  } else if constexpr (CG == 2) {
    cluster_sync_all();
  }
  umma::fence_after_sync();
  if (w == 2) gtmem_dealloc<CG>(tm, kCols);
  if constexpr (EPI == kEpiStats && CG == 1) {
    if (p.ticket != nullptr) {
      // every CTA's partials are out (the epilogue warps' writes, then the barrier above, then the fence)
      int* last = reinterpret_cast<int*>(&tslot);
      __syncthreads();  // tslot has been read by all
      if (t == 0) {
        __threadfence();
        *last = atomicAdd(p.ticket, 1) == (int)gridDim.x - 1;
      }
      __syncthreads();
      if (*last) {
        __threadfence();
        auto red = reinterpret_cast<float2 (*)[kGemmThreads / 32 + 1]>(sm);  // the stages have been consumed
        for (int i0 = 0; i0 < T.m; i0 += 32) {
          join_rows<kGemmThreads / 32>(p.part, T.nt, p.rows_ld, p.at_target, T.m, i0, p.row_idx, p.row_weight,
                                       p.loss_out, p.lse_out, red);
          __syncthreads();
        }
      }
    }
  }
}

// One CTA (or pair) per SM (or pair of SMs), at most one per tile; one cluster per tile where they join.
template <int CG, int BN, int NP, bool A_MN, bool B_MN, int EPI, bool OF32>
cudaError_t gemm_launch(const GemmCall<EPI == kEpiPair ? 2 : 1>& call, int64_t units, int cluster, cudaStream_t s) {
  using S = GemmSmem<CG, BN, NP, EPI>;
  auto kern = k_gemm<CG, BN, NP, A_MN, B_MN, EPI, OF32>;
  cudaError_t e = set_smem_cached(reinterpret_cast<const void*>(kern), (int)S::kBytes, 100);
  if (e != cudaSuccess) return e;
  if (EPI != kEpiJoin) {
    const int sms = sm_count_cached();
    const int64_t most = (sms > 0 ? sms : 152) / CG;
    if (units > most) units = most;
  }
  if (units <= 0) return cudaSuccess;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * cluster));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = S::kBytes;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, call);
}
inline int64_t gemm_tiles(const GemmParams& p, int cg) {
  return (int64_t)((p.m + 128 * cg - 1) / (128 * cg)) * ((p.n + p.bn - 1) / p.bn) * p.splits;
}
template <int CG, int BN, int NP, bool A_MN, bool B_MN, int EPI, bool OF32>
cudaError_t gemm_t(const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  GemmCall<1> call;
  call.p[0] = p;
  call.m[0] = m;
  return gemm_launch<CG, BN, NP, A_MN, B_MN, EPI, OF32>(call, gemm_tiles(p, CG), EPI == kEpiJoin ? p.join : CG, s);
}
template <int CG, int BN, int NP>
cudaError_t gemm_pair_t(const GemmCall<2>& call, cudaStream_t s) {
  const int64_t tiles = gemm_tiles(call.p[0], CG) + gemm_tiles(call.p[1], CG);
  return gemm_launch<CG, BN, NP, false, true, kEpiPair, NP == 3>(call, tiles, CG, s);
}

}  // namespace
}  // namespace bds
