// dense.cu -- the passes around the dense operators' matrix products
// (include/bdscan_dense.h): operand packing, the activation's gradient with
// the bias sums, the sums of a split product, a linear layer of a few rows,
// and the row bookkeeping of the loss. All are single passes over their data,
// bound by memory or by latency.
#include "dense.cuh"
#include "gemm.cuh"

namespace bds {
namespace {

constexpr int kThreads = 256;

// Eight consecutive values at p[at], which lies on a 16-byte boundary.
__device__ __forceinline__ void load8(float (&v)[8], const void* p, int f32, int64_t at) {
  if (f32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = q[0], b = q[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(p) + at);
    const uint32_t e[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(e[i] << 16);
      v[2 * i + 1] = __uint_as_float(e[i] & 0xffff0000u);
    }
  }
}

// The same as they lie in memory: bf16 in half the registers until they are used.
template <bool F32>
struct Raw8 {
  uint4 u[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + at * (F32 ? 4 : 2));
    u[0] = q[0];
    if (F32) u[F32 ? 1 : 0] = q[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t e[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (F32) {
        v[i] = __uint_as_float(e[i]);
      } else {
        v[2 * i] = __uint_as_float(e[i] << 16);
        v[2 * i + 1] = __uint_as_float(e[i] & 0xffff0000u);
      }
    }
    if (F32) {
      const uint4 w = u[F32 ? 1 : 0];
      v[4] = __uint_as_float(w.x), v[5] = __uint_as_float(w.y), v[6] = __uint_as_float(w.z), v[7] = __uint_as_float(w.w);
    }
  }
};

// Eight values from p[at] on, wherever that lies: the 16-byte groups that hold
// them are read whole and shifted into place, two or three wide loads instead of
// eight narrow ones (loss training, 40 rows, 894 x 5824 bf16: 55.4 -> 49.7 us).
// The tensor has `span` elements, starts on a 16-byte boundary and no group that
// reaches past its end is read: there, one element at a time. Values from `n` on
// are zero.
template <bool F32>
struct Any8 {
  static constexpr int kWords = F32 ? 12 : 8;
  uint32_t w[kWords];
  int shift;  // bytes
  __device__ __forceinline__ void load(const void* p, int64_t at, int n, int64_t span) {
    const int64_t first = at * (F32 ? 4 : 2);
    shift = (int)first & 15;
    const int groups = (F32 ? 2 : 1) + (shift != 0 ? 1 : 0);
    const char* q = static_cast<const char*>(p) + (first - shift);
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
    if (first - shift + 16 * groups <= span * (F32 ? 4 : 2)) {
#pragma unroll
      for (int g = 0; g < kWords / 4; ++g) {
        if (g < groups) {
          const uint4 u = *reinterpret_cast<const uint4*>(q + 16 * g);
          w[4 * g] = u.x, w[4 * g + 1] = u.y, w[4 * g + 2] = u.z, w[4 * g + 3] = u.w;
        }
      }
    } else {
      shift = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= n) break;
        if (F32) w[F32 ? j : 0] = __float_as_uint(static_cast<const float*>(p)[at + j]);
        else w[j / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[at + j] << (16 * (j & 1));
      }
    }
  }
  __device__ __forceinline__ void get(float (&v)[8], int n) const {
    uint32_t a[kWords - 2], b[kWords - 3];
#pragma unroll
    for (int i = 0; i < kWords - 2; ++i) a[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < kWords - 3; ++i) b[i] = shift & 4 ? a[i + 1] : a[i];
    if (F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(b[F32 ? j : 0]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t u = __funnelshift_r(b[i], b[i + 1], (shift & 2) * 8);
        v[2 * i] = __uint_as_float(u << 16);
        v[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] : 0.f;
  }
};

// ---- operand packing ----
// A warp converts 256 columns of one row, a lane eight consecutive ones. Operands that TMA can read where
// they lie never come here; the others, fp32 operands and the loss's rows cost
// one read and one write.
__device__ __forceinline__ void pack_store(bf16* d, int64_t plane, int pieces, const float (&v)[8]) {
  if (pieces == 1) {
    *reinterpret_cast<uint4*>(d) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    return;
  }
  __align__(16) bf16 q[3][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) split3(v[j], q[0][j], q[1][j], q[2][j]);
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(d + k * plane) = *reinterpret_cast<const uint4*>(q[k]);
}
// Eight columns of the operand's row from c on.
__device__ __forceinline__ void pack_load(float (&v)[8], const PackParams& p, int64_t row, int c) {
  const int64_t at = row * p.ld + c, span = (p.rows - 1) * p.ld + p.cols;
  const int n = (int)p.cols - c;
  if (p.ld % (p.src_f32 ? 4 : 8) == 0 && n >= 8) {
    load8(v, p.src, p.src_f32, at);
  } else if (p.src_f32) {
    Any8<true> u;
    u.load(p.src, at, n, span);
    u.get(v, n);
  } else {
    Any8<false> u;
    u.load(p.src, at, n, span);
    u.get(v, n);
  }
}
__device__ __forceinline__ void pack_block(const PackParams& p, int64_t block) {
  const int lane = threadIdx.x & 31;
  const int groups = (int)((p.ld_dst + 255) / 256);
  const int64_t idx = block * (kThreads / 32) + (threadIdx.x >> 5);
  const int64_t row = idx / groups;
  const int c0 = (int)(idx - row * groups) * 256;
  if (row >= p.rows) return;
  // debug build: the last element of the warp's row (no barrier follows)
  if (!dguard(kSitePack, (p.pieces - 1) * p.plane + row * p.ld_dst + p.ld_dst - 1, p.dst_extent)) return;
  const int c = c0 + 8 * lane;
  if (c >= p.ld_dst) return;
  float v[8];
  pack_load(v, p, row, c);
  pack_store(p.dst + row * p.ld_dst + c, p.plane, p.pieces, v);
}
int64_t pack_blocks(const PackParams& p) {
  return p.dst == nullptr ? 0 : (p.rows * ((p.ld_dst + 255) / 256) + kThreads / 32 - 1) / (kThreads / 32);
}
// One row's 256 columns from c0 on, to slot `to`: h, and in the backward h times
// the row's scale g.
__device__ __forceinline__ void pack_row(const PackParams& p, int64_t row, int64_t to, float g, int c0) {
  const int c = c0 + 8 * (threadIdx.x & 31);
  if (c >= p.ld_dst) return;
  float v[8];
  pack_load(v, p, row, c);
  pack_store(p.dst + to * p.ld_dst + c, p.plane, p.pieces, v);
  if (p.scaled == nullptr) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= g;
  pack_store(p.scaled + to * p.ld_dst + c, p.plane, p.pieces, v);
}
// Zeros in a slot behind the last row that counts, and in the gradient of a row that does not.
__device__ __forceinline__ void pack_zero_slot(const PackParams& p, int64_t to, int c0) {
  const int c = c0 + 8 * (threadIdx.x & 31);
  if (c >= p.ld_dst) return;
  const float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  pack_store(p.dst + to * p.ld_dst + c, p.plane, p.pieces, v);
  if (p.scaled != nullptr) pack_store(p.scaled + to * p.ld_dst + c, p.plane, p.pieces, v);
}
__device__ __forceinline__ void zero_gradient(const PackParams& p, int64_t row, int c0) {
  const int lane = threadIdx.x & 31, f32 = p.src_f32;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = c0 + 32 * j + lane;
    if (c < p.cols) store1(p.zero, f32, row * p.cols + c, 0.f);
  }
}

// The rows of the loss that count, each to its slot (pos), and zeros behind
// them up to a whole tile of rows; in the backward a second copy scaled by the
// row's weight, and zeros in the gradient of the rows that do not count. A warp
// per 256 columns of a row. Behind them the blocks of an operand to pack.
__global__ void __launch_bounds__(kThreads) k_pack_rows(const PackParams p, const PackParams b, int64_t na) {
  pdl_sync();
  if (blockIdx.x >= na) {
    pack_block(b, blockIdx.x - na);
    return;
  }
  const int groups = (int)((p.ld_dst + 255) / 256);
  const int64_t idx = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int64_t row = idx / groups;
  const int c0 = (int)(idx - row * groups) * 256;
  if (row >= p.rows) {
    const int n = *p.count;
    const int64_t to = n + (row - p.rows);
    if (to < ((n + 255) & ~255)) pack_zero_slot(p, to, c0);
    return;
  }
  const int to = p.pos[row];
  if (to >= 0) pack_row(p, row, to, p.gscale != nullptr ? p.gscale[to] : 0.f, c0);
  else if (p.zero != nullptr) zero_gradient(p, row, c0);
}

// Weight (times dloss) of row i of the loss, and its target: -1 where the row
// does not count.
__device__ __forceinline__ void loss_row(const LossRowsParams& p, int64_t i, float& wt, int64_t& tg) {
  const bool in = i < p.rows;
  tg = in ? p.target[i] : -1;
  wt = in && p.weight != nullptr ? p.weight[i] : 1.f;
  const float dl = in && p.dloss != nullptr ? p.dloss[i] : 1.f;
  if (wt == 0.f || dl == 0.f || tg >= p.vocab || tg < 0) tg = -1;
  wt *= dl;
}
// The slot's bookkeeping of a row that counts, the outputs of one that does not.
__device__ __forceinline__ void loss_row_out(const LossRowsParams& p, int64_t i, int to, float wt, int64_t tg) {
  if (tg >= 0) {
    p.idx[to] = (int)i;
    p.tgt[to] = (int)tg;
    if (p.gscale != nullptr) {
      p.gscale[to] = wt;
      p.lse_c[to] = p.lse_in[i];
    }
  } else if (p.loss != nullptr) {
    p.loss[i] = 0.f;
    p.lse[i] = 0.f;
  }
}

// Numbering and packing in one launch for up to kSmallRows rows: a CTA takes
// eight rows and counts all rows before them by itself (at most eight loads per
// thread, one latency), instead of waiting for a launch of its own.
constexpr int kSmallRows = 2048;
__global__ void __launch_bounds__(kThreads) k_loss_prep(const LossRowsParams l, const PackParams p, const PackParams b,
                                                        int64_t na) {
  pdl_sync();
  if (blockIdx.x >= na) {
    pack_block(b, blockIdx.x - na);
    return;
  }
  __shared__ int wsum[kThreads / 32];
  __shared__ int slot[8];
  __shared__ float scale[8];
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int rows = (int)l.rows, r0 = blockIdx.x * 8, before = min(r0, rows);
  int n = 0;
#pragma unroll
  for (int j = 0; j < kSmallRows / kThreads; ++j) {
    const int i = t + j * kThreads;
    if (i < before) {
      float wt;
      int64_t tg;
      loss_row(l, i, wt, tg);
      n += tg >= 0 ? 1 : 0;
    }
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) wsum[w] = n;
  __syncthreads();
  int at = 0;  // rows that count before this CTA's
#pragma unroll
  for (int k = 0; k < kThreads / 32; ++k) at += wsum[k];
  if (w == 0) {
    float wt = 0.f;
    int64_t tg = -1;
    if (lane < 8) loss_row(l, r0 + lane, wt, tg);
    const uint32_t m = __ballot_sync(0xffffffffu, tg >= 0);
    const int to = at + __popc(m & ((1u << lane) - 1u));
    if (lane < 8) {
      slot[lane] = tg >= 0 ? to : -1;
      scale[lane] = wt;
      if (r0 + lane < rows) loss_row_out(l, r0 + lane, to, wt, tg);
    }
    if (lane == 0 && r0 < rows && r0 + 8 >= rows) {
      l.count[0] = at + __popc(m);
      l.count[1] = 0;  // the ticket of the forward's product
    }
  }
  __syncthreads();
  const int row = r0 + w;
  for (int c0 = 0; c0 < p.ld_dst; c0 += 256) {
    if (row >= rows) {  // these CTAs have counted every row; the first of them may also hold the last rows
      int total = at;
      for (int k = 0; k < 8; ++k) total += slot[k] >= 0 ? 1 : 0;
      const int to = total + (row - rows);
      if (to < ((total + 255) & ~255)) pack_zero_slot(p, to, c0);
    } else if (slot[w] >= 0) {
      pack_row(p, row, slot[w], scale[w], c0);
    } else if (p.zero != nullptr) {
      zero_gradient(p, row, c0);
    }
  }
}

// ---- dz = dy act'(pre), and the column sums for the bias ----
// CTA: 256 columns (a lane holds 8) x one range of rows; its eight warps take
// every eighth row, four bf16 rows of a warp in flight as they lie in memory,
// their arithmetic in a loop of its own (two rows unpacked at once: the training
// step 16384 x 832 x 3328 237.5 us, with this 230). One read of dy and pre and
// one write of dz (16384 x 3328 bf16: 327 MB). The sums are of the unrounded
// products, added in a fixed order: rows of a warp, then warps, then ranges.
constexpr int kDactCols = 256;
template <bool DYF32, bool PREF32>
__device__ __forceinline__ void dact_block(const DactParams& p, int strip, int range) {
  __shared__ float red[8][kDactCols];
  constexpr int kDactFlight = DYF32 ? 2 : 4;  // rows of a warp in flight
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t r0 = p.rows * range / p.ranges, r1 = p.rows * (range + 1) / p.ranges;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const bool aligned = p.ld_dy % (DYF32 ? 4 : 8) == 0 && (p.act == kActNone || p.ld_pre % (PREF32 ? 4 : 8) == 0);
  const int c0 = strip * kDactCols, c = c0 + lane * 8, n = (int)p.cols - c;
  auto grad = [&](float (&e)[8], const float (&z)[8]) {
    if (p.act == kActSilu) {
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] *= act_grad(kActSilu, z[j]);
    } else if (p.act == kActGelu) {
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] *= act_grad(kActGelu, z[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += e[j];
  };
  auto finish = [&](int64_t r, float (&e)[8], const float (&z)[8]) {
    grad(e, z);
    if (p.dz != nullptr) pack_store(p.dz + r * p.ld_dz + c, p.plane, p.pieces, e);
  };
  if (aligned && n >= 8) {
    int64_t r = r0 + w;
    for (; r + 8 * (kDactFlight - 1) < r1; r += 8 * kDactFlight) {
      Raw8<DYF32> e[kDactFlight];
      Raw8<PREF32> z[kDactFlight];
#pragma unroll
      for (int i = 0; i < kDactFlight; ++i) {
        e[i].load(p.dy, (r + 8 * i) * p.ld_dy + c);
        if (p.act != kActNone) z[i].load(p.pre, (r + 8 * i) * p.ld_pre + c);
      }
#pragma unroll 1
      for (int i = 0; i < kDactFlight; ++i) {
        float ev[8], zv[8];
        e[0].get(ev);
        z[0].get(zv);
        finish(r + 8 * i, ev, zv);
#pragma unroll
        for (int j = 0; j + 1 < kDactFlight; ++j) e[j] = e[j + 1], z[j] = z[j + 1];
      }
    }
    for (; r < r1; r += 8) {
      float e[8], z[8];
      load8(e, p.dy, DYF32, r * p.ld_dy + c);
      if (p.act != kActNone) load8(z, p.pre, PREF32, r * p.ld_pre + c);
      finish(r, e, z);
    }
  } else if (n > 0) {
    constexpr int kFlight = DYF32 ? 1 : 2;
    const int64_t dy_span = (p.rows - 1) * p.ld_dy + p.cols, pre_span = (p.rows - 1) * p.ld_pre + p.cols;
    for (int64_t r = r0 + w; r < r1; r += 8 * kFlight) {
      Any8<DYF32> e[kFlight];
      Any8<PREF32> z[kFlight];
#pragma unroll
      for (int i = 0; i < kFlight; ++i) {
        if (r + 8 * i >= r1) break;
        e[i].load(p.dy, (r + 8 * i) * p.ld_dy + c, n, dy_span);
        if (p.act != kActNone) z[i].load(p.pre, (r + 8 * i) * p.ld_pre + c, n, pre_span);
      }
#pragma unroll 1
      for (int i = 0; i < kFlight && r + 8 * i < r1; ++i) {
        float ev[8], zv[8];
        e[0].get(ev, n);
        z[0].get(zv, n);
        finish(r + 8 * i, ev, zv);
#pragma unroll
        for (int j = 0; j + 1 < kFlight; ++j) e[j] = e[j + 1], z[j] = z[j + 1];
      }
    }
  }
  if (p.part == nullptr) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) red[w][j * 32 + lane] = sum[j];
  __syncthreads();
  const int lc = threadIdx.x, col = c0 + (lc & 31) * 8 + (lc >> 5);
  if (col < p.cols) {
    float s = red[0][lc];
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i][lc];
    p.part[(int64_t)range * p.cols + col] = s;
  }
}

// The passes over a call's inputs in one launch: dz first (the longest), then
// the operands that have to be packed.
template <bool DYF32, bool PREF32>
__global__ void __launch_bounds__(kThreads, 3) k_prep(const DactParams d, const PackParams a, const PackParams b,
                                                      int64_t nd, int64_t na) {
  pdl_sync();
  const int64_t block = blockIdx.x;
  if (block < nd) {
    const int strips = (int)((d.cols + kDactCols - 1) / kDactCols);
    dact_block<DYF32, PREF32>(d, (int)(block % strips), (int)(block / strips));
  } else if (block < nd + na) {
    pack_block(a, block - nd);
  } else {
    pack_block(b, block - nd - na);
  }
}
__global__ void __launch_bounds__(kThreads) k_pack(const PackParams a, const PackParams b, int64_t na) {
  pdl_sync();
  const int64_t block = blockIdx.x;
  if (block < na) pack_block(a, block);
  else pack_block(b, block - na);
}

// Sum over row ranges, 32 columns per CTA, eight warps in strides, fixed order.
__global__ void __launch_bounds__(kThreads) k_colsum(const float* part, int ranges, int64_t cols, void* out,
                                                     int out_f32) {
  pdl_sync();
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int r = w; r < ranges; r += 8) s += part[(int64_t)r * cols + c];
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i][lane];
    store1(out, out_f32, c, s);
  }
}

// ---- the sums of a split product ----
// Four columns of one row per SLICES threads: each adds every SLICES-th split, in
// order, with eight loads in flight, and the first adds the slices, in order, and
// ends them as the product's own output step would. With one thread for all 64
// splits of a small output the reads were a chain of latencies (11 us).
template <int SLICES>
__global__ void __launch_bounds__(kThreads) k_split_reduce(const GemmParams p, const float* part, int64_t ld) {
  pdl_sync();
  constexpr int G = kThreads / SLICES;  // groups of four columns per CTA
  __shared__ float4 red[SLICES][G];
  const int64_t groups = ld / 4;
  const int slice = threadIdx.x / G, lg = threadIdx.x % G;
  const int64_t idx = (int64_t)blockIdx.x * G + lg;
  const int64_t row = idx / groups;
  const int c = (int)(idx - row * groups) * 4;
  int m = p.m;
  if (p.rows_axis == 1) m = min(m, *p.rows_dev);
  if (!dguard(kSiteSplitReduce, p.out_last, p.out_extent)) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row < m) {
    const float* at = part + row * ld + c;
    for (int i = slice; i < p.splits; i += 8 * SLICES) {
      float4 q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        q[j] = i + j * SLICES < p.splits ? *reinterpret_cast<const float4*>(at + (i + j * SLICES) * p.split_stride)
                                         : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) s.x += q[j].x, s.y += q[j].y, s.z += q[j].z, s.w += q[j].w;
    }
  }
  if constexpr (SLICES > 1) {
    red[slice][lg] = s;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int k = 1; k < SLICES; ++k) {
      const float4 q = red[k][lg];
      s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
    }
  }
  if (row < m) out4(p, row, c, s);
}

// ---- a linear layer of a few rows ----
// One warp per NC output columns: the weights are streamed once, 16 bytes per
// lane and column, and the rows' x, of which every warp reads all, comes from
// L1. One row is bound by the read of a large w (bf16: 4096 x 50304 6.7 TB/s,
// 832 x 50304 4.9 with launch and tail), by latency else; eight rows of 832 x
// 50304 take 54 us, where the matrix product takes 18 for 24. Sums over k: 32
// lanes in strides, then a butterfly, all in fp32.
template <typename T, int ROWS, int NC, bool VEC>
__global__ void __launch_bounds__(128) k_linear_vec(const VecParams p) {
  pdl_sync();
  constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;  // elements per load
  const int lane = threadIdx.x & 31;
  const int64_t n0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * NC;
  if (n0 >= p.n) return;
  if (!dguard(kSiteLinearVec, (p.rows - 1) * p.ld_y + p.n - 1, p.out_extent)) return;
  const T* x = static_cast<const T*>(p.x);
  const T* w = static_cast<const T*>(p.w);
  float acc[ROWS][NC];
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[r][c] = 0.f;
#pragma unroll 2
  for (int k = lane * E; k < p.k; k += 32 * E) {
    float wv[NC][E];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int64_t n = n0 + c < p.n ? n0 + c : p.n - 1;
      if constexpr (VEC) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4*>(w + n * p.k + k));
        const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
        for (int j = 0; j < E; ++j) wv[c][j] = cvt(e[j]);
      } else {
        wv[c][0] = cvt(w[n * p.k + k]);
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (r < p.rows) {
        float xv[E];
        if constexpr (VEC) {
          const uint4 u = *reinterpret_cast<const uint4*>(x + r * p.ld_x + k);
          const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
          for (int j = 0; j < E; ++j) xv[j] = cvt(e[j]);
        } else {
          xv[0] = cvt(x[r * p.ld_x + k]);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < E; ++j) acc[r][c] = fmaf(xv[j], wv[c][j], acc[r][c]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[r][c] += __shfl_xor_sync(0xffffffffu, acc[r][c], o);
  // lane r * NC + c finishes output (r, c)
  float v = 0.f;
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int c = 0; c < NC; ++c) v = lane == r * NC + c ? acc[r][c] : v;
  const int r = lane / NC;
  const int64_t n = n0 + lane % NC;
  if (lane >= ROWS * NC || r >= p.rows || n >= p.n) return;
  const int f32 = sizeof(T) == 4;
  if (p.bias != nullptr) v += load1(p.bias, f32, n);
  if (p.pre != nullptr) store1(p.pre, f32, (int64_t)r * p.n + n, v);
  v = act_fwd(p.act, v);
  if (p.res != nullptr) v += load1(p.res, p.out_f32, r * p.ld_res + n);
  store1(p.y, p.out_f32, r * p.ld_y + n, v);
}

// ---- rows of the loss ----
// A CTA takes `per` rows (a multiple of 1024). It counts the rows before its
// own, all of them, rather than waiting for another CTA's count: up to 64 CTAs
// re-read at most the 16 bytes per row that the launch reads anyway, from L2.
// Then it numbers its own rows, 1024 at a time. (One CTA for all rows, which
// reads them twice: 21 us at 16384 rows; this 10, from DRAM.)
constexpr int kRowsCtas = 64;
__global__ void __launch_bounds__(1024) k_loss_rows(const LossRowsParams p, int64_t per) {
  pdl_sync();
  constexpr int F = 4;
  __shared__ int wsum[32];
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int64_t begin = blockIdx.x * per, end = min(begin + per, p.rows);
  int n = 0;
  for (int64_t i = t; i < begin; i += 1024 * F) {
    float wt[F];
    int64_t tg[F];
#pragma unroll
    for (int j = 0; j < F; ++j) loss_row(p, i + 1024 * j < begin ? i + 1024 * j : p.rows, wt[j], tg[j]);
#pragma unroll
    for (int j = 0; j < F; ++j) n += tg[j] >= 0 ? 1 : 0;
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) wsum[w] = n;
  __syncthreads();
  int at = __reduce_add_sync(0xffffffffu, wsum[lane]);  // rows before this CTA's
  for (int64_t i0 = begin; i0 < end; i0 += 1024) {
    const int64_t i = i0 + t;
    float wt;
    int64_t tg;
    loss_row(p, i, wt, tg);
    const bool c = tg >= 0;
    const uint32_t m = __ballot_sync(0xffffffffu, c);
    __syncthreads();  // wsum has been read
    if (lane == 0) wsum[w] = __popc(m);
    __syncthreads();
    const int mine = wsum[lane];
    const int before = __reduce_add_sync(0xffffffffu, lane < w ? mine : 0);
    const int to = at + before + __popc(m & ((1u << lane) - 1u));
    at += __reduce_add_sync(0xffffffffu, mine);
    if (i >= p.rows) continue;  // no barrier is skipped: the loop ends for the whole CTA with this round
    p.pos[i] = c ? to : -1;
    loss_row_out(p, i, to, wt, tg);
  }
  if (end == p.rows && t == 0) {
    p.count[0] = at;
    p.count[1] = 0;  // the ticket of the forward's product
  }
}

// The rows' partial maxima and sums joined, 32 rows per CTA.
__global__ void __launch_bounds__(1024) k_loss_combine(const float2* part, int parts, int64_t rows_ld,
                                                       const float* at_target, const int* count, const int* idx,
                                                       const float* weight, float* loss, float* lse) {
  pdl_sync();
  __shared__ float2 red[32][33];
  const int n = *count, i0 = blockIdx.x * 32;
  if (i0 < n) join_rows<32>(part, parts, rows_ld, at_target, n, i0, idx, weight, loss, lse, red);
}

template <typename T, int ROWS, int NC>
void vec_t(const VecParams& p, bool vec, cudaStream_t s) {
  const unsigned grid = (unsigned)((p.n + 4 * NC - 1) / (4 * NC));
  if (vec) launch_pdl(k_linear_vec<T, ROWS, NC, true>, grid, 128, 0, s, p);
  else launch_pdl(k_linear_vec<T, ROWS, NC, false>, grid, 128, 0, s, p);
}
template <typename T>
void vec_rows(const VecParams& p, bool vec, cudaStream_t s) {
  // four columns per warp share its loads of x, once there are columns enough to fill the SMs that way
  const bool wide = p.n >= 8192;
  if (p.rows == 1) wide ? vec_t<T, 1, 4>(p, vec, s) : vec_t<T, 1, 1>(p, vec, s);
  else if (p.rows <= 4) wide ? vec_t<T, 4, 4>(p, vec, s) : vec_t<T, 4, 1>(p, vec, s);
  else wide ? vec_t<T, 8, 4>(p, vec, s) : vec_t<T, 8, 1>(p, vec, s);
}

}  // namespace

int64_t small_loss_rows() { return kSmallRows; }
cudaError_t launch_pack(const PackParams& a, const PackParams& b, cudaStream_t s) {
  const int64_t na = pack_blocks(a), nb = pack_blocks(b);
  if (na + nb == 0) return cudaSuccess;
  launch_pdl(k_pack, dim3((unsigned)(na + nb)), dim3(kThreads), 0, s, a, b, na);
  return cudaGetLastError();
}
cudaError_t launch_loss_prep(const LossRowsParams& l, const PackParams& p, const PackParams& b, cudaStream_t s) {
  const int64_t na = (l.rows + 256 + 7) / 8;
  launch_pdl(k_loss_prep, dim3((unsigned)(na + pack_blocks(b))), dim3(kThreads), 0, s, l, p, b, na);
  return cudaGetLastError();
}
cudaError_t launch_pack_rows(const PackParams& p, const PackParams& b, cudaStream_t s) {
  const int64_t n = (p.rows + 256) * ((p.ld_dst + 255) / 256), na = (n + kThreads / 32 - 1) / (kThreads / 32);
  launch_pdl(k_pack_rows, dim3((unsigned)(na + pack_blocks(b))), dim3(kThreads), 0, s, p, b, na);
  return cudaGetLastError();
}
cudaError_t launch_prep(const DactParams& p, const PackParams& a, const PackParams& b, cudaStream_t s) {
  const int64_t nd = (p.cols + kDactCols - 1) / kDactCols * p.ranges, na = pack_blocks(a), nb = pack_blocks(b);
  const dim3 grid((unsigned)(nd + na + nb));
  if (p.pre_f32) launch_pdl(k_prep<true, true>, grid, dim3(kThreads), 0, s, p, a, b, nd, na);
  else if (p.dy_f32) launch_pdl(k_prep<true, false>, grid, dim3(kThreads), 0, s, p, a, b, nd, na);
  else launch_pdl(k_prep<false, false>, grid, dim3(kThreads), 0, s, p, a, b, nd, na);
  return cudaGetLastError();
}
cudaError_t launch_colsum(const float* part, int ranges, int64_t cols, void* out, int out_f32, cudaStream_t s) {
  launch_pdl(k_colsum, dim3((unsigned)((cols + 31) / 32)), dim3(kThreads), 0, s, part, ranges, cols, out, out_f32);
  return cudaGetLastError();
}
cudaError_t launch_split_reduce(const GemmParams& p, const float* part, cudaStream_t s) {
  const int64_t ld = (p.n + 3) / 4 * 4, n = (int64_t)p.m * (ld / 4);
  auto grid = [&](int slices) { return dim3((unsigned)((n + kThreads / slices - 1) / (kThreads / slices))); };
  if (p.splits > 8) launch_pdl(k_split_reduce<8>, grid(8), dim3(kThreads), 0, s, p, part, ld);
  else launch_pdl(k_split_reduce<1>, grid(1), dim3(kThreads), 0, s, p, part, ld);
  return cudaGetLastError();
}
cudaError_t launch_linear_vec(const VecParams& p, cudaStream_t s) {
  const int e = p.f32 ? 4 : 8;
  const bool vec = p.k % e == 0 && p.ld_x % e == 0;
  if (p.f32) vec_rows<float>(p, vec, s);
  else vec_rows<bf16>(p, vec, s);
  return cudaGetLastError();
}
cudaError_t launch_loss_rows(const LossRowsParams& p, cudaStream_t s) {
  int64_t per = (p.rows + kRowsCtas - 1) / kRowsCtas;
  per = (per + 1023) / 1024 * 1024;
  launch_pdl(k_loss_rows, dim3((unsigned)((p.rows + per - 1) / per)), dim3(1024), 0, s, p, per);
  return cudaGetLastError();
}
cudaError_t launch_loss_combine(const float2* part, int parts, int64_t rows_ld, const float* at_target,
                                const int* count, const int* idx, const float* weight, float* loss, float* lse,
                                int64_t rows, cudaStream_t s) {
  launch_pdl(k_loss_combine, dim3((unsigned)((rows + 31) / 32)), dim3(1024), 0, s, part, parts, rows_ld, at_target,
             count, idx, weight, loss, lse);
  return cudaGetLastError();
}

}  // namespace bds
