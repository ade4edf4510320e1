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

// ---- operand packing ----
// A thread converts four columns of one row. Operands whose rows start on
// 16-byte boundaries are read in place and never come here; the others, fp32
// operands and the loss's gathered rows cost one read and one write.
__global__ void __launch_bounds__(kThreads) k_pack(const PackParams p) {
  pdl_sync();
  const int64_t groups = p.ld_dst / 4;
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = idx / groups;
  const int c = (int)(idx - row * groups) * 4;
  if (row >= p.rows) return;
  int64_t src_row = row;
  bool zero = false;
  if (p.idx != nullptr) {
    const int n = *p.count;
    if (row >= ((n + 255) & ~255)) return;
    zero = row >= n;
    if (!zero) src_row = p.idx[row];
  }
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (!zero) {
    const int64_t at = src_row * p.ld + c;
    if (p.ld % 4 == 0 && c + 3 < p.cols) {
      const float4 q = load4(p.src, p.src_f32, at);
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < p.cols) v[j] = load1(p.src, p.src_f32, at + j);
    }
  }
  bf16* d = p.dst + row * p.ld_dst + c;
  if (p.pieces == 1) {
    *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    return;
  }
  __align__(8) bf16 q[3][4];
#pragma unroll
  for (int j = 0; j < 4; ++j) split3(v[j], q[0][j], q[1][j], q[2][j]);
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(d + k * p.plane) = *reinterpret_cast<const uint2*>(q[k]);
}

// ---- dz = dy act'(pre), and the column sums for the bias ----
// CTA: 128 columns (a warp's lanes hold 4 each) x one range of rows; its eight
// warps take every eighth row. The sums are of the unrounded products, added
// in a fixed order: rows of a warp, then warps, then ranges.
__global__ void __launch_bounds__(kThreads) k_dact(const DactParams p) {
  pdl_sync();
  __shared__ float4 red[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int c = blockIdx.x * 128 + lane * 4;
  const int64_t r0 = p.rows * blockIdx.y / p.ranges, r1 = p.rows * (blockIdx.y + 1) / p.ranges;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool full = c + 3 < p.cols && p.ld_dy % 4 == 0 && (p.act == kActNone || p.ld_pre % 4 == 0);
  for (int64_t r = r0 + w; r < r1; r += 8) {
    if (c >= p.cols) break;
    float e[4] = {0.f, 0.f, 0.f, 0.f};
    if (full) {
      const float4 g = load4(p.dy, p.dy_f32, r * p.ld_dy + c);
      e[0] = g.x, e[1] = g.y, e[2] = g.z, e[3] = g.w;
      if (p.act != kActNone) {
        const float4 z = load4(p.pre, p.pre_f32, r * p.ld_pre + c);
        e[0] *= act_grad(p.act, z.x), e[1] *= act_grad(p.act, z.y);
        e[2] *= act_grad(p.act, z.z), e[3] *= act_grad(p.act, z.w);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < p.cols) {
          e[j] = load1(p.dy, p.dy_f32, r * p.ld_dy + c + j);
          if (p.act != kActNone) e[j] *= act_grad(p.act, load1(p.pre, p.pre_f32, r * p.ld_pre + c + j));
        }
    }
    sum.x += e[0], sum.y += e[1], sum.z += e[2], sum.w += e[3];
    if (p.dz != nullptr) {
      bf16* d = p.dz + r * p.ld_dz + c;
      if (p.pieces == 1) {
        *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]));
      } else {
        __align__(8) bf16 q[3][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split3(e[j], q[0][j], q[1][j], q[2][j]);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(d + k * p.plane) = *reinterpret_cast<const uint2*>(q[k]);
      }
    }
  }
  if (p.part == nullptr) return;
  red[w][lane] = sum;
  __syncthreads();
  if (w == 0 && c < p.cols) {
    float4 s = red[0][lane];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const float4 q = red[i][lane];
      s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
    }
    const float e[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < p.cols) p.part[(int64_t)blockIdx.y * p.cols + c + j] = e[j];
  }
}

// Sum over row ranges, 32 columns per CTA, eight warps in strides, fixed order.
__global__ void __launch_bounds__(kThreads) k_colsum(const float* part, int ranges, int64_t cols, void* out,
                                                     int out_f32) {
  pdl_sync();
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols)
    for (int r = w; r < ranges; r += 8) s += part[(int64_t)r * cols + c];
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += red[i][lane];
    store1(out, out_f32, c, s);
  }
}

// ---- the sums of a split product ----
// A thread adds four columns of one row over the splits, in order, and ends
// them as the product's own output step would.
__global__ void __launch_bounds__(kThreads) k_split_reduce(const GemmParams p, const float* part, int64_t ld) {
  pdl_sync();
  const int64_t groups = ld / 4;
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = idx / groups;
  const int c = (int)(idx - row * groups) * 4;
  int m = p.m;
  if (p.rows_axis == 1) m = min(m, *p.rows_dev);
  if (row >= m) return;
  float4 s = *reinterpret_cast<const float4*>(part + row * ld + c);
  for (int i = 1; i < p.splits; ++i) {
    const float4 q = *reinterpret_cast<const float4*>(part + i * p.split_stride + row * ld + c);
    s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
  }
  float e[4] = {s.x, s.y, s.z, s.w};
  if (p.tma_out && p.vec && c + 3 < p.n && p.row_map == nullptr) {  // rows on 16-byte boundaries
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (p.bias != nullptr) e[j] += load1(p.bias, p.bias_f32, c + j);
    if (p.pre != nullptr) store4(p.pre, p.pre_f32, row * p.ld_pre + c, make_float4(e[0], e[1], e[2], e[3]));
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = act_fwd(p.act, e[j]);
    if (p.res != nullptr) {
      const float4 r = load4(p.res, p.res_f32, row * p.ld_res + c);
      e[0] += r.x, e[1] += r.y, e[2] += r.z, e[3] += r.w;
    }
    store4(p.out, p.out_f32, row * p.ld_out + c, make_float4(e[0], e[1], e[2], e[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < p.n) out1(p, row, c + j, e[j], p.bias != nullptr ? load1(p.bias, p.bias_f32, c + j) : 0.f, 0);
  }
}

// ---- a linear layer of a few rows ----
// One warp per NC output columns: the weights are streamed once, 16 bytes per
// lane and column, and the rows' x, of which every warp reads all, comes from
// L1. Bound by the read of w (6.7 TB/s) for a large w, by latency else. Sums
// over k: 32 lanes in strides, then a butterfly, all in fp32.
template <typename T, int ROWS, int NC, bool VEC>
__global__ void __launch_bounds__(128) k_linear_vec(const VecParams p) {
  pdl_sync();
  constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;  // elements per load
  const int lane = threadIdx.x & 31;
  const int64_t n0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * NC;
  if (n0 >= p.n) return;
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
__device__ __forceinline__ bool row_counts(const int64_t* target, const float* weight, const float* dloss,
                                           int64_t vocab, int64_t i) {
  const int64_t t = target[i];
  return t >= 0 && t < vocab && (weight == nullptr || weight[i] != 0.f) && (dloss == nullptr || dloss[i] != 0.f);
}

// One CTA: each thread counts a run of rows, a scan over the threads gives the
// run's first slot, and the thread fills it in order.
__global__ void __launch_bounds__(1024) k_loss_rows(const LossRowsParams p) {
  pdl_sync();
  __shared__ int wsum[32];
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int64_t per = (p.rows + 1023) / 1024;
  const int64_t r0 = min(p.rows, t * per), r1 = min(p.rows, r0 + per);
  int n = 0;
  for (int64_t i = r0; i < r1; ++i) n += row_counts(p.target, p.weight, p.dloss, p.vocab, i) ? 1 : 0;
  int inc = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) wsum[w] = inc;
  __syncthreads();
  if (w == 0) {
    int v = wsum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    wsum[lane] = v;
  }
  __syncthreads();
  int at = inc - n + (w > 0 ? wsum[w - 1] : 0);
  for (int64_t i = r0; i < r1; ++i) {
    if (row_counts(p.target, p.weight, p.dloss, p.vocab, i)) {
      p.idx[at] = (int)i;
      p.tgt[at] = (int)p.target[i];
      if (p.gscale != nullptr) {
        const float wt = p.weight != nullptr ? p.weight[i] : 1.f;
        p.gscale[at] = p.dloss != nullptr ? wt * p.dloss[i] : wt;
        p.lse_c[at] = p.lse_in[i];
      }
      ++at;
    } else if (p.loss != nullptr) {
      p.loss[i] = 0.f;
      p.lse[i] = 0.f;
    }
  }
  if (t == 1023) *p.count = at;
}

// Joins a row's partial maxima and sums: 32 rows per CTA, eight warps over the
// partials in strides, then the warps in order.
__global__ void __launch_bounds__(kThreads) k_loss_combine(const float2* part, int parts, int64_t rows_ld,
                                                           const float* at_target, const int* count, const int* idx,
                                                           const float* weight, float* loss, float* lse) {
  pdl_sync();
  __shared__ float2 red[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t i = (int64_t)blockIdx.x * 32 + lane;
  if ((int64_t)blockIdx.x * 32 >= *count) return;
  const bool live = i < *count;
  float m = -INFINITY, s = 0.f;
  if (live)
    for (int k = w; k < parts; k += 8) stats_join(m, s, part[(int64_t)k * rows_ld + i]);
  red[w][lane] = make_float2(m, s);
  __syncthreads();
  if (w == 0 && live) {
#pragma unroll
    for (int k = 1; k < 8; ++k) stats_join(m, s, red[k][lane]);
    const float l = (m + log2f(s)) * kLn2;
    const int row = idx[i];
    const float zt = at_target[i];
    // a target that is the excluded entry has probability zero, also where no entry is left
    const float d = zt == -INFINITY ? INFINITY : l - zt;
    lse[row] = l;
    loss[row] = weight != nullptr ? weight[row] * d : d;
  }
}

__global__ void __launch_bounds__(kThreads) k_zero_rows(const int64_t* target, const float* weight,
                                                        const float* dloss, int64_t rows, int64_t vocab,
                                                        unsigned char* dst, int64_t row_bytes) {
  pdl_sync();
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows || row_counts(target, weight, dloss, vocab, row)) return;
  unsigned char* d = dst + row * row_bytes;
  const int lane = threadIdx.x & 31;
  if (row_bytes % 16 == 0) {
    for (int64_t b = lane * 16; b < row_bytes; b += 512) *reinterpret_cast<uint4*>(d + b) = make_uint4(0, 0, 0, 0);
  } else {
    for (int64_t b = lane * 2; b < row_bytes; b += 64) *reinterpret_cast<unsigned short*>(d + b) = 0;
  }
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

cudaError_t launch_pack(const PackParams& p, cudaStream_t s) {
  const int64_t n = p.rows * (p.ld_dst / 4);
  if (n == 0) return cudaSuccess;
  launch_pdl(k_pack, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p);
  return cudaGetLastError();
}
cudaError_t launch_dact(const DactParams& p, cudaStream_t s) {
  launch_pdl(k_dact, dim3((unsigned)((p.cols + 127) / 128), (unsigned)p.ranges), dim3(kThreads), 0, s, p);
  return cudaGetLastError();
}
cudaError_t launch_colsum(const float* part, int ranges, int64_t cols, void* out, int out_f32, cudaStream_t s) {
  launch_pdl(k_colsum, dim3((unsigned)((cols + 31) / 32)), dim3(kThreads), 0, s, part, ranges, cols, out, out_f32);
  return cudaGetLastError();
}
cudaError_t launch_split_reduce(const GemmParams& p, const float* part, cudaStream_t s) {
  const int64_t ld = (p.n + 3) / 4 * 4, n = (int64_t)p.m * (ld / 4);
  launch_pdl(k_split_reduce, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p, part, ld);
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
  launch_pdl(k_loss_rows, dim3(1), dim3(1024), 0, s, p);
  return cudaGetLastError();
}
cudaError_t launch_loss_combine(const float2* part, int parts, int64_t rows_ld, const float* at_target,
                                const int* count, const int* idx, const float* weight, float* loss, float* lse,
                                int64_t rows, cudaStream_t s) {
  launch_pdl(k_loss_combine, dim3((unsigned)((rows + 31) / 32)), dim3(kThreads), 0, s, part, parts, rows_ld, at_target,
             count, idx, weight, loss, lse);
  return cudaGetLastError();
}
cudaError_t launch_zero_rows(const int64_t* target, const float* weight, const float* dloss, int64_t rows,
                             int64_t vocab, void* dst, int64_t row_bytes, cudaStream_t s) {
  launch_pdl(k_zero_rows, dim3((unsigned)((rows + 7) / 8)), dim3(kThreads), 0, s, target, weight, dloss, rows, vocab,
             static_cast<unsigned char*>(dst), row_bytes);
  return cudaGetLastError();
}

}  // namespace bds
