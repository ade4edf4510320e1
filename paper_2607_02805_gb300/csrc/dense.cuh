// dense.cuh -- argument blocks and launchers of the dense operators
// (include/bdscan_dense.h): the tcgen05 matrix product of gemm.cuh and the
// passes around it.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace bds {

// What a product does with its accumulators.
constexpr int kEpiOut = 0;    // residual + act(acc + bias), or a split's partial sums, by TMA
constexpr int kEpiRows = 3;   // the same by plain stores: unaligned or mapped rows
constexpr int kEpiJoin = 4;   // the same, the ranges of k of a tile joined by a cluster
constexpr int kEpiPair = 5;   // two products in one launch, each kEpiOut or kEpiRows without bias, activation and residual
constexpr int kEpiStats = 1;  // running maximum and sum of a row's logits, and the target's logit
constexpr int kEpiDz = 2;     // the loss's gradient at the logits

// A [m][k] or [k][m], B [n][k] or [k][n] come as tensor maps; extents in elements.
struct GemmParams {
  int m, n, k;
  // Rows that count, known on the device only: limits m (1), k (2) or nothing (0).
  const int* rows_dev;
  int rows_axis;
  int bn;         // columns of a tile (a multiple of 32, at most the instance's BN)
  int splits;     // ranges of k, each with its own partial sums
  int join;       // kEpiJoin: CTAs of a tile's cluster, each with a range of k
  int group_m;    // row tiles walked together
  int a_rows;     // rows that a load of A brings (K-major): 128, or what a single smaller tile has, in eights
  int epi, a_mn;  // kEpiPair: kEpiOut or kEpiRows, and how A lies
  int pair_extra; // kEpiPair, problem 0: tiles of problem 1 that take as long as one of its own
  // kEpiOut, kEpiRows: out[row_map ? row_map[i] : i][j]; kEpiOut has res of out's type
  const void* bias;
  const void* res;
  void* out;
  void* pre;
  const int* row_map;
  const float* row_scale;  // with row_map: row i is scaled by row_scale[i]
  int64_t ld_res, ld_out, ld_pre;
  int64_t split_stride;  // elements between the partial sums of two splits
  int bias_f32, res_f32, out_f32, pre_f32;
  int act;
  int vec;               // rows of out, pre and res start on 16-byte boundaries, none is mapped
  int64_t out_last, out_extent;  // last element written and elements of `out` or `part` (debug build)
  // kEpiStats / kEpiDz: rows i are the rows that count; column j is entry v0 + j
  int v0, excluded;
  const int* target;     // [rows] of the rows that count
  float2* part;          // [column tiles][rows] (maximum, sum of exponentials), base 2
  float* at_target;      // [rows]
  int64_t rows_ld;       // rows of `part`
  const float* lse;      // [rows] of the rows that count
  // kEpiStats with few rows: the last CTA to end (by `ticket`, zero before)
  // joins the partial statistics into the outputs; null: launch_loss_combine does
  int* ticket;
  const int* row_idx;
  const float* row_weight;
  float *loss_out, *lse_out;
  // Column sums that a warp without another role finishes on the side (the bias
  // gradient, from launch_prep's partial sums): sum_out[c] = sum of
  // sum_part[0 .. sum_ranges - 1][c]; null: none.
  const float* sum_part;
  void* sum_out;
  int64_t sum_cols;
  int sum_ranges, sum_f32;
  int* flag;             // set by a bounded wait that gave up
};

constexpr int kGemmBk = 64;  // elements of k per stage: one 128-byte swizzled row

// Instances: CG 1 or 2 CTAs per tile, BN columns at most, `pieces` bf16 pieces
// per operand (1: bf16 operands, 3: fp32 operands).
struct GemmCfg {
  int cg, bn, pieces;
  bool a_mn, b_mn;  // operand rows along k (true) or along m / n (false)
  int epi;
  bool out_f32;     // kEpiOut, kEpiRows
};

// Tensor maps of a product; `out` and `pre` for kEpiOut, `out` for kEpiDz.
struct GemmMaps {
  CUtensorMap a, b, out, pre;
};
template <int N>
struct GemmCall {
  GemmMaps m[N];
  GemmParams p[N];
};
// Sums of the partial sums of p.splits splits, then the output step of kEpiOut.
cudaError_t launch_split_reduce(const GemmParams& p, const float* part, cudaStream_t s);

// rows x cols of src (row stride ld) into `pieces` bf16 planes with row stride
// ld_dst (a multiple of 8): the values themselves (bf16), or three pieces whose
// sum they are (fp32).
struct PackParams {
  const void* src;
  int64_t ld, rows, cols;
  __nv_bfloat16* dst;
  int64_t ld_dst, plane;
  int src_f32, pieces;
  int64_t dst_extent;  // elements of dst (debug build)
  // launch_pack_rows only: slot of each row or -1, the number of slots, and in
  // the backward the slots' scales, the scaled copy and the gradient to zero
  const int *pos, *count;
  const float* gscale;
  __nv_bfloat16* scaled;
  void* zero;
};
// One launch for two operands; dst null: nothing to pack.
cudaError_t launch_pack(const PackParams& a, const PackParams& b, cudaStream_t s);
cudaError_t launch_pack_rows(const PackParams& p, const PackParams& b, cudaStream_t s);  // b: one more operand

// dz = dy * act'(pre) in `pieces` bf16 planes, and partial column sums of the
// unrounded values per row range.
struct DactParams {
  const void* dy;
  const void* pre;
  int64_t ld_dy, ld_pre, rows, cols;
  int dy_f32, pre_f32, act, pieces;
  __nv_bfloat16* dz;  // null: sums only
  int64_t ld_dz, plane;
  float* part;  // [ranges][cols], null: no sums
  int ranges;
};
// That and up to two operands to pack, in one launch.
cudaError_t launch_prep(const DactParams& p, const PackParams& a, const PackParams& b, cudaStream_t s);
cudaError_t launch_colsum(const float* part, int ranges, int64_t cols, void* out, int out_f32, cudaStream_t s);

// y = res + act(x w^T + bias) for a few rows, without the tensor cores.
constexpr int kVecRows = 8;
struct VecParams {
  const void *x, *w, *bias, *res;
  void *y, *pre;
  int64_t ld_x, ld_res, ld_y;
  int rows, k, n, act, f32, out_f32;
  int64_t out_extent;  // elements of y (debug build)
};
cudaError_t launch_linear_vec(const VecParams& p, cudaStream_t s);

// The rows of the loss that count (weight, and dloss if given, not zero, and a
// target inside the vocabulary), in order: their number, index, target and
// gradient scale. Rows that do not count get loss = lse = 0 where given.
struct LossRowsParams {
  const int64_t* target;
  const float *weight, *dloss, *lse_in;
  int64_t rows, vocab;
  int *count, *idx, *tgt, *pos;  // count [2]: rows that count, and a zero; pos [rows]: slot, or -1
  float *gscale, *lse_c;
  float *loss, *lse;
};
cudaError_t launch_loss_rows(const LossRowsParams& p, cudaStream_t s);
// launch_loss_rows and launch_pack_rows in one, for up to small_loss_rows() rows.
int64_t small_loss_rows();
cudaError_t launch_loss_prep(const LossRowsParams& l, const PackParams& p, const PackParams& b, cudaStream_t s);
cudaError_t launch_loss_combine(const float2* part, int parts, int64_t rows_ld, const float* at_target,
                                const int* count, const int* idx, const float* weight, float* loss, float* lse,
                                int64_t rows, cudaStream_t s);
int* ssd_wait_flag_ptr();  // ssd.cu

}  // namespace bds
