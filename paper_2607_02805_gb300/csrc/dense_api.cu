// dense_api.cu -- the C ABI of the dense operators (include/bdscan_dense.h):
// argument validation, workspace layout, the choice of tiles and splits, and
// the launch sequences.
#include <cudaTypedefs.h>

#include <cstdio>
#include <cstring>

#include "bdscan_dense.h"
#include "dense.cuh"
#include "params.h"

namespace bds {

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();  // ssd.cu

cudaError_t launch_gemm_nt(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_nn(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_tn(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_nt3(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_nn3(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_tn3(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);
cudaError_t launch_gemm_pair(const GemmCfg&, const GemmCall<2>&, cudaStream_t);
cudaError_t launch_gemm_loss(const GemmCfg&, const GemmParams&, const GemmMaps&, cudaStream_t);

namespace {

int fail_msg(int code, const char* fn, const char* what) {
  char msg[384];
  snprintf(msg, sizeof(msg), "%s: %s", fn, what);
  return api_fail(code, msg);
}
int fail_arg(const char* fn, const char* name, const char* problem) {
  char msg[384];
  snprintf(msg, sizeof(msg), "%s: %s %s", fn, name, problem);
  return api_fail(BDSCAN_ERR_ARG, msg);
}
int cuda_fail(cudaError_t e, const char* fn) { return fail_msg(BDSCAN_ERR_CUDA, fn, cudaGetErrorString(e)); }

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

#define DENSE_REQ(ptr, fn, name)                                               \
  do {                                                                         \
    if ((ptr) == nullptr) return fail_arg(fn, name, "is NULL");                \
    if (!aligned16(ptr)) return fail_arg(fn, name, "is not 16-byte aligned");  \
  } while (0)
#define DENSE_OPT(ptr, fn, name)                                               \
  do {                                                                         \
    if ((ptr) != nullptr && !aligned16(ptr)) return fail_arg(fn, name, "is not 16-byte aligned"); \
  } while (0)

// Sizes above these are refused: extents of tensor maps and row indices are
// 32-bit, and the products of two extents are 64-bit everywhere.
constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxCols = (int64_t)1 << 24;

// A bf16 operand in memory: `rows` rows of `inner` contiguous elements.
struct Operand {
  const void* base;
  int64_t inner, rows, ld;
  int pieces;
  int64_t plane;
};

// Boxes of 64 elements x `box_rows` rows, 128-byte swizzle; elements outside
// the operand read as zero.
bool encode(CUtensorMap* m, const Operand& o, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.rows, (cuuint64_t)o.pieces};
  const int64_t plane = o.pieces > 1 ? o.plane : up(o.ld * 8, 8);  // one piece: never stepped over
  const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)plane * 2};
  const cuuint32_t box[3] = {(cuuint32_t)kGemmBk, (cuuint32_t)box_rows, 1u};
  const cuuint32_t estr[3] = {1u, 1u, 1u};
  return tensor_map_encoder()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.base), dims, strides, box,
                              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The output [planes][rows][cols] as the epilogue stores it: boxes of 32
// rows x 64 bytes.
bool encode_out(CUtensorMap* m, const void* base, int f32, int64_t cols, int64_t rows, int64_t ld, int planes,
                int64_t plane) {
  const int64_t elt = f32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)(ld * elt), (cuuint64_t)((planes > 1 ? plane : ld * 8) * elt)};
  const cuuint32_t box[3] = {f32 ? 16u : 32u, 32u, 1u};
  const cuuint32_t estr[3] = {1u, 1u, 1u};
  return tensor_map_encoder()(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                              const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_64B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Whether rows of `ld` elements start on 16-byte boundaries.
bool rows16(int64_t ld, int f32) { return ld % (f32 ? 4 : 8) == 0; }

// Whether rows of `ld` elements of `dtype` can be read by TMA where they lie.
bool in_place(int dtype, int64_t ld) { return dtype == BDSCAN_BF16 && ld % 8 == 0; }
size_t packed_bytes(int dtype, int64_t rows, int64_t cols) {
  return al256((size_t)rows * up(cols, 8) * 2 * (dtype == BDSCAN_F32 ? 3 : 1));
}

// Tiles and splits of a product of m x n over k. Functions of the sizes only,
// for 152 SMs, so that workspace sizes do not depend on the device.
struct Plan {
  GemmCfg cfg;
  int bn, splits, join, group_m;  // splits > 1: through memory; join > 1: in clusters
  double cost;
};
constexpr int64_t kSms = 152;
// The choice minimises a model of the product's time in clocks. A tile's step
// of 64 k takes the larger of its MMAs (128 x 256 x 16 in 128 clocks per SM)
// and its operands' way from L2 (80 bytes per clock and SM); a tile adds about
// 400 clocks, and the epilogue of the last one 8 per column; the sums of a split
// add a launch and their way to memory and back, a cluster that joins 5000
// clocks; a launch of pairs of CTAs starts 1500 clocks later.
// Over 28 shapes of the three forms (64 to 50,024 rows, both types) its choice
// was the fastest of all candidates or within 5 % of it, except small products,
// which pairs of CTAs started later than it knew: 5.1 us against 4.0.
struct Instance {
  int cg, bn;
};
// Clocks of a tile's step of 64 k. bf16 B with rows along k (b_mn) is loaded in
// whole groups of 64 columns. fp32 loads count at 48 bytes per clock: over 30
// fp32 cases that chose better than 64 or 80 (means of 49.5, 50.3 and 52.7 us),
// since those steps hold the two closer together.
double step_clocks(int64_t m, int cg, int bn, int pieces, bool b_mn) {
  const double mma = 2.0 * bn * (pieces == 3 ? 6 : 1);
  const int64_t cols = b_mn && pieces == 1 ? up(bn / cg, 64) : bn / cg;
  const double load = (pieces == 3 ? 8.0 : 1.6) * (double)((m < 128 ? m : 128) + cols);
  const double least = pieces == 3 ? 800 : 300;  // the stages in flight at a latency of about 1800 clocks
  const double step = mma > load ? mma : load;
  return step > least ? step : least;
}
double product_clocks(const Plan& q, int64_t m, int64_t n, int64_t k) {  // q.cfg.b_mn set
  const int cg = q.cfg.cg;
  const int64_t nk = (k + 63) / 64, tiles = (m + 128 * cg - 1) / (128 * cg) * ((n + q.bn - 1) / q.bn);
  const double step = step_clocks(m, cg, q.bn, q.cfg.pieces, q.cfg.b_mn);
  if (q.join > 1) return 1500 + (nk + q.join - 1) / q.join * step + 8.0 * q.bn + 5000;
  const int64_t waves = (tiles * q.splits + kSms / cg - 1) / (kSms / cg);
  double cost = (cg == 2 ? 3000 : 1500) + waves * ((nk + q.splits - 1) / q.splits * step + 400) + 8.0 * q.bn;
  if (q.splits > 1) cost += 5000 + 8.0 * q.splits * m * n / 3000;
  return cost;
}
// Where the rows that count are known on the device only, m2 and k2 (not zero)
// are the sizes with half of them, and the choice minimises the sum of both.
Plan plan(int64_t m, int64_t n, int64_t k, int pieces, bool may_split, bool b_mn, int64_t m2 = 0, int64_t k2 = 0) {
  static const Instance bf16_any[] = {{2, 256}, {1, 128}}, f32_any[] = {{2, 128}, {1, 128}};
  const Instance* inst = pieces == 3 ? f32_any : bf16_any;
  const int64_t nk = (k + 63) / 64;
  Plan best, q;
  memset(&best, 0, sizeof(best));
  best.cost = -1;
  auto consider = [&]() {
    q.cost = product_clocks(q, m, n, k);
    if (m2 > 0) q.cost += product_clocks(q, m2, n, k2);
    if (best.cost < 0 || q.cost < best.cost) best = q;
  };
  for (int i = 0; i < 2; ++i) {
    const int cg = inst[i].cg;
    if (cg == 2 && m <= 128) continue;
    const int64_t units = kSms / cg, mt = (m + 128 * cg - 1) / (128 * cg);
    for (int bn = inst[i].bn; bn >= 32; bn -= 32) {
      if (bn - 32 >= n) continue;
      const int64_t tiles = mt * ((n + bn - 1) / bn);
      memset(&q, 0, sizeof(q));
      q.cfg.cg = cg;
      q.cfg.bn = inst[i].bn;
      q.cfg.pieces = pieces;
      q.cfg.b_mn = b_mn;
      q.bn = bn;
      q.group_m = cg == 2 ? 8 : 12;
      q.splits = q.join = 1;
      consider();
      if (!may_split) continue;
      for (int waves = 1; waves <= 4; ++waves) {
        int64_t s = units * waves / tiles;
        if (s > nk / 2) s = nk / 2;
        if (s > 64) s = 64;
        if (s <= 1) continue;
        q.splits = (int)s;
        consider();
      }
      q.splits = 1;
      // a cluster per tile, as many as are resident together (fp32 by twos was slower than pairs without a
      // split: 2048 x 448 x 1792 training step 86 us against 82)
      for (int j = 2; cg == 1 && pieces == 1 && j <= 8; j *= 2) {
        if (tiles > (j == 2 ? 76 : j == 4 ? 36 : 15) || nk < 2 * j) break;
        q.join = j;
        consider();
      }
    }
  }
  return best;
}
// Two products in one launch (the gradients of a linear layer or of the head),
// neither of them split: instead of a launch (about 6000 clocks with its start
// and end) and two last waves. Problem 0 is the one with the longer tiles.
struct PairPlan {
  Plan q[2];
  int extra;
  double cost;
};
PairPlan plan_pair(const int64_t (&m)[2], const int64_t (&n)[2], const int64_t (&k)[2], int pieces) {
  static const Instance bf16_any[] = {{2, 256}, {1, 128}}, f32_any[] = {{2, 128}, {1, 128}};
  const Instance* inst = pieces == 3 ? f32_any : bf16_any;
  PairPlan best;
  memset(&best, 0, sizeof(best));
  best.cost = -1;
  for (int i = 0; i < 2; ++i) {
    const int cg = inst[i].cg;
    if (cg == 2 && m[0] <= 128 && m[1] <= 128) continue;
    const double units = (double)(kSms / cg);
    double tile[2][8], count[2][8];
    for (int j = 0; j < 2; ++j)
      for (int c = 0; c < 8; ++c) {
        const int bn = 32 * (c + 1);
        count[j][c] = 0;
        if (bn > inst[i].bn || bn - 32 >= n[j]) continue;
        tile[j][c] = (k[j] + 63) / 64 * step_clocks(m[j], cg, bn, pieces, true) + 400;
        count[j][c] = (double)((m[j] + 128 * cg - 1) / (128 * cg)) * ((n[j] + bn - 1) / bn);
      }
    for (int c = 7; c >= 0; --c)
      for (int d = 7; d >= 0; --d) {
        if (count[0][c] == 0 || count[1][d] == 0 || tile[0][c] < tile[1][d]) continue;
        const double first = (double)(int64_t)((count[0][c] + units - 1) / units) * tile[0][c];
        const double all = (count[0][c] * tile[0][c] + count[1][d] * tile[1][d]) / units + 0.5 * tile[1][d];
        const double one = count[0][c] + count[1][d] <= units ? tile[0][c] : all;
        const double cost = (cg == 2 ? 3000 : 1500) + (first > one ? first : one) + 8.0 * 32 * (c > d ? c + 1 : d + 1);
        if (best.cost >= 0 && cost >= best.cost) continue;
        best.cost = cost;
        const int bn[2] = {32 * (c + 1), 32 * (d + 1)};
        for (int j = 0; j < 2; ++j) {
          best.q[j].cfg.cg = cg;
          best.q[j].cfg.bn = inst[i].bn;
          best.q[j].cfg.pieces = pieces;
          best.q[j].cfg.b_mn = true;
          best.q[j].bn = bn[j];
          best.q[j].splits = best.q[j].join = 1;
          best.q[j].group_m = cg == 2 ? 8 : 12;
        }
        best.extra = (int)(tile[0][c] / tile[1][d] + 0.5);
      }
  }
  return best;
}
// The gradient's products as the calls make them: dx = dz w and dw = dz^T x, one
// launch where that is estimated to be faster.
struct GradPlan {
  Plan x, w;
  PairPlan pair;
  bool one, w_first;
};
GradPlan plan_grad(int64_t rows, int64_t in, int64_t out, int pieces, int64_t rows2 = 0) {
  GradPlan g;
  g.x = plan(rows, in, out, pieces, true, true, rows2, out);
  g.w = plan(out, in, rows, pieces, true, true, rows2 > 0 ? out : 0, rows2);
  const int64_t r = rows2 > 0 ? (rows + rows2 + 1) / 2 : rows;
  const PairPlan wx = plan_pair({out, r}, {in, in}, {r, out}, pieces);
  const PairPlan xw = plan_pair({r, out}, {in, in}, {out, r}, pieces);
  g.w_first = xw.cost < 0 || (wx.cost >= 0 && wx.cost < xw.cost);
  g.pair = g.w_first ? wx : xw;
  const double two = (g.x.cost + g.w.cost) / (rows2 > 0 ? 2 : 1) + 3000;
  g.one = g.pair.cost >= 0 && g.pair.cost < two;
  return g;
}
size_t split_bytes(const Plan& q, int64_t m, int64_t n) {
  return q.splits > 1 ? al256((size_t)q.splits * m * up(n, 4) * 4) : 0;
}

// The geometry of a plan's launch; the caller adds the epilogue's fields.
GemmParams geometry(const Plan& q, int64_t m, int64_t n, int64_t k, int* flag) {
  GemmParams p;
  memset(&p, 0, sizeof(p));
  p.m = (int)m;
  p.n = (int)n;
  p.k = (int)k;
  p.bn = q.bn;
  p.splits = 1;
  p.group_m = q.group_m;
  // rows outside the operand are filled at a row's cost too (24 rows, 832 x 50304, w in L2: 21.8 us by 128, 12.8 by
  // 24); in the last of several tiles, smaller boxes brought nothing (300 x 1024 x 4000: 8.7 us against 7.1)
  p.a_rows = m < 128 ? (int)up(m, 8) : 128;
  p.excluded = -1;
  p.flag = flag;
  return p;
}

// `p.out` has `planes` planes (splits, or pieces of the logits' gradient) of
// `out_rows` rows.
cudaError_t run_product(const Plan& q, const GemmParams& p, const Operand& a, const Operand& b, int planes,
                        int64_t plane, int64_t out_rows, cudaStream_t s) {
  GemmMaps m;
  memset(&m, 0, sizeof(m));
  if (!encode(&m.a, a, q.cfg.a_mn ? kGemmBk : p.a_rows) || !encode(&m.b, b, q.cfg.b_mn ? kGemmBk : q.bn / q.cfg.cg))
    return cudaErrorInvalidValue;
  const int epi = q.cfg.epi;
  if ((epi == kEpiOut || epi == kEpiDz) && !encode_out(&m.out, p.out, p.out_f32, p.n, out_rows, p.ld_out, planes, plane))
    return cudaErrorInvalidValue;
  if (epi == kEpiOut && p.pre != nullptr && !encode_out(&m.pre, p.pre, p.pre_f32, p.n, out_rows, p.ld_pre, 1, 0))
    return cudaErrorInvalidValue;
  const bool f32 = q.cfg.pieces == 3;
  cudaError_t e;
  if (epi == kEpiStats || epi == kEpiDz) e = launch_gemm_loss(q.cfg, p, m, s);
  else if (q.cfg.a_mn) e = f32 ? launch_gemm_tn3(q.cfg, p, m, s) : launch_gemm_tn(q.cfg, p, m, s);
  else if (q.cfg.b_mn) e = f32 ? launch_gemm_nn3(q.cfg, p, m, s) : launch_gemm_nn(q.cfg, p, m, s);
  else e = f32 ? launch_gemm_nt3(q.cfg, p, m, s) : launch_gemm_nt(q.cfg, p, m, s);
  return api_launched(e, s);
}

// A product with the output step of kEpiOut, split over k where the plan says
// so: then the partial sums go to `part` and a second launch ends it. `padded`:
// the output is fp32 in the workspace, its rows padded to 16 bytes.
cudaError_t run_out(Plan q, bool a_mn, bool b_mn, GemmParams p, const Operand& a, const Operand& b, float* part,
                    cudaStream_t s, bool padded = false) {
  q.cfg.a_mn = a_mn;
  q.cfg.b_mn = b_mn;
  // TMA stores whole groups of 16 bytes: a row has to end on such a boundary as
  // well, unless what follows is padding of the workspace
  const int64_t width = padded ? up(p.n, 4) : p.n;
  p.vec = p.row_map == nullptr && rows16(p.ld_out, p.out_f32) && rows16(width, p.out_f32) &&
          (p.pre == nullptr || (rows16(p.ld_pre, p.pre_f32) && rows16(width, p.pre_f32))) &&
          (p.res == nullptr || (p.res_f32 == p.out_f32 && rows16(p.ld_res, p.res_f32)));
  q.cfg.epi = p.vec ? kEpiOut : kEpiRows;
  q.cfg.out_f32 = p.out_f32 != 0;
  if (q.join > 1) {
    q.cfg.epi = kEpiJoin;
    p.join = q.join;
  }
  p.out_last = p.row_map != nullptr ? p.out_extent - 1 : (p.m - 1) * p.ld_out + p.n - 1;
  if (q.splits == 1) return run_product(q, p, a, b, 1, 0, p.m, s);
  GemmParams g = p;
  g.splits = q.splits;
  g.bias = g.res = nullptr;
  g.pre = nullptr;
  g.row_map = nullptr;
  g.out = part;
  g.ld_out = up(p.n, 4);
  g.split_stride = p.m * g.ld_out;
  g.out_f32 = 1;
  q.cfg.epi = kEpiOut;
  q.cfg.out_f32 = true;
  g.act = BDSCAN_ACT_NONE;
  g.out_extent = (int64_t)q.splits * g.split_stride;
  g.out_last = (q.splits - 1) * g.split_stride + (p.m - 1) * g.ld_out + p.n - 1;
  cudaError_t e = run_product(q, g, a, b, q.splits, g.split_stride, p.m, s);
  if (e != cudaSuccess) return e;
  p.splits = q.splits;
  p.split_stride = g.split_stride;
  return api_launched(launch_split_reduce(p, part, s), s);
}

// Both products of a gradient in one launch: px (dz as it lies times w) and pw
// (dz transposed times x).
cudaError_t run_pair(const GradPlan& g, GemmParams px, GemmParams pw, const Operand& dz, const Operand& bx,
                     const Operand& bw, cudaStream_t s) {
  GemmCall<2> call;
  memset(&call, 0, sizeof(call));
  for (int j = 0; j < 2; ++j) {
    const bool w = (j == 0) == g.w_first;
    const Plan& q = g.pair.q[j];
    GemmParams& p = call.p[j];
    p = w ? pw : px;
    p.bn = q.bn;
    p.group_m = q.group_m;
    p.a_mn = w;
    p.pair_extra = g.pair.extra;
    p.epi = p.row_map == nullptr && rows16(p.ld_out, p.out_f32) && rows16(p.n, p.out_f32) ? kEpiOut : kEpiRows;
    p.out_last = p.row_map != nullptr ? p.out_extent - 1 : (p.m - 1) * p.ld_out + p.n - 1;
    GemmMaps& m = call.m[j];
    if (!encode(&m.a, dz, w ? kGemmBk : p.a_rows) || !encode(&m.b, w ? bw : bx, kGemmBk))
      return cudaErrorInvalidValue;
    if (p.epi == kEpiOut && !encode_out(&m.out, p.out, p.out_f32, p.n, p.m, p.ld_out, 1, 0)) return cudaErrorInvalidValue;
  }
  return api_launched(launch_gemm_pair(g.pair.q[0].cfg, call, s), s);
}

// The operand as the products read it: where it lies, or packed into `ws` by
// the launch that gets `p` (dst null: nothing to pack).
Operand operand(PackParams* p, int dtype, const void* src, int64_t rows, int64_t cols, int64_t ld, char* ws) {
  memset(p, 0, sizeof(*p));
  if (in_place(dtype, ld)) return Operand{src, cols, rows, ld, 1, 0};
  p->src = src;
  p->ld = ld;
  p->rows = rows;
  p->cols = cols;
  p->dst = (__nv_bfloat16*)ws;
  p->ld_dst = up(cols, 8);
  p->plane = rows * p->ld_dst;
  p->src_f32 = dtype == BDSCAN_F32;
  p->pieces = p->src_f32 ? 3 : 1;
  p->dst_extent = p->pieces * p->plane;
  return Operand{ws, cols, rows, p->ld_dst, p->pieces, p->plane};
}
const PackParams kNoPack{};

int check_types(int dtype, int out_dtype, const char* fn) {
  if (dtype != BDSCAN_F32 && dtype != BDSCAN_BF16) return fail_msg(BDSCAN_ERR_ARG, fn, "bad dtype");
  if (out_dtype != BDSCAN_F32 && out_dtype != BDSCAN_BF16) return fail_msg(BDSCAN_ERR_ARG, fn, "bad out_dtype");
  if (dtype == BDSCAN_F32 && out_dtype == BDSCAN_BF16)
    return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "f32 inputs with bf16 outputs are not supported");
  return BDSCAN_OK;
}

// ---------------------------------------------------------------------------
// linear
// ---------------------------------------------------------------------------
struct Lin {
  int64_t T, K, N, ld_x, ld_res, ld_y;
  int act, dtype, out, pieces;
};
int check_linear(const bdscan_linear_dims* d, Lin* l, const char* fn) {
  api_begin();
  if (d == nullptr) return fail_msg(BDSCAN_ERR_ARG, fn, "dims is NULL");
  if (d->rows < 0) return fail_msg(BDSCAN_ERR_ARG, fn, "negative rows");
  if (d->d_in <= 0 || d->d_out <= 0) return fail_msg(BDSCAN_ERR_ARG, fn, "d_in and d_out must be positive");
  const int rc = check_types(d->dtype, d->out_dtype, fn);
  if (rc) return rc;
  if (d->act != BDSCAN_ACT_NONE && d->act != BDSCAN_ACT_SILU && d->act != BDSCAN_ACT_GELU)
    return fail_msg(BDSCAN_ERR_ARG, fn, "bad act");
  if (d->rows > kMaxRows || d->d_in > kMaxCols || d->d_out > kMaxCols)
    return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "rows above 2^30, or d_in or d_out above 2^24");
  l->T = d->rows;
  l->K = d->d_in;
  l->N = d->d_out;
  l->ld_x = d->ld_x ? d->ld_x : l->K;
  l->ld_res = d->ld_res ? d->ld_res : l->N;
  l->ld_y = d->ld_y ? d->ld_y : l->N;
  if (l->ld_x < l->K) return fail_msg(BDSCAN_ERR_ARG, fn, "ld_x is below d_in");
  if (l->ld_res < l->N) return fail_msg(BDSCAN_ERR_ARG, fn, "ld_res is below d_out");
  if (l->ld_y < l->N) return fail_msg(BDSCAN_ERR_ARG, fn, "ld_y is below d_out");
  if (l->ld_x > kMaxCols * 64 || l->ld_res > kMaxCols * 64 || l->ld_y > kMaxCols * 64)
    return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "a row stride above 2^30");
  l->act = d->act;
  l->dtype = d->dtype;
  l->out = d->out_dtype;
  l->pieces = d->dtype == BDSCAN_F32 ? 3 : 1;
  return BDSCAN_OK;
}

// Byte offsets of a forward's workspace.
struct LinFwdWs {
  Plan q;
  size_t x, w, part, total;
};
LinFwdWs lin_fwd_ws(const Lin& l) {
  LinFwdWs w;
  memset(&w, 0, sizeof(w));
  if (l.T <= kVecRows) return w;
  w.q = plan(l.T, l.N, l.K, l.pieces, true, false);
  size_t o = 0;
  w.x = o;
  if (!in_place(l.dtype, l.ld_x)) o += packed_bytes(l.dtype, l.T, l.K);
  w.w = o;
  if (!in_place(l.dtype, l.K)) o += packed_bytes(l.dtype, l.N, l.K);
  w.part = o;
  w.total = o + split_bytes(w.q, l.T, l.N);
  return w;
}

// Row ranges of the pass over dy: about six CTAs per SM, 32 rows at least.
int dact_ranges(int64_t rows, int64_t cols) {
  const int64_t strips = (cols + 255) / 256;
  int64_t r = 6 * kSms / strips;
  if (r > (rows + 31) / 32) r = (rows + 31) / 32;
  return (int)(r < 1 ? 1 : r);
}
struct LinBwdWs {
  GradPlan g;
  bool make_dz;  // dz differs from dy, or dy cannot be read by TMA
  size_t x, w, dz, sums, part, total;
  int ranges;
};
LinBwdWs lin_bwd_ws(const Lin& l) {
  LinBwdWs w;
  memset(&w, 0, sizeof(w));
  w.g = plan_grad(l.T, l.K, l.N, l.pieces);
  w.make_dz = l.act != BDSCAN_ACT_NONE || l.out != BDSCAN_BF16 || !in_place(l.out, l.ld_y);
  size_t o = 0;
  w.x = o;
  if (!in_place(l.dtype, l.ld_x)) o += packed_bytes(l.dtype, l.T, l.K);
  w.w = o;
  if (!in_place(l.dtype, l.K)) o += packed_bytes(l.dtype, l.N, l.K);
  w.dz = o;
  if (w.make_dz) o += packed_bytes(l.dtype, l.T, l.N);
  w.sums = o;
  w.ranges = dact_ranges(l.T, l.N);
  o += al256((size_t)w.ranges * l.N * 4);
  w.part = o;
  const size_t a = split_bytes(w.g.x, l.T, l.K), b = split_bytes(w.g.w, l.N, l.K);
  w.total = o + (a > b ? a : b);
  return w;
}

// ---------------------------------------------------------------------------
// loss
// ---------------------------------------------------------------------------
struct Loss {
  int64_t T, K, V, ld_h, excluded;
  int dtype, pieces;
};
int check_loss(const bdscan_lm_loss_dims* d, Loss* l, const char* fn) {
  api_begin();
  if (d == nullptr) return fail_msg(BDSCAN_ERR_ARG, fn, "dims is NULL");
  if (d->rows < 0) return fail_msg(BDSCAN_ERR_ARG, fn, "negative rows");
  if (d->d_model <= 0 || d->vocab <= 0) return fail_msg(BDSCAN_ERR_ARG, fn, "d_model and vocab must be positive");
  const int rc = check_types(d->dtype, d->dtype, fn);
  if (rc) return rc;
  if (d->rows > kMaxRows || d->d_model > kMaxCols || d->vocab > kMaxCols)
    return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "rows above 2^30, or d_model or vocab above 2^24");
  if (d->excluded < -1 || d->excluded >= d->vocab)
    return fail_msg(BDSCAN_ERR_ARG, fn, "excluded is neither -1 nor inside the vocabulary");
  l->T = d->rows;
  l->K = d->d_model;
  l->V = d->vocab;
  l->ld_h = d->ld_h ? d->ld_h : l->K;
  if (l->ld_h < l->K) return fail_msg(BDSCAN_ERR_ARG, fn, "ld_h is below d_model");
  if (l->ld_h > kMaxCols * 64) return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "a row stride above 2^30");
  l->excluded = d->excluded;
  l->dtype = d->dtype;
  l->pieces = d->dtype == BDSCAN_F32 ? 3 : 1;
  return BDSCAN_OK;
}

// The rows that count, gathered: their h (whole tiles of rows), indices,
// targets; in the backward also their gradient scales and log sums and a copy
// of h with the scales applied. The gradient at the logits is kept without the
// scale, as p - 1 at the target and p elsewhere: dh is scaled in fp32 by the
// output step and dw by that copy. (With the scale inside, the entry that
// dominates a row was rounded with its scale, the same way for the whole row.)
struct LossRows {
  size_t count, idx, tgt, pos, gscale, lse, h, scaled, end;
  int64_t rows;  // T rounded up to whole tiles
};
LossRows loss_rows_ws(const Loss& l, bool backward) {
  size_t o = 0;
  LossRows r;
  r.rows = up(l.T, 256);
  const size_t v = al256((size_t)r.rows * 4);
  r.count = o;
  r.idx = o + 256;
  r.tgt = r.idx + v;
  r.pos = r.tgt + v;
  r.gscale = r.pos + v;
  r.lse = r.gscale + v;
  r.h = r.lse + v;
  r.scaled = r.h + packed_bytes(l.dtype, r.rows, l.K);
  r.end = backward ? r.scaled + packed_bytes(l.dtype, r.rows, l.K) : r.scaled;
  return r;
}
// Up to this many rows the product's last CTA joins their statistics, 32 at a
// time in about 2 us each; more rows get a launch of their own, a CTA per 32.
constexpr int64_t kJoinRows = 64;
// How many rows count is known on the device only; any number is right. Tiles and
// splits are chosen for the sum of the model's times with all of them (likelihoods)
// and with half (as a masked objective draws them), for both types and any number
// of rows. Over 318 cases (129 to 4096 rows, four heads, both types, 5, 50 and 100 %
// counting, forward and training) that is 1.9 % above the best of four rules on
// average and 25 % at most; planned for all rows only 3.9 and 71 %. For half alone
// the training step of 256 bf16 rows over 50,021 entries is 76 us with half counting
// (so 85) but 100 with all (91); for all alone, 1000 fp32 rows over 8191 entries take
// 119 us with half counting (111) and 165 with all (173).
int64_t half_rows(const Loss& l) { return (l.T + 1) / 2; }
struct LossFwdWs {
  Plan q;
  LossRows r;
  size_t w, part, at, total;
  int parts;
};
LossFwdWs loss_fwd_ws(const Loss& l) {
  LossFwdWs w;
  memset(&w, 0, sizeof(w));
  w.q = plan(l.T, l.V, l.K, l.pieces, false, false, half_rows(l), l.K);
  w.r = loss_rows_ws(l, false);
  size_t o = w.r.end;
  w.w = o;
  if (!in_place(l.dtype, l.K)) o += packed_bytes(l.dtype, l.V, l.K);
  w.parts = (int)((l.V + w.q.bn - 1) / w.q.bn);
  w.part = o;
  o += al256((size_t)w.parts * w.r.rows * 8);
  w.at = o;
  w.total = o + al256((size_t)w.r.rows * 4);
  return w;
}

// Vocabulary entries per piece of the backward: as many as 512 MiB hold of
// the logits' gradient, in pieces of equal size. Fewer pieces have fewer last
// waves and sums of dh, and each holds memory. Over 30 training steps (4096 to
// 32,768 rows, vocabularies of 32,000 to 128,256 entries, three widths, half or
// all rows counting) 128 MiB are 11.4 % above 512 on average, 256 and 384 4.1 %,
// 1024 1.4 % below: the limit stands where twice as much brings less than 2 %.
constexpr int64_t kPieceBytes = (int64_t)512 << 20;
struct LossBwdWs {
  Plan qz;
  GradPlan g;
  LossRows r;
  size_t w, dz, acc, part, total;
  int64_t piece;  // entries, a multiple of 256 unless there is one piece
  int pieces;
};
LossBwdWs loss_bwd_ws(const Loss& l) {
  LossBwdWs w;
  memset(&w, 0, sizeof(w));
  w.r = loss_rows_ws(l, true);
  int64_t most = kPieceBytes / (w.r.rows * 2 * l.pieces) / 256 * 256;
  if (most < 256) most = 256;
  w.pieces = (int)((l.V + most - 1) / most);
  w.piece = w.pieces == 1 ? l.V : up((l.V + w.pieces - 1) / w.pieces, 256);
  w.pieces = (int)((l.V + w.piece - 1) / w.piece);
  w.qz = plan(l.T, w.piece, l.K, l.pieces, false, false, half_rows(l), l.K);
  w.g = plan_grad(l.T, l.K, w.piece, l.pieces, half_rows(l));
  size_t o = w.r.end;
  w.w = o;
  if (!in_place(l.dtype, l.K)) o += packed_bytes(l.dtype, l.V, l.K);
  w.dz = o;
  o += packed_bytes(l.dtype, w.r.rows, w.piece);
  w.acc = o;
  if (w.pieces > 1) o += al256((size_t)l.T * up(l.K, 4) * 4);
  w.part = o;
  const size_t a = split_bytes(w.g.x, l.T, l.K), b = split_bytes(w.g.w, w.piece, l.K);
  w.total = o + (a > b ? a : b);
  return w;
}

// Numbers the rows that count and gathers their h as an operand; in the
// backward (dh given) also the scaled copy, and zeros in dh where a row does not
// count. `pw`: w, if it has to be packed.
cudaError_t prepare_rows(const Loss& l, const LossRows& r, const LossRowsParams& rp, const void* h, char* ws, void* dh,
                         const PackParams& pw, Operand* o, Operand* scaled, cudaStream_t s) {
  PackParams p;
  memset(&p, 0, sizeof(p));
  p.src = h;
  p.ld = l.ld_h;
  p.rows = l.T;
  p.cols = l.K;
  p.dst = (__nv_bfloat16*)(ws + r.h);
  p.ld_dst = up(l.K, 8);
  p.plane = r.rows * p.ld_dst;
  p.src_f32 = l.dtype == BDSCAN_F32;
  p.pieces = l.pieces;
  p.pos = (const int*)(ws + r.pos);
  p.count = (const int*)(ws + r.count);
  if (dh != nullptr) {
    p.gscale = (const float*)(ws + r.gscale);
    p.scaled = (__nv_bfloat16*)(ws + r.scaled);
    p.zero = dh;
    *scaled = Operand{p.scaled, l.K, r.rows, p.ld_dst, p.pieces, p.plane};
  }
  *o = Operand{p.dst, l.K, r.rows, p.ld_dst, p.pieces, p.plane};
  if (l.T <= small_loss_rows()) return api_launched(launch_loss_prep(rp, p, pw, s), s);
  const cudaError_t e = api_launched(launch_loss_rows(rp, s), s);
  return e != cudaSuccess ? e : api_launched(launch_pack_rows(p, pw, s), s);
}

int check_workspace(const void* ws, size_t have, size_t need, const char* fn) {
  if (need == 0) return BDSCAN_OK;
  DENSE_REQ(ws, fn, "workspace");
  if (have < need) {
    char msg[160];
    snprintf(msg, sizeof(msg), "workspace of %zu bytes, %zu needed", have, need);
    return fail_msg(BDSCAN_ERR_ARG, fn, msg);
  }
  return BDSCAN_OK;
}
int check_device(const char* fn, int** flag) {
  if (tensor_map_encoder() == nullptr)
    return fail_msg(BDSCAN_ERR_UNSUPPORTED, fn, "the driver has no tensor-map encoder");
  *flag = ssd_wait_flag_ptr();
  return *flag != nullptr ? BDSCAN_OK : fail_msg(BDSCAN_ERR_CUDA, fn, "cannot locate the device wait flag");
}

}  // namespace
}  // namespace bds

using namespace bds;

extern "C" {

size_t bdscan_linear_forward_workspace_size(const bdscan_linear_dims* dims) {
  Lin l;
  if (check_linear(dims, &l, "bdscan_linear_forward_workspace_size") != BDSCAN_OK || l.T == 0) return 0;
  return lin_fwd_ws(l).total;
}

int bdscan_linear_forward(const bdscan_linear_dims* dims, const void* x, const void* w, const void* bias,
                          const void* residual, void* pre, void* y, void* workspace, size_t workspace_bytes,
                          void* stream) {
  const char* fn = "bdscan_linear_forward";
  Lin l;
  int rc = check_linear(dims, &l, fn);
  if (rc) return rc;
  if (l.T == 0) return api_ok();
  DENSE_REQ(x, fn, "x");
  DENSE_REQ(w, fn, "w");
  DENSE_OPT(bias, fn, "bias");
  DENSE_OPT(residual, fn, "residual");
  DENSE_OPT(pre, fn, "pre");
  DENSE_REQ(y, fn, "y");
  cudaStream_t s = (cudaStream_t)stream;
  if (l.T <= kVecRows) {
    VecParams v{};
    v.x = x, v.w = w, v.bias = bias, v.res = residual, v.y = y, v.pre = pre;
    v.ld_x = l.ld_x, v.ld_res = l.ld_res, v.ld_y = l.ld_y;
    v.rows = (int)l.T, v.k = (int)l.K, v.n = (int)l.N, v.act = l.act;
    v.f32 = l.dtype == BDSCAN_F32, v.out_f32 = l.out == BDSCAN_F32;
    v.out_extent = (l.T - 1) * l.ld_y + l.N;
    const cudaError_t e = api_launched(launch_linear_vec(v, s), s);
    return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
  }
  const LinFwdWs ws = lin_fwd_ws(l);
  if ((rc = check_workspace(workspace, workspace_bytes, ws.total, fn))) return rc;
  int* flag;
  if ((rc = check_device(fn, &flag))) return rc;
  char* base = (char*)workspace;
  PackParams px, pw;
  const Operand a = operand(&px, l.dtype, x, l.T, l.K, l.ld_x, base + ws.x);
  const Operand b = operand(&pw, l.dtype, w, l.N, l.K, l.K, base + ws.w);
  cudaError_t e = cudaSuccess;
  if (px.dst != nullptr || pw.dst != nullptr) e = api_launched(launch_pack(px, pw, s), s);
  if (e == cudaSuccess) {
    GemmParams p = geometry(ws.q, l.T, l.N, l.K, flag);
    p.bias = bias;
    p.res = residual;
    p.pre = pre;
    p.out = y;
    p.ld_res = l.ld_res;
    p.ld_out = l.ld_y;
    p.ld_pre = l.N;
    p.bias_f32 = p.pre_f32 = l.dtype == BDSCAN_F32;
    p.res_f32 = p.out_f32 = l.out == BDSCAN_F32;
    p.act = l.act;
    p.out_extent = (l.T - 1) * l.ld_y + l.N;
    e = run_out(ws.q, false, false, p, a, b, (float*)(base + ws.part), s);
  }
  return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
}

size_t bdscan_linear_backward_workspace_size(const bdscan_linear_dims* dims) {
  Lin l;
  if (check_linear(dims, &l, "bdscan_linear_backward_workspace_size") != BDSCAN_OK || l.T == 0) return 0;
  return lin_bwd_ws(l).total;
}

int bdscan_linear_backward(const bdscan_linear_dims* dims, const void* x, const void* w, const void* pre,
                           const void* dy, void* dx, void* dw, void* dbias, void* workspace, size_t workspace_bytes,
                           void* stream) {
  const char* fn = "bdscan_linear_backward";
  Lin l;
  int rc = check_linear(dims, &l, fn);
  if (rc) return rc;
  DENSE_OPT(dx, fn, "dx");
  DENSE_OPT(dw, fn, "dw");
  DENSE_OPT(dbias, fn, "dbias");
  cudaStream_t s = (cudaStream_t)stream;
  const size_t elt = l.dtype == BDSCAN_F32 ? 4 : 2;
  if (l.T == 0) {  // sums over no rows
    cudaError_t e = cudaSuccess;
    if (dw != nullptr) e = cudaMemsetAsync(dw, 0, (size_t)l.N * l.K * elt, s);
    if (dbias != nullptr && e == cudaSuccess) e = cudaMemsetAsync(dbias, 0, (size_t)l.N * elt, s);
    return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
  }
  if (dw != nullptr) DENSE_REQ(x, fn, "x");
  if (dx != nullptr) DENSE_REQ(w, fn, "w");
  if (l.act != BDSCAN_ACT_NONE) DENSE_REQ(pre, fn, "pre");
  DENSE_REQ(dy, fn, "dy");
  const LinBwdWs ws = lin_bwd_ws(l);
  if ((rc = check_workspace(workspace, workspace_bytes, ws.total, fn))) return rc;
  int* flag;
  if ((rc = check_device(fn, &flag))) return rc;
  char* base = (char*)workspace;
  float* part = (float*)(base + ws.part);
  cudaError_t e = cudaSuccess;
  const bool products = dx != nullptr || dw != nullptr;
  Operand dz{dy, l.N, l.T, l.ld_y, 1, 0}, ox{}, ow{};
  PackParams px = kNoPack, pw = kNoPack;
  if (dx != nullptr) ow = operand(&pw, l.dtype, w, l.N, l.K, l.K, base + ws.w);
  if (dw != nullptr) ox = operand(&px, l.dtype, x, l.T, l.K, l.ld_x, base + ws.x);
  float* sums = dbias != nullptr ? (float*)(base + ws.sums) : nullptr;
  if ((products && ws.make_dz) || dbias != nullptr) {
    DactParams p;
    memset(&p, 0, sizeof(p));
    p.dy = dy;
    p.pre = pre;
    p.ld_dy = l.ld_y;
    p.ld_pre = l.N;
    p.rows = l.T;
    p.cols = l.N;
    p.dy_f32 = l.out == BDSCAN_F32;
    p.pre_f32 = l.dtype == BDSCAN_F32;
    p.act = l.act;
    p.pieces = l.pieces;
    p.ranges = ws.ranges;
    if (products && ws.make_dz) {
      p.dz = (__nv_bfloat16*)(base + ws.dz);
      p.ld_dz = up(l.N, 8);
      p.plane = l.T * p.ld_dz;
      dz = Operand{p.dz, l.N, l.T, p.ld_dz, l.pieces, p.plane};
    }
    p.part = sums;
    // Large operands are packed by a launch of their own: the gradient's pass leaves room for 24 warps per SM,
    // packing alone has 64 (training 10016 x 1803 -> 560: 131 us against 143; from 2^22 elements on the two ways
    // are within 2 %, and below, the second launch costs up to 10 %).
    if (l.T * l.K + l.N * l.K > ((int64_t)1 << 23) && (px.dst != nullptr || pw.dst != nullptr)) {
      e = api_launched(launch_pack(px, pw, s), s);
      px = pw = kNoPack;
    }
    if (e == cudaSuccess) e = api_launched(launch_prep(p, px, pw, s), s);
    if (e == cudaSuccess && dbias != nullptr && !products)
      e = api_launched(launch_colsum(sums, ws.ranges, l.N, dbias, l.dtype == BDSCAN_F32, s), s);
  } else if (px.dst != nullptr || pw.dst != nullptr) {
    e = api_launched(launch_pack(px, pw, s), s);
  }
  // the first of the products also ends the bias gradient
  auto add_sums = [&](GemmParams* p) {
    if (sums == nullptr) return;
    p->sum_part = sums;
    p->sum_out = dbias;
    p->sum_cols = l.N;
    p->sum_ranges = ws.ranges;
    p->sum_f32 = l.dtype == BDSCAN_F32;
    sums = nullptr;
  };
  GemmParams gx = geometry(ws.g.x, l.T, l.K, l.N, flag), gw = geometry(ws.g.w, l.N, l.K, l.T, flag);
  gx.out = dx;
  gw.out = dw;
  gx.ld_out = gw.ld_out = l.K;
  gx.out_f32 = gw.out_f32 = l.dtype == BDSCAN_F32;
  gx.out_extent = l.T * l.K;
  gw.out_extent = l.N * l.K;
  if (e == cudaSuccess && dx != nullptr && dw != nullptr && ws.g.one) {
    add_sums(ws.g.w_first ? &gw : &gx);
    e = run_pair(ws.g, gx, gw, dz, ow, ox, s);
    return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
  }
  if (e == cudaSuccess && dx != nullptr) {
    add_sums(&gx);
    e = run_out(ws.g.x, false, true, gx, dz, ow, part, s);
  }
  if (e == cudaSuccess && dw != nullptr) {
    add_sums(&gw);
    e = run_out(ws.g.w, true, true, gw, dz, ox, part, s);
  }
  return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
}

size_t bdscan_lm_loss_forward_workspace_size(const bdscan_lm_loss_dims* dims) {
  Loss l;
  if (check_loss(dims, &l, "bdscan_lm_loss_forward_workspace_size") != BDSCAN_OK || l.T == 0) return 0;
  return loss_fwd_ws(l).total;
}

int bdscan_lm_loss_forward(const bdscan_lm_loss_dims* dims, const void* h, const void* w, const int64_t* target,
                           const float* weight, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream) {
  const char* fn = "bdscan_lm_loss_forward";
  Loss l;
  int rc = check_loss(dims, &l, fn);
  if (rc) return rc;
  if (l.T == 0) return api_ok();
  DENSE_REQ(h, fn, "h");
  DENSE_REQ(w, fn, "w");
  DENSE_REQ(target, fn, "target");
  DENSE_OPT(weight, fn, "weight");
  DENSE_REQ(loss, fn, "loss");
  DENSE_REQ(lse, fn, "lse");
  const LossFwdWs ws = loss_fwd_ws(l);
  if ((rc = check_workspace(workspace, workspace_bytes, ws.total, fn))) return rc;
  int* flag;
  if ((rc = check_device(fn, &flag))) return rc;
  cudaStream_t s = (cudaStream_t)stream;
  char* base = (char*)workspace;
  LossRowsParams rp;
  memset(&rp, 0, sizeof(rp));
  rp.target = target;
  rp.weight = weight;
  rp.rows = l.T;
  rp.vocab = l.V;
  rp.count = (int*)(base + ws.r.count);
  rp.idx = (int*)(base + ws.r.idx);
  rp.tgt = (int*)(base + ws.r.tgt);
  rp.pos = (int*)(base + ws.r.pos);
  rp.loss = loss;
  rp.lse = lse;
  Operand a;
  PackParams pw;
  const Operand b = operand(&pw, l.dtype, w, l.V, l.K, l.K, base + ws.w);
  cudaError_t e = prepare_rows(l, ws.r, rp, h, base, nullptr, pw, &a, nullptr, s);
  const bool last_joins = l.T <= kJoinRows && ws.q.cfg.cg == 1;
  if (e == cudaSuccess) {
    Plan q = ws.q;
    q.cfg.epi = kEpiStats;
    GemmParams p = geometry(q, l.T, l.V, l.K, flag);
    p.rows_dev = rp.count;
    p.rows_axis = 1;
    p.target = rp.tgt;
    p.excluded = (int)l.excluded;
    p.part = (float2*)(base + ws.part);
    p.at_target = (float*)(base + ws.at);
    p.rows_ld = ws.r.rows;
    p.out_last = (ws.parts - 1) * p.rows_ld + l.T - 1;
    p.out_extent = ws.parts * p.rows_ld;
    if (last_joins) {
      p.ticket = rp.count + 1;
      p.row_idx = rp.idx;
      p.row_weight = weight;
      p.loss_out = loss;
      p.lse_out = lse;
    }
    e = run_product(q, p, a, b, 1, 0, l.T, s);
  }
  if (e == cudaSuccess && !last_joins)
    e = api_launched(launch_loss_combine((const float2*)(base + ws.part), ws.parts, ws.r.rows,
                                         (const float*)(base + ws.at), rp.count, rp.idx, weight, loss, lse, l.T, s),
                     s);
  return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
}

size_t bdscan_lm_loss_backward_workspace_size(const bdscan_lm_loss_dims* dims) {
  Loss l;
  if (check_loss(dims, &l, "bdscan_lm_loss_backward_workspace_size") != BDSCAN_OK || l.T == 0) return 0;
  return loss_bwd_ws(l).total;
}

int bdscan_lm_loss_backward(const bdscan_lm_loss_dims* dims, const void* h, const void* w, const int64_t* target,
                            const float* weight, const float* lse, const float* dloss, void* dh, void* dw,
                            void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "bdscan_lm_loss_backward";
  Loss l;
  int rc = check_loss(dims, &l, fn);
  if (rc) return rc;
  const size_t elt = l.dtype == BDSCAN_F32 ? 4 : 2;
  cudaStream_t s = (cudaStream_t)stream;
  DENSE_REQ(dw, fn, "dw");
  if (l.T == 0) {
    const cudaError_t e = cudaMemsetAsync(dw, 0, (size_t)l.V * l.K * elt, s);
    return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
  }
  DENSE_REQ(h, fn, "h");
  DENSE_REQ(w, fn, "w");
  DENSE_REQ(target, fn, "target");
  DENSE_OPT(weight, fn, "weight");
  DENSE_REQ(lse, fn, "lse");
  DENSE_OPT(dloss, fn, "dloss");
  DENSE_REQ(dh, fn, "dh");
  const LossBwdWs ws = loss_bwd_ws(l);
  if ((rc = check_workspace(workspace, workspace_bytes, ws.total, fn))) return rc;
  int* flag;
  if ((rc = check_device(fn, &flag))) return rc;
  char* base = (char*)workspace;
  LossRowsParams rp;
  memset(&rp, 0, sizeof(rp));
  rp.target = target;
  rp.weight = weight;
  rp.dloss = dloss;
  rp.lse_in = lse;
  rp.rows = l.T;
  rp.vocab = l.V;
  rp.count = (int*)(base + ws.r.count);
  rp.idx = (int*)(base + ws.r.idx);
  rp.tgt = (int*)(base + ws.r.tgt);
  rp.pos = (int*)(base + ws.r.pos);
  rp.gscale = (float*)(base + ws.r.gscale);
  rp.lse_c = (float*)(base + ws.r.lse);
  Operand a, scaled;
  PackParams pw;
  const Operand b = operand(&pw, l.dtype, w, l.V, l.K, l.K, base + ws.w);
  cudaError_t e = prepare_rows(l, ws.r, rp, h, base, dh, pw, &a, &scaled, s);
  const int64_t ld_dz = up(ws.piece, 8), ld_acc = up(l.K, 4);
  const int f32 = l.dtype == BDSCAN_F32;
  float* part = (float*)(base + ws.part);
  float* acc = (float*)(base + ws.acc);
  for (int i = 0; i < ws.pieces && e == cudaSuccess; ++i) {
    const int64_t v0 = i * ws.piece, n = l.V - v0 < ws.piece ? l.V - v0 : ws.piece;
    Operand bp = b;  // this piece's rows of w
    bp.base = (const char*)b.base + v0 * b.ld * 2;
    bp.rows = n;
    const Operand dz{base + ws.dz, n, ws.r.rows, ld_dz, l.pieces, ws.r.rows * ld_dz};
    // the logits' gradient
    Plan q = ws.qz;
    q.cfg.epi = kEpiDz;
    GemmParams p = geometry(q, l.T, n, l.K, flag);
    p.rows_dev = rp.count;
    p.rows_axis = 1;
    p.target = rp.tgt;
    p.v0 = (int)v0;
    p.excluded = (int)l.excluded;
    p.lse = rp.lse_c;
    p.out = base + ws.dz;
    p.ld_out = ld_dz;
    p.out_last = (l.pieces - 1) * ws.r.rows * ld_dz + (ws.r.rows - 1) * ld_dz + n - 1;
    p.out_extent = l.pieces * ws.r.rows * ld_dz;
    e = run_product(q, p, a, bp, l.pieces, ws.r.rows * ld_dz, ws.r.rows, s);
    // this piece's rows of dw, and its part of dh: fp32 sums over the pieces, the last one writes dh
    const bool last = i + 1 == ws.pieces;
    GemmParams gw = geometry(ws.g.w, n, l.K, ws.r.rows, flag), gh = geometry(ws.g.x, l.T, l.K, n, flag);
    gw.rows_dev = gh.rows_dev = rp.count;
    gw.rows_axis = 2;
    gw.out = (char*)dw + (size_t)v0 * l.K * elt;
    gw.ld_out = l.K;
    gw.out_f32 = f32;
    gw.out_extent = n * l.K;
    gh.rows_axis = 1;
    gh.res = i > 0 ? acc : nullptr;
    gh.ld_res = ld_acc;
    gh.res_f32 = 1;
    gh.out = last ? dh : acc;
    gh.ld_out = last ? l.K : ld_acc;
    gh.out_f32 = last ? f32 : 1;
    gh.row_map = last ? rp.idx : nullptr;
    gh.row_scale = rp.gscale;
    gh.out_extent = last ? l.T * l.K : l.T * ld_acc;
    // With several pieces the rows that count decide how the tiles of the two would have to be dealt, and only the
    // device knows them: 16384 rows, half of them counting, took 1817 us as pairs and 1762 one after the other.
    if (e == cudaSuccess && ws.pieces == 1 && ws.g.one) {
      e = run_pair(ws.g, gh, gw, dz, bp, scaled, s);
    } else {
      if (e == cudaSuccess) e = run_out(ws.g.w, true, true, gw, dz, scaled, part, s);
      if (e == cudaSuccess) e = run_out(ws.g.x, false, true, gh, dz, bp, part, s, !last);
    }
  }
  return e == cudaSuccess ? api_ok() : cuda_fail(e, fn);
}

}  // extern "C"
