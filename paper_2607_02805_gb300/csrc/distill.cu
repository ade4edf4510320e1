// distill.cu -- the passes of the distillation loss (include/bdscan_dense.h)
// around the vocabulary loss's products: which rows count, the student's logits at
// the teacher's entries with the loss, and the gradient at those entries.
//
// q = softmax(teacher / T) over a row's known entries (inside the vocabulary, not
// the excluded one, not minus infinity), p = softmax(h w^T / T) over the whole
// vocabulary, of which the product's epilogue has left partial maxima and sums:
// loss = weight sum_v q_v (log q_v - log p_v). A row has 64 entries at most, two
// per lane; q is formed again from the teacher's logits wherever it is needed.
// Entries of the same id are one entry of the vocabulary, with their shares added.
#include "dense.cuh"
#include "gemm.cuh"

namespace bds {
namespace {

constexpr int kThreads = 256, kRowWarps = kThreads / 32;

// A row's entries, lane l those at l and l + 32: id (-1 where not known), q and log2 q.
struct Entries {
  int id[2];
  float q[2], l2[2];
};
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ void load_ids(Entries& e, float (&t)[2], const DistillParams& p, int64_t row) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 32 * k;
    const int64_t id = j < p.top ? p.ids[row * p.top + j] : -1;
    t[k] = j < p.top ? p.teacher[row * p.top + j] : -INFINITY;
    e.id[k] = id >= 0 && id < p.vocab && id != p.excluded && t[k] != -INFINITY ? (int)id : -1;
  }
}
__device__ __forceinline__ void load_entries(Entries& e, const DistillParams& p, int64_t row) {
  float t[2];
  load_ids(e, t, p, row);
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (e.id[k] >= 0) m = fmaxf(m, t[k]);
  m = warp_max(m);
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    e.l2[k] = (t[k] - m) * p.scale2;  // NaN stays, and plus infinity becomes that
    e.q[k] = e.id[k] >= 0 ? ex2(e.l2[k]) : 0.f;
    s += e.q[k];
  }
  s = warp_sum(s);
  const float l2 = log2f(s), r = 1.f / s;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    e.q[k] *= r;
    e.l2[k] -= l2;
  }
}

// The shares of an entry's id in all places, and their logarithm in base 2.
__device__ __forceinline__ void merge_ids(Entries& e, float (&share)[2], int top) {
  const int lane = threadIdx.x & 31;
  // no two lanes with the same id: an entry that is not known stands for itself
  const int own[2] = {e.id[0] >= 0 ? e.id[0] : -1 - lane, e.id[1] >= 0 ? e.id[1] : -1 - lane};
  bool twice = __popc(__match_any_sync(0xffffffffu, own[0])) > 1;
  if (top > 32) {
    twice |= __popc(__match_any_sync(0xffffffffu, own[1])) > 1;
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
      const int id = __shfl_sync(0xffffffffu, e.id[0], j);
      twice |= id >= 0 && id == e.id[1];
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) share[k] = e.q[k];
  if (!__any_sync(0xffffffffu, twice)) return;
  share[0] = share[1] = 0.f;
  int times[2] = {0, 0};
  for (int j = 0; j < top; ++j) {
    const int id = __shfl_sync(0xffffffffu, j < 32 ? e.id[0] : e.id[1], j & 31);
    const float q = __shfl_sync(0xffffffffu, j < 32 ? e.q[0] : e.q[1], j & 31);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (id == e.id[k]) share[k] += q, ++times[k];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (times[k] > 1) e.l2[k] = log2f(share[k]);
}

// p - q of an entry, from the student's logit there.
__device__ __forceinline__ float entry_grad(const DistillParams& p, float z, float lse, float share) {
  return ex2(fmaf(z, p.scale, -lse) * kLog2e) - share;
}

// Which part of a row's scale g = weight dloss / T its gradient at the logits
// takes before it is rounded to bf16; h, in the copy that the product for dw
// reads, takes the rest, b. Two ways, whose roundings are worked out at the
// entries (those of p - q elsewhere are small and many):
//   the mantissa of g: b is a power of two, so that h stays as it is, and every
//     entry is rounded by itself. Good where several entries count.
//   a factor near one that makes the largest entry exact: the row that one entry
//     dominates would be off by that entry's rounding as a whole. h times b is
//     rounded instead, by 2^-16 / 3 * 0.54 in square, element by element.
// (With the second rounding always there, dw was off by 2.9e-3 where the plain
// form, rounded once, is by 1.7e-3; so by 2.4e-3.)
// Where few rows count, the entries' rows of dw come from k_distill_dw, and only dh
// reads their rounded gradients: there the best of a lane's factor each is taken
// too, and what h loses does not count.
__device__ __forceinline__ float rounding(float v) {
  const float d = __bfloat162float(__float2bfloat16_rn(v)) - v;
  return d * d;
}
__device__ __forceinline__ float pick_scale(const Entries& e, const float (&s)[2], float g, bool few, int top) {
  if (!isfinite(g) || g == 0.f) return 1.f;
  int exp2;
  const float mant = 2.f * frexpf(g, &exp2);
  float x = 0.f, size = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (e.id[k] >= 0) x = fmaxf(x, fabsf(s[k])), size = fmaf(s[k], s[k], size);
  x = warp_max(x);
  size = warp_sum(size);
  if (!(x > 1e-30f) || !isfinite(x)) return mant;
  const float one = __bfloat162float(__float2bfloat16_rn(x)) / x;
  float err_m = 0.f, err_1 = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (e.id[k] >= 0) err_m += rounding(s[k] * mant), err_1 += rounding(s[k] * one);
  err_m = warp_sum(err_m) / (mant * mant);
  err_1 = warp_sum(err_1);
  if (few) {
    const float mine = ex2((float)(threadIdx.x & 31) / 32.f), r = 1.f / (mine * mine);
    float err = 0.f;
    for (int j = 0; j < top; ++j) {
      const float v = __shfl_sync(0xffffffffu, j < 32 ? s[0] : s[1], j & 31);  // zero where not known
      err += rounding(v * mine) * r;
    }
    const float best = -warp_max(-err);
    const float of = __shfl_sync(0xffffffffu, mine, __ffs(__ballot_sync(0xffffffffu, err == best)) - 1 & 31);
    if (best < err_m && best < err_1) return of;
  } else {
    err_1 += 0x1p-16f / 3.f * 0.54f * size;
  }
  return err_1 < err_m ? one : mant;
}

// Rows of 32 U from `first` on whose scales are not zero, by the lane. The loads are unconditional, so that all are in
// flight.
template <int U>
__device__ __forceinline__ int some_scales(const DistillParams& p, int64_t first) {
  const int64_t r0 = first + (threadIdx.x & 31), last = p.rows - 1;
  float a[U], b[U];
#pragma unroll
  for (int u = 0; u < U; ++u) a[u] = b[u] = 1.f;
  if (p.weight != nullptr) {
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = p.weight[min(r0 + 32 * u, last)];
  }
  if (p.dloss != nullptr) {
#pragma unroll
    for (int u = 0; u < U; ++u) b[u] = p.dloss[min(r0 + 32 * u, last)];
  }
  int c = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) c += (r0 + 32 * u <= last) & (a[u] != 0.f) & (b[u] != 0.f);
  return c;
}
// Whether up to kFewRows rows count, by a bound that all warps agree on: rows whose scales are not zero (some may know
// no entry). The warps of a call of many are done with its first rows, c of the lane's among them; where they are few,
// few warps go through all.
constexpr int kFirstScales = 8;
__device__ __forceinline__ bool few_scales(const DistillParams& p, int c) {
  constexpr int U = 32;
  int n = __reduce_add_sync(0xffffffffu, c);
  for (int64_t first = 32 * kFirstScales; n <= kFewRows && first < p.rows; first += 32 * U)
    n += __reduce_add_sync(0xffffffffu, some_scales<U>(p, first));
  return n <= kFewRows;
}

// A warp per row: the gradient at its entries, which k_distill_dz puts in place
// piece by piece of the vocabulary, and what it takes of the row's scale.
__global__ void __launch_bounds__(kThreads) k_distill_grad(const DistillParams p) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  if (!dguard(kSiteDistill, row, p.rows)) return;
  const float wt = p.weight != nullptr ? p.weight[row] : 1.f, dl = p.dloss != nullptr ? p.dloss[row] : 1.f;
  const float g = wt * (dl * p.scale);  // may be zero where neither is
  const int scales = p.row_scale != nullptr ? some_scales<kFirstScales>(p, 0) : 0;
  Entries e;
  float share[2], s[2] = {0.f, 0.f};
  load_entries(e, p, row);
  // the rows that count, as loss_row() has them
  if (wt == 0.f || dl == 0.f || !__any_sync(0xffffffffu, e.id[0] >= 0 || e.id[1] >= 0)) return;
  merge_ids(e, share, p.top);
  const float lse = p.lse_in[row];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (e.id[k] >= 0) s[k] = entry_grad(p, p.z_in[row * p.top + lane + 32 * k], lse, share[k]);
  const float a = p.row_scale != nullptr ? pick_scale(e, s, g, few_scales(p, scales), p.top) : 1.f;
  if (lane == 0 && p.row_scale != nullptr) p.row_scale[row] = a;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (lane + 32 * k < p.top) p.grad[row * p.top + lane + 32 * k] = a * s[k];
}

// A row's products with J rows of w (null: none), by a warp, J loads of w and one of the row in flight.
template <typename T, bool VEC, int J>
__device__ __forceinline__ void dot_rows(float (&s)[J], const T* a, const T* const (&b)[J], int k) {
  constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < J; ++j) s[j] = 0.f;
#pragma unroll 2
  for (int i = lane * E; i < k; i += 32 * E) {
    if constexpr (VEC) {
      const uint4 u = *reinterpret_cast<const uint4*>(a + i);
      uint4 v[J];
#pragma unroll
      for (int j = 0; j < J; ++j)
        v[j] = b[j] != nullptr ? *reinterpret_cast<const uint4*>(b[j] + i) : make_uint4(0, 0, 0, 0);
      const T* x = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const T* y = reinterpret_cast<const T*>(&v[j]);
#pragma unroll
        for (int q = 0; q < E; ++q) s[j] = fmaf(cvt(x[q]), cvt(y[q]), s[j]);
      }
    } else {
      const float x = cvt(a[i]);
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (b[j] != nullptr) s[j] = fmaf(x, cvt(b[j][i]), s[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < J; ++j) s[j] = warp_sum(s[j]);
}

// WPR warps per row that counts: the student's logits at the row's entries, four
// of them per warp at a time (rows of w come from L2 mostly), the partial
// statistics joined, and the loss, formed in base 2 before anything is rounded at
// the logits' own size. It is a chain of latencies: with many rows one warp each
// (8192 rows, 32 entries of 832 bf16, 436 MB), a CTA each where there are few.
template <typename T, bool VEC, int WPR>
__global__ void __launch_bounds__(kThreads) k_distill_join(const DistillParams p) {
  pdl_sync();
  constexpr int J = 4, R = kRowWarps / WPR;
  __shared__ float2 red[kRowWarps];
  __shared__ float zs[R][64];
  const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % WPR, r = (threadIdx.x >> 5) / WPR;
  const int slot = blockIdx.x * R + r;
  if (slot >= *p.count) return;  // all warps of the row
  const int64_t row = p.idx[slot];
  if (!dguard(kSiteDistill, row * p.top + p.top - 1, p.rows * p.top)) return;
  Entries e;
  float t[2];
  load_ids(e, t, p, row);
  const T* h = static_cast<const T*>(p.h) + row * p.ld_h;
  for (int j0 = J * w; j0 < p.top; j0 += J * WPR) {
    const T* at[J];
    float z[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int id = __shfl_sync(0xffffffffu, j0 + j < 32 ? e.id[0] : e.id[1], (j0 + j) & 31);
      at[j] = id >= 0 && j0 + j < p.top ? static_cast<const T*>(p.w) + (int64_t)id * p.d_model : nullptr;
    }
    dot_rows<T, VEC, J>(z, h, at, p.d_model);
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (lane == j && j0 + j < p.top) zs[r][j0 + j] = at[j] != nullptr ? z[j] : 0.f;  // 0 times a NaN of h is NaN
  }
  float m = -INFINITY, s = 0.f;
  for (int k = w * 32 + lane; k < p.parts; k += 32 * WPR) stats_join(m, s, p.part[(int64_t)k * p.rows_ld + slot]);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    stats_join(m, s, make_float2(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o)));
  if constexpr (WPR > 1) {
    static_assert(R == 1, "the barrier is the CTA's");
    if (lane == 0) red[w] = make_float2(m, s);
    __syncthreads();
    if (w != 0) return;
    m = red[0].x, s = red[0].y;
#pragma unroll
    for (int k = 1; k < WPR; ++k) stats_join(m, s, red[k]);
  } else {
    __syncwarp();
  }
  float share[2];
  load_entries(e, p, row);
  merge_ids(e, share, p.top);
  const float l2 = log2f(s);
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 32 * k;
    if (j < p.top) {
      const float z = zs[r][j];
      p.z[row * p.top + j] = z;
      // an entry too unlikely for fp32 adds nothing
      if (e.id[k] >= 0 && e.q[k] != 0.f) sum = fmaf(e.q[k], e.l2[k] - (fmaf(z, p.scale2, -m) - l2), sum);
    }
  }
  sum = warp_sum(sum);
  if (lane == 0) {
    const float d = sum < 0.f ? 0.f : sum * kLn2;  // no divergence is below zero; a NaN stays
    p.loss[row] = p.weight != nullptr ? p.weight[row] * d : d;
    p.lse[row] = (m + l2) * kLn2;
  }
}

// The gradient at the logits of the entries inside a piece of the vocabulary,
// over what the product's epilogue left there: rounded once, from the row's own
// logit. A thread per entry; those of an id that comes twice write the same value.
__global__ void __launch_bounds__(kThreads) k_distill_dz(const DistillParams p) {
  pdl_sync();
  const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x, slot = x / p.top;
  if (slot >= *p.count) return;
  if (!dguard(kSiteDistill, (p.pieces - 1) * p.plane + slot * p.ld_dz + p.n - 1, p.dz_extent)) return;
  const int64_t at = (int64_t)p.idx[slot] * p.top + (x - slot * p.top);
  const int64_t id = p.ids[at], to = id - p.v0;
  if (id < 0 || id == p.excluded || to < 0 || to >= p.n || p.teacher[at] == -INFINITY) return;
  float v = p.grad[at];
  bf16* d = p.dz + slot * p.ld_dz + to;
  for (int i = 0; i < p.pieces; ++i) {
    const float part = p.pieces == 1 ? v : bf16_part(v);
    d[i * p.plane] = __float2bfloat16_rn(part);
    v -= part;
  }
}

// Where up to kFewRows rows count, the rows of dw at their entries once more, from
// the gradients before any rounding: dw[v] = sum_r g_r (p - q)_rv h_r, with what
// the products read where v is no entry of row r. Over many rows the roundings of
// g (p - q) and of the scaled copy of h are as likely up as down; few do not
// average them out. dw's error over the plain form's (rounded once), the largest of
// 24 draws of 24 entries of 21,707, whatever the number of rows in the call:
//   rows that count      1     5    16    20    32    48   128
//   by the products   1.64  1.51  1.57  1.49  1.43  1.41  1.36
//   with this         1.02  1.12  1.03  1.03  1.02
// (64 entries of 5000: 1.59 to 1.42, so 1.27 to 1.13.) From 32 rows on the error no
// longer falls much, and the time rises: a step of 256 rows, 448 x 50021, takes 92 us
// with 5 rows (without 88), 113 with 32 of 64 entries (98), and the 2 us of an empty
// launch, 93.6 for 91.2, where more rows count.
// A CTA takes four entries of a row, looks for their ids among all known ones, and
// reads h once for the four: a chain of six latencies. Several entries of one id
// write the same sums.
constexpr int kDwEntries = 4;
__global__ void __launch_bounds__(kThreads) k_distill_dw(const DistillParams p) {
  pdl_sync();
  constexpr int M = kDwEntries;
  __shared__ float coef[M][kFewRows], scale[kFewRows];
  __shared__ bool own[M][kFewRows];  // coef is that of the row's own entry
  __shared__ int index[kFewRows];
  static_assert(M * kFewRows <= kThreads, "a thread per gradient");
  static_assert(kFewRows % 8 == 0, "coef[] in eights");
  const int t = threadIdx.x, groups = (p.top + M - 1) / M, slot = blockIdx.x / groups, j0 = blockIdx.x % groups * M;
  // read without waiting for the count: both have room for a tile of rows
  const int mine = t < kFewRows ? p.idx[t] : 0;
  const float by = t < kFewRows ? p.gscale[t] : 0.f;
  const int count = *p.count;
  if (count > kFewRows || slot >= count) return;
  if (t < count) index[t] = mine, scale[t] = by;
  if (t < M * kFewRows) own[t / kFewRows][t % kFewRows] = false;
  __syncthreads();
  int to[M];  // this piece's columns of the four, -1 where it is not known or not there
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int64_t at = (int64_t)index[slot] * p.top + min(j0 + m, p.top - 1), id = p.ids[at];
    const bool known = p.teacher[at] != -INFINITY && id != p.excluded && id >= p.v0 && id < p.v0 + p.n;
    to[m] = known ? (int)(id - p.v0) : -1;
  }
  if ((to[0] & to[1] & to[2] & to[3]) < 0) return;  // none; the whole CTA
  // what the products read, and over it the rows' own entries
  float read = 0.f;
#pragma unroll
  for (int m = 0; m < M; ++m)
    if (to[m] >= 0 && t / kFewRows == m && t % kFewRows < count) {
      const int64_t at = t % kFewRows * p.ld_dz + to[m];
      if (dguard(kSiteDistill, at, p.dz_extent)) read = __bfloat162float(p.dz[at]);
    }
#pragma unroll 2
  for (int x = t; x < count * p.top; x += kThreads) {
    const int r = x / p.top;
    const int64_t at = (int64_t)index[r] * p.top + (x - r * p.top), id = p.ids[at] - p.v0;
    const float teacher = p.teacher[at], grad = p.grad[at];
#pragma unroll
    for (int m = 0; m < M; ++m)
      if (to[m] >= 0 && id == to[m] && teacher != -INFINITY) coef[m][r] = grad * scale[r], own[m][r] = true;
  }
  __syncthreads();
  if (t < M * kFewRows && t % kFewRows < count && !own[t / kFewRows][t % kFewRows])
    coef[t / kFewRows][t % kFewRows] = read * scale[t % kFewRows];
  __syncthreads();
  const bf16* h = static_cast<const bf16*>(p.h);
  bf16* out = static_cast<bf16*>(p.dw);
  constexpr int U = 2, K = 8;  // columns of a thread, and rows of them in flight
  for (int c0 = t; c0 < p.d_model; c0 += U * kThreads) {
    float sum[M][U] = {};
    for (int k0 = 0; k0 < count; k0 += K) {
      float v[K][U];  // no branch between the loads and their use: all are in flight
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const bf16* row = h + index[min(k0 + k, count - 1)] * p.ld_h;
#pragma unroll
        for (int u = 0; u < U; ++u) v[k][u] = __bfloat162float(row[min(c0 + u * kThreads, p.d_model - 1)]);
      }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const float by = coef[m][k0 + k];
#pragma unroll
          for (int u = 0; u < U; ++u) sum[m][u] = k0 + k < count ? fmaf(by, v[k][u], sum[m][u]) : sum[m][u];
        }
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * kThreads;
        if (to[m] >= 0 && c < p.d_model) out[(p.v0 + to[m]) * (int64_t)p.d_model + c] = __float2bfloat16_rn(sum[m][u]);
      }
  }
}

}  // namespace

cudaError_t launch_distill_dw(const DistillParams& p, cudaStream_t s) {
  const int64_t slots = p.rows < kFewRows ? p.rows : kFewRows;
  const int64_t groups = (p.top + kDwEntries - 1) / kDwEntries;
  launch_pdl(k_distill_dw, dim3((unsigned)(slots * groups)), dim3(kThreads), 0, s, p);
  return cudaGetLastError();
}
cudaError_t launch_distill_grad(const DistillParams& p, cudaStream_t s) {
  launch_pdl(k_distill_grad, dim3((unsigned)((p.rows + kRowWarps - 1) / kRowWarps)), dim3(kThreads), 0, s, p);
  return cudaGetLastError();
}
namespace {
template <typename T, bool VEC>
void join_t(const DistillParams& p, cudaStream_t s) {
  // 8192 of 16384 rows, 32 entries of 832 bf16: a CTA per row 145 us, two warps 111, one 97; 2048 rows, 16 entries: 18
  // by CTAs, 14 by warps; 1024 rows 11 and 12. A warp takes four entries in turn, so that it needs the more rows beside
  // it the more entries.
  if (p.rows >= 2048 && p.rows >= 64 * p.top)
    launch_pdl(k_distill_join<T, VEC, 1>, dim3((unsigned)((p.rows + 7) / 8)), dim3(kThreads), 0, s, p);
  else
    launch_pdl(k_distill_join<T, VEC, 8>, dim3((unsigned)p.rows), dim3(kThreads), 0, s, p);
}
}  // namespace
cudaError_t launch_distill_join(const DistillParams& p, int f32, cudaStream_t s) {
  const int e = f32 ? 4 : 8;
  const bool vec = p.d_model % e == 0 && p.ld_h % e == 0;
  if (f32) vec ? join_t<float, true>(p, s) : join_t<float, false>(p, s);
  else vec ? join_t<bf16, true>(p, s) : join_t<bf16, false>(p, s);
  return cudaGetLastError();
}
cudaError_t launch_distill_dz(const DistillParams& p, cudaStream_t s) {
  launch_pdl(k_distill_dz, dim3((unsigned)((p.rows * p.top + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p);
  return cudaGetLastError();
}

}  // namespace bds
