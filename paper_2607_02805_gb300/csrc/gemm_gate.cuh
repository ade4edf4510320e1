// gemm_gate.cuh -- the epilogue of a gated layer's products, for gemm.cuh, which
// includes it before its kernel.
//
// A warp holds CW = BN / 8 columns of the gate g and the same of the other
// projection u, 16 at a time, a thread one row of them.
//   forward: y = act(g) u
//   gradient: dg = dy u act'(g), du = dy act(g), from dy in the place of a
//   residual; g and u have been computed again, so that they enter unrounded (a
//   saved bf16 copy would add a third rounding beside those of dg, du and of the
//   result, and costs two passes over 2 n columns).
// Rows on 16-byte boundaries come and leave in units of 32 rows x CW columns
// through the warp's shared memory, in the swizzle of the map's box; others
// (kEpiGateRows, kEpiGateDzRows) through the same memory as fp32, 16 columns at
// a time, by plain loads and stores of 16 lanes per row.
//
// Every wait has a poll limit; a warp that gives up leaves its loop and says so.
#pragma once

namespace bds {
namespace {

__device__ __forceinline__ void act_both(int act, float z, float& a, float& d) {
  if (act == kActNone) {
    a = z, d = 1.f;
    return;
  }
  // the argument is clamped and 0 z added as in act_grad
  float s, k;
  const float c = act == kActSilu ? fminf(fmaxf(z, -100.f), 100.f) : fminf(fmaxf(z, -16.f), 16.f);
  if (act == kActSilu) {
    s = rcp_f(1.f + ex2(silu_arg(c)));
    k = 1.f;
  } else {
    s = rcp_f(1.f + ex2(gelu_arg(c)));
    k = fmaf(6.f * kGeluA * kGeluB, c * c, 2.f * kGeluA);
  }
  a = z * s;
  d = fmaf(0.f, z, s * (1.f + c * (1.f - s) * k));
}
// Address of 16-byte piece j of a row in a unit of PR pieces per row.
template <int PR>
__device__ __forceinline__ unsigned char* unit_at(unsigned char* unit, int row, int j) {
  return unit + row * (16 * PR) + 16 * (PR == 4 ? j ^ ((row >> 1) & 3) : j ^ ((row >> 2) & 1));
}
// The unit of `res` at (row0, col): lane l holds piece l % PR of rows l / PR + 32 / PR j. Rows end on 16-byte
// boundaries, so that no piece reaches past column n.
template <int PR, int ELT>
__device__ __forceinline__ void load_unit(uint4 (&raw)[PR], const GemmParams& p, int64_t row0, int col, int n) {
  const int lane = threadIdx.x & 31, c = col + 16 / ELT * (lane % PR);
#pragma unroll
  for (int j = 0; j < PR; ++j) {
    const int64_t r = row0 + 32 / PR * j + lane / PR;
    raw[j] = r < p.m && c < n ? *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(p.res) +
                                                                (r * p.ld_res + c) * ELT)
                              : make_uint4(0, 0, 0, 0);
  }
}
// 16 columns from col on of 32 rows, those of them below row + left and column n, into a row per thread, and back.
template <bool F32>
__device__ __forceinline__ void rows_in(float (&v)[16], const GemmParams& p, int64_t row0, int col, int n,
                                        unsigned char* stg) {
  const int lane = threadIdx.x & 31, cl = lane & 15;
  float* f = reinterpret_cast<float*>(stg);
  const int64_t row = row0 + (lane >> 4);
  const int left = col + cl < n ? (int)min((int64_t)32, p.m - row) : 0;
  float e[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) e[i] = 2 * i < left ? load1(p.res, F32, (row + 2 * i) * p.ld_res + col + cl) : 0.f;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = 2 * i + (lane >> 4);
    f[r * 16 + 4 * ((cl >> 2) ^ ((r >> 1) & 3)) + (cl & 3)] = e[i];
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float4 q = *reinterpret_cast<const float4*>(f + lane * 16 + 4 * (j ^ ((lane >> 1) & 3)));
    v[4 * j] = q.x, v[4 * j + 1] = q.y, v[4 * j + 2] = q.z, v[4 * j + 3] = q.w;
  }
}
// PIECES: to as many planes of bf16, `plane` elements apart, the largest piece of what is left of the value each.
template <bool F32, int PIECES = 1>
__device__ __forceinline__ void rows_out(void* out, int64_t ld, int64_t m, int64_t row0, int col, int n, int at,
                                         const float (&v)[16], unsigned char* stg, int64_t plane = 0) {
  const int lane = threadIdx.x & 31, cl = lane & 15;
  float* f = reinterpret_cast<float*>(stg);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<float4*>(f + lane * 16 + 4 * (j ^ ((lane >> 1) & 3))) =
        make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  __syncwarp();
  if (col + cl < n) {
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 2 * i + (lane >> 4);
      y[i] = f[r * 16 + 4 * ((cl >> 2) ^ ((r >> 1) & 3)) + (cl & 3)];
    }
    const int64_t row = row0 + (lane >> 4);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      float part[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) part[i] = PIECES == 1 ? y[i] : bf16_part(y[i]);
      const int left = (int)min((int64_t)32, m - row);
      store_rows<F32>(static_cast<bf16*>(out) + k * plane, row, ld, at + col + cl, left, part);
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] -= part[i];
    }
  }
  __syncwarp();
}
// Bias of 16 columns from col on, added to them.
template <bool F32, bool ROWS>
__device__ __forceinline__ void gate_bias(float (&v)[16], const GemmParams& p, int col, int n, int at) {
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (col + i < n) v[i] += load1(p.bias, F32, at + col + i);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (col + 4 * j >= n) continue;  // whole pieces: n is a multiple of four
      const float4 b = load4(p.bias, F32, at + col + 4 * j);
      v[4 * j] += b.x, v[4 * j + 1] += b.y, v[4 * j + 2] += b.z, v[4 * j + 3] += b.w;
    }
  }
}
// Sums over the lanes, column by column: lane l ends with column l / 2.
__device__ __forceinline__ float colsum16(float (&v)[16]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int half = 8; half >= 1; half >>= 1) {
    const bool hi = (lane & (2 * half)) != 0;
#pragma unroll
    for (int j = 0; j < half; ++j) {
      const float give = hi ? v[j] : v[j + half], keep = hi ? v[j + half] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, 2 * half);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}
// Columns 16 hf .. + 15 of a thread's row to its place in a unit of bf16.
template <int PR>
__device__ __forceinline__ void unit_put(unsigned char* unit, int hf, const float (&v)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
    *reinterpret_cast<uint4*>(unit_at<PR>(unit, threadIdx.x & 31, 2 * hf + j)) =
        make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]),
                   pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
}
template <int CG, int BN, int NP, int EPI, int NA, typename SCHED>
__device__ __forceinline__ bool gate_epilogue(const GemmParams& p, const GemmMaps& maps, const SCHED& sched,
                                              uint32_t tm, unsigned char* stage, uint64_t* accfull, uint64_t* accempty,
                                              int rank) {
  using S = GemmSmem<CG, BN, NP, EPI>;
  constexpr bool FLUSH = NP == 3, F32 = NP == 3;
  constexpr bool DZ = EPI == kEpiGateDz || EPI == kEpiGateDzRows;
  constexpr bool ROWS = EPI == kEpiGateRows || EPI == kEpiGateDzRows;
  constexpr int CW = BN / 8, NH = CW / 16;
  static_assert(!FLUSH || NH == 1, "fp32 sums of 16 columns of both");
  constexpr int ELT = F32 ? 4 : 2, PR = CW * ELT / 16;  // pieces per row of a unit of dy or y
  constexpr int PZ = CW / 8;                            // of a unit of bf16
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, ew = w - 4, quarter = ew >> 2;
  const uint32_t lanes = tm + ((uint32_t)(32 * (w & 3)) << 16);
  unsigned char* stg = stage + ew * S::kUnit;
  const int n = p.n >> 1, h = p.bn >> 1, c0 = CW * quarter;
  const bool mine = c0 < h;  // small tiles have fewer columns than the sixteen warps
  auto first_row = [&](const Tile& x) { return (int64_t)x.tm * 128 * CG + rank * 128 + 32 * (w & 3); };
  uint4 raw[PR];
  auto ahead = [&](const Tile& x) {
    if constexpr (DZ && !ROWS) {
      if (mine) load_unit<PR, ELT>(raw, p, first_row(x), x.tn * h + c0, n);
    }
  };
  bool ok = true;
  uint32_t job = 0;
  Tile x, nx;
  bool another = sched.get(p, p, 0, nx);
  if (another) ahead(nx);
  for (int i = 0; another;) {
    x = nx;
    another = sched.get(p, p, ++i, nx);
    const int col0 = x.tn * h + c0;
    const bool live = mine && col0 < n;  // uniform over the warp
    const int64_t row0 = first_row(x);
    float g[16], u[16];
    auto release = [&]() {
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) leader_arrive<CG>(&accempty[job % NA]);
      ++job;
    };
    if constexpr (FLUSH) {
#pragma unroll
      for (int j = 0; j < 16; ++j) g[j] = u[j] = 0.f;
      for (int k = x.k0; k < x.k1; ++k) {
        if (!(ok = warp_wait(&accfull[job % NA], (job / NA) & 1))) break;
        umma::fence_after_sync();
        if (live) {
          __syncwarp();  // TMEM is read by whole warps
          float a[16], b[16];
          umma::tmem_ld16x2(lanes + job % NA * BN + c0, a, lanes + job % NA * BN + h + c0, b);
#pragma unroll
          for (int j = 0; j < 16; ++j) g[j] += a[j], u[j] += b[j];
        }
        release();
      }
    } else {
      ok = warp_wait(&accfull[job % NA], (job / NA) & 1);
      umma::fence_after_sync();
    }
    if (!ok) break;
    if (!live) {
      if (!FLUSH) release();
      if (another) ahead(nx);
      continue;
    }
    if constexpr (!ROWS) {
      if (lane == 0) tma_store_wait_read();
      __syncwarp();
    }
    if constexpr (DZ && !ROWS) {
#pragma unroll
      for (int j = 0; j < PR; ++j)
        *reinterpret_cast<uint4*>(unit_at<PR>(stg, 32 / PR * j + lane / PR, lane % PR)) = raw[j];
      __syncwarp();
      if (another) ahead(nx);
    }
#pragma unroll
    for (int hf = 0; hf < NH; ++hf) {
      const int col = col0 + 16 * hf;
      if constexpr (!FLUSH) {
        __syncwarp();  // TMEM is read by whole warps
        const uint32_t at = lanes + job % NA * BN + (uint32_t)(c0 + 16 * hf);
        umma::tmem_ld16x2(at, g, at + (uint32_t)h, u);
        if (hf == NH - 1) release();
      }
      if (p.bias != nullptr) {
        gate_bias<F32, ROWS>(g, p, col, n, 0);
        gate_bias<F32, ROWS>(u, p, col, n, n);
      }
      if constexpr (!DZ) {
        if (p.act == kActSilu) {
#pragma unroll
          for (int j = 0; j < 16; j += 2) sigmoid_mul2<silu_arg>(g[j], g[j + 1]);
        } else if (p.act == kActGelu) {
#pragma unroll
          for (int j = 0; j < 16; j += 2) sigmoid_mul2<gelu_arg>(g[j], g[j + 1]);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) g[j] *= u[j];
        if constexpr (ROWS) {
          rows_out<F32>(p.out, p.ld_out, p.m, row0, col, n, 0, g, stg);
        } else if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<float4*>(unit_at<PR>(stg, lane, j)) =
                make_float4(g[4 * j], g[4 * j + 1], g[4 * j + 2], g[4 * j + 3]);
        } else {
          unit_put<PR>(stg, hf, g);
        }
      } else {
        float e[16];
        if constexpr (ROWS) {
          rows_in<F32>(e, p, row0, col, n, stg);
        } else if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float4 q = *reinterpret_cast<const float4*>(unit_at<PR>(stg, lane, j));
            e[4 * j] = q.x, e[4 * j + 1] = q.y, e[4 * j + 2] = q.z, e[4 * j + 3] = q.w;
          }
          __syncwarp();  // the pieces of dz overwrite it
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            add8(f, *reinterpret_cast<const uint4*>(unit_at<PR>(stg, lane, 2 * hf + j)));
#pragma unroll
            for (int k = 0; k < 8; ++k) e[8 * j + k] = f[k];
          }
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          float a, d;
          act_both(p.act, g[j], a, d);
          g[j] = e[j] * u[j] * d;
          u[j] = e[j] * a;
        }
        if (p.colsum != nullptr && row0 < p.m) {
          // Rows behind the last one add nothing: dy = 0 there is not enough, since below 128 rows their accumulators
          // come from rows of A that no load has written, and zero times a NaN left there is NaN.
          const bool in = row0 + lane < p.m;
          float sg[16], su[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) sg[j] = in ? g[j] : 0.f, su[j] = in ? u[j] : 0.f;
          const float a = colsum16(sg), b = colsum16(su);
          const int c = col + (lane >> 1);
          if (c < n) p.colsum[(row0 >> 5) * p.n + c + (lane & 1) * n] = (lane & 1) ? b : a;
        }
        if constexpr (ROWS) {
          rows_out<false, NP>(p.out, p.ld_out, p.m, row0, col, n, 0, g, stg, p.split_stride);
          rows_out<false, NP>(p.out, p.ld_out, p.m, row0, col, n, n, u, stg, p.split_stride);
          continue;
        }
        // the pieces of both gradients (fp32: the largest of what is left, three times)
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          float dg[16], du[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            dg[j] = g[j], du[j] = u[j];
            if constexpr (NP == 3) {
              dg[j] = bf16_part(g[j]), du[j] = bf16_part(u[j]);
              g[j] -= dg[j], u[j] -= du[j];
            }
          }
          if constexpr (NP == 3) {
            unsigned char* at = stg + 2048 * (k & 1);
            if (k == 2) {  // the first piece's two stores have read this half
              if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 2;\n" ::: "memory");
              __syncwarp();
            }
            unit_put<PZ>(at, 0, dg);
            unit_put<PZ>(at + 1024, 0, du);
            umma::fence_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_3d(&maps.out, col0, (int)row0, k, umma::smem_u32(at));
              tma_store_3d(&maps.pre, col0, (int)row0, k, umma::smem_u32(at + 1024));
            }
          } else {
            unit_put<PZ>(stg, hf, dg);
            unit_put<PZ>(stg + 2048, hf, du);
          }
        }
      }
    }
    if constexpr (!ROWS && !(DZ && NP == 3)) {
      umma::fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        tma_store_3d(&maps.out, col0, (int)row0, 0, umma::smem_u32(stg));
        if constexpr (DZ) tma_store_3d(&maps.pre, col0, (int)row0, 0, umma::smem_u32(stg + 2048));
      }
    }
  }
  if (!ROWS && lane == 0) tma_store_wait_read();  // the stores themselves end with the grid
  return ok;
}

}  // namespace
}  // namespace bds
