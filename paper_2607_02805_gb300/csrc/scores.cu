// scores.cu -- token scores (include/bdscan_dense.h): per row of logits / T the
// log probability of a token, the entropy of the distribution and its likeliest
// entries, and the gradient of the logits. Kernels and C ABI.
//
// With c = log2(e) / T, m = max z and d_v = c (z_v - m): s = sum 2^d_v, t = sum
// 2^d_v d_v, log p_v = ln2 (d_v - log2 s), entropy ln2 (log2 s - t / s). The
// difference comes first, so that logits of the type's lowest value do not
// overflow. One pass: a thread keeps the maximum of what it has seen and s, t
// relative to it, and rescales them once per batch of four 16-byte loads.
//
// The likeliest entries come without sorting. The threads of a CTA form 64
// groups; the top-th largest of the groups' maxima is a bound that at least
// `top` entries reach, and only groups that reach it can hold one. Those read
// their entries again (from L2) and list what reaches the bound, on average
// little more than `top`; the rank of each in the list, by value and then by
// lower index, is its place in the output. Rows with so many equal entries that
// the list overflows are searched once per place instead.
//
// One CTA per row. Where that leaves SMs idle, a cluster of CTAs shares a row:
// each leaves its statistics and its own likeliest entries in the first one's
// shared memory.
#include <cstdio>
#include <cstring>

#include "bdscan_dense.h"
#include "debug.cuh"
#include "device.cuh"
#include "params.h"

namespace bds {
namespace {

constexpr int kMaxTop = 64;
constexpr int kGroups = 64;
constexpr int kList = 512;     // entries of a CTA's list; eight CTAs' kMaxTop each
constexpr int kMaxParts = 8;   // CTAs of a row's cluster
constexpr int kNone = 1 << 30; // stands for the index of a place without an entry, another for each place
static_assert(kMaxParts * kMaxTop <= kList, "the first CTA lists what the others found");

struct ScoresParams {
  const void* logits;
  const int64_t* token;
  float *logp, *entropy, *top_logp;
  float2* stats;
  int64_t* top_ids;
  int64_t rows, ld;
  int vocab, excluded, top;
  float scale;  // log2(e) / T
  // backward
  void* dlogits;
  int64_t ld_out;
  const float2* stats_in;
  const float *entropy_in, *dlogp, *dentropy;
  float inv_t;
  int parts;
};

// Two fp32 values in a register pair, for the packed instructions.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// 16 bytes of logits as they lie in memory.
template <typename T>
struct Vec {
  static constexpr int E = 16 / (int)sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ void load(const uint4* at) {
    const uint4 u = __ldg(at);
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  }
  __device__ __forceinline__ float2 two(int j) const {  // entries 2 j and 2 j + 1
    if constexpr (E == 4) return make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
    else return make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
  }
  __device__ __forceinline__ void none() {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = E == 4 ? 0xff800000u : 0xff80ff80u;
  }
  __device__ __forceinline__ void exclude(int k) {  // entry k becomes minus infinity
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (E == 4) {
        if (i == k) w[i] = 0xff800000u;
      } else {
        if (2 * i == k) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
        if (2 * i + 1 == k) w[i] = (w[i] & 0xffffu) | 0xff800000u;
      }
    }
  }
};
// The largest of U groups; NaN is passed over.
template <typename T, int U>
__device__ __forceinline__ float vec_max(const Vec<T> (&q)[U]) {
  if constexpr (Vec<T>::E == 4) {
    float m = __uint_as_float(q[0].w[0]);
#pragma unroll
    for (int i = 1; i < 4 * U; ++i) m = fmaxf(m, __uint_as_float(q[i / 4].w[i % 4]));
    return m;
  } else {
    auto bits = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    __nv_bfloat162 m = bits(q[0].w[0]);
#pragma unroll
    for (int i = 1; i < 4 * U; ++i) m = __hmax2(m, bits(q[i / 4].w[i % 4]));
    const float2 f = __bfloat1622float2(m);
    return fmaxf(f.x, f.y);
  }
}

// A row as 16-byte groups: `lead` entries before the first boundary, `n` groups, `tail` entries behind the last.
template <typename T>
struct Row {
  static constexpr int E = Vec<T>::E;
  const T* at;
  int lead, n, tail;
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t ld, int vocab) {
    at = static_cast<const T*>(base) + row * ld;
    const int off = (int)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T));
    lead = min(vocab, off == 0 ? 0 : E - off);
    n = (vocab - lead) / E;
    tail = vocab - lead - n * E;
  }
  __device__ __forceinline__ const uint4* group(int i) const { return reinterpret_cast<const uint4*>(at + lead) + i; }
  __device__ __forceinline__ int first(int i) const { return lead + i * E; }  // entry index of group i
};

// The entries of part `part` of `parts` of a row that this thread of THREADS
// takes: batch(U groups, the first's number; the others follow in steps of
// THREADS), one(value, index) at the ends of the row. The excluded entry is minus
// infinity, and so is what fills up the last batch.
template <typename T, int THREADS, int U, typename FV, typename FB>
__device__ __forceinline__ void for_entries(const Row<T>& r, int part, int parts, int excluded, FV one, FB batch) {
  constexpr int E = Vec<T>::E;
  const int t = threadIdx.x;
  const int a = (int)((int64_t)r.n * part / parts), b = (int)((int64_t)r.n * (part + 1) / parts);
  int i = a + t;
  for (; i < b; i += U * THREADS) {
    Vec<T> q[U];
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (i + j * THREADS < b) q[j].load(r.group(i + j * THREADS));
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int at = r.first(i + j * THREADS);
      if (i + j * THREADS >= b) q[j].none();
      else if ((unsigned)(excluded - at) < (unsigned)E) q[j].exclude(excluded - at);
    }
    batch(q, i);
  }
  // the few entries before and behind the groups, by threads of the first and the last part
  if (part == 0 && t < r.lead) one(t == excluded ? -INFINITY : cvt(r.at[t]), t);
  if (part == parts - 1 && t < r.tail) {
    const int at = r.lead + r.n * E + t;
    one(at == excluded ? -INFINITY : cvt(r.at[at]), at);
  }
}

// ---- statistics ----
struct Stat {
  float m, s, t;  // maximum, sum 2^d, sum 2^d d with d = c (z - m)
};
// What is subtracted: nothing where there is no maximum, so that minus infinity stays that.
__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }
// Moves s and t to a maximum that is not smaller.
__device__ __forceinline__ void stat_move(Stat& a, float m, float c) {
  if (a.m == -INFINITY) {  // nothing so far (or NaN, which no maximum shows)
    a.t = a.s;
  } else {
    const float by = fmaxf((a.m - m) * c, -1e30f), f = ex2(by);
    a.t = f * fmaf(a.s, by, a.t);
    a.s *= f;
  }
  a.m = m;
}
// d is clamped in its product with 2^d, so that minus infinity adds zero.
__device__ __forceinline__ void stat_add(Stat& a, float v, float c) {
  if (v > a.m) stat_move(a, v, c);
  const float d = (v - ref_of(a.m)) * c, e = ex2(d);
  a.s += e;
  a.t = fmaf(e, fmaxf(d, -200.f), a.t);
}
template <typename T, int U>
__device__ __forceinline__ void stat_add(Stat& a, const Vec<T> (&q)[U], float c) {
  const float m = vec_max(q);
  if (m > a.m) stat_move(a, m, c);
  const float ref = -ref_of(a.m);
  const f32x2 mm = pair(ref, ref), cc = pair(c, c);
  f32x2 s = pair(a.s, 0.f), t = pair(a.t, 0.f);
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int k = 0; k < Vec<T>::E / 2; ++k) {
      const float2 v = q[j].two(k);
      const float2 d = halves(mul2(add2(pair(v.x, v.y), mm), cc));
      const f32x2 e = pair(ex2(d.x), ex2(d.y));
      s = add2(s, e);
      t = fma2(e, pair(fmaxf(d.x, -200.f), fmaxf(d.y, -200.f)), t);
    }
  a.s = halves(s).x + halves(s).y;
  a.t = halves(t).x + halves(t).y;
}

__device__ __forceinline__ uint32_t my_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t first_cta(const void* p) {  // the same place in the cluster's first CTA
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  return r;
}
__device__ __forceinline__ void put_cluster(uint32_t at, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(at), "f"(v) : "memory");
}
__device__ __forceinline__ void put_cluster(uint32_t at, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;\n" ::"r"(at), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }

// Whether entry (v, i) comes before (w, j).
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

template <int THREADS>
struct ScoresSmem {
  float gmax[kGroups];
  Stat warp[THREADS / 32];
  float lv[kList], pv[kList];  // the list, and what the parts of a row found
  int li[kList], pi[kList];
  Stat part[kMaxParts];
  int count;
};

// The `top` first entries of the list in order: emit(place, value, index), then minus infinity for what is missing.
template <int THREADS, typename F>
__device__ __forceinline__ void rank_list(const float* lv, const int* li, int n, int top, F emit) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const float v = lv[i];
    const int at = li[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += before(lv[j], li[j], v, at) ? 1 : 0;
    if (rank < top) emit(rank, v, at);
  }
  for (int i = threadIdx.x; i < top; i += THREADS)
    if (i >= n) emit(i, -INFINITY, kNone);
}

template <typename T, int THREADS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_scores(const ScoresParams p) {
  pdl_sync();
  constexpr int E = Vec<T>::E, U = 4, W = THREADS / 32;
  __shared__ ScoresSmem<THREADS> sm;
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  const int parts = CLUSTER ? p.parts : 1, part = CLUSTER ? (int)my_rank() : 0;
  const int64_t row = CLUSTER ? blockIdx.x / parts : blockIdx.x;
  if (!dguard(kSiteScores, row * p.ld + p.vocab - 1, (p.rows - 1) * p.ld + p.vocab)) return;
  if (CLUSTER) cluster_arrive();
  int64_t token = p.token != nullptr ? p.token[row] : 0;
  if (token < 0 || token >= p.vocab) {  // a row that does not count (the same for its whole cluster)
    if (part == 0) {
      if (t == 0) {
        if (p.logp != nullptr) p.logp[row] = 0.f;
        if (p.entropy != nullptr) p.entropy[row] = 0.f;
        if (p.stats != nullptr) p.stats[row] = make_float2(0.f, 0.f);
      }
      for (int i = t; i < p.top; i += THREADS) {
        p.top_ids[row * p.top + i] = -1;
        p.top_logp[row * p.top + i] = -INFINITY;
      }
    }
    if (CLUSTER) cluster_wait();
    return;
  }
  const Row<T> r(p.logits, row, p.ld, p.vocab);
  const float c = p.scale;
  float zt = 0.f;
  if (t == 0 && part == 0 && p.token != nullptr) zt = token == p.excluded ? -INFINITY : cvt(r.at[token]);
  auto each_of = [&](auto f) {  // a batch entry by entry
    return [&r, f](const Vec<T>(&q)[U], int i) {
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int k = 0; k < E / 2; ++k) {
          const float2 v = q[j].two(k);
          f(v.x, r.first(i + j * THREADS) + 2 * k);
          f(v.y, r.first(i + j * THREADS) + 2 * k + 1);
        }
    };
  };
  Stat a = {-INFINITY, 0.f, 0.f};
  for_entries<T, THREADS, U>(
      r, part, parts, p.excluded, [&](float v, int) { stat_add(a, v, c); },
      [&](const Vec<T>(&q)[U], int) { stat_add(a, q, c); });

  // the groups' maxima, then the CTA's
  constexpr int G = THREADS / kGroups;  // threads of a group
  float m = a.m;
#pragma unroll
  for (int o = 1; o < G; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float gm = m;
  if (t % G == 0) sm.gmax[t / G] = gm;
  if (t == 0) sm.count = 0;
  __syncthreads();
  const float g0 = sm.gmax[lane], g1 = sm.gmax[lane + 32];
  m = fmaxf(g0, g1);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  // all threads' sums relative to that, added in a fixed order
  stat_move(a, m, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
  if (lane == 0) sm.warp[w] = a;
  if (p.top > 0) {
    // the bound: the top-th largest of the groups' maxima (every warp finds it for itself)
    int r0 = 0, r1 = 0;
#pragma unroll 8
    for (int j = 0; j < kGroups; ++j) {
      const float q = sm.gmax[j];
      r0 += before(q, j, g0, lane) ? 1 : 0;
      r1 += before(q, j, g1, lane + 32) ? 1 : 0;
    }
    float tau = r0 == p.top - 1 ? g0 : r1 == p.top - 1 ? g1 : -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) tau = fmaxf(tau, __shfl_xor_sync(0xffffffffu, tau, o));
    if (gm >= tau && a.m != -INFINITY) {
      auto keep = [&](float v, int at) {
        if (v >= tau && v != -INFINITY) {
          const int to = atomicAdd(&sm.count, 1);
          if (to < kList) sm.lv[to] = v, sm.li[to] = at;
        }
      };
      for_entries<T, THREADS, U>(r, part, parts, p.excluded, keep, each_of(keep));
    }
  }
  __syncthreads();
  // the part's sums (every thread: the same)
  a = sm.warp[0];
#pragma unroll
  for (int k = 1; k < W; ++k) a.s += sm.warp[k].s, a.t += sm.warp[k].t;
  int n = sm.count;
  if (p.top > 0 && n > kList) {
    // many equal entries: place by place the first entry behind the last one found
    float pv = INFINITY;
    int pi = -1;
    for (int k = 0; k < p.top; ++k) {
      float bv = -INFINITY;
      int bi = 0x7fffffff;
      auto see = [&](float v, int at) {
        if (v != -INFINITY && before(pv, pi, v, at) && before(v, at, bv, bi)) bv = v, bi = at;
      };
      for_entries<T, THREADS, U>(r, part, parts, p.excluded, see, each_of(see));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, bv, o);
        const int at = __shfl_xor_sync(0xffffffffu, bi, o);
        if (before(v, at, bv, bi)) bv = v, bi = at;
      }
      __syncthreads();
      if (lane == 0) sm.lv[kMaxTop + w] = bv, sm.li[kMaxTop + w] = bi;
      __syncthreads();
      bv = sm.lv[kMaxTop], bi = sm.li[kMaxTop];
      for (int j = 1; j < W; ++j)
        if (before(sm.lv[kMaxTop + j], sm.li[kMaxTop + j], bv, bi)) bv = sm.lv[kMaxTop + j], bi = sm.li[kMaxTop + j];
      if (t == 0) sm.lv[k] = bv, sm.li[k] = bv == -INFINITY ? kNone + k : bi;
      pv = bv, pi = bi;
    }
    n = p.top;
    __syncthreads();
  }
  const float *lv = sm.lv;
  const int* li = sm.li;
  if constexpr (CLUSTER) {
    cluster_wait();  // the first CTA has begun
    if (t == 0) {
      const uint32_t to = first_cta(&sm.part[part]);
      put_cluster(to, a.m);
      put_cluster(to + 4, a.s);
      put_cluster(to + 8, a.t);
    }
    const uint32_t tv = first_cta(&sm.pv[part * p.top]), ti = first_cta(&sm.pi[part * p.top]);
    rank_list<THREADS>(sm.lv, sm.li, n, p.top, [&](int k, float v, int at) {
      put_cluster(tv + 4 * k, v);
      put_cluster(ti + 4 * k, v == -INFINITY ? kNone + part * p.top + k : at);
    });
    cluster_arrive();
    cluster_wait();
    if (part != 0) return;
    a = sm.part[0];
    for (int k = 1; k < parts; ++k) {
      Stat q = sm.part[k];
      const float nm = fmaxf(a.m, q.m);
      stat_move(a, nm, c);
      stat_move(q, nm, c);
      a.s += q.s, a.t += q.t;
    }
    lv = sm.pv, li = sm.pi;
    n = parts * p.top;
  }
  // nothing left: no entry has a probability; NaN or plus infinity anywhere: everything is NaN
  const float l2 = log2f(a.s), ln = l2 * kLn2;
  const bool bad = isnan(a.s);
  auto logp = [&](float z) {
    const float d = fmaf(z - a.m, p.inv_t, -ln);
    return bad ? a.s : z == -INFINITY ? z : d > 0.f ? 0.f : d;
  };
  if (t == 0) {
    if (p.logp != nullptr) p.logp[row] = logp(zt);
    const float h = (l2 - a.t / a.s) * kLn2;
    if (p.entropy != nullptr) p.entropy[row] = a.m == -INFINITY && !bad ? 0.f : h < 0.f ? 0.f : h;
    if (p.stats != nullptr) p.stats[row] = make_float2(bad ? a.s : a.m, ln);
  }
  if (p.top > 0) {
    float* lo = p.top_logp + row * p.top;
    int64_t* id = p.top_ids + row * p.top;
    rank_list<THREADS>(lv, li, n, p.top, [&](int k, float v, int at) {
      if (k < p.top) lo[k] = logp(v), id[k] = bad || v == -INFINITY ? -1 : at;
    });
  }
}

// ---- gradient of the logits ----
// dz_v = -p_v (dlogp + dentropy (entropy + log p_v)) / T, at the token plus dlogp
// / T: one read and one write, with p from the forward's statistics.
template <typename T>
__global__ void __launch_bounds__(256) k_scores_bwd(const ScoresParams p) {
  pdl_sync();
  constexpr int E = Vec<T>::E, THREADS = 256;
  const int t = threadIdx.x, part = (int)(blockIdx.x % p.parts);
  const int64_t row = blockIdx.x / p.parts;
  if (!dguard(kSiteScores, row * p.ld_out + p.vocab - 1, (p.rows - 1) * p.ld_out + p.vocab)) return;
  T* out = static_cast<T*>(p.dlogits) + row * p.ld_out;
  const int64_t token = p.token != nullptr ? p.token[row] : 0;
  const float2 st = p.stats_in[row];
  const bool counts = token >= 0 && token < p.vocab && st.x != -INFINITY;
  const Row<T> r(p.logits, row, p.ld, p.vocab);
  const float ls = st.y * kLog2e, ref = ref_of(st.x);
  const float dl = (p.dlogp != nullptr ? p.dlogp[row] : 0.f) * p.inv_t;
  const float dh = (p.dentropy != nullptr ? p.dentropy[row] : 0.f) * p.inv_t;
  const float base = dl + (p.dentropy != nullptr ? dh * p.entropy_in[row] : 0.f), slope = dh * kLn2;
  auto grad = [&](float z, int at) {
    const float d = (z - ref) * p.scale - ls;
    float g = -ex2(d) * fmaf(slope, fmaxf(d, -200.f), base);
    if (p.token != nullptr && at == (int)token) g += dl;
    return at == p.excluded || !counts ? 0.f : g;
  };
  const int a = (int)((int64_t)p.vocab * part / p.parts), b = (int)((int64_t)p.vocab * (part + 1) / p.parts);
  for (int i = a + t; i < b; i += THREADS) out[i] = to_out<T>(grad(counts ? cvt(r.at[i]) : 0.f, i));
}

template <typename T, int THREADS>
cudaError_t scores_t(const ScoresParams& p, cudaStream_t s) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * p.parts));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = p.parts > 1 ? 2 : 1;
  return p.parts > 1 ? cudaLaunchKernelEx(&cfg, k_scores<T, THREADS, true>, p)
                     : cudaLaunchKernelEx(&cfg, k_scores<T, THREADS, false>, p);
}

int fail(int code, const char* fn, const char* what) {
  char msg[384];
  snprintf(msg, sizeof(msg), "%s: %s", fn, what);
  return api_fail(code, msg);
}
int fail_ptr(const char* fn, const char* name, const char* problem) {
  char msg[128];
  snprintf(msg, sizeof(msg), "%s %s", name, problem);
  return fail(BDSCAN_ERR_ARG, fn, msg);
}
#define SCORES_REQ(ptr, fn, name)                                                                      \
  do {                                                                                                 \
    if ((ptr) == nullptr) return fail_ptr(fn, name, "is NULL");                                        \
    if (((uintptr_t)(ptr)&15u) != 0) return fail_ptr(fn, name, "is not 16-byte aligned");              \
  } while (0)
#define SCORES_OPT(ptr, fn, name)                                                                      \
  do {                                                                                                 \
    if (((uintptr_t)(ptr)&15u) != 0) return fail_ptr(fn, name, "is not 16-byte aligned");              \
  } while (0)

int check_scores(const bdscan_token_scores_dims* d, ScoresParams* p, const char* fn) {
  api_begin();
  memset(p, 0, sizeof(*p));
  if (d == nullptr) return fail(BDSCAN_ERR_ARG, fn, "dims is NULL");
  if (d->rows < 0) return fail(BDSCAN_ERR_ARG, fn, "negative rows");
  if (d->vocab <= 0) return fail(BDSCAN_ERR_ARG, fn, "vocab must be positive");
  if (d->dtype != BDSCAN_F32 && d->dtype != BDSCAN_BF16) return fail(BDSCAN_ERR_ARG, fn, "bad dtype");
  if (d->top < 0) return fail(BDSCAN_ERR_ARG, fn, "negative top");
  if (d->excluded < -1 || d->excluded >= d->vocab)
    return fail(BDSCAN_ERR_ARG, fn, "excluded is neither -1 nor inside the vocabulary");
  // 2^-20 .. 2^20: what is beyond would leave fp32 with ordinary logits
  if (!(d->temperature >= 0x1p-20f && d->temperature <= 0x1p20f))
    return fail(BDSCAN_ERR_ARG, fn, "temperature is not between 2^-20 and 2^20");
  if (d->top > kMaxTop) return fail(BDSCAN_ERR_UNSUPPORTED, fn, "top above 64");
  if (d->rows > ((int64_t)1 << 27) || d->vocab > ((int64_t)1 << 24))
    return fail(BDSCAN_ERR_UNSUPPORTED, fn, "rows above 2^27 or vocab above 2^24");
  p->ld = d->ld_logits ? d->ld_logits : d->vocab;
  p->ld_out = d->ld_dlogits ? d->ld_dlogits : d->vocab;
  if (p->ld < d->vocab) return fail(BDSCAN_ERR_ARG, fn, "ld_logits is below vocab");
  if (p->ld_out < d->vocab) return fail(BDSCAN_ERR_ARG, fn, "ld_dlogits is below vocab");
  if (p->ld > ((int64_t)1 << 30) || p->ld_out > ((int64_t)1 << 30))
    return fail(BDSCAN_ERR_UNSUPPORTED, fn, "a row stride above 2^30");
  p->rows = d->rows;
  p->vocab = (int)d->vocab;
  p->excluded = (int)d->excluded;
  p->top = d->top;
  p->inv_t = 1.f / d->temperature;
  p->scale = kLog2e / d->temperature;
  p->parts = 1;
  return BDSCAN_OK;
}
int done(cudaError_t e, const char* fn, cudaStream_t s) {
  e = api_launched(e, s);
  return e == cudaSuccess ? api_ok() : fail(BDSCAN_ERR_CUDA, fn, cudaGetErrorString(e));
}

}  // namespace
}  // namespace bds

using namespace bds;

extern "C" {

int bdscan_token_scores_forward(const bdscan_token_scores_dims* dims, const void* logits, const int64_t* token,
                                float* logp, float* entropy, float* stats, int64_t* top_ids, float* top_logp,
                                void* stream) {
  const char* fn = "bdscan_token_scores_forward";
  ScoresParams p;
  const int rc = check_scores(dims, &p, fn);
  if (rc) return rc;
  if (p.rows == 0) return api_ok();
  SCORES_REQ(logits, fn, "logits");
  SCORES_OPT(token, fn, "token");
  if (token != nullptr) SCORES_REQ(logp, fn, "logp");
  else if (logp != nullptr) return fail(BDSCAN_ERR_ARG, fn, "logp without token");
  SCORES_OPT(entropy, fn, "entropy");
  SCORES_OPT(stats, fn, "stats");
  if (p.top > 0) {
    SCORES_REQ(top_ids, fn, "top_ids");
    SCORES_REQ(top_logp, fn, "top_logp");
  }
  p.logits = logits;
  p.token = token;
  p.logp = logp;
  p.entropy = entropy;
  p.stats = (float2*)stats;
  p.top_ids = top_ids;
  p.top_logp = top_logp;
  const bool small = p.vocab <= 4096;
  // a row's cluster: as many CTAs as leave no SM idle, each with 2048 entries at least
  while (p.parts < kMaxParts && p.rows * p.parts < 152 && p.vocab >= 2048 * 2 * p.parts) p.parts *= 2;
  cudaStream_t s = (cudaStream_t)stream;
  const bool f32 = dims->dtype == BDSCAN_F32;
  const cudaError_t e = small ? (f32 ? scores_t<float, 128>(p, s) : scores_t<bf16, 128>(p, s))
                              : (f32 ? scores_t<float, 512>(p, s) : scores_t<bf16, 512>(p, s));
  return done(e, fn, s);
}

int bdscan_token_scores_backward(const bdscan_token_scores_dims* dims, const void* logits, const int64_t* token,
                                 const float* stats, const float* entropy, const float* dlogp, const float* dentropy,
                                 void* dlogits, void* stream) {
  const char* fn = "bdscan_token_scores_backward";
  ScoresParams p;
  const int rc = check_scores(dims, &p, fn);
  if (rc) return rc;
  if (p.rows == 0) return api_ok();
  SCORES_REQ(logits, fn, "logits");
  SCORES_OPT(token, fn, "token");
  SCORES_REQ(stats, fn, "stats");
  SCORES_OPT(dlogp, fn, "dlogp");
  SCORES_OPT(dentropy, fn, "dentropy");
  if (dlogp != nullptr && token == nullptr) return fail(BDSCAN_ERR_ARG, fn, "dlogp without token");
  if (dentropy != nullptr) SCORES_REQ(entropy, fn, "entropy");
  SCORES_REQ(dlogits, fn, "dlogits");
  p.logits = logits;
  p.token = token;
  p.stats_in = (const float2*)stats;
  p.entropy_in = entropy;
  p.dlogp = dlogp;
  p.dentropy = dentropy;
  p.dlogits = dlogits;
  while (p.parts < 64 && p.rows * p.parts < 608 && p.vocab >= 2048 * p.parts) p.parts *= 2;
  cudaStream_t s = (cudaStream_t)stream;
  const dim3 grid((unsigned)(p.rows * p.parts)), block(256);
  const cudaError_t e = dims->dtype == BDSCAN_F32 ? launch_pdl(k_scores_bwd<float>, grid, block, 0, s, p)
                                                  : launch_pdl(k_scores_bwd<bf16>, grid, block, 0, s, p);
  return done(e, fn, s);
}

}  // extern "C"
