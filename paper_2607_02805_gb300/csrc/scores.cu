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
// The likeliest entries come without sorting. The threads of a CTA form 128
// groups; the top-th largest of the groups' maxima is a bound that at least
// `top` entries reach, and only groups that reach it can hold one. A warp each
// reads such a group's entries again (from L2) and lists what reaches the bound:
// of independent entries -128 log(1 - top / 128) on average, 17 for 16 and 89
// for 64. The rank of each in the list, by value and then by lower index, is its
// place in the output. Rows with so many equal entries that the list overflows
// are searched once per place instead (16384 rows of 50304 equal bf16 logits with
// 16 entries: 9.5 ms).
//
// One CTA per row, six of 256 threads per SM. Where that leaves SMs idle, a
// cluster of CTAs shares a row: each leaves its statistics and its own likeliest
// entries in the first one's shared memory. 16384 rows of 50304 bf16 (1.65 GB):
// 240 us without likeliest entries, the copy rate, 260 with one, 300 with 16 (an
// eighth of each row read again, and its latency), 473 with 64. The gradient is
// one read and one write at the copy rate (477 us).
#include <cstdio>
#include <cstring>

#include "bdscan_dense.h"
#include "debug.cuh"
#include "device.cuh"
#include "overlap.h"
#include "params.h"
#include "ssd_common.cuh"

namespace bds {
namespace {

constexpr int kMaxTop = 64;
constexpr int kGroups = 128;
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
  // The larger of the first or the second half.
  __device__ __forceinline__ float half_max(int h) const {
    if constexpr (E == 4) {
      return fmaxf(__uint_as_float(w[2 * h]), __uint_as_float(w[2 * h + 1]));
    } else {
      const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w[2 * h]),
                                       *reinterpret_cast<const __nv_bfloat162*>(&w[2 * h + 1]));
      const float2 f = __bfloat1622float2(m);
      return fmaxf(f.x, f.y);
    }
  }
  // Which entries, not minus infinity, are `tau` or more.
  __device__ __forceinline__ uint32_t reach(float tau) const {
    uint32_t hit = 0;
#pragma unroll
    for (int k = 0; k < E / 2; ++k) {
      const float2 v = two(k);
      hit |= (v.x >= tau && v.x != -INFINITY ? 1u : 0u) << 2 * k | (v.y >= tau && v.y != -INFINITY ? 2u : 0u) << 2 * k;
    }
    return hit;
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
  __device__ __forceinline__ int begin(int part, int parts) const { return (int)((int64_t)n * part / parts); }
  __device__ __forceinline__ void exclude(Vec<T>& q, int i, int excluded) const {
    if ((unsigned)(excluded - first(i)) < (unsigned)E) q.exclude(excluded - first(i));
  }
};

// The entries of part `part` of `parts` of a row that this thread of THREADS
// takes: batch(U groups or one, the first's number; the others follow in steps of
// THREADS), one(value, index) at the ends of the row. The excluded entry is minus
// infinity.
template <typename T, int THREADS, int U, typename FV, typename FB>
__device__ __forceinline__ void for_entries(const Row<T>& r, int part, int parts, int excluded, FV one, FB batch) {
  constexpr int E = Vec<T>::E;
  const int t = threadIdx.x;
  const int a = r.begin(part, parts), b = r.begin(part + 1, parts);
  int i = a + t;
  // whole batches, then single groups
  for (; i + (U - 1) * THREADS < b; i += U * THREADS) {
    Vec<T> q[U];
#pragma unroll
    for (int j = 0; j < U; ++j) q[j].load(r.group(i + j * THREADS));
#pragma unroll
    for (int j = 0; j < U; ++j) r.exclude(q[j], i + j * THREADS, excluded);
    batch(q, i);
  }
  for (; i < b; i += THREADS) {
    Vec<T> q[1];
    q[0].load(r.group(i));
    r.exclude(q[0], i, excluded);
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
__device__ __forceinline__ void stat_sum(Stat& a, const Vec<T> (&q)[U], float c) {  // none above a.m
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
template <typename T, int U>
__device__ __forceinline__ void stat_add(Stat& a, const Vec<T> (&q)[U], float c) {
  const float m = vec_max(q);
  if (m > a.m) stat_move(a, m, c);
  stat_sum(a, q, c);
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
// Each thread by itself: what comes before may have left the warp's threads at different places, and the aligned forms
// would count such a warp more than once.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;\n" ::: "memory"); }

// Keys that order like the floats they stand for (one zero); 0 is below all.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// A bound that the top-th largest of a warp's N values per lane reaches, and no
// more than it: the values' keys, taken off one by one. In their last bits the
// keys carry their place, so that no two are equal and a round is a maximum, a
// reduction and N selects (with a ballot for the first of equal keys a round took
// twice as long); the bound is the key without them. Minus infinity (where there
// are fewer values than `top`) and NaN count as none.
template <int N>
__device__ __forceinline__ float take_off(const float (&v)[N], int top) {
  constexpr uint32_t kPlace = 32 * N - 1;
  const int lane = threadIdx.x & 31;
  uint32_t keys[N], bound = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) keys[k] = v[k] > -INFINITY ? (key_of(v[k]) & ~kPlace) | (uint32_t)(N * lane + k) : 0u;
  for (int i = 0; i < top; ++i) {
    uint32_t mine = keys[0];
#pragma unroll
    for (int k = 1; k < N; ++k) mine = max(mine, keys[k]);
    bound = __reduce_max_sync(0xffffffffu, mine);
#pragma unroll
    for (int k = 0; k < N; ++k) keys[k] = keys[k] == bound ? 0u : keys[k];
  }
  return bound != 0 ? of_key(bound & ~kPlace) : -INFINITY;
}
// Whether entry (v, i) comes before (w, j).
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

template <int THREADS>
struct ScoresSmem {
  alignas(16) float gmax[kGroups];
  Stat warp[THREADS / 32];
  float lv[kList], pv[kList];  // the list, and what the parts of a row found
  int li[kList], pi[kList];
  Stat part[kMaxParts];
  float tau[kGroups / 32];
  int sel[kGroups];  // groups that reach the bound
  int count, selected;
};

// The outputs of a row from its statistics. Nothing left: no entry has a
// probability. NaN or plus infinity anywhere: everything is NaN.
struct RowOut {
  const ScoresParams& p;
  int64_t row;
  float m, s, ln;
  bool bad;
  __device__ __forceinline__ RowOut(const ScoresParams& p_, int64_t row_, const Stat& a)
      : p(p_), row(row_), m(a.m), s(a.s), ln(log2f(a.s) * kLn2), bad(isnan(a.s)) {}
  __device__ __forceinline__ float logp(float z) const {
    const float d = fmaf(z - m, p.inv_t, -ln);
    return bad ? s : z == -INFINITY ? z : d > 0.f ? 0.f : d;
  }
  // by one thread; zt: the token's logit
  __device__ __forceinline__ void scores(const Stat& a, float zt) const {
    if (p.logp != nullptr) p.logp[row] = logp(zt);
    const float h = (log2f(s) - a.t / s) * kLn2;
    if (p.entropy != nullptr) p.entropy[row] = m == -INFINITY && !bad ? 0.f : h < 0.f ? 0.f : h;
    if (p.stats != nullptr) p.stats[row] = make_float2(bad ? s : m, ln);
  }
  __device__ __forceinline__ void place(int k, float v, int at) const {
    p.top_logp[row * p.top + k] = logp(v);
    p.top_ids[row * p.top + k] = bad || v == -INFINITY ? -1 : at;
  }
};
// Of a row that does not count, by thread t of n.
__device__ __forceinline__ void out_none(const ScoresParams& p, int64_t row, int t, int n) {
  if (t == 0) {
    if (p.logp != nullptr) p.logp[row] = 0.f;
    if (p.entropy != nullptr) p.entropy[row] = 0.f;
    if (p.stats != nullptr) p.stats[row] = make_float2(-INFINITY, 0.f);  // as of a row without entries: no gradient
  }
  for (int i = t; i < p.top; i += n) {
    p.top_ids[row * p.top + i] = -1;
    p.top_logp[row * p.top + i] = -INFINITY;
  }
}

// The `top` first entries of the list in order: emit(place, value, index), then minus infinity for what is missing.
template <int THREADS, typename F>
__device__ __forceinline__ void rank_list(const float* lv, const int* li, int n, int top, F emit) {
  const int t = threadIdx.x % THREADS;
  if (THREADS >= 128 && 2 * n <= THREADS) {  // a short list: four or two lanes of a warp per entry
    const int lanes = 4 * n <= THREADS ? 4 : 2, i = t / lanes;
    float v = 0.f;
    int at = 0, rank = 0;
    if (i < n) {
      v = lv[i], at = li[i];
#pragma unroll 4
      for (int j = t % lanes; j < n; j += lanes) rank += before(lv[j], li[j], v, at) ? 1 : 0;
    }
    __syncwarp();
    rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    const int more = __shfl_xor_sync(0xffffffffu, rank, 2);
    if (lanes == 4) rank += more;
    if (i < n && t % lanes == 0 && rank < top) emit(rank, v, at);
    for (int k = n + t; k < top; k += THREADS) emit(k, -INFINITY, kNone);
    return;
  }
  for (int i = t; i < n; i += THREADS) {
    const float v = lv[i];
    const int at = li[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += before(lv[j], li[j], v, at) ? 1 : 0;
    if (rank < top) emit(rank, v, at);
  }
  for (int i = t; i < top; i += THREADS)
    if (i >= n) emit(i, -INFINITY, kNone);
}

template <typename T, int THREADS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, CLUSTER ? 512 / THREADS : 1536 / THREADS) k_scores(const ScoresParams p) {
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
    if (part == 0) out_none(p, row, t, THREADS);
    if (CLUSTER) cluster_wait();
    return;
  }
  const Row<T> r(p.logits, row, p.ld, p.vocab);
  const float c = p.scale;
  float zt = 0.f;
  if (t == 0 && part == 0 && p.token != nullptr) zt = token == p.excluded ? -INFINITY : cvt(r.at[token]);
  auto each_of = [&](auto f) {  // a batch entry by entry
    return [&r, f](const auto& q, int i) {
#pragma unroll
      for (int j = 0; j < (int)(sizeof(q) / sizeof(Vec<T>)); ++j)
#pragma unroll
        for (int k = 0; k < E / 2; ++k) {
          const float2 v = q[j].two(k);
          f(v.x, r.first(i + j * THREADS) + 2 * k);
          f(v.y, r.first(i + j * THREADS) + 2 * k + 1);
        }
    };
  };
  Stat a = {-INFINITY, 0.f, 0.f};
  // a part of a row that is shared fits the threads' registers mostly: it is not read again then
  constexpr int NR = CLUSTER ? 8 : 1;
  Vec<T> held[NR];
  const bool hold = CLUSTER && r.begin(part + 1, parts) - r.begin(part, parts) <= NR * THREADS;
  if (hold) {
    const int begin = r.begin(part, parts) + t, end = r.begin(part + 1, parts);
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      if (begin + j * THREADS < end) held[j].load(r.group(begin + j * THREADS));
      else held[j].none();
    }
#pragma unroll
    for (int j = 0; j < NR; ++j) r.exclude(held[j], begin + j * THREADS, p.excluded);
    stat_add(a, held, c);
    if (part == 0 && t < r.lead && t != p.excluded) stat_add(a, cvt(r.at[t]), c);
    const int last = r.lead + r.n * E + t;
    if (part == parts - 1 && t < r.tail && last != p.excluded) stat_add(a, cvt(r.at[last]), c);
  } else {
    for_entries<T, THREADS, U>(
        r, part, parts, p.excluded, [&](float v, int) { stat_add(a, v, c); },
        [&](const auto& q, int) { stat_add(a, q, c); });
  }

  // the groups' maxima, then the CTA's
  constexpr int G = THREADS / kGroups;  // threads of a group
  float m = a.m;
#pragma unroll
  for (int o = 1; o < G; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (t % G == 0) sm.gmax[t / G] = m;
  if (t == 0) sm.count = sm.selected = 0;
  __syncthreads();
  const float4 g4 = reinterpret_cast<const float4*>(sm.gmax)[lane];
  m = fmaxf(fmaxf(g4.x, g4.y), fmaxf(g4.z, g4.w));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  // The bound, the top-th largest of the groups' maxima. For few places one warp takes the maxima off, while the others
  // wait (issue slots are what many rows share); for many a thread per group counts those above its own, and the bound
  // is the smallest that fewer than `top` exceed. A row that several CTAs share has the SMs to itself, and the count is
  // sooner done (16 entries of one row 7.4 us, by taking off 7.9).
  constexpr int kTakeOff = CLUSTER ? 4 : 32;
  if (p.top > 0 && p.top <= kTakeOff) {
    if (w == 0) {
      const float four[4] = {g4.x, g4.y, g4.z, g4.w};
      const float tau = take_off(four, p.top);
      if (lane < kGroups / 32) sm.tau[lane] = tau;
    }
  } else if (p.top > 0 && t < kGroups) {
    const float of = sm.gmax[t];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < kGroups / 4; ++j) {
      const float4 q = reinterpret_cast<const float4*>(sm.gmax)[j];
      above += (q.x > of) + (q.y > of) + (q.z > of) + (q.w > of);
    }
    float tau = above < p.top ? of : INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) tau = fminf(tau, __shfl_xor_sync(0xffffffffu, tau, o));
    if (lane == 0) sm.tau[w] = tau;
  }
  // all threads' sums relative to the maximum, added in a fixed order
  stat_move(a, m, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
  if (lane == 0) sm.warp[w] = a;
  __syncthreads();
  if (p.top > 0) {
    float tau = sm.tau[0];
#pragma unroll
    for (int k = 1; k < kGroups / 32; ++k) tau = fminf(tau, sm.tau[k]);
    auto keep = [&](float v, int at) {
      if (v >= tau && v != -INFINITY) {
        const int to = atomicAdd(&sm.count, 1);
        if (to < kList) sm.lv[to] = v, sm.li[to] = at;
      }
    };
    if (hold) {
      const int begin = r.begin(part, parts) + t;
#pragma unroll
      for (int j = 0; j < NR; ++j) {
        const Vec<T> one[1] = {held[j]};
        if (vec_max(one) < tau) continue;
        for (uint32_t hit = held[j].reach(tau); hit != 0; hit &= hit - 1) {
          const int i = r.first(begin + j * THREADS) + __ffs(hit) - 1;
          keep(cvt(r.at[i]), i);
        }
      }
    } else {
      // the groups that reach it, listed in any order; all threads share their entries (a warp those of its own groups:
      // 16384 x 50304 with 16 entries 327 us, 2048 x 131072 fp32 211; so 316 and 189, by the rest of that time)
      if (t < kGroups && sm.gmax[t] >= tau && sm.gmax[t] != -INFINITY) sm.sel[atomicAdd(&sm.selected, 1)] = t;
      __syncthreads();
      const int begin = r.begin(part, parts), end = r.begin(part + 1, parts), ns = sm.selected;
      const int per = (end - begin + THREADS - 1) / THREADS * G;  // 16-byte groups of each, the last ones past the end
      int k = per > 0 ? t / per : ns, e = t - k * per;  // group and its e-th
      const int dk = per > 0 ? THREADS / per : 0, de = THREADS - dk * per;
      while (k < ns) {
        Vec<T> q[U];
        int at[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          at[j] = k < ns ? begin + sm.sel[k] * G + e % G + e / G * THREADS : end;
          if (at[j] < end) q[j].load(r.group(at[j]));
          k += dk, e += de;
          if (e >= per) e -= per, ++k;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
          if (at[j] >= end) continue;
          r.exclude(q[j], at[j], p.excluded);
          const Vec<T> one[1] = {q[j]};
          if (vec_max(one) < tau) continue;
          for (uint32_t hit = q[j].reach(tau); hit != 0; hit &= hit - 1) {
            const int i = r.first(at[j]) + __ffs(hit) - 1;
            keep(cvt(r.at[i]), i);
          }
        }
      }
    }
    if (part == 0 && t < r.lead && t != p.excluded) keep(cvt(r.at[t]), t);
    const int last = r.lead + r.n * E + t;
    if (part == parts - 1 && t < r.tail && last != p.excluded) keep(cvt(r.at[last]), last);
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
  if constexpr (CLUSTER) {
    __syncthreads();
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
    __syncthreads();
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
  }
  const RowOut out(p, row, a);
  if (t == 0) out.scores(a, zt);
  if (p.top > 0) {
    const float* lv = sm.lv;
    const int* li = sm.li;
    if constexpr (CLUSTER) {
      // The parts' lists again as one. Of long ones first those that reach a bound: as many of each list as add up to
      // `top` do (one row, 64 entries: 24 us ranking all 512).
      lv = sm.pv, li = sm.pi;
      n = parts * p.top;
      if (n > 128) {
        const int deep = (p.top + parts - 1) / parts - 1;
        float tau = sm.pv[deep];
        for (int q = 1; q < parts; ++q) tau = fminf(tau, sm.pv[q * p.top + deep]);
        if (t == 0) sm.count = 0;
        __syncthreads();
        for (int x = t; x < n; x += THREADS) {
          if (!(sm.pv[x] >= tau) || sm.pv[x] == -INFINITY) continue;
          const int to = atomicAdd(&sm.count, 1);
          sm.lv[to] = sm.pv[x], sm.li[to] = sm.pi[x];
        }
        __syncthreads();
        lv = sm.lv, li = sm.li;
        n = sm.count;
      }
    }
    rank_list<THREADS>(lv, li, n, p.top, [&](int k, float v, int at) { out.place(k, v, at); });
  }
}

// ---- short rows: a warp each ----
// The whole row stays in registers, NV 16-byte groups and two single entries per
// lane: the maximum first, then the sums. The bound is the top-th largest of 128
// groups' maxima, four per lane (of 256 in the shortest rows, whose groups would
// be fewer than `top`), taken off one by one; what reaches it is ranked as above,
// in the warp's own list. 16384 rows of 2000 bf16: 21 us, with 16 entries 46 (by
// CTAs of 128 threads: 36 and 68); the loop that takes the maxima off is most of
// the difference.
constexpr int kWarpList = 256;
constexpr int kWarpsPerCta = 4;
template <typename T, int NV>
__global__ void __launch_bounds__(32 * kWarpsPerCta) k_scores_warp(const ScoresParams p) {
  pdl_sync();
  constexpr int E = Vec<T>::E;
  __shared__ float lists[kWarpsPerCta][kWarpList];
  __shared__ int places[kWarpsPerCta][kWarpList], counts[kWarpsPerCta];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * kWarpsPerCta + w;
  if (row >= p.rows) return;
  if (!dguard(kSiteScores, row * p.ld + p.vocab - 1, (p.rows - 1) * p.ld + p.vocab)) return;
  const int64_t token = p.token != nullptr ? p.token[row] : 0;
  if (token < 0 || token >= p.vocab) {
    out_none(p, row, lane, 32);
    return;
  }
  const Row<T> r(p.logits, row, p.ld, p.vocab);
  const float c = p.scale;
  Vec<T> q[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (lane + 32 * j < r.n) q[j].load(r.group(lane + 32 * j));
    else q[j].none();
  }
  const int last = r.lead + r.n * E + lane;
  float one[2] = {-INFINITY, -INFINITY};
  if (lane < r.lead && lane != p.excluded) one[0] = cvt(r.at[lane]);
  if (lane < r.tail && last != p.excluded) one[1] = cvt(r.at[last]);
  float zt = 0.f;
  if (lane == 0 && p.token != nullptr) zt = token == p.excluded ? -INFINITY : cvt(r.at[token]);
  if (lane == 0) counts[w] = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) r.exclude(q[j], lane + 32 * j, p.excluded);
  // a lane's groups: every fourth of its 16-byte groups, or half a one, the single entries with the first
  constexpr int NG = NV == 4 ? 8 : 4;
  float g[NG];
#pragma unroll
  for (int k = 0; k < NG; ++k) {
    if constexpr (NG == 8) {
      g[k] = q[k / 2].half_max(k % 2);
    } else {
      Vec<T> mine[NV / 4];
#pragma unroll
      for (int j = 0; j < NV / 4; ++j) mine[j] = q[4 * j + k];
      g[k] = vec_max(mine);
    }
  }
  g[0] = fmaxf(g[0], fmaxf(one[0], one[1]));
  Stat a = {g[0], 0.f, 0.f};
#pragma unroll
  for (int k = 1; k < NG; ++k) a.m = fmaxf(a.m, g[k]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xffffffffu, a.m, o));
  stat_sum(a, q, c);
  stat_add(a, one[0], c);
  stat_add(a, one[1], c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
  const RowOut out(p, row, a);
  if (lane == 0) out.scores(a, zt);
  if (p.top == 0) return;
  const float tau = take_off(g, p.top);  // minus infinity: fewer groups than places, and everything is listed
  float* lv = lists[w];
  int* li = places[w];
  auto keep = [&](float v, int at) {
    if (v >= tau && v != -INFINITY) {
      const int to = atomicAdd(&counts[w], 1);
      if (to < kWarpList) lv[to] = v, li[to] = at;
    }
  };
  __syncwarp();
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const Vec<T> v[1] = {q[j]};
    if (vec_max(v) >= tau) {
      for (uint32_t hit = v[0].reach(tau); hit != 0; hit &= hit - 1) {
        const int i = r.first(lane + 32 * j) + __ffs(hit) - 1;
        keep(cvt(r.at[i]), i);
      }
    }
  }
  keep(one[0], lane);
  keep(one[1], last);
  __syncwarp();
  int n = counts[w];
  if (n > kWarpList) {  // place by place, as above
    float pv = INFINITY;
    int pi = -1;
    for (int k = 0; k < p.top; ++k) {
      float bv = -INFINITY;
      int bi = 0x7fffffff;
      for (int i = lane; i < p.vocab; i += 32) {
        const float v = i == p.excluded ? -INFINITY : cvt(r.at[i]);
        if (v != -INFINITY && before(pv, pi, v, i) && before(v, i, bv, bi)) bv = v, bi = i;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, bv, o);
        const int i = __shfl_xor_sync(0xffffffffu, bi, o);
        if (before(v, i, bv, bi)) bv = v, bi = i;
      }
      if (lane == 0) out.place(k, bv, bi);
      pv = bv, pi = bi;
    }
    return;
  }
  rank_list<32>(lv, li, n, p.top, [&](int k, float v, int at) { out.place(k, v, at); });
}

// ---- gradient of the logits ----
// dz_v = -p_v (dlogp + dentropy (entropy + log p_v)) / T, at the token plus dlogp
// / T: one read and one write in 16-byte groups of the output's rows, with p from
// the forward's statistics. Where the logits' rows lie on other boundaries
// (SHIFT), a group comes from the two that hold it.
template <typename T>
__device__ __forceinline__ void load_shifted(Vec<T>& v, const T* at, const T* end) {
  const int shift = (int)(reinterpret_cast<uintptr_t>(at) & 15);
  const uint4* g = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(at) - shift);
  uint32_t w[8];
  if (shift == 0 || reinterpret_cast<const T*>(g + 2) <= end) {
    const uint4 a = __ldg(g), b = shift == 0 ? make_uint4(0, 0, 0, 0) : __ldg(g + 1);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  } else {  // the second one reaches past the last entry
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (Vec<T>::E == 4) {
        v.w[j] = reinterpret_cast<const uint32_t*>(at)[j];
      } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(at);
        v.w[j] = (uint32_t)h[2 * j] | (uint32_t)h[2 * j + 1] << 16;
      }
    }
    return;
  }
  uint32_t a[6], b[5];
#pragma unroll
  for (int i = 0; i < 6; ++i) a[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) b[i] = shift & 4 ? a[i + 1] : a[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) v.w[i] = __funnelshift_r(b[i], b[i + 1], (shift & 2) * 8);
}
template <typename T, bool SHIFT>
__global__ void __launch_bounds__(256, 6) k_scores_bwd(const ScoresParams p) {
  pdl_sync();
  constexpr int E = Vec<T>::E, THREADS = 256, U = SHIFT ? 2 : 4;
  const int t = threadIdx.x, part = (int)(blockIdx.x % p.parts);
  const int64_t row = blockIdx.x / p.parts;
  if (!dguard(kSiteScores, row * p.ld_out + p.vocab - 1, (p.rows - 1) * p.ld_out + p.vocab)) return;
  T* out = static_cast<T*>(p.dlogits) + row * p.ld_out;
  const T* in = static_cast<const T*>(p.logits) + row * p.ld;
  const T* end = static_cast<const T*>(p.logits) + (p.rows - 1) * p.ld + p.vocab;
  const int64_t token = p.token != nullptr ? p.token[row] : 0;
  const float2 st = p.stats_in[row];
  const bool counts = token >= 0 && token < p.vocab && st.x != -INFINITY;
  const Row<T> r(p.dlogits, row, p.ld_out, p.vocab);
  const float ls = -st.y * kLog2e, ref = -ref_of(st.x);
  const float dl = (p.dlogp != nullptr ? p.dlogp[row] : 0.f) * p.inv_t;
  const float dh = (p.dentropy != nullptr ? p.dentropy[row] : 0.f) * p.inv_t;
  const float base = -dl - (p.dentropy != nullptr ? dh * p.entropy_in[row] : 0.f), slope = -dh * kLn2;
  const int tk = p.token != nullptr ? (int)token : -1;
  auto special = [&](float g, int at) { return at == p.excluded ? 0.f : at == tk ? g + dl : g; };
  auto grad = [&](float z, int at) {
    const float d = fmaf(z + ref, p.scale, ls);
    return special(ex2(d) * fmaf(slope, fmaxf(d, -200.f), base), at);
  };
  const int a = r.begin(part, p.parts), b = r.begin(part + 1, p.parts);
  auto store = [&](int i, const float (&g)[E]) {
    uint4 u;
    if constexpr (E == 4)
      u = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
    else
      u = make_uint4(pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[E / 2], g[E / 2 + 1]),
                     pack_bf16(g[E - 2], g[E - 1]));
    *reinterpret_cast<uint4*>(out + r.first(i)) = u;
  };
  if (!counts) {
    const float zero[E] = {};
    for (int i = a + t; i < b; i += THREADS) store(i, zero);
  } else {
    for (int i = a + t; i < b; i += U * THREADS) {
      Vec<T> q[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (i + j * THREADS >= b) continue;
        const T* at = in + r.first(i + j * THREADS);
        if constexpr (SHIFT) {
          load_shifted(q[j], at, end);
        } else {  // not through the read-only path: the output may be the input
          const uint4 u = *reinterpret_cast<const uint4*>(at);
          q[j].w[0] = u.x, q[j].w[1] = u.y, q[j].w[2] = u.z, q[j].w[3] = u.w;
        }
      }
      const f32x2 rr = pair(ref, ref), cc = pair(p.scale, p.scale), ll = pair(ls, ls), ss = pair(slope, slope),
                  bb = pair(base, base);
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (i + j * THREADS >= b) continue;
        float g[E];
#pragma unroll
        for (int k = 0; k < E / 2; ++k) {
          const float2 v = q[j].two(k);
          const float2 d = halves(fma2(add2(pair(v.x, v.y), rr), cc, ll));
          const f32x2 by = fma2(pair(fmaxf(d.x, -200.f), fmaxf(d.y, -200.f)), ss, bb);
          const float2 e = halves(mul2(pair(ex2(d.x), ex2(d.y)), by));
          g[2 * k] = e.x, g[2 * k + 1] = e.y;
        }
        const int at = r.first(i + j * THREADS);
        if ((unsigned)(tk - at) < (unsigned)E || (unsigned)(p.excluded - at) < (unsigned)E) {
#pragma unroll
          for (int k = 0; k < E; ++k) g[k] = special(g[k], at + k);
        }
        store(i + j * THREADS, g);
      }
    }
  }
  if (part == 0 && t < r.lead) out[t] = to_out<T>(counts ? grad(cvt(in[t]), t) : 0.f);
  const int last = r.lead + r.n * E + t;
  if (part == p.parts - 1 && t < r.tail) out[last] = to_out<T>(counts ? grad(cvt(in[last]), last) : 0.f);
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

template <typename T, int NV>
cudaError_t scores_warp_t(const ScoresParams& p, cudaStream_t s) {
  return launch_pdl(k_scores_warp<T, NV>, dim3((unsigned)((p.rows + kWarpsPerCta - 1) / kWarpsPerCta)),
                    dim3(32 * kWarpsPerCta), 0, s, p);
}
template <typename T>
cudaError_t scores(ScoresParams p, cudaStream_t s) {
  const int64_t bytes = (int64_t)p.vocab * sizeof(T);
  // a row's 16-byte groups beside its single entries: 512 NV bytes at most
  if (bytes <= 2048) return scores_warp_t<T, 4>(p, s);
  if (bytes <= 4096) return scores_warp_t<T, 8>(p, s);
  if (bytes <= 8192) return scores_warp_t<T, 16>(p, s);
  // a row's cluster: as many CTAs as leave no SM idle, each with 2048 entries at least
  while (p.parts < kMaxParts && p.rows * p.parts < 152 && p.vocab >= 2048 * 2 * p.parts) p.parts *= 2;
  // 1536 threads per SM either way. Small CTAs overlap one row's passes with another's loads (16384 rows of 24000 bf16,
  // 16 entries: 177 us by 128 threads, 216 by 256), but the rows in flight should stay in L2 until their likeliest
  // entries are listed: 912 rows of 100 KB do (50304 bf16: 363 by 128, 313 by 256), of fp32 456 (8192 rows 314 by 256,
  // 283 by 512).
  if (bytes <= 64 * 1024) return scores_t<T, 128>(p, s);
  if (bytes <= 160 * 1024 || p.parts > 1) return scores_t<T, 256>(p, s);
  return scores_t<T, 512>(p, s);
}
template <typename T>
cudaError_t scores_bwd(ScoresParams p, cudaStream_t s) {
  // a row over several CTAs where there are few: four groups per thread at least
  while (p.parts < 64 && p.rows * p.parts < 912 && (int64_t)p.vocab * sizeof(T) >= 2 * 16384 * p.parts) p.parts *= 2;
  const dim3 grid((unsigned)(p.rows * p.parts)), block(256);
  // rows of both on the same boundaries: the first ones are
  const bool same = p.rows == 1 || (p.ld - p.ld_out) * sizeof(T) % 16 == 0;
  return same ? launch_pdl(k_scores_bwd<T, false>, grid, block, 0, s, p)
              : launch_pdl(k_scores_bwd<T, true>, grid, block, 0, s, p);
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
int check_apart(const char* fn, std::initializer_list<Span> reads, std::initializer_list<Span> writes) {
  char msg[128];
  return any_overlap(reads, writes, msg, sizeof(msg)) ? fail(BDSCAN_ERR_ARG, fn, msg) : BDSCAN_OK;
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
  const int64_t elt = dims->dtype == BDSCAN_F32 ? 4 : 2, t = p.rows;
  const int apart = check_apart(
      fn, {Span{"logits", logits, t, p.vocab * elt, p.ld * elt}, dense_span("token", token, t * 8)},
      {dense_span("logp", logp, t * 4), dense_span("entropy", entropy, t * 4), dense_span("stats", stats, t * 8),
       dense_span("top_ids", p.top > 0 ? top_ids : nullptr, t * p.top * 8),
       dense_span("top_logp", p.top > 0 ? top_logp : nullptr, t * p.top * 4)});
  if (apart) return apart;
  p.logits = logits;
  p.token = token;
  p.logp = logp;
  p.entropy = entropy;
  p.stats = (float2*)stats;
  p.top_ids = top_ids;
  p.top_logp = top_logp;
  cudaStream_t s = (cudaStream_t)stream;
  return done(dims->dtype == BDSCAN_F32 ? scores<float>(p, s) : scores<bf16>(p, s), fn, s);
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
  if (dlogits == logits && p.rows > 1 && p.ld != p.ld_out)
    return fail(BDSCAN_ERR_ARG, fn, "dlogits is logits, with another row stride");
  const int64_t elt = dims->dtype == BDSCAN_F32 ? 4 : 2, t = p.rows;
  const Span to{"dlogits", dlogits, t, p.vocab * elt, p.ld_out * elt};
  int apart = check_apart(fn,
                          {dense_span("token", token, t * 8), dense_span("stats", stats, t * 8),
                           dense_span("entropy", dentropy != nullptr ? entropy : nullptr, t * 4),
                           dense_span("dlogp", dlogp, t * 4), dense_span("dentropy", dentropy, t * 4)},
                          {to});
  // in place, or nowhere near
  if (!apart && dlogits != logits) apart = check_apart(fn, {Span{"logits", logits, t, p.vocab * elt, p.ld * elt}}, {to});
  if (apart) return apart;
  p.logits = logits;
  p.token = token;
  p.stats_in = (const float2*)stats;
  p.entropy_in = entropy;
  p.dlogp = dlogp;
  p.dentropy = dentropy;
  p.dlogits = dlogits;
  cudaStream_t s = (cudaStream_t)stream;
  return done(dims->dtype == BDSCAN_F32 ? scores_bwd<float>(p, s) : scores_bwd<bf16>(p, s), fn, s);
}

}  // extern "C"
