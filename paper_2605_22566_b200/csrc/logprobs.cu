// Log probabilities of given tokens, the entropy and the most likely tokens of rows of logits, in one pass over them.
//
// With m the largest logit seen so far, a thread keeps l = sum 2^d and s = sum d 2^d of d = (x - m) log2 e over its part of the
// row (both relative to m, and moved when m does); then lse = m + ln l and the entropy, sum p (lse - x), is
// ln 2 (log2 l - s / l): no second pass, and no difference of large numbers where one token has nearly everything.
// d is x log2 e - c in one fused step, two entries at a time; c, m log2 e rounded, is what all of a row's d are relative to, so
// its rounding cancels.  Where that rounding is no small number (a largest logit beyond 1e6) d is (x - m) log2 e.
// Masked entries are held to -1.2e38, so that d and its product with p = 0 are numbers.
//
// The k most likely: where n warps of a CTA each have m lanes whose largest logit so far reaches t, n m logits do, so with n m > k
// nothing below t can be among them.  The warps tell each other these levels (m lanes') through shared memory, with no barrier (a
// level that is read late is lower, which is right too), and a logit above the n-th largest of them goes to a list; the largest of a
// lane's round is compared, so that this costs little where nothing happens.  On 128 000 normal values some 20 to 200 get there.
// At the end the list has every logit above the last t.  If those are k, its k largest are the answer (each counts those above it); if
// not, the others are the first ones equal to t, and are looked for from the row's start.  More than the list holds (a row
// that rises from end to end): a second pass in steps that it cannot overrun, cut to k in between.
//
// A warp brings its own pieces of the row to shared memory, in rounds of 4 KB, one on the way while it works on another, and waits for no other warp
// (rounds of loads into registers leave room for half the warps).
//
// A row is one CTA's, or that of a cluster, whose first CTA joins the parts through shared memory.
//
// Measured: 2048 rows of 128 000 bf16 logits 100.5 us, 5.2 TB/s, 64 % of the issue slots (5 instructions an entry, exponentials at half the
// special-function unit's rate; ex2.approx, two units in the last place) and HBM at 80 % of a copy's; 256 rows 21 us, two rows on most multiprocessors and 44 % of the slots; one row 8.0 us, latency.
#include <algorithm>

#include "tc_device.cuh"
#include "gf_internal.h"
#include "rounds.h"

namespace gf {
namespace {

constexpr int kMinThreads = 128, kMaxThreads = 256, kMaxTop = 32, kMaxCluster = 8;
constexpr int kList = 1024;      // candidates that the list has room for
constexpr int kAhead = 8;        // vectors that a lane takes at a time
constexpr int kStages = 2;       // such rounds that a warp has on the way
constexpr int kRound = 32 * kAhead;
constexpr int kMargin = 4;       // so many more than k reach a level, so that logits equal to it seldom have to be looked for
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf(), kNan = __builtin_nanf("");
constexpr uint32_t kLowest = 0x007fffffu;  // order of minus infinity

typedef unsigned long long Key;  // 0: none

struct Stats { float m, l, s; };

struct Shared {
  Key list[kList];
  Key best[kMaxTop];             // the k largest, descending, after a cut
  Key bound[kMaxThreads / 32];
  uint32_t level[kMaxThreads / 32];  // order of the logit that enough lanes of the warp reach
  uint32_t common;                   // the highest of what the warps have made of all levels
  int before[kMaxThreads / 32 + 1];
  uint64_t full[kMaxThreads / 32][kStages];
  Stats stats[kMaxThreads / 32];
  Stats part;                    // the CTA's
  Key join[kMaxCluster * kMaxTop];
  int count, kept;
};

// Order of a value: larger values, larger numbers; both zeros alike; NaN below everything.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0u;
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  if (order == 0u) return kNan;
  return __uint_as_float((order & 0x80000000u) ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ Key key_of(float x, int64_t index) { return (Key)order_of(x) << 32 | (uint32_t)~(uint32_t)index; }

constexpr float kFar = 1e6f, kLag = 4.f;

// (x - m) log2 e, relative to the same c wherever |m| is not far.
__device__ __forceinline__ float diff(float x, float m) { return fabsf(m) < kFar ? fmaf(x, kLog2e, -(m * kLog2e)) : (x - m) * kLog2e; }

__device__ __forceinline__ void stats_move(Stats& a, float m) {  // to the reference m >= a.m
  if (a.m != kNegInf) {
    // (what a reference stands for is its c where it is not far, itself times log2 e where it is)
    const bool near_a = fabsf(a.m) < kFar, near_m = fabsf(m) < kFar;
    const float ca = __fmul_rn(a.m, kLog2e), cm = __fmul_rn(m, kLog2e);
    const float d = near_a ? (near_m ? ca - cm : fmaf(-m, kLog2e, ca)) : near_m ? fmaf(a.m, kLog2e, -cm) : (a.m - m) * kLog2e;
    const float e = fmaxf(d, -1000.f), f = fast_exp2(e);
    a.s = f * (a.s + a.l * e);
    a.l *= f;
  }
  a.m = m;
}
// The sum over a warp's lanes, in all of them: to the largest reference first.
__device__ __forceinline__ Stats stats_sum(Stats a) {
  float m = a.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (a.m < m) stats_move(a, m);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a.l += __shfl_xor_sync(0xffffffffu, a.l, d);
    a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
  }
  return a;
}
// The larger one, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// One more logit, at most a.m; any value.
__device__ __forceinline__ void stats_add(Stats& a, float x) {
  if (a.m == kNegInf) {
    if (x != x) a.l = x;
    return;
  }
  const float d = diff(x, a.m), p = fast_exp2(d);
  a.l += p;
  a.s = fmaf(p, fmaxf(d, -1000.f), a.s);
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void get(uint4 v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static constexpr uint32_t kNothing = 0xff800000u;  // minus infinity in every entry
  static __device__ __forceinline__ void word(uint32_t w, float (&x)[1]) { x[0] = __uint_as_float(w); }
  // the largest of a round; NaN only where there is nothing else
  static __device__ __forceinline__ float largest(const uint4 (&v)[kAhead]) {
    float x[4];
    get(v[0], x);
    float top = fmax3(fmaxf(x[0], x[1]), x[2], x[3]);
#pragma unroll
    for (int u = 1; u < kAhead; ++u) {
      get(v[u], x);
      top = fmax3(fmax3(top, x[0], x[1]), x[2], x[3]);
    }
    return top;
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ uint32_t held(uint32_t w) {
    return __float_as_uint(max_nan(__uint_as_float(w), -1.2e38f));
  }
  static __device__ __forceinline__ uint4 held(uint4 v) { return make_uint4(held(v.x), held(v.y), held(v.z), held(v.w)); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void get(uint4 v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void word(uint32_t w, float (&x)[2]) {
    x[0] = __uint_as_float(w << 16);
    x[1] = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
  static constexpr uint32_t kNothing = 0xff80ff80u;
  static __device__ __forceinline__ float largest(const uint4 (&v)[kAhead]) {
    __nv_bfloat162 t = pair(v[0].x);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (u > 0) t = __hmax2(t, pair(v[u].x));
      t = __hmax2(t, pair(v[u].y));
      t = __hmax2(t, pair(v[u].z));
      t = __hmax2(t, pair(v[u].w));
    }
    return fmaxf(__low2float(t), __high2float(t));
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ uint32_t held(uint32_t w) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0xfeb4feb4u));  // -1.2e38
    return r;
  }
  static __device__ __forceinline__ uint4 held(uint4 v) { return make_uint4(held(v.x), held(v.y), held(v.z), held(v.w)); }
};

// The k largest of the list's first n keys to its front, in descending order.  All threads; n is theirs alike.
__device__ void rank(Shared& sm, int n, int k, int32_t* status) {
  if (!GF_CHECK(n >= 0 && n <= kList && k <= kMaxTop, status, 702)) n = 0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const Key x = sm.list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += sm.list[j] > x;
    if (above < k) sm.best[above] = x;
  }
  __syncthreads();
  const int m = min(n, k);
  for (int i = threadIdx.x; i < m; i += blockDim.x) sm.list[i] = sm.best[i];
  if (threadIdx.x == 0) sm.count = m;
  __syncthreads();
}

// Keeps of the list the keys whose value's order is above `order`, then ranks them.
__device__ void cut_above(Shared& sm, int k, uint32_t order, int32_t* status) {
  constexpr int kOwn = kList / kMinThreads;
  const int n = sm.count;
  if (threadIdx.x == 0) sm.kept = 0;
  Key own[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    own[j] = i < n ? sm.list[i] : 0;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kOwn; ++j)
    if ((uint32_t)(own[j] >> 32) > order) {
      const int at = atomicAdd(&sm.kept, 1);
      if (GF_CHECK(at < kList, status, 703)) sm.list[at] = own[j];
    }
  __syncthreads();
  rank(sm, sm.kept, k, status);
}

// Publishes the largest order that `enough` lanes of the warp reach with their largest logit so far (it never falls).
__device__ __forceinline__ void publish(Shared& sm, float seen, int enough) {
  const int lane = threadIdx.x & 31;
  const uint32_t b = __float_as_uint(seen);  // (a number, so the plain form of order_of)
  uint32_t mine = b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
  for (int j = 1; j < enough; ++j) {
    const uint32_t holders = __ballot_sync(0xffffffffu, mine == __reduce_max_sync(0xffffffffu, mine));
    if (lane == __ffs(holders) - 1) mine = 0;
  }
  const uint32_t level = __reduce_max_sync(0xffffffffu, mine);
  if (lane == 0 && level > kLowest) *(volatile uint32_t*)&sm.level[threadIdx.x >> 5] = level;
}
// The `nth` largest of all warps' levels, as a value: nth * enough lanes reach it.
__device__ __forceinline__ float common_level(Shared& sm, int nth, int warps) {
  const int lane = threadIdx.x & 31;
  uint32_t mine = lane < warps ? *(volatile uint32_t*)&sm.level[lane] : 0u, level;
  if (2 * nth <= warps) {
    for (int j = 1; j < nth; ++j) {
      const uint32_t holders = __ballot_sync(0xffffffffu, mine == __reduce_max_sync(0xffffffffu, mine));
      if (lane == __ffs(holders) - 1) mine = 0u;
    }
    level = __reduce_max_sync(0xffffffffu, mine);
  } else {
    if (lane >= warps) mine = 0xffffffffu;
    for (int j = nth; j < warps; ++j) {
      const uint32_t holders = __ballot_sync(0xffffffffu, mine == __reduce_min_sync(0xffffffffu, mine));
      if (lane == __ffs(holders) - 1) mine = 0xffffffffu;
    }
    level = __reduce_min_sync(0xffffffffu, mine);
  }
  return value_of(level);
}

// Cuts the list to its k largest keys, in descending order, and raises the threshold to the k-th.  All threads.
__device__ void cut(Shared& sm, int k, Key& least, int32_t* status) {
  const int tid = threadIdx.x, lane = tid & 31, warps = blockDim.x >> 5;
  int n = min(sm.count, kList);
  __syncthreads();
  if (n > kMaxThreads) {
    // A bound from below first: where every warp has `each` keys that reach it, k do.
    Key mine = 0;
    for (int i = tid; i < n; i += blockDim.x) mine = max(mine, sm.list[i]);
    const int each = (k + warps - 1) / warps;
    Key level = 0;
    for (int j = 0; j < each; ++j) {
      Key top = mine;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
      if (mine == top) mine = 0;
      level = top;
    }
    if (lane == 0) sm.bound[tid >> 5] = level;
    if (tid == 0) sm.kept = 0;
    __syncthreads();
    Key bound = sm.bound[0];
    for (int w = 1; w < warps; ++w) bound = min(bound, sm.bound[w]);
    // (read by all before any place is written)
    constexpr int kOwn = kList / kMinThreads;
    Key own[kOwn];
    int have = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = tid + j * blockDim.x;
      own[j] = i < n ? sm.list[i] : 0;
      have += own[j] >= bound && own[j] != 0;
    }
    __syncthreads();
    if (have) {
      int at = atomicAdd(&sm.kept, have);
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (own[j] >= bound && own[j] != 0 && GF_CHECK(at < kList, status, 704)) sm.list[at++] = own[j];
    }
    __syncthreads();
    n = sm.kept;
  }
  rank(sm, n, k, status);
  if (n >= k) least = sm.best[k - 1];
  __syncthreads();
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ Key peer_key(const Key* p, uint32_t rank) {
  Key x;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(x) : "r"(peer_addr(p, rank)) : "memory");
  return x;
}
__device__ __forceinline__ float peer_float(const float* p, uint32_t rank) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(peer_addr(p, rank)) : "memory");
  return x;
}

// The k largest of a CTA's part from what was listed, to best; how many there are.  All threads.
template <typename T, typename P>
__device__ int finish(Shared& sm, int k, float least, const P& p, int loose, int my_loose, int vocab, int warps, int32_t* status) {
  constexpr int kN = Vec<T>::n;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, threads = blockDim.x;
  const int n = sm.count;
  if (n <= threads) {
    const Key mine = tid < n ? sm.list[tid] : 0;
    if (__syncthreads_count((uint32_t)(mine >> 32) > order_of(least)) >= k) {
      int above = 0;
      if (mine != 0) {
#pragma unroll 4
        for (int j = 0; j < n; ++j) above += sm.list[j] > mine;
        if (above < k) sm.best[above] = mine;
      }
      __syncthreads();
      return k;
    }
  }
  const T* x = p.x;
  const int head = p.head, tail = p.tail, v0 = p.v0, v1 = p.v1;
  if (n > kList) {
    Key bound = 0;
    cut(sm, k, bound, status);
    // (what the first pass listed is met again: from an empty list, against a key that k of them reach)
    if (tid == 0) sm.count = 0;
    __syncthreads();
    auto again = [&](bool mine, float v, int64_t index) {
      if (sm.count > kList - threads) cut(sm, k, bound, status);
      __syncthreads();
      const Key key = mine ? key_of(v, index) : 0;
      if (mine && key >= bound) {
        const int at = atomicAdd(&sm.count, 1);
        if (GF_CHECK(at < kList && index >= 0 && index < vocab, status, 705)) sm.list[at] = key;
      }
      __syncthreads();
    };
    again(tid < loose, tid < loose ? Vec<T>::one(x + my_loose) : 0.f, my_loose);
#pragma unroll 1
    for (int base = v0; base < v1; base += threads)
#pragma unroll 1
      for (int i = 0; i < kN; ++i) {
        const int64_t at = head + (int64_t)(base + tid) * kN + i;
        again(base + tid < v1, base + tid < v1 ? Vec<T>::one(x + at) : 0.f, at);
      }
    cut(sm, k, bound, status);
    return sm.count;
  }
  cut_above(sm, k, order_of(least), status);
  // the others: the first ones equal to `least`, and behind them, where nothing is left but NaN, the first of those
  for (int nan = 0; nan < 2 && sm.count < k; ++nan) {
    auto same = [&](float v) { return nan ? v != v : v == least; };
    // in the order of the row: the entries before the vectors, theirs, those behind
    auto take = [&](uint32_t found, int64_t first) {  // `found`: which of the thread's entries, from index `first` on
      const int here = __popc(found);
      int upto = here;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      const int have = sm.count;
      if (lane == 31) sm.before[wid] = upto;
      __syncthreads();
      int at = have + upto - here, all = have;
      for (int w = 0; w < warps; ++w) {
        if (w < wid) at += sm.before[w];
        all += sm.before[w];
      }
      for (; found && at < k; found &= found - 1, ++at) sm.list[at] = key_of(nan ? kNan : least, first + (__ffs(found) - 1));
      __syncthreads();
      if (tid == 0) sm.count = min(all, k);
      __syncthreads();
    };
    if (loose) take(tid < head && same(Vec<T>::one(x + tid)) ? 1u : 0u, tid);
    for (int base = v0; base < v1 && sm.count < k; base += threads) {
      uint32_t found = 0;
      if (base + tid < v1) {
        float e[kN];
        Vec<T>::get(__ldg(p.xv + base + tid), e);
#pragma unroll
        for (int i = 0; i < kN; ++i) found |= (same(e[i]) ? 1u : 0u) << i;
      }
      take(found, head + (int64_t)(base + tid) * kN);
    }
    if (loose && sm.count < k) take(tid < vocab - tail && same(Vec<T>::one(x + tail + tid)) ? 1u : 0u, tail + tid);
  }
  const int have = sm.count;
  for (int i = tid; i < have; i += threads) sm.best[i] = sm.list[i];
  __syncthreads();
  return have;
}

// Where the part of a row that a CTA has lies: 16-byte vectors from the row's first aligned entry on, v0 .. v1 of them the CTA's, a
// warp's first round from `first` on, `len` long, the next `stride` further.  The entries before and behind the vectors go one by one.
template <typename T>
struct Place {
  const T* x;
  const uint4* xv;
  int head, tail, v0, v1, first, len, stride;
  __device__ __forceinline__ Place(const T* row, int vocab, int part, int parts, int warp, int warps) : x(row) {
    head = min(vocab, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
    const int vecs = (vocab - head) / Vec<T>::n;
    tail = head + vecs * Vec<T>::n;
    const int each = (vecs + parts - 1) / parts;
    v0 = min(vecs, part * each);
    v1 = min(vecs, v0 + each);
    len = v1 - v0 >= kRound * warps ? kRound : (v1 - v0 + warps - 1) / warps;  // (short parts: every warp has some)
    first = v0 + warp * len;
    stride = warps * len;
    xv = reinterpret_cast<const uint4*>(x + head);
  }
};

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 3) k_token_logprobs(const T* __restrict__ logits, int64_t row_stride, int vocab, int parts,
                                                                const int32_t* __restrict__ tokens, int k, float* __restrict__ logprob,
                                                                float* __restrict__ entropy, float* __restrict__ lse_out,
                                                                int32_t* __restrict__ top_ids, float* __restrict__ top_logprobs, int32_t* status) {
  constexpr int kN = Vec<T>::n, kPer = kN / 4;  // entries of a vector, of a word
  static_assert(kAhead * 4 == 32, "a lane's round is 32 words");
  __shared__ Shared sm;
  extern __shared__ __align__(128) uint4 ring[];  // [warps][kStages][kRound]
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int part = parts > 1 ? (int)cluster_rank() : 0;
  const int64_t row = blockIdx.x / parts;
  const Place<T> p(logits + row * row_stride, vocab, part, parts, wid, warps);
  const T* __restrict__ x = p.x;
  const int head = p.head, tail = p.tail, v0 = p.v0, v1 = p.v1;
  // (three quarters of the warps: the least of all levels lies lower than that which all but two reach with more lanes)
  const int want = k + kMargin, most_warps = warps - warps / 4, enough = (want + most_warps - 1) / most_warps, nth = (want + enough - 1) / enough;
  // Lane 0 brings the warp's rounds.
  uint4* my_ring = ring + wid * kStages * kRound;
  int bring_at = p.first;  // the next round's first vector
  Rounds rounds;           // (a lane's own waits; lane 0 starts the copies)
  auto bring = [&] {
    if (bring_at >= v1) return;
    const uint32_t bytes = (uint32_t)min(p.len, v1 - bring_at) * 16u;
    if (!GF_CHECK(bring_at >= 0 && bytes <= kRound * 16u && head + (int64_t)bring_at * kN + bytes / sizeof(T) <= vocab, status, 701)) return;
    uint64_t* full = &sm.full[wid][rounds.started % kStages];
    mbar_arrive_expect_tx(full, bytes);
    bulk_g2s(my_ring + (rounds.started % kStages) * kRound, p.xv + bring_at, bytes, full);
    rounds.start();
    bring_at += p.stride;
  };
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&sm.full[wid][i], 1);
    mbar_fence_init();
    for (int i = 0; i < kStages; ++i) bring();
  }
  __syncwarp();

  Stats st{kNegInf, 0.f, 0.f};
  float least = kNegInf;  // more than k logits of the CTA's part reach it, or minus infinity
  auto push = [&](float v, int64_t index) {
    const int at = atomicAdd(&sm.count, 1);
    if (at < kList) sm.list[at] = key_of(v, index);
  };
  if (lane == 0) sm.level[wid] = kLowest;
  if (tid == 0) {
    sm.count = 0;
    sm.common = kLowest;
  }
  // asked for here, used at the row's end
  int token = -1;
  float given = 0.f;
  if (tid == 0 && part == 0 && tokens != nullptr) {
    token = tokens[row];
    if (token >= 0 && token < vocab) given = Vec<T>::one(x + token);
  }
  const int loose = part == 0 ? head + (vocab - tail) : 0;  // the entries that no vector holds: the first CTA's
  const int my_loose = tid < head ? tid : tail + (tid - head);
  float loose_value = kNegInf;
  if (tid < loose) {
    loose_value = Vec<T>::one(x + my_loose);
    if (loose_value > st.m) st.m = loose_value;
    stats_add(st, loose_value);
  }
  uint64_t l2 = 0ull, s2 = 0ull;  // l and s of the vectors, two halves
  auto fold = [&] {
    float lo, hi;
    f2_unpack(l2, lo, hi);
    st.l += lo + hi;
    f2_unpack(s2, lo, hi);
    st.s += lo + hi;
    l2 = s2 = 0ull;
  };
  float seen = st.m;  // the thread's largest logit; st.m, what its sums are relative to, follows when it is left far behind
  int round = 0;
  for (int base = v0; base < v1; base += p.stride, ++round) {
    const int begin = base + (p.first - v0), end = min(v1, begin + p.len);
    const uint4* piece = my_ring + (rounds.landed % kStages) * kRound;
    if (begin < v1) rounds.waited(rounds.ok && mbar_wait(&sm.full[wid][rounds.landed % kStages], (rounds.landed / kStages) & 1u, status));
    __syncwarp();
    uint4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u] = piece[u * 32 + lane];
    if (begin + kRound > end) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (begin + u * 32 + lane >= end) raw[u] = make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
    }
    const float most = Vec<T>::largest(raw);
    seen = fmaxf(seen, most);
    if (seen > st.m + kLag || st.m == kNegInf) {  // (a lag of 4 leaves a sum's terms below 2^6 and costs 2^-24 of it in the entropy)
      fold();
      if (seen > st.m) stats_move(st, seen);
    }
    if (k > 0) {
      if (round == 0 || round == 2 || (round & 7) == 5) {  // (a level rises less and less)
        publish(sm, seen, enough);
        if (round == 0) __syncthreads();  // (nothing is listed before all warps have one)
        const float level = common_level(sm, nth, warps);
        if (lane == 0) atomicMax(&sm.common, order_of(level));
        least = level;
      } else {
        least = value_of(*(volatile uint32_t*)&sm.common);
      }
      if (round == 0 && loose_value > least) push(loose_value, my_loose);
    }
    bool near = __all_sync(0xffffffffu, fabsf(st.m) < kFar || st.m == kNegInf);
    if (!near) {  // (lanes that have seen nothing but a mask's low values: the largest of the warp will do for them)
      float m = seen;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      near = fabsf(m) < kFar;
      if (near && st.m < m) {
        fold();
        stats_move(st, m);
      }
    }
    if (near) {
      const float c = st.m == kNegInf ? 0.f : -(st.m * kLog2e);  // (no logit with a probability yet: any reference will do)
      const uint64_t cc = f2_pack(c, c), ee = f2_pack(kLog2e, kLog2e);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float e[kN];
        Vec<T>::get(Vec<T>::held(raw[u]), e);
#pragma unroll
        for (int i = 0; i < kN; i += 2) {
          const uint64_t d2 = f2_fma(f2_pack(e[i], e[i + 1]), ee, cc);
          float d0, d1;
          f2_unpack(d2, d0, d1);
          const uint64_t p2 = f2_pack(fast_exp2(d0), fast_exp2(d1));
          l2 = f2_add(l2, p2);
          s2 = f2_fma(p2, d2, s2);
        }
      }
    } else {
      const bool far = fabsf(st.m) >= kFar && st.m != kNegInf;
      const float m = far ? -st.m : 0.f, c = far || st.m == kNegInf ? 0.f : -(st.m * kLog2e);
      const uint64_t mm = f2_pack(m, m), cc = f2_pack(c, c), ee = f2_pack(kLog2e, kLog2e);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float e[kN];
        Vec<T>::get(raw[u], e);
#pragma unroll
        for (int i = 0; i < kN; i += 2) {
          float d0, d1;
          f2_unpack(f2_fma(f2_add(f2_pack(e[i], e[i + 1]), mm), ee, cc), d0, d1);
          d0 = max_nan(d0, -1000.f);
          d1 = max_nan(d1, -1000.f);
          const uint64_t p2 = f2_pack(fast_exp2(d0), fast_exp2(d1));
          l2 = f2_add(l2, p2);
          s2 = f2_fma(p2, f2_pack(d0, d1), s2);
        }
      }
    }
    if (k > 0) {
      // a lane that has a logit above the least: the warp looks at its entries, 32 words of them
      for (uint32_t who = __ballot_sync(0xffffffffu, most > least); who; who &= who - 1) {
        const int at = (lane >> 2) * 32 + __ffs(who) - 1;
        float e[kPer];
        Vec<T>::word(reinterpret_cast<const uint32_t*>(piece + at)[lane & 3], e);
        if (begin + at < end) {
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (e[i] > least) push(e[i], head + (int64_t)(begin + at) * kN + (lane & 3) * kPer + i);
        }
      }
    }
    __syncwarp();
    if (lane == 0 && rounds.ok && begin < v1) bring();
  }
  fold();
  st = stats_sum(st);
  if (lane == 0) sm.stats[wid] = st;
  __syncthreads();
  int have = 0;  // the largest of the CTA's part: best[0 .. have)
  if (k > 0) {
    if (v0 >= v1) {  // a row that is no longer than its loose entries
      if (tid < loose && loose_value > kNegInf) push(loose_value, my_loose);
      __syncthreads();
    }
    least = value_of(sm.common);
    have = finish<T>(sm, k, least, p, loose, my_loose, vocab, warps, status);
  }

  if (wid == 0) {
    st = stats_sum(lane < warps ? sm.stats[lane] : Stats{kNegInf, 0.f, 0.f});
  }
  if (parts > 1) {
    if (tid == 0) sm.part = st;
    for (int i = have + tid; i < k; i += threads) sm.best[i] = 0;
    __syncthreads();
    cluster_sync();
    if (part == 0) {
      if (wid == 0) {
        st = Stats{kNegInf, 0.f, 0.f};
        if (lane < parts) {
          st.m = peer_float(&sm.part.m, lane);
          st.l = peer_float(&sm.part.l, lane);
          st.s = peer_float(&sm.part.s, lane);
        }
        st = stats_sum(st);
      }
      if (k > 0) {
        Key mine = 0;
        if (tid < parts * k) sm.join[tid] = mine = peer_key(&sm.best[tid % k], tid / k);
        __syncthreads();
        int above = 0;
        if (mine != 0)
          for (int j = 0; j < parts * k; ++j) above += sm.join[j] > mine;
        __syncthreads();
        if (mine != 0 && above < k) sm.list[above] = mine;  // (not to best, which the others may still read)
      }
    }
    __syncthreads();
    cluster_sync();  // nobody leaves while its shared memory is read
  }
  if (wid == 0 && part == 0) {
    // l is NaN where a logit is; nothing but minus infinity leaves l = 0
    if (st.m == -kNegInf) st.l = kNan;
    // (log probabilities relative to m: lse itself may be too large to hold ln l)
    const float log_sum = logf(st.l), lse = st.l == 0.f ? kNegInf : st.m + log_sum;
    auto of = [&](float v) { return lse == kNegInf ? lse : (fabsf(v) < kFar ? diff(v, st.m) * kLn2 : v - st.m) - log_sum; };
    if (lane == 0) {
      if (logprob != nullptr) logprob[row] = token == -1 ? 0.f : token < 0 || token >= vocab ? kNan : of(given);
      if (entropy != nullptr) entropy[row] = st.l == 0.f ? 0.f : log_sum - kLn2 * (st.s / st.l);
      if (lse_out != nullptr) lse_out[row] = lse;
    }
    if (lane < k) {
      const Key key = (parts > 1 ? sm.list : sm.best)[lane];
      if (top_ids != nullptr && GF_CHECK((int32_t)~(uint32_t)key >= 0 && (int32_t)~(uint32_t)key < vocab, status, 706)) top_ids[row * k + lane] = (int32_t)~(uint32_t)key;
      if (top_logprobs != nullptr) top_logprobs[row * k + lane] = of(value_of((uint32_t)(key >> 32)));
    }
  }
  if (lane == 0)  // where it gave up, its copies on the way land before the memory is another's
    for (uint32_t i = rounds.landed; i < rounds.started; ++i) mbar_drain(&sm.full[wid][i % kStages], (i / kStages) & 1u, status);
}

}  // namespace

int launch_token_logprobs(const void* logits, int fp32, int64_t stride, int rows, int vocab, const int32_t* tokens, int top, float* logprob,
                          float* entropy, float* lse, int32_t* top_ids, float* top_logprobs, int num_sms, int32_t* status, cudaStream_t st) {
  // CTAs per row: as many as two per multiprocessor, with parts of 4096 entries and more, or three, which are all at work at once, with
  // parts long enough for their joins (128 000 entries: 100 rows 15.6 us with two, 13.6 with three; 32 000: 9.0 and 11.0; 256 rows
  // with two parts each, not all at once: 27.1 in place of 21.3).
  int parts = 1;
  while (parts < kMaxCluster && vocab / (parts * 2) >= 4096 &&
         (int64_t)rows * parts * 2 <= (vocab / (parts * 2) >= 32000 ? 3 : 2) * num_sms) parts *= 2;
  const int per_vec = fp32 ? 4 : 8, vecs = vocab / parts / per_vec;
  const int threads = vecs < 256 ? kMinThreads : kMaxThreads;
  const size_t smem = (size_t)(threads / 32) * kStages * kRound * 16;
  static bool done[2][kMaxDevices];
  if (!(fp32 ? ensure_dynamic_smem(k_token_logprobs<float>, kMaxThreads / 32 * kStages * kRound * 16, done[0])
             : ensure_dynamic_smem(k_token_logprobs<__nv_bfloat16>, kMaxThreads / 32 * kStages * kRound * 16, done[1])))
    return -1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * parts));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  const cudaError_t e = fp32 ? cudaLaunchKernelEx(&cfg, k_token_logprobs<float>, (const float*)logits, stride, vocab, parts, tokens, top, logprob,
                                                  entropy, lse, top_ids, top_logprobs, status)
                             : cudaLaunchKernelEx(&cfg, k_token_logprobs<__nv_bfloat16>, (const __nv_bfloat16*)logits, stride, vocab, parts, tokens,
                                                  top, logprob, entropy, lse, top_ids, top_logprobs, status);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace gf
