// Log probabilities of given tokens, the entropy and the most likely tokens of rows of logits, in one pass over them.
//
// With m the largest logit seen so far, a thread keeps l = sum 2^d and s = sum d 2^d of d = (x - m) log2 e over its part of the
// row (both relative to m, and moved when m does); then lse = m + ln l and the entropy, sum p (lse - x), is
// ln 2 (log2 l - s / l): no second pass, and no difference of large numbers where one token has nearly everything.
//
// The k most likely: every logit gets a 64-bit key, its value's order above the complement of its index, so that keys differ and
// equal values rank by the lower index.  A threshold that at least k keys of the CTA's part reach is known after each thread's first
// vector; from then on a vector's maximum is compared with it, and only what reaches it goes to a list in shared memory, which is
// cut to its k largest (each counts the keys above it) when it has grown, which raises the threshold.  On 128 000 normal
// values some 100 to 200 get there.
//
// A row is one CTA's, or that of a cluster, whose first CTA joins the parts through shared memory.
#include "gf_device.cuh"
#include "gf_internal.h"

namespace gf {
namespace {

constexpr int kMinThreads = 128, kMaxThreads = 512, kMaxTop = 32, kMaxCluster = 8;
constexpr int kList = 2048;      // candidates that the list has room for
constexpr int kCutAt = 256;      // it is cut when it holds more than this
constexpr int kAhead = 4;        // vectors that a thread asks for at a time
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();

typedef unsigned long long Key;  // 0: none

struct Stats { float m, l, s; };

struct Shared {
  Key list[kList];
  Key best[kMaxTop];             // the k largest, descending, after a cut
  Key bound[kMaxThreads / 32];
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
  if (order == 0u) return __int_as_float(0x7fffffff);
  return __uint_as_float((order & 0x80000000u) ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ Key key_of(float x, int64_t index) { return (Key)order_of(x) << 32 | (uint32_t)~(uint32_t)index; }

__device__ __forceinline__ void stats_move(Stats& a, float m) {  // to the reference m >= a.m
  if (a.m != kNegInf) {
    const float d = fmaxf((a.m - m) * kLog2e, -1000.f), f = fast_exp2(d);
    a.s = f * (a.s + a.l * d);
    a.l *= f;
  }
  a.m = m;
}
__device__ __forceinline__ Stats stats_join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  if (a.m < m) stats_move(a, m);
  if (b.m < m) stats_move(b, m);
  a.l += b.l;
  a.s += b.s;
  return a;
}
// One more logit, at most a.m.  (A difference below -1000 has no probability left; the product with it has to stay a number.)
__device__ __forceinline__ void stats_add(Stats& a, float x) {
  const float d = fmaxf((x - a.m) * kLog2e, -1000.f), p = fast_exp2(d);
  a.l += x == x ? p : x;
  a.s = fmaf(p, d, a.s);
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void get(uint4 v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
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
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};

// Cuts the list to its k largest keys, in descending order, and raises the threshold to the k-th.  All threads.
__device__ void cut(Shared& sm, int k, Key& least) {
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
        if (own[j] >= bound && own[j] != 0) sm.list[at++] = own[j];
    }
    __syncthreads();
    n = sm.kept;
  }
  for (int i = tid; i < n; i += blockDim.x) {
    const Key x = sm.list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += sm.list[j] > x;
    if (above < k) sm.best[above] = x;
  }
  __syncthreads();
  const int m = min(n, k);
  for (int i = tid; i < m; i += blockDim.x) sm.list[i] = sm.best[i];
  if (tid == 0) sm.count = m;
  if (m == k) least = sm.best[k - 1];
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

template <typename T>
__global__ void __launch_bounds__(kMaxThreads) k_token_logprobs(const T* __restrict__ logits, int64_t stride, int vocab, int parts,
                                                                const int32_t* __restrict__ tokens, int k, float* __restrict__ logprob,
                                                                float* __restrict__ entropy, float* __restrict__ lse_out,
                                                                int32_t* __restrict__ top_ids, float* __restrict__ top_logprobs) {
  constexpr int kN = Vec<T>::n;
  __shared__ Shared sm;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int64_t row = blockIdx.x / parts;
  const int part = parts > 1 ? (int)cluster_rank() : 0;
  const T* __restrict__ x = logits + row * stride;
  // 16-byte vectors from the row's first aligned entry on; the entries before and behind them go one by one
  const int head = min(vocab, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int vecs = (vocab - head) / kN, tail = head + vecs * kN;
  const int v0 = (int)((int64_t)vecs * part / parts), v1 = (int)((int64_t)vecs * (part + 1) / parts);
  const uint4* __restrict__ xv = reinterpret_cast<const uint4*>(x + head);
  if (tid == 0) sm.count = 0;
  __syncthreads();

  Stats st{kNegInf, 0.f, 0.f};
  Key least = 0;  // a key of the CTA's part that k of its keys reach, or 0
  float least_value = kNegInf;
  auto push = [&](Key key) {
    const int at = atomicAdd(&sm.count, 1);
    if (at < kList) sm.list[at] = key;
  };
  auto consider = [&](float v, int64_t index) {
    const Key key = key_of(v, index);
    if (key >= least) push(key);
  };
  auto add_stats = [&](const float (&e)[kN]) {
    float top = e[0];
#pragma unroll
    for (int i = 1; i < kN; ++i) top = fmaxf(top, e[i]);
    if (top > st.m) stats_move(st, top);
    if (st.m != kNegInf) {
#pragma unroll
      for (int i = 0; i < kN; ++i) stats_add(st, e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (e[i] != e[i]) st.l = e[i];
    }
    return top;
  };

  if (k > 0 && v1 - v0 >= threads) {
    // the first threshold, from the largest of every thread's first vector
    float e[kN];
    Vec<T>::get(xv[v0 + tid], e);
    Key mine = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) mine = max(mine, key_of(e[i], head + (int64_t)(v0 + tid) * kN + i));
    const int each = (k + warps - 1) / warps;
    Key level = 0;
    for (int j = 0; j < each; ++j) {
      Key top = mine;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
      if (mine == top) mine = 0;
      level = top;
    }
    if (lane == 0) sm.bound[wid] = level;
    __syncthreads();
    least = sm.bound[0];
    for (int w = 1; w < warps; ++w) least = min(least, sm.bound[w]);
    least_value = (uint32_t)(least >> 32) ? value_of((uint32_t)(least >> 32)) : kNegInf;
  }

  // the entries that no vector holds
  if (part == 0 && tid < head + (vocab - tail)) {
    const int i = tid < head ? tid : tail + (tid - head);
    const float v = Vec<T>::one(x + i);
    if (v > st.m) stats_move(st, v);
    if (st.m != kNegInf) stats_add(st, v);
    else if (v != v) st.l = v;
    if (k > 0) consider(v, i);
  }
  for (int base = v0; base < v1; base += kAhead * threads) {
    if (k > 0) {
      __syncthreads();
      const int before = sm.count;
      if (before > kCutAt) {
        cut(sm, k, least);
        least_value = (uint32_t)(least >> 32) ? value_of((uint32_t)(least >> 32)) : kNegInf;
      }
    }
    uint4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = base + u * threads + tid;
      raw[u] = v < v1 ? __ldg(xv + v) : make_uint4(0u, 0u, 0u, 0u);
    }
    const int start = k > 0 ? *(volatile int*)&sm.count : 0;
    if (k > 0) __syncthreads();
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = base + u * threads + tid;
      if (v < v1) {
        float e[kN];
        Vec<T>::get(raw[u], e);
        const float top = add_stats(e);
        if (k > 0 && !(top < least_value)) {
#pragma unroll
          for (int i = 0; i < kN; ++i) consider(e[i], head + (int64_t)v * kN + i);
        }
      }
    }
    if (k > 0) {
      __syncthreads();
      if (sm.count > kList) {
        // more reached the threshold than the list holds: once more from where this round began, one entry of each thread at a time
        __syncthreads();
        if (tid == 0) sm.count = start;
        __syncthreads();
#pragma unroll 1
        for (int u = 0; u < kAhead; ++u) {
          const int v = base + u * threads + tid;
#pragma unroll 1
          for (int i = 0; i < kN; ++i) {
            if (sm.count > kList - threads) {
              cut(sm, k, least);
              least_value = (uint32_t)(least >> 32) ? value_of((uint32_t)(least >> 32)) : kNegInf;
            }
            __syncthreads();
            if (v < v1) consider(Vec<T>::one(x + head + (int64_t)v * kN + i), head + (int64_t)v * kN + i);
            __syncthreads();
          }
        }
      }
    }
  }

  // the CTA's part
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    Stats o;
    o.m = __shfl_xor_sync(0xffffffffu, st.m, d);
    o.l = __shfl_xor_sync(0xffffffffu, st.l, d);
    o.s = __shfl_xor_sync(0xffffffffu, st.s, d);
    st = stats_join(st, o);
  }
  if (lane == 0) sm.stats[wid] = st;
  __syncthreads();
  if (k > 0) cut(sm, k, least);
  if (tid == 0) {
    st = sm.stats[0];
    for (int w = 1; w < warps; ++w) st = stats_join(st, sm.stats[w]);
    sm.part = st;
  }
  __syncthreads();
  if (parts > 1) {
    if (k > 0)
      for (int i = sm.count + tid; i < kMaxTop; i += threads) sm.best[i] = 0;
    __syncthreads();
    cluster_sync();
    if (part == 0) {
      if (tid < 32) {
        Stats a{kNegInf, 0.f, 0.f};
        for (int p = 0; p < parts; ++p) {
          Stats b;
          b.m = peer_float(&sm.part.m, p); b.l = peer_float(&sm.part.l, p); b.s = peer_float(&sm.part.s, p);
          a = stats_join(a, b);
        }
        st = a;
      }
      if (k > 0) {
        for (int i = tid; i < parts * k; i += threads) sm.join[i] = peer_key(&sm.best[i % k], i / k);
        __syncthreads();
        for (int i = tid; i < parts * k; i += threads) {
          const Key key = sm.join[i];
          int above = 0;
          for (int j = 0; j < parts * k; ++j) above += sm.join[j] > key;
          if (key != 0 && above < k) sm.list[above] = key;
        }
      }
    }
    __syncthreads();
    cluster_sync();  // nobody leaves while its shared memory is read
    if (part != 0) return;
  } else if (tid < 32) {
    st = sm.part;
  }
  if (tid >= 32) return;
  // l is NaN where a logit is; nothing but minus infinity leaves l = 0
  if (st.m == -kNegInf) st.l = __int_as_float(0x7fffffff);
  // (log probabilities relative to m: lse itself may be too large to hold ln l)
  const float log_sum = logf(st.l), lse = st.l == 0.f ? kNegInf : st.m + log_sum;
  auto of = [&](float v) { return lse == kNegInf ? lse : v - st.m - log_sum; };
  if (lane == 0) {
    const int token = tokens != nullptr ? tokens[row] : -1;
    if (logprob != nullptr) {
      float lp = 0.f;
      if (token != -1) {
        if (token < 0 || token >= vocab) lp = __int_as_float(0x7fffffff);
        else lp = of(Vec<T>::one(x + token));
      }
      logprob[row] = lp;
    }
    if (entropy != nullptr) entropy[row] = st.l == 0.f ? 0.f : log_sum - kLn2 * (st.s / st.l);
    if (lse_out != nullptr) lse_out[row] = lse;
  }
  for (int i = lane; i < k; i += 32) {
    const Key key = sm.list[i];
    if (top_ids != nullptr) top_ids[row * k + i] = (int32_t)~(uint32_t)key;
    if (top_logprobs != nullptr) top_logprobs[row * k + i] = of(value_of((uint32_t)(key >> 32)));
  }
}

}  // namespace

int launch_token_logprobs(const void* logits, int fp32, int64_t stride, int rows, int vocab, const int32_t* tokens, int top, float* logprob,
                          float* entropy, float* lse, int32_t* top_ids, float* top_logprobs, int num_sms, cudaStream_t st) {
  // CTAs per row: until two per multiprocessor have work, a part not below 4096 entries
  int parts = 1;
  while (parts < kMaxCluster && (int64_t)rows * parts * 2 <= 2 * num_sms && vocab / (parts * 2) >= 4096) parts *= 2;
  const int per_vec = fp32 ? 4 : 8, vecs = vocab / parts / per_vec;
  const int threads = vecs >= 1024 ? 512 : vecs >= 256 ? 256 : 128;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * parts));
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  const cudaError_t e = fp32 ? cudaLaunchKernelEx(&cfg, k_token_logprobs<float>, (const float*)logits, stride, vocab, parts, tokens, top, logprob,
                                                  entropy, lse, top_ids, top_logprobs)
                             : cudaLaunchKernelEx(&cfg, k_token_logprobs<__nv_bfloat16>, (const __nv_bfloat16*)logits, stride, vocab, parts, tokens,
                                                  top, logprob, entropy, lse, top_ids, top_logprobs);
  return e == cudaSuccess ? 1 : -1;
}

}  // namespace gf
