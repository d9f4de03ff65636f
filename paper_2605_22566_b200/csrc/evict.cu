// Eviction by accumulated attention weight: the kept tokens of one node's state become the state of another.
//
// Per (node, layer, KV head) the kept tokens are the first and last few (as many as the caller protects) and
// then those with the largest weight, ties to the lower index, m in all; they keep their order.  Two kernels:
//
//   k_select  one CTA per (entry, layer, head).  32-bit keys have the weights' order; the key of rank m is found from
//             its top bits down, then one ordered pass writes the kept indices and carries the weights to the
//             destination's slots.  The choice is a function of the weights alone: integer counts, and ranks from
//             scans.  Up to kHeldTokens tokens, what a CTA's registers hold, the keys stay there and two bits cost a
//             count over them (the search ends when nothing is left to decide); longer nodes are read five times,
//             from L2, by a radix select of eight bits a pass, still by one CTA.
//   k_gather  copies the kept rows, in the 4-bit layout by moving the codes of whole tokens (the values are
//             not touched).  Rows of the last tile past the end become zeros, as every writer of the pools
//             leaves them.
//
// Four nodes of 6000 to 8192 tokens, two layers of 8 heads of 128, half kept: chosen in 17 us (64 CTAs, bound by their
// chain of sixteen counts; a radix select with counts in shared memory 30), copied in 31 us (146 MB, 4.7 TB/s).  300
// tokens: 7.5 us in one launch.  One node, half kept, chosen in 15 us with 8192 tokens, 34 with one more, 119 with 32 768 and
// 600 with 131 072 (copied in 13, 13, 44 and 85): there a pass is 16 or 8 CTAs' walk over the weights.
//
// The destination is another node, so nothing is read after it was overwritten and both kernels spread over
// everything at once.
#include "kv4_device.cuh"

namespace gf {
namespace {

constexpr int kSelectThreads = 512;
constexpr int kHeldKeys = 16, kHeldTokens = kHeldKeys * kSelectThreads;  // keys a thread keeps
// Up to so many kept tokens per entry, one round of two tiles, the CTA that chose the rows copies them too, which saves
// a launch (120 of 300 tokens: 12.3 us instead of 13.3, 128 in 4 bits 14.3 instead of 17.4).  More rounds would leave the
// copy to a CTA per layer and head where a launch spreads it (255 of 300 tokens: 14.3 instead of 15.3 still).
constexpr int kOneLaunch = 2 * kTile;
constexpr int kGatherThreads = 256;  // 64 rows, 32 at a time, of eight 16-byte pieces

// Keys in the order of the weights; NaN counts as the least, -0 as +0.  Protected tokens get the largest
// key, which no weight has.
__device__ __forceinline__ uint32_t key_of(float w, int t, int n, int first, int last) {
  if (t < first || t >= n - last) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The key of rank `need` (from the top) among the keys the CTA holds, and how many of its equals are kept.
__device__ __forceinline__ void select_held(const uint32_t (&key)[kHeldKeys], int n, uint32_t& pick, uint32_t& need) {
  constexpr int kWarps = kSelectThreads / 32;
  static_assert(kHeldKeys * 32 < 1024 && kWarps <= 32, "a warp's three counts are packed, ten bits each");
  __shared__ uint32_t count_s[2][kWarps];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  uint32_t prefix = 0, above = 0, at_least = (uint32_t)n;  // keys above the candidates, and those with them
  // two bits at a time (keys past the end are 0 and never counted: no trial is 0)
  for (int shift = 30; shift >= 0 && at_least != need; shift -= 2) {
    const uint32_t one = prefix | (1u << shift), two = prefix | (2u << shift), three = prefix | (3u << shift);
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) {
      if (i * kSelectThreads >= n) break;
      c += (key[i] >= one ? 1u : 0u) + (key[i] >= two ? 1u << 10 : 0u) + (key[i] >= three ? 1u << 20 : 0u);
    }
    c = __reduce_add_sync(0xffffffffu, c);
    uint32_t* count = count_s[(shift >> 1) & 1];
    if (lane == 0) count[wid] = c;
    __syncthreads();
    c = lane < kWarps ? count[lane] : 0u;
    const uint32_t c1 = __reduce_add_sync(0xffffffffu, c & 1023u), c2 = __reduce_add_sync(0xffffffffu, (c >> 10) & 1023u),
                   c3 = __reduce_add_sync(0xffffffffu, c >> 20);
    // the digit of the key of rank `need`
    if (c3 >= need) {
      prefix = three;
      at_least = c3;
    } else if (c2 >= need) {
      prefix = two;
      at_least = c2;
      above = c3;
    } else if (c1 >= need) {
      prefix = one;
      at_least = c1;
      above = c2;
    } else {
      above = c1;
    }
  }
  // either every bit is known, or exactly the keys >= prefix are kept: then all of prefix's equals are
  pick = prefix;
  need = at_least == need ? (uint32_t)n : need - above;
}

// The same where they are too many, digit by digit.
template <typename KeyAt>
__device__ __forceinline__ void select_radix(KeyAt&& key_at, int n, uint32_t& pick, uint32_t& need) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t pick_s, need_s;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelectThreads) hist[i] = 0u;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    // (lanes with the same digit count together: weights share their high digits, and many are equal)
    for (int base = 0; base < n; base += kSelectThreads) {
      const int t = base + tid;
      const uint32_t key = t < n ? key_at(t) : 0u;
      const bool on = t < n && (key & mask) == prefix;
      if (!__any_sync(0xffffffffu, on)) continue;
      const uint32_t digit = on ? (key >> shift) & 255u : 256u, same = __match_any_sync(0xffffffffu, digit);
      if (on && (same & ((1u << lane) - 1u)) == 0u) atomicAdd(&hist[digit], (uint32_t)__popc(same));
    }
    __syncthreads();
    if (wid == 0) {  // counts from the top: lane l owns bins 255 - 8 l .. 248 - 8 l
      uint32_t c[8], local = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { c[i] = hist[255 - 8 * lane - i]; local += c[i]; }
      uint32_t incl = local;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      uint32_t above = incl - local;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above < need && need <= above + c[i]) { pick_s = 255u - 8u * lane - i; need_s = need - above; }
        above += c[i];
      }
    }
    __syncthreads();
    prefix |= pick_s << shift;
    need = need_s;
  }
  pick = prefix;
}

// What one (entry, layer, head) keeps: the indices to out, the weights from src to dst.  Executed by the whole CTA.
__device__ __forceinline__ void select_kept(const EvictEntry& e, const float* src, float* dst, int32_t* out) {
  constexpr int kWarps = kSelectThreads / 32;
  const int n = e.len, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  auto key_at = [&](int t) { return key_of(src[t], t, n, e.first, e.last); };
  uint32_t pick, need = (uint32_t)e.keep;  // of the tokens whose key is `pick`, the first `need` are kept
  const uint32_t below = (1u << lane) - 1u;
  // Writes what is kept of 512 tokens (this thread's key of token t); g and q: how many greater and equal ones the
  // warps before this one have.
  auto write = [&](uint32_t key, float w, int t, int g, int q) {
    const bool gt = t < n && key > pick, eq = t < n && key == pick;
    g += __popc(__ballot_sync(0xffffffffu, gt) & below);
    q += __popc(__ballot_sync(0xffffffffu, eq) & below);
    if (gt || (eq && q < (int)need)) {
      const int at = g + min(q, (int)need);
      out[at] = t;
      dst[at] = w;
    }
  };
  if (n <= kHeldTokens) {
    __shared__ uint32_t before_s[kHeldKeys * kWarps];  // by (512 tokens, warp): equal ones, and greater ones in the high half
    __shared__ uint32_t total_s[kWarps];
    uint32_t key[kHeldKeys];
    float w[kHeldKeys];
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) w[i] = i * kSelectThreads + tid < n ? src[i * kSelectThreads + tid] : 0.f;
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) key[i] = i * kSelectThreads + tid < n ? key_of(w[i], i * kSelectThreads + tid, n, e.first, e.last) : 0u;
    select_held(key, n, pick, need);
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) {
      const int t = i * kSelectThreads + tid;
      const uint32_t gt = __ballot_sync(0xffffffffu, t < n && key[i] > pick), eq = __ballot_sync(0xffffffffu, t < n && key[i] == pick);
      if (lane == 0) before_s[i * kWarps + wid] = (uint32_t)__popc(gt) << 16 | (uint32_t)__popc(eq);
    }
    __syncthreads();
    // exclusive scan (both halves stay below 2^16)
    static_assert(kHeldKeys * kWarps <= kSelectThreads && kHeldTokens < 65536, "a thread scans one count, of 16 bits each");
    const uint32_t own = tid < kHeldKeys * kWarps ? before_s[tid] : 0u;
    uint32_t incl = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) total_s[wid] = incl;
    __syncthreads();
    const uint32_t warps = __reduce_add_sync(0xffffffffu, lane < wid ? total_s[lane & (kWarps - 1)] : 0u);
    if (tid < kHeldKeys * kWarps) before_s[tid] = warps + incl - own;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) {
      if (i * kSelectThreads >= n) break;
      const uint32_t b = before_s[i * kWarps + wid];
      write(key[i], w[i], i * kSelectThreads + tid, (int)(b >> 16), (int)(b & 0xffffu));
    }
    return;
  }
  __shared__ int32_t wsum[2][kWarps];
  select_radix(key_at, n, pick, need);
  int greater = 0, equal = 0;  // before this chunk
  for (int base = 0; base < n; base += kSelectThreads) {
    const int t = base + tid;
    const uint32_t key = t < n ? key_at(t) : 0u;
    const uint32_t gt = __ballot_sync(0xffffffffu, t < n && key > pick), eq = __ballot_sync(0xffffffffu, t < n && key == pick);
    if (lane == 0) { wsum[0][wid] = __popc(gt); wsum[1][wid] = __popc(eq); }
    __syncthreads();
    int g = greater, q = equal;
    for (int i = 0; i < kWarps; ++i) {
      if (i < wid) { g += wsum[0][i]; q += wsum[1][i]; }
      greater += wsum[0][i];
      equal += wsum[1][i];
    }
    write(key, t < n ? src[t] : 0.f, t, g, q);
    __syncthreads();
  }
}

template <int D>
__device__ __forceinline__ void gather_tile16(const char* src_head, char* dst_tile, int src_tile0, int count, const int32_t* idx, int tid) {
  constexpr uint32_t kTileBytes = 2 * kTile * D * 2;
  constexpr int kBlocks = 2 * (D / 64);  // K's column blocks, then V's
  // eight neighbouring threads share a 128-byte line; a thread has two rows, every block of them: all its loads are
  // issued before its stores
  const uint32_t chunk = tid & 7;
  uint4 v[2][kBlocks];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = (tid >> 3) + 32 * h, t = row < count ? idx[row] : -1;
    const char* from = src_head + (uint64_t)(src_tile0 + (t < 0 ? 0 : t) / kTile) * kTileBytes + swz128(t & (kTile - 1), chunk);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
      v[h][i] = t < 0 ? make_uint4(0u, 0u, 0u, 0u) : *reinterpret_cast<const uint4*>(from + i * (kTile * 128));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
      *reinterpret_cast<uint4*>(dst_tile + i * (kTile * 128) + swz128((tid >> 3) + 32 * h, chunk)) = v[h][i];
}

template <int D>
__device__ __forceinline__ void gather_tile4(const char* src_head, char* dst_tile, int src_tile0, int count, const int32_t* idx, int tid) {
  constexpr int NG = D / kGroup4;
  constexpr uint32_t kTileBytes = kv4_tile_bytes(D), kPart = kv4_part_bytes(D), kCodes = kv4_code_bytes(D);
  const int lane = tid & 31, wid = tid >> 5, l4 = lane & 3, l8 = lane >> 2;
  // a warp per (part, block of 16 tokens, group): every lane builds its 16 bytes from its tokens' pieces
#pragma unroll
  for (int job = wid; job < 2 * 4 * NG; job += kGatherThreads / 32) {
    const int g = job % NG, b = job / NG % 4, which = job / NG / 4;
    const char* part = src_head + which * kPart;
    uint4 acc = make_uint4(0u, 0u, 0u, 0u);
    if (which == 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {  // K: tokens l8 + 8 j; a token's codes are nibbles j' and j' + 2, j' = bit 3 of its place
        const int row = b * 16 + l8 + 8 * j;
        if (row >= count) continue;
        const int t = idx[row], in = t & (kTile - 1);
        const uint4 w = reinterpret_cast<const uint4*>(part + (uint64_t)(src_tile0 + t / kTile) * kTileBytes)[((in >> 4) * NG + g) * 32 + (in & 7) * 4 + l4];
        const int from = 4 * ((in >> 3) & 1), to = 4 * j;
        acc.x |= ((w.x >> from) & 0x0f0f0f0fu) << to;
        acc.y |= ((w.y >> from) & 0x0f0f0f0fu) << to;
        acc.z |= ((w.z >> from) & 0x0f0f0f0fu) << to;
        acc.w |= ((w.w >> from) & 0x0f0f0f0fu) << to;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // V: tokens 2 l4 + (k & 1) + 8 (k / 2); a token's codes are one byte of every word
        const int row = b * 16 + 2 * l4 + (k & 1) + 8 * (k >> 1);
        if (row >= count) continue;
        const int t = idx[row], in = t & (kTile - 1);
        const uint4 w = reinterpret_cast<const uint4*>(part + (uint64_t)(src_tile0 + t / kTile) * kTileBytes)[((in >> 4) * NG + g) * 32 + l8 * 4 + ((in & 7) >> 1)];
        const int from = 16 * (in & 1) + 8 * ((in >> 3) & 1), to = 16 * (k & 1) + 8 * (k >> 1);
        acc.x |= ((w.x >> from) & 0xffu) << to;
        acc.y |= ((w.y >> from) & 0xffu) << to;
        acc.z |= ((w.z >> from) & 0xffu) << to;
        acc.w |= ((w.w >> from) & 0xffu) << to;
      }
    }
    reinterpret_cast<uint4*>(dst_tile + which * kPart)[(b * NG + g) * 32 + lane] = acc;
  }
  for (int i = tid; i < 2 * kTile * NG; i += kGatherThreads) {
    const int g = i % NG, row = i / NG % kTile, which = i / NG / kTile;
    uint32_t sl = 0u;
    if (row < count) {
      const int t = idx[row];
      sl = reinterpret_cast<const uint32_t*>(src_head + (uint64_t)(src_tile0 + t / kTile) * kTileBytes + which * kPart + kCodes)[(t & (kTile - 1)) * NG + g];
    }
    reinterpret_cast<uint32_t*>(dst_tile + which * kPart + kCodes)[row * NG + g] = sl;
  }
}

// Tile `tile` of what one (entry, layer, head) keeps; by kGatherThreads threads.
template <int D>
__device__ __forceinline__ void gather_tile(const EvictEntry& e, const PoolGeom& pool16, const PoolGeom& pool4, int layer, int head, int tile,
                                            const int32_t* kept_of_head, int tid) {
  const int32_t* idx = kept_of_head + tile * kTile;
  const int count = min(kTile, e.keep - tile * kTile);
  const PoolGeom& pool = e.four ? pool4 : pool16;
  char* head_base = pool.base + (uint64_t)layer * pool.layer_stride + (uint64_t)head * pool.head_stride;
  char* dst = head_base + (uint64_t)(e.dst_tile0 + tile) * pool.tile_bytes;
  if (e.four) gather_tile4<D>(head_base, dst, e.src_tile0, count, idx, tid);
  else gather_tile16<D>(head_base, dst, e.src_tile0, count, idx, tid);
}

// kGather: the CTA also copies the rows that it chose, two tiles at a time.
template <int D, bool kGather>
__global__ void __launch_bounds__(kSelectThreads) k_select(const EvictBatch batch, const PoolGeom pool16, const PoolGeom pool4,
                                                           float* __restrict__ weights, int64_t layer_slots, int64_t slots,
                                                           int num_kv_heads, int32_t* kept, int32_t* node_len, int32_t* node_off) {
  const EvictEntry e = batch.entry[blockIdx.y];
  if (e.fresh && blockIdx.x == 0 && threadIdx.x == 0) {
    node_len[e.node] = e.keep;
    node_off[e.node] = (int32_t)e.dst_slot;
  }
  if (e.keep == 0) return;
  const int layer = blockIdx.x / num_kv_heads, head = blockIdx.x % num_kv_heads;
  float* w = weights + layer * layer_slots + head * slots;
  int32_t* out = kept + e.kept_off + (int64_t)blockIdx.x * e.keep;
  select_kept(e, w + e.src_slot, w + e.dst_slot, out);
  if (kGather) {
    static_assert(kSelectThreads == 2 * kGatherThreads, "two tiles at a time");
    __syncthreads();
    for (int tile = threadIdx.x / kGatherThreads; tile * kTile < e.keep; tile += 2)
      gather_tile<D>(e, pool16, pool4, layer, head, tile, out, threadIdx.x % kGatherThreads);
  }
}

template <int D>
__global__ void __launch_bounds__(kGatherThreads) k_gather(const EvictBatch batch, const PoolGeom pool16, const PoolGeom pool4,
                                                           int num_kv_heads, const int32_t* __restrict__ kept) {
  const EvictEntry e = batch.entry[blockIdx.z];
  const int tile = blockIdx.x;
  if (tile * kTile >= e.keep) return;
  const int layer = blockIdx.y / num_kv_heads, head = blockIdx.y % num_kv_heads;
  gather_tile<D>(e, pool16, pool4, layer, head, tile, kept + e.kept_off + (int64_t)blockIdx.y * e.keep, threadIdx.x);
}

}  // namespace

int launch_evict(const PoolGeom& pool16, const PoolGeom& pool4, const EvictBatch& batch, int num_layers, int num_kv_heads,
                 int head_dim, float* weights, int64_t slots, int32_t* kept, const GraphDev& g, cudaStream_t st) {
  int most = 0;
  for (int i = 0; i < batch.count; ++i) most = batch.entry[i].keep > most ? batch.entry[i].keep : most;
  const unsigned lh = (unsigned)(num_layers * num_kv_heads);
  const dim3 select_grid(lh, batch.count);
  auto select = [&](auto kernel) {
    kernel<<<select_grid, kSelectThreads, 0, st>>>(batch, pool16, pool4, weights, slots * num_kv_heads, slots, num_kv_heads, kept, g.node_len, g.node_off);
  };
  int launched = 1;
  if (most <= kOneLaunch) {
    if (head_dim == 128) select(k_select<128, true>);
    else select(k_select<64, true>);
  } else {
    select(k_select<64, false>);  // (the choice does not depend on the head's size)
    const dim3 grid((unsigned)((most + kTile - 1) / kTile), lh, batch.count);
    if (head_dim == 128) k_gather<128><<<grid, kGatherThreads, 0, st>>>(batch, pool16, pool4, num_kv_heads, kept);
    else k_gather<64><<<grid, kGatherThreads, 0, st>>>(batch, pool16, pool4, num_kv_heads, kept);
    ++launched;
  }
  return cudaGetLastError() == cudaSuccess ? launched : -1;
}

}  // namespace gf
