// Nodes that grow: the token slots of a batch's new tokens from the requests' lengths, and the new K/V rows put into
// the pool.
//
// Request r has held_r tokens in its node and gets count_r more; its rows in the batch start at the sum of the counts
// before it, and row i of them goes to the slot off(node_r) + held_r + i.  All of it stays on the device: the node's new
// length is written where the table builder reads it.  Every row of an open node at or beyond its length is zero in
// every layer (gf_node_kv_open clears the extent, a call that takes tokens back clears theirs), so that the tails of
// its tiles contribute exact zeros to P*V as everywhere in the pool.
#include <algorithm>

#include "gf_device.cuh"
#include "gf_internal.h"

namespace gf {
namespace {

constexpr int kSlotThreads = 256, kSlotRequests = 32;  // requests per CTA, at most

__device__ __forceinline__ char* chunk_at(const PoolGeom& pool, int layer, int head, int slot, int chunk, int value) {
  const uint32_t row = (uint32_t)slot & (kTile - 1);
  return pool.base + (uint64_t)layer * pool.layer_stride + (uint64_t)head * pool.head_stride +
         (uint64_t)(slot / kTile) * pool.tile_bytes + (value ? pool.tile_bytes >> 1 : 0u) +
         (uint32_t)(chunk >> 3) * (kTile * 128u) + swz128(row, (uint32_t)chunk & 7u);
}

// Zeros in the rows [from, to) of the pool, (layer, head) pairs first .. last, by all threads of the CTA (256): 2 * chunks neighbouring
// threads a row.
__device__ void clear_rows(const PoolGeom& pool, int heads, int chunks, int from, int to, int first, int last, int32_t* status) {
  if (!GF_CHECK(from >= 0 && (from >= to || (uint32_t)((to - 1) / kTile) < pool.cap_tiles), status, 501)) return;
  const int per_row = 2 * chunks, c = threadIdx.x % per_row, value = c >= chunks;
  for (int j = first + threadIdx.x / per_row; j < last; j += 256 / per_row) {
    const int layer = j / heads, head = j - layer * heads;
    for (int slot = from; slot < to; ++slot)
      *reinterpret_cast<uint4*>(chunk_at(pool, layer, head, slot, c - value * chunks, value)) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// A CTA has `per` requests, one where multiprocessors are left (what taken-back tokens leave to clear is much: 131 KB a token of 32 layers with 8
// heads): it adds up the counts of those before them and looks for its nodes among theirs (each CTA by itself: 8 bytes a request from L2, against
// a launch or a chain of CTAs; so the work grows with the square of the requests: 4096 take 11.5 us, 16 384 64, 65 536 600), one warp checks its requests and sets their lengths, and all threads write the slots.
// Latency-bound: a chain of four dependent loads; with the rows' copy 3.9 us for one request, 4.6 for 256.  256 requests that take back 4 tokens of
// 32 layers: 29 us (134 MB of zeros); one request's are one CTA's, 2.1 us a token: 1024 of 32 layers 2.1 ms.
__global__ void __launch_bounds__(kSlotThreads) k_append_slots(GraphDev g, PoolGeom pool, int layers, int heads, int chunks, int num_requests, int per,
                                                               const int32_t* __restrict__ node, const int32_t* __restrict__ held,
                                                               const int32_t* __restrict__ count, int num_new, int32_t* __restrict__ slots,
                                                               int32_t* __restrict__ lens, int32_t* status) {
  __shared__ long long warp_sums[kSlotThreads / 32];
  __shared__ int s_begin[kSlotRequests + 1], s_slot[kSlotRequests], s_from[kSlotRequests], s_to[kSlotRequests];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  __shared__ int s_node[kSlotRequests];
  __shared__ uint32_t s_twice;  // bit i: a request before has request i's node
  const int r0 = blockIdx.x * per;
  long long before = 0;
  uint32_t twice = 0;
  if (tid == 0) s_twice = 0;
  if (per == 1) {
    const int own = num_requests > 0 ? node[r0] : -1;
    for (int r = tid; r < r0; r += kSlotThreads) {
      before += max(count[r], 0);
      twice |= node[r] == own;
    }
  } else {
    if (tid < per) s_node[tid] = r0 + tid < num_requests ? node[r0 + tid] : -1;
    __syncthreads();
    for (int r = tid; r < r0; r += kSlotThreads) {
      before += max(count[r], 0);
      const int v = node[r];
      for (int i = 0; i < per; ++i) twice |= (uint32_t)(v == s_node[i]) << i;
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
  if (lane == 0) warp_sums[wid] = before;
  __syncthreads();
  if (twice) atomicOr(&s_twice, twice);
  __syncthreads();
  if (wid == 0) {
    long long begin = 0;
#pragma unroll
    for (int w = 0; w < kSlotThreads / 32; ++w) begin += warp_sums[w];
    const int r = r0 + lane;
    const bool mine = lane < per && r < num_requests;
    const int c = mine ? count[r] : 0, v = mine ? node[r] : -1;
    const bool known = v >= 0 && v < g.num_nodes;
    const int room = known ? g.node_room[v] : -1, now = known ? g.node_len[v] : 0;
    const int h = !mine ? 0 : held != nullptr ? held[r] : now;
    long long end = max(c, 0);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, end, d);
      if (lane >= d) end += y;
    }
    end += begin;
    const long long first = end - max(c, 0);
    int why = GF_OK;
    const uint32_t alike = __match_any_sync(0xffffffffu, v);  // (by all lanes, whatever is known of theirs)
    const bool again = ((alike & ((1u << lane) - 1u)) | (s_twice >> lane & 1u)) != 0;
    if (mine) {
      if (again || room < 0 || c < 0 || h < 0 || h > now || end > num_new) why = GF_ERR_INVALID_ARG;
      else if ((long long)h + c > room) why = GF_ERR_CAPACITY;
      if (why != GF_OK) atomicCAS(status + kStatusReport, 0, why);
    }
    const bool ok = mine && why == GF_OK && GF_CHECK(g.node_off[v] >= 0 && (int64_t)g.node_off[v] + room <= (int64_t)pool.cap_tiles * kTile, status, 502);
    if (ok) g.node_len[v] = h + c;
    if (mine && lens != nullptr) lens[r] = ok ? h + c : -1;
    const int off = ok ? g.node_off[v] : 0;
    s_slot[lane] = ok ? off + h : -1;
    // tokens taken back; none of a request that is left out (whose held and count may be anything)
    const bool back = ok && now > h + c;
    s_from[lane] = back ? off + h + c : 0;
    s_to[lane] = back ? off + now : 0;
    s_begin[lane] = (int)min(first, (long long)num_new);
    if (lane == 31) s_begin[32] = (int)min(end, (long long)num_new);
  }
  __syncthreads();
  for (int t = s_begin[0] + tid, i = 0; t < s_begin[per]; t += kSlotThreads) {
    while (t >= s_begin[i + 1]) ++i;
    if (!GF_CHECK(t >= 0 && t < num_new && i < per, status, 503)) break;
    slots[t] = s_slot[i] < 0 ? -1 : s_slot[i] + (t - s_begin[i]);
  }
  if (r0 + per >= num_requests)  // rows behind the last request's
    for (int t = s_begin[per] + tid; t < num_new; t += kSlotThreads) slots[t] = -1;
  for (int i = 0; i < per; ++i)
    if (s_to[i] > s_from[i]) clear_rows(pool, heads, chunks, s_from[i], s_to[i], 0, layers * heads, status);
}

// One layer's new rows from the caller's layout to their slots: 16 bytes of K and of V per step of a thread, a few tokens per
// CTA.  15 800 tokens of 8 heads of 128 entries: 20 us, 130 MB asked for, there and back, at 6.4 TB/s; L2 takes in most of what is written (counters: 65 MB read and 16 of
// 65 written by the kernel's end, DRAM at 49 %), so what bounds it is loads on the way, not HBM alone.
__global__ void __launch_bounds__(256) k_kv_append(PoolGeom pool, int layer, int heads, int chunk_bits, int num_new, int per_cta,
                                                   const int32_t* __restrict__ slots, const char* __restrict__ k, int64_t k_stride,
                                                   const char* __restrict__ v, int64_t v_stride, int32_t* status) {
  const int t0 = blockIdx.x * per_cta, per_token = heads << chunk_bits;
  const int n = min(per_cta, num_new - t0) * per_token;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) {
    const int t = i / per_token, at = i - t * per_token;
    const int slot = slots[t0 + t];
    const uint4 kv = *reinterpret_cast<const uint4*>(k + (int64_t)(t0 + t) * k_stride + at * 16);
    const uint4 vv = *reinterpret_cast<const uint4*>(v + (int64_t)(t0 + t) * v_stride + at * 16);
    if (slot < 0) continue;
    if ((uint32_t)(slot / kTile) >= pool.cap_tiles) {
      atomicCAS(status + kStatusReport, 0, (int)GF_ERR_INVALID_ARG);
      continue;
    }
    const int head = at >> chunk_bits, c = at & ((1 << chunk_bits) - 1);
    *reinterpret_cast<uint4*>(chunk_at(pool, layer, head, slot, c, 0)) = kv;
    *reinterpret_cast<uint4*>(chunk_at(pool, layer, head, slot, c, 1)) = vv;
  }
}

// Zeros in a whole extent, every layer and head.  With the two words of the node: 1088 tokens of 32 layers of 8 heads of 128 27 us, 8256 156 us (1.08 GB at 6.9 TB/s).
__global__ void __launch_bounds__(256) k_clear_extent(PoolGeom pool, int rows, int tile0, int tiles, int32_t* status) {
  if (!GF_CHECK(tile0 >= 0 && (uint32_t)(tile0 + tiles) <= pool.cap_tiles, status, 504)) return;
  const uint64_t n = (uint64_t)tiles * (pool.tile_bytes / 16);
  for (int j = blockIdx.y; j < rows; j += gridDim.y) {
    uint4* p = reinterpret_cast<uint4*>(pool.base + (uint64_t)j * pool.head_stride + (uint64_t)tile0 * pool.tile_bytes);
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) p[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// The end of a node's growth: zeros in what is left of its last tile, a CTA per layer, then its length: 6 to 8 us, two launches.
__global__ void __launch_bounds__(256) k_clear_tail(GraphDev g, PoolGeom pool, int heads, int chunks, int node, int n_tokens, int32_t* status) {
  const int off = g.node_off[node], end = min(g.node_len[node], (n_tokens + kTile - 1) / kTile * kTile);
  clear_rows(pool, heads, chunks, off + n_tokens, off + end, blockIdx.x * heads, (blockIdx.x + 1) * heads, status);
}
__global__ void k_close_node(GraphDev g, int node, int n_tokens, int32_t* status) {
  if (g.node_len[node] < n_tokens) atomicCAS(status + kStatusReport, 0, (int)GF_ERR_INVALID_ARG);
  g.node_len[node] = n_tokens;
  g.node_room[node] = -1;
}

}  // namespace

int launch_append_slots(const GraphDev& g, const PoolGeom& pool, int layers, int heads, int head_dim, int num_requests, const int32_t* node,
                        const int32_t* held, const int32_t* count, int num_new, int32_t* slots, int32_t* lens, int num_sms, int32_t* status,
                        cudaStream_t st) {
  const int per = std::min(kSlotRequests, std::max(1, num_requests / (2 * num_sms)));
  const int ctas = num_requests > 0 ? (num_requests + per - 1) / per : 1;  // (no request: the rows' -1 are left)
  k_append_slots<<<ctas, kSlotThreads, 0, st>>>(g, pool, layers, heads, head_dim / 8, num_requests, per, node, held, count, num_new, slots, lens,
                                                status);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int launch_kv_append(const PoolGeom& pool, int layer, int heads, int head_dim, int num_new, const int32_t* slots, const void* k,
                     int64_t k_stride, const void* v, int64_t v_stride, int num_sms, int32_t* status, cudaStream_t st) {
  // tokens per CTA: one while that leaves multiprocessors without work, up to eight
  int per_cta = num_new / (num_sms * 8);
  per_cta = per_cta < 1 ? 1 : per_cta > 8 ? 8 : per_cta;
  k_kv_append<<<(num_new + per_cta - 1) / per_cta, 256, 0, st>>>(pool, layer, heads, head_dim == 128 ? 4 : 3, num_new, per_cta, slots,
                                                                (const char*)k, k_stride * 2, (const char*)v, v_stride * 2, status);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int launch_clear_extent(const PoolGeom& pool, int layers, int heads, int tile0, int tiles, int32_t* status, cudaStream_t st) {
  if (tiles <= 0) return 0;
  const long long rows = (long long)layers * heads, blocks = (long long)tiles * (pool.tile_bytes / 16) / 1024;
  k_clear_extent<<<dim3((unsigned)(blocks < 64 ? blocks : 64), (unsigned)(rows < 65535 ? rows : 65535)), 256, 0, st>>>(pool, (int)rows, tile0, tiles, status);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int launch_close_node(const GraphDev& g, const PoolGeom& pool, int layers, int heads, int head_dim, int node, int n_tokens, int32_t* status,
                      cudaStream_t st) {
  k_clear_tail<<<layers, 256, 0, st>>>(g, pool, heads, head_dim / 8, node, n_tokens, status);
  if (cudaGetLastError() != cudaSuccess) return -1;
  k_close_node<<<1, 1, 0, st>>>(g, node, n_tokens, status);
  return cudaGetLastError() == cudaSuccess ? 2 : -1;
}

}  // namespace gf
