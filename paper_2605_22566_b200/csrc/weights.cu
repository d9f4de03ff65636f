// Accumulated attention weights: how much of a decode batch's attention every resident token received.
//
//   w[kvh][slot(t)] (+)= sum over the requests r that share t's segment and the query heads h of KV head kvh
//                        of exp(scale q_rh . k_t - lse_rh)
//
// with lse from the decode call of the same step, so one pass over K is enough and no probability is ever
// stored.  It is a reduction over query rows for a fixed token, so a work unit is one 64-token tile of one
// segment and KV head with ALL the rows that share it: every slot has one writer, which adds in a fixed
// order, and the result does not depend on scheduling (no atomics).
//
// A warp keeps the tile's K in registers as MMA operands (bf16 values, or the codes c - 8 of a 4-bit
// state, which are exact in bf16), read straight from global memory, and walks the rows eight at a time:
// S^T = K Q^T, exp2 against the row's lse, sums per token in registers; at the end a shuffle over the
// four lanes that share a token and one read-modify-write of 64 floats.
#include "kv4_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 128;
constexpr int kBuckets = 1024;  // runs of segments whose tile counts are summed in shared memory

struct Params {
  const char* layer16;
  const char* layer4;
  uint64_t head_stride16, head_stride4;
  uint32_t tile_bytes16;
  int32_t kv4_tile0, cap16, cap4;
  const Header* hdr;
  const int32_t* seg_node;
  const int32_t* seg_len;
  const int32_t* seg_off;
  const int32_t* grp_ptr;
  const int32_t* grp_req;
  const int32_t* node_res;
  const __nv_bfloat16* q;
  const float* lse;
  float* weights;
  int64_t slots;
  int32_t slot_cap, num_pairs, num_requests;
  int32_t num_q_heads, num_kv_heads, gqa, accumulate;
  float scale_log2;
  int32_t* status;
};

// The tile's K as A operands: a[b][ks] holds tokens 16 b + l8 (+ 8) and, inside a run of 32 entries, the
// entries 8 l4 .. 8 l4 + 7 (the same permutation of the MMA's k as the queries below).
template <int D>
__device__ __forceinline__ void load_tile16(uint32_t (&a)[4][D / 16][4], const char* tile, int lane) {
  const uint32_t l4 = lane & 3, l8 = lane >> 2;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t row = b * 16 + l8 + 8 * h;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint32_t chunk = l4 + 4 * x;
        const uint4 v = *reinterpret_cast<const uint4*>(tile + (chunk >> 3) * (kTile * 128u) + swz128(row, chunk & 7u));
        a[b][2 * x][h] = v.x;
        a[b][2 * x][2 + h] = v.y;
        a[b][2 * x + 1][h] = v.z;
        a[b][2 * x + 1][2 + h] = v.w;
      }
    }
}
template <int D>
__device__ __forceinline__ void load_tile4(uint32_t (&a)[4][D / 16][4], const char* tile, int lane) {
  constexpr int NG = D / kGroup4;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint4 v = reinterpret_cast<const uint4*>(tile)[(b * NG + g) * 32 + lane];
      kv4_expand(a[b][4 * g], v.x);
      kv4_expand(a[b][4 * g + 1], v.y);
      kv4_expand(a[b][4 * g + 2], v.z);
      kv4_expand(a[b][4 * g + 3], v.w);
    }
}

// Adds the rows [0, rows) of the group to sum[b][h] (tokens 16 b + l8 + 8 h, this lane's two columns).
template <int D, bool k4>
__device__ __forceinline__ void walk_rows(const Params& p, const uint32_t (&a)[4][D / 16][4], const char* tile, int grp_begin,
                                          int rows, int kvh, int lane, float (&sum)[4][2]) {
  constexpr int NG = D / kGroup4, KS = D / 16;
  const int l4 = lane & 3, l8 = lane >> 2, g = p.gqa;
  uint32_t sl[4][2][NG];  // a 4-bit state's (s, lo) of this lane's tokens
  if (k4) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(tile + kv4_code_bytes(D));
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 0; x < NG; ++x) sl[b][h][x] = w[(b * 16 + l8 + 8 * h) * NG + x];
  }
  for (int row0 = 0; row0 < rows; row0 += 8) {
    // this lane's query row (operand) and its two columns' lse
    uint32_t qf[KS][2];
    {
      const int row = row0 + l8;
      const bool ok = row < rows;
      int req = ok ? p.grp_req[GF_CLAMP(grp_begin + row / g, p.num_pairs, p.status, 131)] : 0;
      req = GF_CLAMP(req, p.num_requests, p.status, 132);
      const uint4* qrow = reinterpret_cast<const uint4*>(p.q + ((size_t)req * p.num_q_heads + kvh * g + row % g) * D);
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint4 v = ok ? qrow[4 * x + l4] : make_uint4(0u, 0u, 0u, 0u);
        qf[2 * x][0] = v.x;
        qf[2 * x][1] = v.y;
        qf[2 * x + 1][0] = v.z;
        qf[2 * x + 1][1] = v.w;
      }
    }
    float off[2];  // -lse in log2 units; a row that does not exist counts for nothing
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = row0 + l4 * 2 + c;
      const bool ok = row < rows;
      int req = ok ? p.grp_req[GF_CLAMP(grp_begin + row / g, p.num_pairs, p.status, 133)] : 0;
      req = GF_CLAMP(req, p.num_requests, p.status, 134);
      off[c] = ok ? -1.4426950408889634f * p.lse[(size_t)req * p.num_q_heads + kvh * g + row % g] : -INFINITY;
    }
    float qsum[NG][2];
    if (k4) {
#pragma unroll
      for (int x = 0; x < NG; ++x) {
        const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_bf16(acc, ones, qf[x * 4 + kk][0], qf[x * 4 + kk][1]);
        qsum[x][0] = acc[0];
        qsum[x][1] = acc[1];
      }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      if (k4) {
#pragma unroll
        for (int x = 0; x < NG; ++x) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) mma_bf16(acc, a[b][x * 4 + kk], qf[x * 4 + kk][0], qf[x * 4 + kk][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float sc = kv4_s(sl[b][e >> 1][x]), z = fmaf(8.5f, sc, kv4_lo(sl[b][e >> 1][x]));
            s[e] = fmaf(acc[e], sc, fmaf(qsum[x][e & 1], z, s[e]));
          }
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) mma_bf16(s, a[b][ks], qf[ks][0], qf[ks][1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[b][e >> 1] += fast_exp2(fmaf(s[e], p.scale_log2, off[e & 1]));
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_weights(const Params p) {
  __shared__ int32_t start[kBuckets + 1];  // tiles of the segments before the bucket
  __shared__ int32_t warp_tot[kThreads / 32];
  chain_enter();
  if (!tables_usable(*p.hdr, p.slot_cap)) return;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int S = p.hdr->num_segments;
  const int per = (S + kBuckets - 1) / kBuckets;  // segments per bucket
  {
    // exclusive scan of the buckets' tile counts: a thread owns a run of buckets
    constexpr int kRun = kBuckets / kThreads;
    int cnt[kRun], local = 0;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const int b0 = min(S, (tid * kRun + i) * per), b1 = min(S, b0 + per);
      cnt[i] = 0;
      for (int s = b0; s < b1; ++s) cnt[i] += (p.seg_len[s] + kTile - 1) / kTile;
      local += cnt[i];
    }
    int incl = local;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 31) warp_tot[wid] = incl;
    __syncthreads();
    int run = incl - local;
    for (int w = 0; w < wid; ++w) run += warp_tot[w];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      start[tid * kRun + i] = run;
      run += cnt[i];
    }
    if (tid == kThreads - 1) start[kBuckets] = run;
    __syncthreads();
  }
  const long long units = (long long)start[kBuckets] * p.num_kv_heads;
  for (long long u = (long long)blockIdx.x * (kThreads / 32) + wid; u < units; u += (long long)gridDim.x * (kThreads / 32)) {
    const int ti = (int)(u / p.num_kv_heads), kvh = (int)(u % p.num_kv_heads);
    int lo = 0, hi = kBuckets;  // the last bucket that starts at or before the tile
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= ti) lo = mid; else hi = mid;
    }
    int seg = lo * per, at = start[lo];
    while (true) {
      const int n = (p.seg_len[seg] + kTile - 1) / kTile;
      if (ti < at + n) break;
      at += n;
      ++seg;
    }
    // a state kept as base + residual has no slots of its own
    if (p.node_res[p.seg_node[seg]] >= 0) continue;
    const int tok0 = (ti - at) * kTile, nv = min(kTile, p.seg_len[seg] - tok0);
    const int slot0 = p.seg_off[seg] + tok0, tile_index = slot0 / kTile;
    const int gb = p.grp_ptr[seg], rows = (p.grp_ptr[seg + 1] - gb) * p.gqa;
    float sum[4][2];
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b][0] = sum[b][1] = 0.f;
    uint32_t a[4][D / 16][4];
    if (tile_index < p.kv4_tile0) {
      const char* tile = p.layer16 + (uint64_t)kvh * p.head_stride16 + (uint64_t)GF_CLAMP(tile_index, p.cap16, p.status, 135) * p.tile_bytes16;
      load_tile16<D>(a, tile, lane);
      walk_rows<D, false>(p, a, tile, gb, rows, kvh, lane, sum);
    } else {
      const char* tile = p.layer4 + (uint64_t)kvh * p.head_stride4 + (uint64_t)GF_CLAMP(tile_index - p.kv4_tile0, p.cap4, p.status, 136) * kv4_tile_bytes(D);
      load_tile4<D>(a, tile, lane);
      walk_rows<D, true>(p, a, tile, gb, rows, kvh, lane, sum);
    }
    float* w = p.weights + (int64_t)kvh * p.slots + slot0;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v = sum[b][h];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        const int t = b * 16 + (lane >> 2) + 8 * h;
        if ((lane & 3) == 0 && t < nv) w[t] = p.accumulate ? w[t] + v : v;
      }
  }
}

}  // namespace

int launch_weights(const PoolGeom& pool16, const PoolGeom& pool4, const AttnShape& sh, const TablesDev& t, int layer, const void* q,
                   const float* lse, int accumulate, float* weights, int64_t slots, int32_t* status, cudaStream_t st) {
  Params p;
  p.layer16 = pool16.base + (uint64_t)layer * pool16.layer_stride;
  p.layer4 = pool4.base ? pool4.base + (uint64_t)layer * pool4.layer_stride : nullptr;
  p.head_stride16 = pool16.head_stride;
  p.head_stride4 = pool4.head_stride;
  p.tile_bytes16 = pool16.tile_bytes;
  p.kv4_tile0 = t.kv4_tile0;
  p.cap16 = (int32_t)pool16.cap_tiles;
  p.cap4 = (int32_t)pool4.cap_tiles;
  p.hdr = t.hdr;
  p.seg_node = t.seg_node;
  p.seg_len = t.seg_len;
  p.seg_off = t.seg_off;
  p.grp_ptr = t.grp_ptr;
  p.grp_req = t.grp_req;
  p.node_res = t.node_res;
  p.q = (const __nv_bfloat16*)q;
  p.lse = lse;
  p.weights = weights;
  p.slots = slots;
  p.slot_cap = t.slot_cap;
  p.num_pairs = t.num_pairs_in;
  p.num_requests = t.num_requests;
  p.num_q_heads = sh.num_q_heads;
  p.num_kv_heads = sh.num_kv_heads;
  p.gqa = sh.num_q_heads / sh.num_kv_heads;
  p.accumulate = accumulate;
  p.scale_log2 = sh.scale_log2;
  p.status = status;
  const dim3 grid((unsigned)(2 * t.num_sms));
  if (sh.head_dim == 128) launch_chained(k_weights<128>, grid, dim3(kThreads), 0, st, p);
  else launch_chained(k_weights<64>, grid, dim3(kThreads), 0, st, p);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace gf
