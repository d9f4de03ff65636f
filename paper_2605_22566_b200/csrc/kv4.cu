// Node states held in 4 bits: put there from bf16 (k_kv4_write) and read back as the values that the
// codes stand for (k_kv4_read).  Format and layout: kv4_device.cuh.
//
// Both are streams: 2 bytes of bf16 per entry on one side, 0.5625 on the other, nothing reused, so they are
// bound by HBM (and by the launch, for a short node).  A warp works on one block of 16 tokens of one KV
// head and one group of 64 entries, K or V: 2 KB of bf16, 512 bytes of codes.  The layout gives every lane
// 16-byte runs on both sides, so nothing goes through shared memory; a token's least and largest entry are
// found with shuffles among the lanes that hold it.
#include "kv4_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void unpack8(float (&x)[8], const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// (s, lo) of a group from its extremes.  hi / 16 - lo / 16 cannot overflow; the scaling is exact.
__device__ __forceinline__ uint32_t group_word(float lo, float hi) {
  const __nv_bfloat16 s = __float2bfloat16_rn(__fsub_rn(hi * 0.0625f, lo * 0.0625f));
  return (uint32_t)__bfloat16_as_ushort(s) | (__float_as_uint(lo) & 0xffff0000u);
}
// floor((x - lo) / s) within 0..15.  The division is rounded correctly, so no quotient below a whole number
// reaches it (x, lo and s have 8 significant bits each).
__device__ __forceinline__ uint32_t code_of(float x, uint32_t sl) {
  const float s = kv4_s(sl);
  if (!(s > 0.f)) return 0u;
  const float c = floorf(__fdiv_rn(__fsub_rn(x * 0.0625f, kv4_lo(sl) * 0.0625f), s) * 16.f);
  return (uint32_t)fminf(fmaxf(c, 0.f), 15.f);
}

// Where block `b16` (16 tokens), group `grp` of a node's K or V part of one head lies.
__device__ __forceinline__ char* block_codes(char* head_base, int tile0, uint32_t tile_bytes, int b16, int grp, int groups,
                                             uint32_t part) {
  return head_base + (uint64_t)(tile0 + (b16 >> 2)) * tile_bytes + part + (uint32_t)((b16 & 3) * groups + grp) * 512u;
}
__device__ __forceinline__ uint32_t* token_word(char* head_base, int tile0, uint32_t tile_bytes, int token, int grp, int groups,
                                                uint32_t part, uint32_t code_bytes) {
  return reinterpret_cast<uint32_t*>(head_base + (uint64_t)(tile0 + token / kTile) * tile_bytes + part + code_bytes) +
         (token & (kTile - 1)) * groups + grp;
}

template <int D>
__global__ void __launch_bounds__(kThreads) k_kv4_write(char* __restrict__ layer_base, uint64_t head_stride, int tile0,
                                                        const __nv_bfloat16* __restrict__ k,
                                                        const __nv_bfloat16* __restrict__ v, int n_tokens, int n_pad,
                                                        int num_kv_heads, int32_t* node_len, int32_t* node_off, int node,
                                                        int token_off) {
  constexpr int kGroups = D / kGroup4;
  constexpr uint32_t kTileBytes = kv4_tile_bytes(D), kCodes = kv4_code_bytes(D);
  if (node_len != nullptr && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    node_len[node] = n_tokens;
    node_off[node] = token_off;
  }
  const int lane = threadIdx.x & 31, l4 = lane & 3, l8 = lane >> 2;
  const long long jobs = (long long)(n_pad / 16) * num_kv_heads * kGroups;
  const uint32_t part = blockIdx.y ? kv4_part_bytes(D) : 0u;
  for (long long job = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5; job < jobs;
       job += ((long long)gridDim.x * kThreads) >> 5) {
    const int grp = (int)(job % kGroups);
    const int head = (int)(job / kGroups % num_kv_heads);
    const int b16 = (int)(job / kGroups / num_kv_heads);
    char* head_base = layer_base + (uint64_t)head * head_stride;
    uint32_t word[4] = {0u, 0u, 0u, 0u};
    if (blockIdx.y == 0) {
      // K: two tokens (l8, l8 + 8), 16 entries of each
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int token = b16 * 16 + l8 + 8 * j;
        uint4 raw[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
        if (token < n_tokens) {
          const uint4* src = reinterpret_cast<const uint4*>(k + ((long long)token * num_kv_heads + head) * D + grp * kGroup4);
          raw[0] = src[l4];
          raw[1] = src[4 + l4];
        }
        float x[2][8];
        unpack8(x[0], raw[0]);
        unpack8(x[1], raw[1]);
        float lo = x[0][0], hi = x[0][0];
#pragma unroll
        for (int e = 0; e < 16; ++e) { lo = fminf(lo, x[e >> 3][e & 7]); hi = fmaxf(hi, x[e >> 3][e & 7]); }
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
          lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
          hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        }
        const uint32_t sl = group_word(lo, hi);
#pragma unroll
        for (int e = 0; e < 16; ++e)  // e = 4 kk + 2 (j / 2) + half
          word[e >> 2] |= code_of(x[e >> 3][e & 7], sl) << (16 * (e & 1) + 4 * (j + 2 * ((e >> 1) & 1)));
        if (l4 == 0) *token_word(head_base, tile0, kTileBytes, token, grp, kGroups, part, kCodes) = sl;
      }
    } else {
      // V: four tokens (2 l4 + half + 8 t8), 8 entries of each
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int half = t & 1, t8 = t >> 1;
        const int token = b16 * 16 + 2 * l4 + half + 8 * t8;
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        if (token < n_tokens)
          raw = reinterpret_cast<const uint4*>(v + ((long long)token * num_kv_heads + head) * D + grp * kGroup4)[l8];
        float x[8];
        unpack8(x, raw);
        float lo = x[0], hi = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) { lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]); }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
          hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        }
        const uint32_t sl = group_word(lo, hi);
#pragma unroll
        for (int e = 0; e < 8; ++e)  // e = 2 kk + (j & 1)
          word[e >> 1] |= code_of(x[e], sl) << (16 * half + 4 * ((e & 1) + 2 * t8));
        if (l8 == 0) *token_word(head_base, tile0, kTileBytes, token, grp, kGroups, part, kCodes) = sl;
      }
    }
    reinterpret_cast<uint4*>(block_codes(head_base, tile0, kTileBytes, b16, grp, kGroups, part))[lane] =
        make_uint4(word[0], word[1], word[2], word[3]);
  }
}

__device__ __forceinline__ float value_of(uint32_t code, uint32_t sl) {
  return __fmaf_rn(kv4_s(sl), (float)code + 0.5f, kv4_lo(sl));
}

template <int D>
__global__ void __launch_bounds__(kThreads) k_kv4_read(const char* __restrict__ layer_base, uint64_t head_stride, int tile0,
                                                       __nv_bfloat16* __restrict__ k, __nv_bfloat16* __restrict__ v,
                                                       int n_tokens, int num_kv_heads) {
  constexpr int kGroups = D / kGroup4;
  constexpr uint32_t kTileBytes = kv4_tile_bytes(D), kCodes = kv4_code_bytes(D);
  const int lane = threadIdx.x & 31, l4 = lane & 3, l8 = lane >> 2;
  const long long jobs = (long long)((n_tokens + 15) / 16) * num_kv_heads * kGroups;
  const uint32_t part = blockIdx.y ? kv4_part_bytes(D) : 0u;
  for (long long job = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5; job < jobs;
       job += ((long long)gridDim.x * kThreads) >> 5) {
    const int grp = (int)(job % kGroups);
    const int head = (int)(job / kGroups % num_kv_heads);
    const int b16 = (int)(job / kGroups / num_kv_heads);
    char* head_base = const_cast<char*>(layer_base) + (uint64_t)head * head_stride;
    const uint4 codes = reinterpret_cast<const uint4*>(block_codes(head_base, tile0, kTileBytes, b16, grp, kGroups, part))[lane];
    const uint32_t word[4] = {codes.x, codes.y, codes.z, codes.w};
    if (blockIdx.y == 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int token = b16 * 16 + l8 + 8 * j;
        if (token >= n_tokens) continue;
        const uint32_t sl = *token_word(head_base, tile0, kTileBytes, token, grp, kGroups, part, kCodes);
        uint32_t out[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // entries e = 2 i, 2 i + 1
          const uint32_t w = word[i >> 1] >> (4 * (j + 2 * (i & 1)));
          out[i] = pack_bf16(value_of(w & 15u, sl), value_of((w >> 16) & 15u, sl));
        }
        uint4* dst = reinterpret_cast<uint4*>(k + ((long long)token * num_kv_heads + head) * D + grp * kGroup4);
        dst[l4] = make_uint4(out[0], out[1], out[2], out[3]);
        dst[4 + l4] = make_uint4(out[4], out[5], out[6], out[7]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int half = t & 1, t8 = t >> 1;
        const int token = b16 * 16 + 2 * l4 + half + 8 * t8;
        if (token >= n_tokens) continue;
        const uint32_t sl = *token_word(head_base, tile0, kTileBytes, token, grp, kGroups, part, kCodes);
        uint32_t out[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // entries 2 i, 2 i + 1
          const uint32_t w = word[i] >> (16 * half + 8 * t8);
          out[i] = pack_bf16(value_of(w & 15u, sl), value_of((w >> 4) & 15u, sl));
        }
        reinterpret_cast<uint4*>(v + ((long long)token * num_kv_heads + head) * D + grp * kGroup4)[l8] =
            make_uint4(out[0], out[1], out[2], out[3]);
      }
    }
  }
}

unsigned stream_blocks(int blocks16, int num_kv_heads, int head_dim, int num_sms) {
  const long long jobs = (long long)blocks16 * num_kv_heads * (head_dim / kGroup4);
  const long long blocks = (jobs + kThreads / 32 - 1) / (kThreads / 32), most = (long long)num_sms * 16;
  return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace

int launch_kv4_write(const PoolGeom& pool, int layer, int num_kv_heads, int head_dim, int tile0, const void* k,
                     const void* v, int n_tokens, const GraphDev* set, int node, int token_off, int num_sms, cudaStream_t st) {
  if (n_tokens <= 0) return 0;
  const int n_pad = (n_tokens + kTile - 1) / kTile * kTile;
  const dim3 grid(stream_blocks(n_pad / 16, num_kv_heads, head_dim, num_sms), 2, 1);
  auto go = [&](auto kernel) {
    kernel<<<grid, kThreads, 0, st>>>(pool.base + (uint64_t)layer * pool.layer_stride, pool.head_stride, tile0,
                                      (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, n_tokens, n_pad, num_kv_heads,
                                      set ? set->node_len : nullptr, set ? set->node_off : nullptr, node, token_off);
  };
  if (head_dim == 128) go(k_kv4_write<128>);
  else go(k_kv4_write<64>);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int launch_kv4_read(const PoolGeom& pool, int layer, int num_kv_heads, int head_dim, int tile0, void* k, void* v,
                    int n_tokens, int num_sms, cudaStream_t st) {
  if (n_tokens <= 0) return 0;
  const dim3 grid(stream_blocks((n_tokens + 15) / 16, num_kv_heads, head_dim, num_sms), 2, 1);
  auto go = [&](auto kernel) {
    kernel<<<grid, kThreads, 0, st>>>(pool.base + (uint64_t)layer * pool.layer_stride, pool.head_stride, tile0,
                                      (__nv_bfloat16*)k, (__nv_bfloat16*)v, n_tokens, num_kv_heads);
  };
  if (head_dim == 128) go(k_kv4_read<128>);
  else go(k_kv4_read<64>);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace gf
