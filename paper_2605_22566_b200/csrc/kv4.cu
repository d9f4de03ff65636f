// Node states held in 4 bits: put there from bf16 (k_kv4_write) and read back as the values that the
// codes stand for (k_kv4_read).  Format and layout: kv4_device.cuh.
//
// Both are streams: 2 bytes of bf16 per entry on one side, 0.5625 on the other, nothing reused.  32 768 tokens of 8 heads
// of 128, 172 MB either way: read in 29 us (5.9 TB/s, bound by HBM), written in 48 us (3.6 TB/s; 113 us with divisions).
// The write issues 31.8 M warp instructions, 15 per entry, which fill 66 % of its issue slots; in the rest its
// 29 warps per SM (64 registers) wait for the rows of their next block, which are asked for when the one before is
// coded.  A short node costs its launch.
// A warp works on one block of 16 tokens of one KV
// head and one group of 64 entries, K or V: 2 KB of bf16, 512 bytes of codes.  The layout gives every lane
// 16-byte runs on both sides, so nothing goes through shared memory; a token's least and largest entry are
// found with shuffles among the lanes that hold it.
#include "kv4_device.cuh"
#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The least entry and, negated, the greatest of two pairs that hold the least and the greatest of a run: one pair of
// bf16, so that one minimum (and one shuffle) serves both from here on.
__device__ __forceinline__ uint32_t ends_of(uint32_t lo2, uint32_t hi2) {
  hi2 ^= 0x80008000u;
  return min_pair(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));
}

__device__ __forceinline__ uint64_t f2_fma_rz(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// A group's numbers as the coding of its entries takes them.  Everything is scaled by 1/16, which is exact and keeps
// hi - lo from overflowing; a group whose s is below 2^-96 by 2^60 instead, exact too (its entries are below 2^-80: they
// differ by at least a bf16 step), so that s, which goes down to 2^-133, has a reciprocal in fp32.
struct GroupCoder {
  uint32_t word;   // (s, lo) as stored
  float unit;      // 1/16 or 2^60
  float low, cell; // -lo unit, s unit
  float inv;       // a little more than 1 / cell; 0 where s is 0
  __device__ __forceinline__ explicit GroupCoder(uint32_t ends) {  // see ends_of
    const float lo = __uint_as_float(ends << 16), hi = -__uint_as_float(ends & 0xffff0000u);
    const __nv_bfloat16 s = __float2bfloat16_rn(__fsub_rn(hi * 0.0625f, lo * 0.0625f));
    word = (uint32_t)__bfloat16_as_ushort(s) | (__float_as_uint(lo) & 0xffff0000u);
    unit = __bfloat162float(s) > 0.f && __bfloat162float(s) < 0x1p-96f ? 0x1p60f : 0.0625f;
    low = lo * -unit;
    cell = __bfloat162float(s) * unit;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(cell));  // within 2^-23, the factor is 1 + 2^-21
    inv = cell > 0.f ? __fmul_ru(inv, 1.0000005f) : 0.f;
  }
  // The codes of N bf16 pairs, floor((x - lo) / s) within 0..15, one in each half of out[i].  x - lo is rounded towards
  // zero: fp32 holds every whole number of cells, so the rounded difference lies in the cell of the true one (rounded
  // to nearest, one within 2^-24 below a border came to lie on it).  (s is the one of the true hi - lo too: where that
  // difference is not exact in fp32, the smaller of the two numbers is below 2^-16 of the larger, which is then
  // the bf16 number nearest to it either way.)  The quotient from the
  // reciprocal is never below the true one and less than 2^-19 of it above, so its whole part is the code or,
  // where a whole number lies between the two, one more: then the remainder (exact: an FMA on a small
  // whole number and two short numbers) is negative.  That is rare, and put right behind a vote.
  template <int N>
  __device__ __forceinline__ void codes(const uint32_t (&pair)[N], uint32_t (&out)[N]) const {
    const uint64_t magic = f2_pack(8388608.f, 8388608.f), minus = f2_pack(-8388608.f, -8388608.f), unit2 = f2_pack(unit, unit);
    const uint64_t l2 = f2_pack(low, low), i2 = f2_pack(inv, inv), c2 = f2_pack(-cell, -cell);
    uint32_t sign = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t x = f2_pack(__uint_as_float(pair[i] << 16), __uint_as_float(pair[i] & 0xffff0000u));
      const uint64_t r = f2_fma_rz(x, unit2, l2);
      uint64_t t, u;
      asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(r), "l"(i2));
      asm("add.rm.f32x2 %0, %1, %2;" : "=l"(u) : "l"(t), "l"(magic));  // 2^23 + the whole part: it stands in the low bits
      const uint64_t rem = f2_fma(f2_add(u, minus), c2, r);
      uint32_t u0, u1, r0, r1;
      asm("mov.b64 {%0, %1}, %2;" : "=r"(u0), "=r"(u1) : "l"(u));
      asm("mov.b64 {%0, %1}, %2;" : "=r"(r0), "=r"(r1) : "l"(rem));
      sign |= r0 | r1;
      out[i] = __byte_perm(u0, u1, 0x5410);
    }
    if (__any_sync(0xffffffffu, (sign >> 31) != 0u)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float r0 = __fmaf_rz(__uint_as_float(pair[i] << 16), unit, low), r1 = __fmaf_rz(__uint_as_float(pair[i] & 0xffff0000u), unit, low);
        if (fmaf(-(float)(out[i] & 0xffffu), cell, r0) < 0.f) out[i] -= 1u;
        if (fmaf(-(float)(out[i] >> 16), cell, r1) < 0.f) out[i] -= 0x10000u;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) asm("min.u16x2 %0, %0, %1;" : "+r"(out[i]) : "r"(0x000f000fu));
  }
};

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
  const uint32_t jobs = (uint32_t)(n_pad / 16) * num_kv_heads * kGroups;  // (a pool of 2^31 such blocks would be 10^12 bytes)
  const uint32_t part = blockIdx.y ? kv4_part_bytes(D) : 0u;
  for (uint32_t job = (blockIdx.x * kThreads + threadIdx.x) >> 5; job < jobs; job += (gridDim.x * kThreads) >> 5) {
    const int grp = (int)(job % kGroups), b16 = (int)(job / kGroups / (uint32_t)num_kv_heads);
    const int head = (int)(job / kGroups - (uint32_t)b16 * num_kv_heads);
    char* head_base = layer_base + (uint64_t)head * head_stride;
    uint32_t word[4] = {0u, 0u, 0u, 0u};
    if (blockIdx.y == 0) {
      // K: two tokens (l8, l8 + 8), 16 entries of each
      uint4 raw[2][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int token = b16 * 16 + l8 + 8 * j;
        raw[j][0] = raw[j][1] = make_uint4(0u, 0u, 0u, 0u);
        if (token < n_tokens) {
          const uint4* src = reinterpret_cast<const uint4*>(k + ((long long)token * num_kv_heads + head) * D + grp * kGroup4);
          raw[j][0] = src[l4];
          raw[j][1] = src[4 + l4];
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t x[8] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w, raw[j][1].x, raw[j][1].y, raw[j][1].z, raw[j][1].w};
        uint32_t lo2 = x[0], hi2 = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) { lo2 = min_pair(lo2, x[i]); hi2 = max_pair(hi2, x[i]); }
        uint32_t ends = ends_of(lo2, hi2);
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) ends = min_pair(ends, __shfl_xor_sync(0xffffffffu, ends, d));
        const GroupCoder coder(ends);
        uint32_t c[8];
        coder.codes(x, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) word[i >> 1] += c[i] << (4 * (j + 2 * (i & 1)));  // entries e = 2 i, 2 i + 1
        if (l4 == 0) *token_word(head_base, tile0, kTileBytes, b16 * 16 + l8 + 8 * j, grp, kGroups, part, kCodes) = coder.word;
      }
    } else {
      // V: four tokens (2 l4 + half + 8 t8), 8 entries of each
      uint4 raw[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int token = b16 * 16 + 2 * l4 + (t & 1) + 8 * (t >> 1);
        raw[t] = make_uint4(0u, 0u, 0u, 0u);
        if (token < n_tokens)
          raw[t] = reinterpret_cast<const uint4*>(v + ((long long)token * num_kv_heads + head) * D + grp * kGroup4)[l8];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t x[4] = {raw[t].x, raw[t].y, raw[t].z, raw[t].w};
        uint32_t lo2 = x[0], hi2 = x[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) { lo2 = min_pair(lo2, x[i]); hi2 = max_pair(hi2, x[i]); }
        uint32_t ends = ends_of(lo2, hi2);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) ends = min_pair(ends, __shfl_xor_sync(0xffffffffu, ends, d));
        const GroupCoder coder(ends);
        uint32_t c[4];
        coder.codes(x, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) word[i] += ((c[i] | (c[i] >> 12)) & 0xffu) << (16 * (t & 1) + 8 * (t >> 1));  // entries 2 i, 2 i + 1
        if (l8 == 0)
          *token_word(head_base, tile0, kTileBytes, b16 * 16 + 2 * l4 + (t & 1) + 8 * (t >> 1), grp, kGroups, part, kCodes) = coder.word;
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
  const uint32_t jobs = (uint32_t)((n_tokens + 15) / 16) * num_kv_heads * kGroups;
  const uint32_t part = blockIdx.y ? kv4_part_bytes(D) : 0u;
  for (uint32_t job = (blockIdx.x * kThreads + threadIdx.x) >> 5; job < jobs; job += (gridDim.x * kThreads) >> 5) {
    const int grp = (int)(job % kGroups), b16 = (int)(job / kGroups / (uint32_t)num_kv_heads);
    const int head = (int)(job / kGroups - (uint32_t)b16 * num_kv_heads);
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
