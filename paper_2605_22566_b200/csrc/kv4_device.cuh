// The 4-bit node states: format, layout and the device pieces that read and write it.
//
// Format.  64 neighbouring entries of one (token, KV head) form a group with two bf16 numbers: lo, the
// group's least value, and s, the bf16 nearest to (hi - lo) / 16.  An entry x has the code
// c = floor((x - lo) / s) held within 0..15 (0 where s is 0) and stands for lo + s (c + 1/2), the middle of
// its cell (lo itself where s is 0); 4.5 bits per entry.  A group's numbers belong to one token, so that a
// score is a sum of exact products: q . k = sum over groups of s (q . (c - 8)) + (lo + 8.5 s) (sum of q),
// with c - 8 exact in bf16.
//
// Layout.  A tile holds 64 tokens of one KV head: the K part, then the V part; a part is its codes, then
// one 32-bit word (s in the low half, lo in the high half) per (token, group).  The codes lie in the order
// in which a warp's MMA operands take them: for every block of 16 tokens and every group, lane l owns 16
// consecutive bytes (four words of eight codes), so that a warp reads a block with one 16-byte load per
// lane, and word kk unpacks into the four A registers of MMA number kk.  Register j is nibble j of the low
// half and nibble j of the high half.  With l4 = l % 4 and l8 = l / 4:
//   K (A = K, tokens are rows):     token 16 b + l8 + 8 (j & 1), entry 32 (e / 8) + 8 l4 + e % 8 of the group
//                                   with e = 4 kk + 2 (j / 2) + half
//   V (A = V^T, entries are rows):  token 16 b + 2 l4 + half + 8 (j / 2), entry 8 l8 + 2 kk + (j & 1) of the group
// The order of the entries inside a group is a permutation of the MMA's k (for K) or of its rows (for V),
// chosen so that a lane's entries are 16-byte runs of the caller's rows, of the queries and of the output.
#pragma once
#include "gf_device.cuh"
#include "gf_internal.h"

namespace gf {

constexpr int kGroup4 = 64;  // entries that share one (s, lo) pair

__host__ __device__ constexpr uint32_t kv4_code_bytes(int head_dim) { return (uint32_t)kTile * head_dim / 2; }
__host__ __device__ constexpr uint32_t kv4_part_bytes(int head_dim) {
  return kv4_code_bytes(head_dim) + (uint32_t)kTile * (head_dim / kGroup4) * 4;
}
__host__ __device__ constexpr uint32_t kv4_tile_bytes(int head_dim) { return 2 * kv4_part_bytes(head_dim); }

// Four A registers (bf16 pairs) of c - 8 from one word of codes: 0x4300 | c is the bf16 number 128 + c.
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w) {
  uint32_t r = (w & 0x000f000fu) | 0x43004300u;
  asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x43084308u));
  return r;
}
__device__ __forceinline__ void kv4_expand(uint32_t (&a)[4], uint32_t w) {
  a[0] = kv4_pair(w);
  a[1] = kv4_pair(w >> 4);
  a[2] = kv4_pair(w >> 8);
  a[3] = kv4_pair(w >> 12);
}
__device__ __forceinline__ float kv4_s(uint32_t sl) { return __uint_as_float(sl << 16); }
__device__ __forceinline__ float kv4_lo(uint32_t sl) { return __uint_as_float(sl & 0xffff0000u); }

// A code in the low bits of an fp16 pattern is the subnormal number c 2^-24, one nibble up 16 c 2^-24.  What undoes them:
constexpr float kUnit0 = 16777216.f, kUnit1 = 1048576.f;
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// 2^(t - e) for the exponent e of x (2^e <= x < 2^(e + 1)), held within 2^-100 .. 2^100 (2^100 for x = 0).
__device__ __forceinline__ float pow2_to(float x, int t) {
  const int e = (int)(__float_as_uint(x) >> 23) - 127;
  return __uint_as_float((uint32_t)(min(100, max(-100, t - e)) + 127) << 23);
}
// 1 / x for a power of two x within 2^-126 .. 2^126.
__device__ __forceinline__ float pow2_inverse(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }

}  // namespace gf
