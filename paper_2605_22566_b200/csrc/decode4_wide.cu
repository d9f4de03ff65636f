// K2 over node states held in 4 bits, widely shared chunks: decode on tcgen05 tensor cores.
//
// A unit is a chunk of a 4-bit segment and up to 128 stacked query rows (request x GQA head) of the requests that
// share it.  The codes are expanded once per unit instead of once per 16 rows (decode4.cu), into shared memory, and
// S = Q K^T and O += P C run as tcgen05 MMAs with accumulators in tensor memory:
//   S_rt = sum over groups G of  q_rG . (s_tG (c_tG - 8))  +  (sum of q_rG) (lo_tG + 8.5 s_tG)
// K's scales are part of the operand, exact in fp16 (the second term takes a few entries more, see sums_offset), so that a
// score costs its thread one multiplication.  That needs a token's groups to be of about one size (see kNearGroups);
// a tile with a token whose groups are not gets one S per group and two multiplications.  V's operand are the codes, fp16
// subnormals c 2^-24 and 16 c 2^-24 (exact), with one accumulator per group of 64 entries, because values of different
// tokens may lie any power of two apart:
//   O_rG = sum over tokens of  (p_rt s_tG) c_tG  +  sum of  p_rt (lo_tG + s_tG / 2)
// A thread owns a query row: it takes the 32 scores of a step from tensor memory, exponentiates, applies the
// tokens' scales (tables in shared memory, read as broadcasts), keeps l and the second term of O in fp32, and puts
// p s f over the scores as fp16, one P per group.  Reference, f and roundings are those of decode4.cu.
//
// Two CTAs per SM, whose phases fill each other's gaps.  Roles by warp:
//   warps 0-3  softmax, a row per thread; at the end of a unit its fp32 partial
//   warps 4-7  the unit's queries (fp16 times a power of two per row), then a block of 16 tokens
//              each of every tile: codes and scale tables
//   warp 8     claims units, streams their tiles as they lie in the pool (bulk copies, three in flight)
//   warp 9     one thread issues the MMAs  (warps 10 and 11 only complete the group whose registers are handed over)
// Every wait is bounded; a warp whose wait gave up leaves its role, and so do the others.
//
// 1024 requests, 608 units of mostly 128 rows, 8776 tiles of 64 tokens: 137 us (the 16-row kernel takes 170 for the
// same), 4 of them since every tile is asked whether its groups lie apart.  The tensor pipe is busy 16 % of the time, the
// schedulers issue in 44 % of their cycles.  Bound by the latency of one softmax warp per scheduler and CTA, two CTAs
// being what tensor memory holds, and by shared memory: the scales' broadcasts, four wavefronts for 16 bytes, cost 600 of
// a step's 2000 cycles, the MMAs' operands 400.  Measured on the way: K as codes, its scales applied to the scores, 7 us
// more; K as values rounded to fp16, 13 less, but lse in fp32 lost bits to it; steps of a whole tile with one S, 23 more:
// an MMA or a commit costs its issuing thread 60 cycles, and there they stood between two softmaxes.
#include "kv4_device.cuh"
#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 384;
// Registers per thread after the roles' split, of the 80 that two CTAs of 384 threads leave; the shares of the three
// groups of four warps add up to what the CTA was launched with.
constexpr int kLaunchRegs = 80, kSoftmaxRegs = 120, kExpandRegs = 72, kControlRegs = 48;
static_assert(kSoftmaxRegs + kExpandRegs + kControlRegs == 3 * kLaunchRegs, "setmaxnreg draws on the launch's registers");  // (see the launch)
// What a warp gets of a kernel that needs `regs` per thread: registers are handed out by eights.
constexpr int allocated_regs(int regs) { return (regs + 7) / 8 * 8; }
static_assert(allocated_regs(72) == 72 && allocated_regs(73) == 80 && allocated_regs(80) == 80, "");
constexpr int kRows = 128;
constexpr int kUnits = 4, kStages = 3;
constexpr int kSub = 32;  // tokens per step of the softmax: half a tile

struct Params {
  const char* pool_layer;
  uint64_t head_stride;
  int32_t tile_base;  // index of the 4-bit pool's first tile among all tiles
  const Item* items;
  const int32_t* list;  // the handle's unit lists (see TablesDev::wide_list)
  const int32_t* grp_ptr;
  const int32_t* grp_req;
  const __nv_bfloat16* q;
  float* part_o;
  float* part_ml;
  int32_t* status;
  int32_t* counters;  // [0] next unit, [1] CTAs finished; both zero between launches
  const Header* hdr;
  int32_t slot_cap, num_q_heads, num_kv_heads, gqa;
  float scale_log2;
  int32_t cap_tiles, num_pairs, num_requests;
};

struct __align__(16) Unit {
  int32_t rows;  // -1: no more units
  int32_t grp_begin, part_base, kvh, tok_count, ntile, pad0, pad1;
};

// s and z = lo + s / 2 of a tile's V, [group][token]; what undoes the powers of two that K's tokens were multiplied by, per
// group; and by block of 16 tokens whether the two groups have powers of their own.
struct Scales { float s[2][kTile], z[2][kTile], k[2][kTile]; int32_t apart[4]; };
// A token's groups share a power of two where their largest entries lie within 2^8 of each other: s, whose eight bits
// begin at 2^-12 of its group's largest entry or above (entries are bf16), then stands at 2^-12 or above in the smaller
// group, and s (c - 8) and lo + 8.5 s keep their bits in fp16.
constexpr int kNearGroups = 8;

template <int D>
struct Smem {
  static constexpr int CB = D / 64;
  unsigned char q[CB][kRows * 128];       // fp16, 128-byte-swizzled rows of 64 entries
  unsigned char k[CB][kTile * 128];       // codes of a tile, K-major
  unsigned char v[CB][kTile * 128];       // and MN-major: both are rows of a token's 64 entries
  unsigned char q_sum[kRows * 32];        // 16 more entries of K's and Q's rows, for the term without codes (see sums_offset)
  unsigned char k_mid[CB][kTile * 32];    // of the first S, and of the second one where the groups have one each
  unsigned char stage[kStages][kv4_tile_bytes(D)];
  Scales scales[kStages];                 // of tile n at n % kStages
  float row_scale[kRows];                 // softmax scale over the row's power of two
  Unit unit[kUnits];
  uint32_t tmem_base;
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  uint64_t stage_full[kStages], stage_empty[kStages];
  uint64_t s_full[2], p_full[2], o_full[2];  // by step parity
  uint64_t q_full, q_empty, k_full, v_full, o_empty, mmas_done;
};
static_assert(2 * (sizeof(Smem<128>) + 1024) <= 228 * 1024, "two CTAs share an SM's shared memory, of which each takes 1 KB more");
constexpr int kUnitReaders = 4 + 4 + 1;

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t phase, const Params& p) { return mbar_wait(bar, phase & 1, p.status); }
// A pair of barriers that steps use in turn.
__device__ __forceinline__ bool wait_step(uint64_t (&bar)[2], int step, const Params& p) { return wait(&bar[step & 1], (uint32_t)step >> 1, p); }
// The term without codes, (sum of q_rG) (lo_tG + 8.5 s_tG), as more entries of the same product: two fp16 numbers hold 22
// bits of either factor (the sum to 2^-33 of its row's largest entry, where that is coarser), which is a 2^-21 of the
// term, of the size of the fp32 sum's own roundings; a group takes four entries, (qh, qh, ql, ql) times (zh, zl, zh, zl).
// Rows of 16 entries
// without a swizzle: eight rows of 16 bytes, twice, per 256 bytes; entries 8..15 stay zero.
__device__ __forceinline__ uint32_t sums_offset(uint32_t row, uint32_t group) { return (row >> 3) * 256 + (row & 7) * 16 + group * 8; }
__device__ __forceinline__ uint64_t sums_desc(uint32_t saddr) {  // lbo: 128 bytes to the next 8 entries, sbo: 256 to the next 8 rows
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(256 >> 4) << 32) | ((uint64_t)1 << 46);
}
// x as the sum of two fp16 numbers.
__device__ __forceinline__ void split_f16(float x, __half& hi, __half& lo) {
  hi = __float2half_rn(x);
  lo = __float2half_rn(x - __half2float(hi));
}
__device__ __forceinline__ uint32_t pair_of(__half a, __half b) { return (uint32_t)__half_as_ushort(a) | (uint32_t)__half_as_ushort(b) << 16; }
// Instruction descriptor: D fp32, A and B fp16.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

template <int D, typename F>
__device__ __forceinline__ void for_units(Smem<D>& sm, const Params& p, int lane, F&& body) {
  for (int n = 0;; ++n) {
    if (!wait(&sm.unit_full[n % kUnits], n / kUnits, p)) return;
    const Unit u = sm.unit[n % kUnits];
    if (u.rows < 0) return;
    if (!body(n, u)) return;
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.unit_empty[n % kUnits]);
  }
}

// ---- warp 8: units and their tiles ---------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void stream_units(Smem<D>& sm, const Params& p, int num_units, int& tile) {
  int n = 0;
  for (int u = blockIdx.x; u < num_units; ++n) {
    const int next = atomicAdd(&p.counters[0], 1) + (int)gridDim.x;  // (its result is needed one unit later)
    const Item it = p.items[GF_CLAMP(p.list[GF_CLAMP(p.hdr->kv4_wide_first + u / p.num_kv_heads, p.slot_cap, p.status, 141)], p.slot_cap, p.status, 142)];
    Unit x{};
    x.grp_begin = it.grp_begin;
    x.rows = min(kRows, (p.grp_ptr[it.seg + 1] - it.grp_begin) * p.gqa);
    x.part_base = it.part_base;
    x.kvh = u % p.num_kv_heads;
    x.tok_count = it.tok_count;
    x.ntile = (it.tok_count + kTile - 1) / kTile;
    if (n >= kUnits && !wait(&sm.unit_empty[n % kUnits], n / kUnits - 1, p)) return;
    sm.unit[n % kUnits] = x;
    mbar_arrive(&sm.unit_full[n % kUnits]);
    const char* src = p.pool_layer + (uint64_t)x.kvh * p.head_stride +
                      (uint64_t)GF_CLAMP(it.tile0 - p.tile_base, p.cap_tiles, p.status, 143) * kv4_tile_bytes(D);
    for (int t = 0; t < x.ntile; ++t, src += kv4_tile_bytes(D)) {
      const int st = tile % kStages;
      if (tile >= kStages && !wait(&sm.stage_empty[st], tile / kStages - 1, p)) return;
      mbar_arrive_expect_tx(&sm.stage_full[st], kv4_tile_bytes(D));
      bulk_g2s(sm.stage[st], src, kv4_tile_bytes(D), &sm.stage_full[st]);
      ++tile;
    }
    u = next;
  }
  if (n >= kUnits && !wait(&sm.unit_empty[n % kUnits], n / kUnits - 1, p)) return;
  sm.unit[n % kUnits].rows = -1;
  mbar_arrive(&sm.unit_full[n % kUnits]);
}
template <int D>
__device__ __forceinline__ void produce(Smem<D>& sm, const Params& p, int num_units, int lane) {
  if (lane != 0) return;
  int tile = 0;
  stream_units(sm, p, num_units, tile);
  for (int t = max(0, tile - kStages); t < tile; ++t) mbar_drain(&sm.stage_full[t % kStages], (t / kStages) & 1, p.status);
}

// ---- warps 4-7: queries and codes --------------------------------------------------------------------------
// 32 query rows of the warp: fp16 times a power of two per row.
template <int D>
__device__ __forceinline__ void load_queries(Smem<D>& sm, const Params& p, const Unit& u, int row0, int lane) {
  constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;  // lanes per row, rows per load
  const int g = p.gqa, own = row0 + lane;
  int at = -1;  // the lane's own row among the queries' rows
  if (own < u.rows) {
    const int req = GF_CLAMP(p.grp_req[GF_CLAMP(u.grp_begin + own / g, p.num_pairs, p.status, 144)], p.num_requests, p.status, 145);
    at = req * p.num_q_heads + u.kvh * g + own % g;
  }
  const int chunk = lane % kLanes;
#pragma unroll
  for (int j0 = 0; j0 < kLanes; j0 += 8) {
    uint4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int from = __shfl_sync(0xffffffffu, at, (j0 + j) * kAtOnce + lane / kLanes);
      v[j] = from >= 0 ? reinterpret_cast<const uint4*>(p.q + (size_t)from * D)[chunk] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = row0 + (j0 + j) * kAtOnce + lane / kLanes;
      const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
      float big = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) big = fmax3(big, fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u)));
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
      const float mul = pow2_to(big, 14);
      uint32_t h[4];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = pack_f16(__uint_as_float(w[i] << 16) * mul, __uint_as_float(w[i] & 0xffff0000u) * mul);
        const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        sum += r.x + r.y;
      }
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (chunk % 8 == 0) {
        __half hi, lo;
        split_f16(sum * 0x1p-6f, hi, lo);  // up to 2^15; the other factor has the 2^6
        *reinterpret_cast<uint2*>(sm.q_sum + sums_offset(row, chunk / 8)) = make_uint2(pair_of(hi, hi), pair_of(lo, lo));
      }
      *reinterpret_cast<uint4*>(sm.q[chunk / 8] + swz128(row, chunk % 8)) = make_uint4(h[0], h[1], h[2], h[3]);
      if (chunk == 0) sm.row_scale[row] = p.scale_log2 * pow2_inverse(mul);
    }
  }
}

// Block b (16 tokens) of a tile's K: s (c - 8), which eleven bits hold (eight of s, three of c - 8), times a power of two
// that brings the token's largest value (or each group's, see kNearGroups) to 2^8..2^9; and lo + 8.5 s beside it.  1024 + c
// and 1024 + 16 c are fp16 patterns with the code in their low bits.
template <int D>
__device__ __forceinline__ void expand_k(Smem<D>& sm, Scales& to, const char* part, int b, int lane) {
  constexpr int NG = D / kGroup4;
  const int l4 = lane & 3, l8 = lane >> 2, own = b * 16 + (lane & 15);
  // a token's numbers per lane (twice)
  float s[NG], lo[NG], big[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const uint32_t sl = reinterpret_cast<const uint32_t*>(part + kv4_code_bytes(D))[own * NG + g];
    s[g] = kv4_s(sl);
    lo[g] = kv4_lo(sl);
    big[g] = fmaxf(fabsf(lo[g]), fabsf(fmaf(16.f, s[g], lo[g])));
  }
  bool apart = false;
  if (NG == 2) {
    const float least = fminf(big[0], big[NG - 1]), most = fmaxf(big[0], big[NG - 1]);
    apart = __any_sync(0xffffffffu, least > 0.f && (__float_as_uint(most) >> 23) - (__float_as_uint(least) >> 23) > kNearGroups);
    if (!apart) big[0] = big[NG - 1] = most;
    if (lane == 0) to.apart[b] = apart;
  }
  uint32_t step[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float mul = pow2_to(big[g], 8);
    step[g] = pack_f16(s[g] * mul, s[g] * mul);
    if (lane < 16) {
      __half hi, rest;
      split_f16(fmaf(8.5f, s[g], lo[g]) * (mul * 64.f), hi, rest);
      const uint32_t z = pair_of(hi, rest);
      const bool second = g == 1 && apart;
      *reinterpret_cast<uint2*>(sm.k_mid[0] + sums_offset(own, g)) = second ? make_uint2(0u, 0u) : make_uint2(z, z);
      if (g == 1) *reinterpret_cast<uint2*>(sm.k_mid[NG - 1] + sums_offset(own, g)) = second ? make_uint2(z, z) : make_uint2(0u, 0u);
      to.k[g][own] = pow2_inverse(mul);
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const uint4 c = reinterpret_cast<const uint4*>(part)[(b * NG + g) * 32 + lane];
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t mask = h ? 0x00f000f0u : 0x000f000fu, row = b * 16 + l8 + 8 * h, token = __shfl_sync(0xffffffffu, step[g], l8 + 8 * h);
      const __half2 by = *reinterpret_cast<const __half2*>(&token);
      uint32_t x[8];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t code = ((e ? w[kk] >> 8 : w[kk]) & mask) | 0x64006400u;
          const __half2 c2 = *reinterpret_cast<const __half2*>(&code);
          const __half2 v = __hmul2(h ? __hfma2(c2, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hadd2(c2, __float2half2_rn(-1032.f)), by);
          x[2 * kk + e] = *reinterpret_cast<const uint32_t*>(&v);
        }
      *reinterpret_cast<uint4*>(sm.k[g] + swz128(row, l4)) = make_uint4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<uint4*>(sm.k[g] + swz128(row, 4 + l4)) = make_uint4(x[4], x[5], x[6], x[7]);
    }
  }
}

// Block b of V: a token's codes are one byte of every word; even entries in units of 2^-24, odd ones of 2^-20.
template <int D>
__device__ __forceinline__ void expand_v(Smem<D>& sm, const char* part, int b, int lane) {
  constexpr int NG = D / kGroup4;
  const int l4 = lane & 3, l8 = lane >> 2;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const uint4 c = reinterpret_cast<const uint4*>(part)[(b * NG + g) * 32 + lane];
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {  // token 2 l4 + (t & 1) + 8 (t / 2): byte 2 (t & 1) + t / 2
      const uint32_t row = b * 16 + 2 * l4 + (t & 1) + 8 * (t >> 1), byte = 2 * (t & 1) + (t >> 1);
      uint32_t x[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) x[kk] = __byte_perm(w[kk], 0u, 0x4040u | byte | (byte << 8)) & 0x00f0000fu;
      *reinterpret_cast<uint4*>(sm.v[g] + swz128(row, l8)) = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
}

// The scales of block b of V: a token and a group per lane.
template <int D>
__device__ __forceinline__ void expand_scales(Scales& to, const char* part, int b, int lane) {
  constexpr int NG = D / kGroup4;
  const int t = b * 16 + (lane & 15), g = lane >> 4;
  if (g >= NG) return;
  const uint32_t sl = reinterpret_cast<const uint32_t*>(part + kv4_code_bytes(D))[t * NG + g];
  const float s = kv4_s(sl);
  to.s[g][t] = s;
  to.z[g][t] = fmaf(0.5f, s, kv4_lo(sl));
}

template <int D>
__device__ __forceinline__ void expand(Smem<D>& sm, const Params& p, int w, int lane) {
  int tile = 0, step = 0;  // the next one, and its first step
  for_units(sm, p, lane, [&](int n, const Unit& u) {
    // the unit before has its last scores, and its rows' scales have been read
    if (n > 0 && (!wait_step(sm.s_full, step - 1, p) || !wait(&sm.q_empty, n - 1, p))) return false;
    load_queries(sm, p, u, w * 32, lane);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.q_full);
    for (int left = u.tok_count; left > 0; left -= kTile, ++tile) {
      const int st = tile % kStages;
      if (!wait(&sm.stage_full[st], tile / kStages, p)) return false;
      const char* at = reinterpret_cast<const char*>(sm.stage[st]);
      if (tile > 0 && !wait_step(sm.s_full, step - 1, p)) return false;  // K of the tile before has been read
      // (scales: tile - 1 and tile - 2 may still be in the softmax, tile - 3 not)
      expand_scales<D>(sm.scales[st], at + kv4_part_bytes(D), w, lane);
      expand_k<D>(sm, sm.scales[st], at, w, lane);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.k_full);
      if (tile > 0 && !wait_step(sm.o_full, step - 1, p)) return false;  // and V
      expand_v<D>(sm, at + kv4_part_bytes(D), w, lane);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sm.v_full);
        mbar_arrive(&sm.stage_empty[st]);
      }
      step += left > kSub ? 2 : 1;
    }
    return true;
  });
}

// ---- warp 9: MMAs ----------------------------------------------------------------------------------------
// Tensor memory: S of step i at columns 32 (i % 2), the second group's at 64 + 32 (i % 2) where it has one of its own, P of
// group g over 16 g of the first; O of group g at 128 + 64 g.  The scores of a step are formed while the softmax works on
// the step before.  (MMAs run in the order of their issue: P of step i has been read when S of step i + 2 is written.
// Each commit takes the issuing thread as long as an MMA, 60 cycles, so there are two per step and every role takes them
// for what it waits for.)
template <int D>
__device__ __forceinline__ bool any_apart(const Scales& s) {
  const int4 x = *reinterpret_cast<const int4*>(s.apart);
  return D == 128 && (x.x | x.y | x.z | x.w) != 0;
}
template <int D>
__device__ __forceinline__ void issue_scores(Smem<D>& sm, uint32_t tmem, uint32_t buf, uint32_t sub, bool apart) {
  constexpr uint32_t idesc = idesc_f16(kRows, kSub, false);
#pragma unroll
  for (int g = 0; g < D / kGroup4; ++g) {
    const uint64_t qd = tc_smem_desc(smem_u32(sm.q[g]), 0, 1024), kd = tc_smem_desc(smem_u32(sm.k[g]), 0, 1024) + sub * (kSub * 128 >> 4);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)  // 16 entries each
      umma_ss(tmem + 32 * buf + (apart ? 64 * g : 0), qd + 2 * ks, kd + 2 * ks, idesc, (apart ? 0 : g) + ks > 0 ? 1u : 0u);
  }
  umma_ss(tmem + 32 * buf, sums_desc(smem_u32(sm.q_sum)), sums_desc(smem_u32(sm.k_mid[0]) + sub * (kSub * 32)), idesc, 1u);
  if (apart) umma_ss(tmem + 64 + 32 * buf, sums_desc(smem_u32(sm.q_sum)), sums_desc(smem_u32(sm.k_mid[D / kGroup4 - 1]) + sub * (kSub * 32)), idesc, 1u);
  tc_commit(&sm.s_full[buf]);
}
template <int D>
__device__ __forceinline__ void issue_mmas(Smem<D>& sm, const Params& p, int lane) {
  constexpr uint32_t idesc_o = idesc_f16(kRows, kGroup4, true);
  const uint32_t tmem = __shfl_sync(0xffffffffu, sm.tmem_base, 0);  // (the shuffles tell that every lane has the same)
  int step = 0, tile = 0;  // the unit's first
  for_units(sm, p, lane, [&](int n, const Unit& u) {
    const int steps = __shfl_sync(0xffffffffu, (u.tok_count + kSub - 1) / kSub, 0);
    if (!wait(&sm.q_full, n, p)) return false;
    bool apart = false;  // of the tile whose scores are formed
    for (int i = -1; i < steps; ++i) {
      const uint32_t next = step + i + 1;
      if (i + 1 < steps) {  // the next step's scores
        if ((i + 1) % 2 == 0) {
          if (!wait(&sm.k_full, tile + (i + 1) / 2, p)) return false;
          apart = any_apart<D>(sm.scales[(tile + (i + 1) / 2) % kStages]);
        }
        tc_fence_after_sync();
        if (lane == 0) issue_scores<D>(sm, tmem, next & 1, (i + 1) & 1, apart);
        __syncwarp();
      }
      if (i < 0) continue;
      const uint32_t buf = (step + i) & 1;
      if (i == 0 && n > 0 && !wait(&sm.o_empty, n - 1, p)) return false;  // the unit before has read its O
      if (i % 2 == 0 && !wait(&sm.v_full, tile + i / 2, p)) return false;
      if (!wait_step(sm.p_full, step + i, p)) return false;
      tc_fence_after_sync();
      if (lane == 0) {
#pragma unroll
        for (int g = 0; g < D / kGroup4; ++g) {
          const uint64_t vd = tc_smem_desc(smem_u32(sm.v[g]), 0, 1024) + (i & 1) * (kSub * 128 >> 4);
#pragma unroll
          for (int ks = 0; ks < kSub / 16; ++ks)  // 16 token rows = 2048 bytes per MMA
            umma_ts(tmem + 128 + 64 * g, tmem + 32 * buf + 16 * g + 8 * ks, vd + ks * (2048 >> 4), idesc_o, (i > 0 || ks > 0) ? 1u : 0u);
        }
        tc_commit(&sm.o_full[buf]);
      }
      __syncwarp();
    }
    step += steps;
    tile += (steps + 1) / 2;
    return true;
  });
  if (lane == 0) {  // (every MMA is waited for already, unless a wait gave up)
    tc_commit(&sm.mmas_done);
    mbar_drain(&sm.mmas_done, 0, p.status);
  }
}

// ---- warps 0-3: softmax ------------------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void softmax(Smem<D>& sm, const Params& p, int warp, int lane) {
  constexpr int NG = D / kGroup4;
  const int row = warp * 32 + lane;
  const uint32_t lanes = sm.tmem_base + ((uint32_t)(warp * 32) << 16);
  int step = 0, tile0 = 0;
  for_units(sm, p, lane, [&](int n, const Unit& u) {
    if (!wait(&sm.q_full, n, p)) return false;
    const float scale = sm.row_scale[row];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.q_empty);
    float top = -INFINITY;    // the reference's score, in log2 units
    float f[2] = {1.f, 1.f};  // as in decode4.cu
    uint64_t l2 = 0, oz[2] = {0, 0};
    for (int left = u.tok_count, i = 0; left > 0; left -= kSub, ++i, ++step) {
      // this step's tokens: scales as float4 of group g's tokens 4 k .. + 3
      const Scales& vs = sm.scales[(tile0 + i / 2) % kStages];
      const int at = (i & 1) * kSub;
      auto quad = [&](const float (&a)[2][kTile], int g, int k) { return *reinterpret_cast<const float4*>(&a[g][at + 4 * k]); };
      auto half = [](const float4& v, int h) { return h ? f2_pack(v.z, v.w) : f2_pack(v.x, v.y); };
      const uint32_t cols = lanes + 32 * (step & 1);
      if (!wait_step(sm.s_full, step, p)) return false;
      tc_fence_after_sync();
      // the largest s per group (not negative: its bits order as it does)
      float big_s[2];
#pragma unroll
      for (int g = 0; g < NG; ++g) big_s[g] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(vs.s[g][at + lane])));
      // scores of token pairs, in units of 1 / scale
      uint64_t x[kSub / 2];
      {
        uint32_t a[kSub];
        tmem_ld32(cols, a);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < kSub / 4; ++k) {
          const float4 f = quad(vs.k, 0, k);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            x[2 * k + h] = f2_mul(f2_pack(__uint_as_float(a[4 * k + 2 * h]), __uint_as_float(a[4 * k + 2 * h + 1])), half(f, h));
        }
      }
      if (any_apart<D>(vs)) {  // the second group's
#pragma unroll
        for (int c0 = 0; c0 < kSub; c0 += 16) {
          uint32_t a[16];
          tmem_ld16(cols + 64 + c0, a);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 f = quad(vs.k, 1, c0 / 4 + k);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint64_t& to = x[c0 / 2 + 2 * k + h];
              to = f2_fma(f2_pack(__uint_as_float(a[4 * k + 2 * h]), __uint_as_float(a[4 * k + 2 * h + 1])), half(f, h), to);
            }
          }
        }
      }
      if (left < kSub) {
#pragma unroll
        for (int k = 0; k < kSub / 2; ++k) {
          float lo, hi;
          f2_unpack(x[k], lo, hi);
          x[k] = f2_pack(2 * k < left ? lo : -INFINITY, 2 * k + 1 < left ? hi : -INFINITY);
        }
      }
      float m = -INFINITY, m1 = -INFINITY;
#pragma unroll
      for (int k = 0; k < kSub / 2; k += 2) {
        float lo, hi;
        f2_unpack(x[k], lo, hi);
        m = fmax3(m, lo, hi);
        f2_unpack(x[k + 1], lo, hi);
        m1 = fmax3(m1, lo, hi);
      }
      m = fmaxf(m, m1) * scale;
      bool move = m > top + 8.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) move |= big_s[g] * f[g] > 128.f;
      if (__any_sync(0xffffffffu, move)) {
        if (i > 0 && !wait_step(sm.o_full, step - 1, p)) return false;  // the products so far are in O
        tc_fence_after_sync();
        const float new_top = fmaxf(top, m), r = fast_exp2(top - new_top);  // (0 for the unit's first step)
        top = new_top;
        const uint64_t r2 = f2_pack(r, r);
        l2 = f2_mul(l2, r2);
        float big[2] = {0.f, 0.f};  // the row's largest p s of the step
#pragma unroll
        for (int k = 0; k < kSub / 2; ++k) {
          float lo, hi;
          f2_unpack(x[k], lo, hi);
          lo = fast_exp2(fmaf(lo, scale, -top));
          hi = fast_exp2(fmaf(hi, scale, -top));
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const float2 s2 = *reinterpret_cast<const float2*>(&vs.s[g][at + 2 * k]);
            big[g] = fmax3(big[g], lo * s2.x, hi * s2.y);
          }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          oz[g] = f2_mul(oz[g], r2);
          const float inv = pow2_inverse(f[g]), fn = pow2_to(fmaxf(4.f * inv * r, big[g]), 2), ratio = fn * r * inv;
          f[g] = fn;
          if (i > 0) {
#pragma unroll
            for (int c0 = 64 * g; c0 < 64 * g + 64; c0 += 16) {
              uint32_t o[16];
              tmem_ld16(lanes + 128 + c0, o);
              tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * ratio);
              tmem_st16(lanes + 128 + c0, o);
            }
          }
        }
      }
      // p, l, the second term of O, and p s f over the scores
      const uint64_t scale2 = f2_pack(scale, scale), ref2 = f2_pack(-top, -top), f0 = f2_pack(f[0], f[0]), f1 = f2_pack(f[1], f[1]);
#pragma unroll
      for (int c0 = 0; c0 < kSub; c0 += 16) {
        uint32_t pk[2][8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int kk = c0 / 4 + k;
          const float4 s0 = quad(vs.s, 0, kk), z0 = quad(vs.z, 0, kk);
          float4 s1, z1;
          if (NG == 2) { s1 = quad(vs.s, 1, kk); z1 = quad(vs.z, 1, kk); }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float lo, hi;
            f2_unpack(f2_fma(x[(c0 + 4 * k + 2 * h) >> 1], scale2, ref2), lo, hi);
            const uint64_t pr = f2_pack(fast_exp2(lo), fast_exp2(hi));
            l2 = f2_add(l2, pr);
            oz[0] = f2_fma(pr, half(z0, h), oz[0]);
            f2_unpack(f2_mul(f2_mul(pr, f0), half(s0, h)), lo, hi);
            pk[0][2 * k + h] = pack_f16(lo, hi);
            if (NG == 2) {
              oz[1] = f2_fma(pr, half(z1, h), oz[1]);
              f2_unpack(f2_mul(f2_mul(pr, f1), half(s1, h)), lo, hi);
              pk[1][2 * k + h] = pack_f16(lo, hi);
            }
          }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) tmem_st8(cols + 16 * g + c0 / 2, pk[g]);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.p_full[step & 1]);
    }
    tile0 += u.ntile;
    // the unit's partial
    if (!wait_step(sm.o_full, step - 1, p)) return false;
    tc_fence_after_sync();
    const int slot = u.part_base + row / p.gqa;
    const bool ok = row < u.rows && GF_CHECK(slot < p.slot_cap, p.status, 146);
    const size_t ph = ok ? (size_t)slot * p.num_q_heads + u.kvh * p.gqa + row % p.gqa : 0;
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += 32) {
      uint32_t o[32];
      tmem_ld32(lanes + 128 + c0, o);
      tmem_wait_ld();
      float z, zhi;
      f2_unpack(oz[c0 / kGroup4], z, zhi);
      z += zhi;
      const float inv = pow2_inverse(f[c0 / kGroup4]);
      if (ok) {
        float4* to = reinterpret_cast<float4*>(p.part_o + ph * D + c0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(__uint_as_float(o[4 * i + e]) * inv, (e & 1) ? kUnit1 : kUnit0, z);
          to[i] = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.o_empty);
    float l, lhi;
    f2_unpack(l2, l, lhi);
    if (ok) *reinterpret_cast<float2*>(p.part_ml + ph * 2) = make_float2(top, l + lhi);
    return true;
  });
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_decode4_wide(const Params p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kUnits; ++i) { mbar_init(&sm.unit_full[i], 1); mbar_init(&sm.unit_empty[i], kUnitReaders); }
    for (int i = 0; i < kStages; ++i) { mbar_init(&sm.stage_full[i], 1); mbar_init(&sm.stage_empty[i], 4); }
    mbar_init(&sm.q_full, 4);
    mbar_init(&sm.k_full, 4);
    mbar_init(&sm.v_full, 4);
    mbar_init(&sm.o_empty, 4);
    mbar_init(&sm.q_empty, 4);
    for (int i = 0; i < 2; ++i) { mbar_init(&sm.s_full[i], 1); mbar_init(&sm.p_full[i], 4); mbar_init(&sm.o_full[i], 1); }
    mbar_init(&sm.mmas_done, 1);
    mbar_fence_init();
  }
  chain_enter();
  const int num_units = tables_usable(*p.hdr, p.slot_cap) ? p.hdr->kv4_wide * p.num_kv_heads : 0;
  if (num_units > 0) {  // uniform over the launch
    for (int i = threadIdx.x; i < (int)sizeof(sm.q_sum) / 16; i += kThreads) reinterpret_cast<uint4*>(sm.q_sum)[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = threadIdx.x; i < (int)sizeof(sm.k_mid) / 16; i += kThreads) reinterpret_cast<uint4*>(sm.k_mid)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    if (warp == 9) tmem_alloc(&sm.tmem_base, 256);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp < 4) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
      softmax<D>(sm, p, warp, lane);
    } else if (warp < 8) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kExpandRegs));
      expand<D>(sm, p, warp - 4, lane);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kControlRegs));
      if (warp == 8) produce<D>(sm, p, num_units, lane);
      if (warp == 9) issue_mmas<D>(sm, p, lane);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 9) tmem_dealloc(sm.tmem_base, 256);
  }
  // the last CTA to run out of work re-arms the counters for the next launch
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&p.counters[1], 1) == (int)gridDim.x - 1) {
      p.counters[0] = 0;
      p.counters[1] = 0;
    }
  }
}

}  // namespace

int launch_decode4_wide(const PoolGeom& pool, const AttnShape& sh, const TablesDev& t, int units, int layer, const void* q,
                        int32_t* status, bool chained, cudaStream_t st) {
  if (units == 0) return 0;
  Params p;
  p.pool_layer = pool.base + (uint64_t)layer * pool.layer_stride;
  p.head_stride = pool.head_stride;
  p.tile_base = t.kv4_tile0;
  p.items = t.items;
  p.list = t.wide_list;
  p.grp_ptr = t.grp_ptr;
  p.grp_req = t.grp_req;
  p.q = (const __nv_bfloat16*)q;
  p.part_o = t.part_o;
  p.part_ml = t.part_ml;
  p.status = status;
  p.counters = status + kStatusKv4WideQueue;
  p.hdr = t.hdr;
  p.slot_cap = t.slot_cap;
  p.num_q_heads = sh.num_q_heads;
  p.num_kv_heads = sh.num_kv_heads;
  p.gqa = sh.num_q_heads / sh.num_kv_heads;
  p.scale_log2 = sh.scale_log2;
  p.cap_tiles = (int32_t)pool.cap_tiles;
  p.num_pairs = t.num_pairs_in;
  p.num_requests = t.num_requests;
  const long long work = units < 0 ? (1ll << 40) : (long long)units * sh.num_kv_heads, most = 2ll * t.num_sms;
  const dim3 grid((unsigned)(work < most ? work : most));
  auto go = [&](auto kernel, size_t smem, bool (&optin)[kMaxDevices]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    if (dev >= kMaxDevices || !optin[dev]) {
      // (a build that gives the kernel fewer registers would leave the roles waiting for their shares)
      cudaFuncAttributes attr;
      if (cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || allocated_regs(attr.numRegs) != kLaunchRegs) return false;
    }
    if (!ensure_dynamic_smem(kernel, smem, optin)) return false;
    if (chained) launch_chained(kernel, grid, dim3(kThreads), smem, st, p);
    else kernel<<<grid, dim3(kThreads), smem, st>>>(p);  // behind an event of another stream
    return true;
  };
  static bool optin[2][kMaxDevices] = {};
  if (!(sh.head_dim == 128 ? go(k_decode4_wide<128>, sizeof(Smem<128>), optin[0]) : go(k_decode4_wide<64>, sizeof(Smem<64>), optin[1]))) return -1;
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace gf
