// A projection that all rows share, with a low-rank adapter of each row's own:
//   y[t] = W x[t] + scale_a B_a (A_a x[t]),  a the row's adapter.
//
// W x: tcgen05 MMAs with the output features as the MMA's rows (128 of W at a time, K-major) and up to 256 rows of x as its
// columns, so that one row and thousands go the same way; both operands come by TMA in stages of 64 entries of K, the sums stay in
// tensor memory in fp32.  256 rows and more: two CTAs share a tile of 256 features (cta_group::2).  Few rows leave few tiles: then a cluster of CTAs shares a tile, each with a part of K, and
// joins its parts through shared memory in a fixed order.
//
// The adapters are more entries of K.  For every adapter that rows of a tile of x name (a slot of the tile), h = scale_a A_a x is a
// [rows, rank] operand with zeros in the other rows, and B_a, [features, rank], stands beside W: the sums go on over the tile's
// slots, in the same pipeline, and nothing is left for the warps that take them out of tensor memory.  h is held in two bf16
// numbers, its nearest and the nearest of what is left (off by 2^-17 of it at most: less than a result's rounding unless W x nearly takes the adapter's part away), and
// multiplied twice; for results in fp32 in three (2^-26), the least first and into an empty accumulator.
// A x goes the same way as W x: the rows of the A of 8, 4 or 2 slots (of rank 16, 32, 64) stand in W's place, for all rows of the tile, and
// what comes out is kept where row and slot belong together and written as those operands.
// Three launches: the slots, A x, W x; only the copies behind a tile's last entry of W wait for the second.  (Few rows: the first two are
// one, k_adapter_rows.)
//
// Results in fp32: tensor memory's sums are cut off, not rounded, where an MMA adds to them, each of its products at some 2^-24 of the sum (measured, K = 4096: 4.4e-6 of the
// result with products of either sign, 1e-4 with products of one; 32 768: 5e-4), so every 8 stages they are taken out and added, rounded, to sums that stand beside
// them; 2.4e-7 (one sign) to 5e-7 is left at any K.  (Those sums in registers spilled.)  Results in bf16 take them out once: a take-out in between stops the MMAs
// (8192 rows 380 us in place of 275), for digits that their rounding, 4e-3, takes away.
//
// Measured, 4096 -> 6144 in bf16: one row 11.4 us, where W alone is 7.8 of HBM (launch, the first copies and the join of 6 parts are the rest); 256 rows 20.1,
// with 64 adapters of rank 16 37 (their stages are half as many as W's, in 96 CTAs: clusters of 6 do not all find room); 8192 rows 275 us, 1500
// TFLOP/s, tensor pipe 85 % busy.  64 rows of 4096 -> 128 000 in fp32: 176 to 190 us, 5.7 to 6.2 TB/s of W and results.
//
// (The same sums on the CUDA cores, while the MMAs ran, took 568 us for 8192 rows with adapters of rank 16 and 1143 of rank 64,
// where W x alone took 295: their reads of B and h wait behind the copies' traffic.)
#include <cuda.h>

#include <algorithm>

#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kFeat = 128;        // output features of a tile
constexpr int kStep = 64;         // entries of K in a stage
constexpr int kThreads = 256;
constexpr int kWideThreads = 384; // with eight warps that take the sums out
constexpr int kChunk = 8;         // fp32 results: stages after which the sums are taken out
constexpr int kPanel = 8;         // tiles of x that the tiles of W go over together, so that those at work at once read few rows of either:
                                  // 8192 rows of 4096 -> 28672 take 1530 us with 1, 1230 with 8
constexpr int kGroup = 8;         // rows of x that are taken out of tensor memory together

// The slots of the tiles of x, in the caller's scratch.
struct Slots {
  int32_t* count;        // [row_tiles]
  int32_t* adapter;      // [row_tiles][most]
  int32_t* of_row;       // [rows] a row's slot in its tile, -1: none
  const float* scale;    // [num_adapters] or null
  char* h;               // [row_tiles][most][numbers][nt][padded rank], read by TMA like the others
  int most;
  int numbers;           // that h is held in: 2 or 3
  int rank, padded;      // padded: 16, 32 or 64
  uint32_t block;        // bytes of one [nt][padded]
};

struct ProjectArgs {
  int rows, in_dim, out_dim, nt;        // nt: rows of x in a tile
  int feat_tiles, row_tiles, stages;
  int pair;                             // stages that share their barriers: 1 or 2
  int two;                              // two CTAs a tile
  int splits;                           // CTAs that share a tile
  uint32_t tmem_cols, acc_cols;         // allocated; from one accumulator to the next
  int accs;                             // accumulators: 1 or 2
  uint32_t sum_cols;                    // fp32: where the sums stand
  Slots slots;
  void* y;
  int64_t y_stride;
  int y_fp32, y_vec;                    // y_vec: four neighbouring results can be stored at once
  int32_t* status;
  // what a single result is worked out from (rework)
  const __nv_bfloat16 *w, *x, *b;
  int64_t w_stride, x_stride;
  const int32_t* adapter;               // [rows] as given
  int num_adapters;
};

// kTwo: the CTA is one of two that work on one tile with MMAs of both (cta_group::2), the even one, which issues them, the leader.  Each brings
// its own half of either operand; all of a stage's bytes count on the leader's barrier, whose address in the cluster `bar` is.
template <bool kTwo>
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (kTwo)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
template <bool kTwo>
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if constexpr (kTwo)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
// The address in the cluster of CTA `rank`'s copy of what is at p here.
__device__ __forceinline__ uint32_t at_rank(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// An arrival at another CTA's barrier; what this thread has done is seen there (kRelease), or it has done nothing that is to be.  (A thread with
// copies on the way waits for long in a release: 1500 cycles a stage.)
template <bool kRelease>
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  if constexpr (kRelease) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <bool kTwo>
__device__ __forceinline__ void tmem_take(uint32_t* dst_smem, uint32_t ncols) {
  if constexpr (kTwo) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tmem_alloc(dst_smem, ncols);
  }
}
template <bool kTwo>
__device__ __forceinline__ void tmem_give(uint32_t taddr, uint32_t ncols) {
  if constexpr (kTwo) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
  else tmem_dealloc(taddr, ncols);
}
// The barrier gets one arrival when all MMAs issued so far have ended; or that of both CTAs (mask: theirs in the cluster) does.
template <bool kTwo>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (kTwo) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
  else tc_commit(bar);
}
template <bool kTwo>
__device__ __forceinline__ void commit_both(uint64_t* bar, uint16_t mask) {
  if constexpr (kTwo)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"(mask) : "memory");
  else tc_commit(bar);
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

// Shared-memory matrix descriptor of a K-major operand whose rows are `row_bytes` (32, 64 or 128) long and swizzled over that many.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, int row_bytes) {
  const uint64_t kind = row_bytes == 128 ? 2 : row_bytes == 64 ? 4 : 6;
  return (tc_smem_desc(saddr, 0, 8 * row_bytes) & ~((uint64_t)7 << 61)) | kind << 61;
}
__device__ __forceinline__ uint64_t bf16x2_to_f2(uint32_t v) { return f2_pack(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }

// Four MMAs along a stage's 64 entries of K, 32 bytes apart in both operands.  (In one block: the issuing thread is alone on its
// scheduler, and with few rows of x its instructions between the MMAs are what takes the time.)
#define GF_MMA4(GROUP)                                                           \
  "{\n\t.reg .pred p, t;\n\t.reg .b64 a, b;\n\t"                                \
  "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"                           \
  "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], %1, %2, %3, p;\n\t"         \
  "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"                                  \
  "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a, b, %3, t;\n\t"           \
  "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"                                  \
  "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a, b, %3, t;\n\t"           \
  "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"                                  \
  "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a, b, %3, t;\n\t}"
template <bool kTwo>
__device__ __forceinline__ void mma4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kTwo) asm volatile(GF_MMA4("2")::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
  else asm volatile(GF_MMA4("1")::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
#undef GF_MMA4
template <bool kTwo>
__device__ __forceinline__ void mma1(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kTwo)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(a_desc),
                 "l"(b_desc), "r"(idesc), "r"(accumulate)
                 : "memory");
  else umma_ss(d_tmem, a_desc, b_desc, idesc, accumulate);
}

__device__ __forceinline__ void store_y(const ProjectArgs& a, int row, int feat, float v) {
  if (feat < a.out_dim && row >= 0 && row < a.rows) {
    const int64_t at = (int64_t)row * a.y_stride + feat;
    if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
    else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
  }
}

// A feature's results for kGroup rows from `row` on.
__device__ __forceinline__ void store_rows(const ProjectArgs& a, int row, int feat, const uint32_t (&r)[kGroup]) {
  const int64_t at = (int64_t)row * a.y_stride + feat;
  const int n = min(kGroup, a.rows - row);
  if (a.y_fp32) {
    float* y = static_cast<float*>(a.y) + at;
#pragma unroll
    for (int j = 0; j < kGroup; ++j, y += a.y_stride)
      if (j < n) *y = __uint_as_float(r[j]);
  } else {
    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + at;
#pragma unroll
    for (int j = 0; j < kGroup; ++j, y += a.y_stride)
      if (j < n) *y = __float2bfloat16_rn(__uint_as_float(r[j]));
  }
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
// Whether a feature's row of a slot's B, of all slots of a tile of x, has an entry that is no finite number.
__device__ __forceinline__ bool spoiled(const ProjectArgs& a, int row_tile, int feat) {
  const int32_t* which = a.slots.adapter + (int64_t)row_tile * a.slots.most;
  const int n = __ldcg(a.slots.count + row_tile), pieces = a.slots.rank / 8;
  auto none = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
  bool found = false;
  for (int i0 = 0; i0 < n; i0 += 8) {
    const uint4* row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row[i] = reinterpret_cast<const uint4*>(a.b + ((int64_t)__ldcg(which + min(i0 + i, n - 1)) * a.out_dim + feat) * a.slots.rank);
    for (int c = 0; c < pieces; ++c) {
      uint4 w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __ldg(row[i] + c);
#pragma unroll
      for (int i = 0; i < 8; ++i) found = found || none(w[i].x) || none(w[i].y) || none(w[i].z) || none(w[i].w);
    }
  }
  return found;
}
// Results that came out of the MMAs as no finite numbers, by the warp that stored them.  Every row of a tile meets the B
// of each of its slots, times zero where the slot is another's, and an infinity or a NaN there makes a NaN of that: where the feature has one, such results are
// worked out anew, each from what belongs to it; the others are what the formula gives.  Bit i of `where` stands for the kGroup rows from row0 + i kGroup step on (of
// those below `end`), with `feats` features from the lane's `feat` on.  The lanes share K: 8 results in some 20 us at K = 4096
// (1024 rows of 4096 -> 6144 under 12 adapters of rank 64: 0.8 ms in place of 0.1 for one such entry, 43 ms where an adapter has nothing else).
__device__ __noinline__ void rework(const ProjectArgs& a, int row_tile, uint32_t where, int row0, int step, int end, int feat, int feats) {
  const Slots& sl = a.slots;
  const int lane = threadIdx.x & 31, n = __ldcg(sl.count + row_tile);
  const int32_t* which = sl.adapter + (int64_t)row_tile * sl.most;
  __syncwarp();  // (the lanes read what others have stored)
  for (int f = feat; f < feat + feats; ++f) {
    for (uint32_t lanes = __ballot_sync(0xffffffffu, f < a.out_dim && spoiled(a, row_tile, f)); lanes; lanes &= lanes - 1) {
      const int of = __ffs(lanes) - 1, col = __shfl_sync(0xffffffffu, f, of);
      const uint4* wr = reinterpret_cast<const uint4*>(a.w + col * a.w_stride);
      for (uint32_t groups = where; groups; groups &= groups - 1) {
        const int first = row0 + (__ffs(groups) - 1) * kGroup * step, mine = first + (lane & (kGroup - 1)) * step;
        bool wrong = lane < kGroup && mine < end;
        if (wrong) {
          const int64_t at = (int64_t)mine * a.y_stride + col;
          wrong = !finite(a.y_fp32 ? static_cast<float*>(a.y)[at] : __bfloat162float(static_cast<__nv_bfloat16*>(a.y)[at]));
        }
        const uint32_t todo = __ballot_sync(0xffffffffu, wrong);
        if (todo == 0) continue;
        float sum[kGroup] = {};
        for (int k = lane; k < a.in_dim / 8; k += 32) {
          const uint4 p = __ldg(wr + k);
          const uint64_t p0 = bf16x2_to_f2(p.x), p1 = bf16x2_to_f2(p.y), p2 = bf16x2_to_f2(p.z), p3 = bf16x2_to_f2(p.w);
#pragma unroll
          for (int j = 0; j < kGroup; ++j) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(a.x + min(first + j * step, end - 1) * a.x_stride) + k);
            float lo, hi;
            f2_unpack(f2_fma(p0, bf16x2_to_f2(q.x), f2_fma(p1, bf16x2_to_f2(q.y), f2_fma(p2, bf16x2_to_f2(q.z), f2_fma(p3, bf16x2_to_f2(q.w), 0ull)))), lo, hi);
            sum[j] += lo + hi;
          }
        }
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
          const int row = min(first + j * step, end - 1), id = a.adapter[row];
          int own = -1;  // the row's slot
          for (int i0 = 0; i0 < n && own < 0; i0 += 32) {
            const uint32_t here = __ballot_sync(0xffffffffu, i0 + lane < n && __ldcg(which + min(i0 + lane, n - 1)) == id);
            if (here) own = i0 + __ffs(here) - 1;
          }
          if (own >= 0) {
            const __nv_bfloat16* b = a.b + ((int64_t)id * a.out_dim + col) * sl.rank;
            const char* h = sl.h + ((int64_t)row_tile * sl.most + own) * sl.numbers * sl.block + (int64_t)(row - row_tile * a.nt) * sl.padded * 2;
            for (int i = lane; i < sl.rank; i += 32) {
              float value = 0.f;
              for (int c = 0; c < sl.numbers; ++c) value += __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(h + c * sl.block)[i]);
              sum[j] = fmaf(__bfloat162float(b[i]), value, sum[j]);
            }
          }
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], d);
          if (lane == j && (todo >> j & 1u)) store_y(a, mine, col, sum[j]);
        }
      }
    }
  }
}

// (a warp's lanes together; every warp of every CTA of the cluster takes part in each barrier)
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// What a launch is: W x alone, W x with the adapters behind it, or A x for the adapters.
enum { kPlain = 0, kWith = 1, kDown = 2 };

// Four results of a row at features f .. f + 3.
__device__ __forceinline__ void store_y4(const ProjectArgs& a, int row, int f, float4 v) {
  const int64_t at = (int64_t)row * a.y_stride + f;
  if (a.y_vec && f + 3 < a.out_dim) {
    if (a.y_fp32) *reinterpret_cast<float4*>(static_cast<float*>(a.y) + at) = v;
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.y) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  } else {
    store_y(a, row, f, v.x);
    store_y(a, row, f + 1, v.y);
    store_y(a, row, f + 2, v.z);
    store_y(a, row, f + 3, v.w);
  }
}
// Where the results of row `m` of a tile of A's go: into a slot's operands, scaled.
struct HPlace {
  char* at;      // the slot's first operand; null: no slot, or beyond the rank's padding
  int slot, r;   // the slot, the rank
  float scale;   // 0 beyond the rank
  __device__ HPlace() : at(nullptr), slot(-1), r(0), scale(0.f) {}
  __device__ HPlace(const Slots& sl, int row_tile, int first_slot, int slots, int m) {
    const int j = m / sl.padded;
    r = m - j * sl.padded;
    slot = first_slot + j;
    at = slot < slots ? sl.h + ((int64_t)row_tile * sl.most + slot) * sl.numbers * sl.block : nullptr;
    scale = 0.f;
    if (at != nullptr && r < sl.rank) scale = sl.scale != nullptr ? __ldg(sl.scale + __ldcg(sl.adapter + (int64_t)row_tile * sl.most + slot)) : 1.f;
  }
};
// v's next number: the nearest bf16 to it; v becomes what is left.  (Nothing is left of an infinity, or a NaN.)
__device__ __forceinline__ __nv_bfloat16 take_number(float& v) {
  const __nv_bfloat16 n = __float2bfloat16_rn(v);
  v = fabsf(v) <= 3.3895e38f ? v - __bfloat162float(n) : 0.f;
  return n;
}
// Four results of neighbouring ranks of a row; zeros where the row is another slot's.  The numbers stand, and are added, from the least to the first:
// an MMA cuts each of its products off at some 2^-24 of the sum that is there, and behind the first number's sum most of the third's would be gone.
__device__ __forceinline__ void store_h(const Slots& sl, const HPlace& p, int row_in_tile, int row_slot, float4 v) {
  if (p.at == nullptr) return;
  const bool mine = row_slot == p.slot && p.r < sl.rank;  // (ranks are multiples of 8)
  v.x = mine ? v.x * p.scale : 0.f;
  v.y = mine ? v.y * p.scale : 0.f;
  v.z = mine ? v.z * p.scale : 0.f;
  v.w = mine ? v.w * p.scale : 0.f;
  char* at = p.at + (row_in_tile * sl.padded + p.r) * 2;
  for (int i = 0; i < sl.numbers; ++i) {
    __align__(8) __nv_bfloat16 n[4] = {take_number(v.x), take_number(v.y), take_number(v.z), take_number(v.w)};
    *reinterpret_cast<uint2*>(at + (sl.numbers - 1 - i) * sl.block) = *reinterpret_cast<uint2*>(n);
  }
}

// Shared memory: the ring of stages (kFeat rows of W, then nt rows of x, 128 bytes each, 128-byte swizzle; a stage of the
// adapters holds a slot's B and as many of its h's numbers as are 128 bytes a row, or two slots of rank 16 with both their numbers),
// which a cluster uses again for its parts of the sums; behind it the barriers.
// Warp 0 issues the copies, warp 1 the MMAs, warps 4 to 7 take the sums out; the parts of a cluster are joined by all.
// kExact: results in fp32, whose sums are taken out by so many warps: 4, or 8 for the tiles of 256 rows, for which tensor memory holds no second
// accumulator to go on in meanwhile.  0: results in bf16.
// kTwo: two CTAs, neighbours in a cluster, share a tile of 256 features and 256 rows of x.  Each has 128 of the features, so its own accumulator, but
// brings only 128 of the rows: what the MMAs read of a stage comes from both, 32 KB a CTA and stage in place of 48, so that there are six stages on
// the way in place of four.  8192 rows of 4096 -> 6144: 277 us, one CTA a tile 319; of 4096 -> 28672: 1192 (1614 TFLOP/s) and 1432.
template <int kMode, int kExact, bool kTwo>
__global__ void __launch_bounds__(kExact == 8 ? kWideThreads : kThreads, kExact == 8 ? 1 : 2) k_project(
    const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap b_map,
    const __grid_constant__ CUtensorMap h_map, const __grid_constant__ ProjectArgs a) {
  constexpr int kWarps = (kExact == 8 ? kWideThreads : kThreads) / 32, kTakers = kWarps - 4, kCtas = kTwo ? 2 : 1, kTileFeat = kFeat * kCtas;
  extern __shared__ __align__(1024) char smem_raw[];
  char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t w_bytes = kFeat * 128u, x_bytes = (uint32_t)a.nt / kCtas * 128u, stage_bytes = w_bytes + x_bytes;
  const bool rounds = kMode == kDown || a.splits > 1;  // the results leave through shared memory, a tile at a time
  const uint32_t ring = max(stage_bytes * a.stages, rounds ? (uint32_t)a.nt * kFeat * 4u : 0u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + ring);
  uint64_t* empty = full + a.stages;
  uint64_t* acc_full = empty + a.stages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* drained = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  uint32_t* gave_up = tmem_slot + 1;  // the CTA has; what a cluster does next goes by those of all its CTAs, so that none leaves alone
  volatile uint32_t* odd_ones = gave_up + 1;  // a result was no finite number (in shared memory: there is no register to spare)
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
  const int size = a.splits * kCtas;  // of a cluster
  const int group = blockIdx.x / size, groups = gridDim.x / size, rank = blockIdx.x - group * size, part = rank / kCtas, half = rank - part * kCtas;
  const bool leader = half == 0;
  const uint16_t both = (uint16_t)(3u << (part * kCtas));
  const int tiles = a.feat_tiles * a.row_tiles;
  const int steps_all = (a.in_dim + kStep - 1) / kStep;
  int step0 = (int)((int64_t)steps_all * part / a.splits), step1 = (int)((int64_t)steps_all * (part + 1) / a.splits);
  const Slots& sl = a.slots;
  const int h_row = sl.padded * 2;                       // bytes of a row of h, and of B's
  const uint32_t b_bytes = kFeat * (uint32_t)h_row, h_bytes = sl.block / kCtas;  // of a slot's B, of a number of its h
  const int per_tile = kMode == kDown ? kFeat / sl.padded : 1;  // slots whose A a tile takes
  auto slots_of = [&](int row_tile) {
    const int n = *(volatile int32_t*)(sl.count + row_tile);
    return GF_CHECK(n >= 0 && n <= sl.most && row_tile < a.row_tiles, a.status, 601) ? n : 0;
  };
  auto adapter_at = [&](const int32_t* which, int i) { return GF_CLAMP(__ldcg(which + i), a.num_adapters, a.status, 602); };  // of a tile's slot i
  // The tiles of a CTA or cluster: features f of W (or slots, from f * per_tile on) and rows r of x.  Those of A x are only as many as there
  // are slots, so a tile of x is left when they end.
  struct Tile { int index, f, r, slots; };
  const int f_step = max(1, groups / a.row_tiles);
  auto more = [&](const Tile& t) { return kMode == kDown ? t.r < a.row_tiles : t.index < tiles; };
  auto settle = [&](Tile& t) {
    if (kMode == kDown) {
      while (t.r < a.row_tiles && t.f * per_tile >= t.slots) {
        t.r += groups;
        t.f = 0;
        t.slots = t.r < a.row_tiles ? slots_of(t.r) : 0;
      }
    } else {
      const int panel = t.index / (a.feat_tiles * kPanel), i = t.index - panel * a.feat_tiles * kPanel, n = min(kPanel, a.row_tiles - panel * kPanel);
      t.f = i / n;
      t.r = panel * kPanel + i - t.f * n;
    }
  };
  auto start = [&] {
    Tile t{group, group / a.row_tiles, group % a.row_tiles, 0};
    if (kMode == kDown) t.slots = slots_of(t.r);
    settle(t);
    return t;
  };
  auto advance = [&](Tile& t) {
    t.index += groups;
    t.f += f_step;
    settle(t);
  };
  if (tid == 0) {
    for (int i = 0; i < a.stages; ++i) { mbar_init(full + i, a.pair); mbar_init(empty + i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, kTakers * kCtas); }
    mbar_init(drained, 1);
    *gave_up = 0;
    *odd_ones = 0;
    mbar_fence_init();
  }
  if (wid == 1) tmem_take<kTwo>(tmem_slot, a.tmem_cols);
  tc_fence_before_sync();
  __syncthreads();
  if (kTwo) cluster_sync_all();  // (the other one's barriers are there)
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  if (kMode == kDown) {
    // (the slots are there when all CTAs of the kernel before have ended; those of the next may start when all of these have begun)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }

  // the stages of n slots
  constexpr int kNumbers = kExact ? 3 : 2;
  const bool two_slots = kNumbers == 2 && h_row == 32;
  const int per_stage = h_row == 128 ? 1 : h_row == 64 ? 2 : 4;  // numbers
  const int a_slot = h_row == 128 ? kNumbers : h_row == 64 ? (kNumbers + 1) / 2 : 1;
  auto slot_stages = [&](int n) { return two_slots ? (n + 1) / 2 : n * a_slot; };

  const int odd = a.pair - 1;  // (a stage's barriers are those at s >> odd)
  int s = 0;           // the role's stage and its phase
  uint32_t phase = 0;
  uint32_t used = 0, phases = 0;  // stages that copies have been issued for, and the last phase of each
  int done = 0;                   // accumulators: tiles, or their chunks
  auto acc_at = [&] { return a.accs == 2 ? done & 1 : 0; };
  auto acc_phase = [&] { return (uint32_t)(a.accs == 2 ? done >> 1 : done) & 1u; };
  auto give_acc = [&] {  // to the thread that issues the MMAs
    if (kTwo) arrive_at<true>(at_rank(acc_empty + acc_at(), part * kCtas));
    else mbar_arrive(acc_empty + acc_at());
  };
  bool ok = true, waited = kMode != kWith;
  // a warp that takes sums out: row m of the tile of W, columns col0 .. col0 + cols (rows of x)
  const int m = (wid & 3) * 32 + lane, cols = kTakers == 8 ? a.nt / 2 : a.nt, col0 = kTakers == 8 && wid >= 8 ? cols : 0;
  const uint32_t lanes = tmem + ((uint32_t)((wid & 3) * 32) << 16);
  // W x of a CTA by itself goes through its tiles in one round, so that the roles run ahead of each other.  A cluster takes a round per tile, and
  // so does A x, whose results are short pieces for places far apart (stored as they come from tensor memory: 31 us for 256 rows).
  Tile now = start();
  while (more(now)) {
    // A x: where there are more than half as many tiles left in a tile of x as the cluster has CTAs, they take one each, with all of K.
    bool whole = false, idle = false;
    if (kMode == kDown) {
      const int left = ((now.slots + per_tile - 1) / per_tile - now.f + f_step - 1) / f_step;
      whole = 2 * left > a.splits;
      idle = whole && part >= left;
      step0 = whole ? 0 : steps_all * part / a.splits;
      step1 = whole ? steps_all : steps_all * (part + 1) / a.splits;
      if (whole) now.f += part * f_step;
    }
    if (idle) {
    } else if (wid == 0) {
      if (lane == 0) {
        // (the leader passes on to the other CTA what it has waited for)
        auto free = [&] {
          if ((s & odd) != 0) return true;
          if (!mbar_wait(empty + (s >> odd), phase ^ 1u, a.status)) return false;
          if (kTwo && leader && (used >> s & 1u)) arrive_at<false>(at_rank(empty + (s >> odd), part * kCtas + 1));
          return true;
        };
        auto next = [&] {
          used |= 1u << s;
          phases = (phases & ~(1u << s)) | phase << s;
          if (++s == a.stages) { s = 0; phase ^= 1u; }
        };
        auto full_at = [&] { return kTwo ? at_rank(full + (s >> odd), part * kCtas) : smem_u32(full + (s >> odd)); };
        auto expect = [&](uint32_t bytes) { if (leader) mbar_arrive_expect_tx(full + (s >> odd), bytes * kCtas); };
        for (Tile t = now; more(t) && ok; advance(t)) {
          const int f = t.f, f0 = f * kTileFeat + half * kFeat, row_tile = t.r, t0 = row_tile * a.nt, mine0 = t0 + half * (a.nt / kCtas);
          const int32_t* which = sl.adapter + (int64_t)row_tile * sl.most;
          int s0 = 0, s1 = 0, ids[8];
          if (kMode == kWith && waited) s1 = slots_of(row_tile);  // (asked for here, used behind the loop)
          if (kMode == kDown) {
            s1 = min(per_tile, t.slots - f * per_tile);
#pragma unroll
            for (int j = 0; j < 8; ++j) ids[j] = j < s1 ? adapter_at(which, f * per_tile + j) : 0;
          }
          for (int k = step0; k < step1; ++k) {
            if (!(ok = free())) break;
            char* at = smem + s * stage_bytes;
            const uint32_t bar = full_at();
            if (kMode == kDown) {
              expect(s1 * sl.rank * 128u + x_bytes);
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (j < s1) tma_load_2d<kTwo>(at + j * sl.padded * 128, &w_map, k * kStep, ids[j] * sl.rank, bar);
            } else {
              expect(stage_bytes);
              tma_load_2d<kTwo>(at, &w_map, k * kStep, f0, bar);
            }
            tma_load_2d<kTwo>(at + w_bytes, &x_map, k * kStep, mine0, bar);
            next();
          }
          if (kMode == kWith && ok) {
            if (!waited) {
              asm volatile("griddepcontrol.wait;" ::: "memory");  // the slots' operands are the kernel's before this one
              waited = true;
              s1 = slots_of(row_tile);
            }
            s0 = s1 * part / a.splits;
            s1 = s1 * (part + 1) / a.splits;
            int ahead[2] = {s0 < s1 ? adapter_at(which, s0) : 0, s0 + 1 < s1 ? adapter_at(which, s0 + 1) : 0};  // of the next two slots
            int y = (row_tile * sl.most + s0) * kNumbers * a.nt + half * (a.nt / kCtas);  // of the next number of h
            for (int i = s0; i < s1 && ok;) {
              const int id = ahead[0], id2 = ahead[1], taken = two_slots && i + 1 < s1 ? 2 : 1;
              i += taken;
              ahead[0] = taken == 2 ? (i < s1 ? adapter_at(which, i) : 0) : id2;
              ahead[1] = i + 1 < s1 ? adapter_at(which, i + 1) : 0;
              for (int j = 0; j < taken * kNumbers;) {
                if (!(ok = free())) break;
                char* at = smem + s * stage_bytes;
                const uint32_t bar = full_at();
                const int n = two_slots ? taken * kNumbers : min(per_stage, kNumbers - j);
                expect(taken * b_bytes + n * h_bytes);
                tma_load_3d<kTwo>(at, &b_map, 0, f0, id, bar);
                if (taken == 2) tma_load_3d<kTwo>(at + b_bytes, &b_map, 0, f0, id2, bar);
                for (int q = 0; q < n; ++q, y += a.nt) tma_load_2d<kTwo>(at + w_bytes + q * h_bytes, &h_map, 0, y, bar);
                j += n;
                next();
              }
            }
          }
          if (ok && (s & odd) != 0) {  // the next tile's begin with a pair: the other one of this passes empty
            if (leader) mbar_arrive(full + (s >> odd));
            next();
          }
          if (rounds) break;
        }
        // nothing of its own is on the way when it leaves, also where it gave up
        for (int i = 0; i < a.stages && leader; i += a.pair)
          if (used >> i & 1u) mbar_drain(full + (i >> odd), phases >> i & 1u, a.status);
      }
    } else if (wid == 1) {
      if (lane == 0 && leader) {
        const uint32_t idesc = tc_idesc_bf16(kTileFeat, a.nt, false);
        const uint64_t first_desc = tc_smem_desc(smem_u32(smem), 0, 1024);  // (its address is the low field, which the ring does not overrun)
        bool ready = false;  // the next pair has been seen to be full
        auto filled = [&] {
          if ((s & odd) != 0) return true;
          const bool there = ready || mbar_wait(full + (s >> odd), phase, a.status);
          tc_fence_after_sync();
          return there;
        };
        auto peek = [&] {    // (before a stage's MMAs, so that the answer is there behind them)
          if ((s & odd) != odd) return;
          const bool wraps = s + 1 == a.stages;
          ready = mbar_try_wait(full + (wraps ? 0 : (s + 1) >> odd), wraps ? phase ^ 1u : phase);
        };
        auto next = [&] {
          if ((s & odd) == odd) commit<kTwo>(empty + (s >> odd));
          if (++s == a.stages) { s = 0; phase ^= 1u; }
        };
        for (Tile t = now; more(t) && ok; advance(t)) {
          const int row_tile = t.r;
          int s0 = 0, s1 = 0;
          if (kMode == kWith && waited) s1 = slots_of(row_tile);
          uint32_t d = 0;
          int in_acc = 0;  // stages in the accumulator
          auto open = [&] {
            in_acc = 0;
            d = tmem + acc_at() * a.acc_cols;
            const bool got = mbar_wait(acc_empty + acc_at(), acc_phase() ^ 1u, a.status);
            tc_fence_after_sync();
            return got;
          };
          auto chunk = [&] {  // the next stage's accumulator
            if (kExact && in_acc == kChunk) {
              commit_both<kTwo>(acc_full + acc_at(), both);
              ++done;
              if (!open()) return false;
            }
            ++in_acc;
            return true;
          };
          if (!(ok = open())) break;
          int k = step0;
          if (a.pair == 2) {  // in few instructions
            const uint32_t stage_desc = stage_bytes >> 4, x_desc = w_bytes >> 4;
            for (; k + 2 <= step1; k += 2) {
              if (!(ok = filled() && chunk())) break;
              ++in_acc;
              const uint64_t wd = first_desc + (uint32_t)s * stage_desc;
              mma4<kTwo>(d, wd, wd + x_desc, idesc, in_acc > 2);
              const bool wraps = s + 2 == a.stages;
              ready = mbar_try_wait(full + (wraps ? 0 : (s >> 1) + 1), wraps ? phase ^ 1u : phase);
              mma4<kTwo>(d, wd + stage_desc, wd + (stage_desc + x_desc), idesc, 1);
              commit<kTwo>(empty + (s >> 1));
              s = wraps ? 0 : s + 2;
              phase ^= wraps;
            }
          }
          for (; k < step1 && ok; ++k) {
            if (!(ok = filled() && chunk())) break;
            const uint64_t wd = first_desc + (uint64_t)((uint32_t)s * stage_bytes >> 4);
            peek();
            mma4<kTwo>(d, wd, wd + (w_bytes >> 4), idesc, in_acc > 1);
            next();
          }
          if (kMode == kWith && ok) {
            if (!waited) {
              asm volatile("griddepcontrol.wait;" ::: "memory");
              waited = true;
              s1 = slots_of(row_tile);
            }
            s0 = s1 * part / a.splits;
            s1 = s1 * (part + 1) / a.splits;
            const int stages = slot_stages(s1 - s0);
            if (kExact && stages > 0 && in_acc > 0) in_acc = kChunk;  // (to an empty accumulator: h's last number would be lost beside W x)
            for (int i = 0; i < stages; ++i) {
              if (!(ok = filled() && chunk())) break;
              const uint32_t at = smem_u32(smem + s * stage_bytes), ht = at + w_bytes;
              peek();
              // the numbers of h in this stage, each with its slot's B
              const uint32_t on = in_acc > 1;
              if (h_row == 128) {
                mma4<kTwo>(d, operand_desc(at, 128), operand_desc(ht, 128), idesc, on);
              } else if (h_row == 64) {
                const uint64_t bd = operand_desc(at, 64), hd = operand_desc(ht, 64), hd2 = operand_desc(ht + h_bytes, 64);
                mma1<kTwo>(d, bd, hd, idesc, on);
                mma1<kTwo>(d, bd + 2, hd + 2, idesc, 1);
                if (kNumbers == 2 || (i & 1) == 0) {
                  mma1<kTwo>(d, bd, hd2, idesc, 1);
                  mma1<kTwo>(d, bd + 2, hd2 + 2, idesc, 1);
                }
              } else if (kNumbers == 2) {
                const uint64_t bd = operand_desc(at, 32), bd2 = operand_desc(at + b_bytes, 32), hd = operand_desc(ht, 32);
                const uint64_t next_h = h_bytes >> 4;
                mma1<kTwo>(d, bd, hd, idesc, on);
                mma1<kTwo>(d, bd, hd + next_h, idesc, 1);
                if (s0 + 2 * i + 1 < s1) {
                  mma1<kTwo>(d, bd2, hd + 2 * next_h, idesc, 1);
                  mma1<kTwo>(d, bd2, hd + 3 * next_h, idesc, 1);
                }
              } else {
                const uint64_t bd = operand_desc(at, 32), hd = operand_desc(ht, 32);
#pragma unroll
                for (int j = 0; j < kNumbers; ++j) mma1<kTwo>(d, bd, hd + j * (h_bytes >> 4), idesc, on || j > 0);
              }
              next();
            }
          }
          if ((s & odd) != 0) {
            commit<kTwo>(empty + (s >> odd));
            if (++s == a.stages) { s = 0; phase ^= 1u; }
            ready = false;
          }
          commit_both<kTwo>(acc_full + acc_at(), both);
          ++done;
          if (rounds) break;
        }
        if (!ok) {  // (otherwise the tiles' own waits have seen the last of them)
          commit<kTwo>(drained);
          mbar_drain(drained, 0, a.status);
        }
      }
    } else if (wid >= 4) {
      if (kMode == kWith && !waited) {
        asm volatile("griddepcontrol.wait;" ::: "memory");  // (what is written here may be read by kernels before)
        waited = true;
      }
      for (Tile t = now; more(t); advance(t)) {
        const int f = t.f, row_tile = t.r, t0 = row_tile * a.nt;
        auto wait_sums = [&] {
          ok = __all_sync(0xffffffffu, ok && mbar_wait(acc_full + acc_at(), acc_phase(), a.status));
          tc_fence_after_sync();
          return ok;
        };
        auto sums_taken = [&] {
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) give_acc();
          ++done;
        };
        uint32_t from = lanes + acc_at() * a.acc_cols + col0;
        if (kExact) {
          int chunks = (step1 - step0 + kChunk - 1) / kChunk;
          if (kMode == kWith) {
            const int n = slots_of(row_tile);
            chunks += (slot_stages(n * (part + 1) / a.splits - n * part / a.splits) + kChunk - 1) / kChunk;
          }
          const uint32_t sums = lanes + a.sum_cols + col0;
          for (int c = 0; c < chunks && wait_sums(); ++c) {
            from = lanes + acc_at() * a.acc_cols + col0;
            for (int g = 0; g < cols; g += kGroup) {
              uint32_t r[kGroup], q[kGroup];
              tmem_ld8(from + g, r);
              if (c > 0) tmem_ld8(sums + g, q);
              tmem_wait_ld();
              if (c > 0) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(q[j]));
              }
              tmem_st8(sums + g, r);
            }
            tmem_wait_st();
            sums_taken();
          }
          from = sums;
        } else {
          wait_sums();
        }
        if (!ok || rounds) break;  // (joined below, by the whole cluster)
        const int feat = f * kTileFeat + half * kFeat + m;
        uint64_t nothing = 0ull;  // results times zero, in two halves: NaN where one is no finite number
        for (int g = col0; g < col0 + cols && t0 + g < a.rows; g += kGroup) {
          uint32_t r[kGroup];
          tmem_ld8(from + (g - col0), r);
          tmem_wait_ld();
          if (feat < a.out_dim) store_rows(a, t0 + g, feat, r);
          if (kMode == kWith) {
#pragma unroll
            for (int j = 0; j < kGroup; j += 2) nothing = f2_fma(f2_pack(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), 0ull, nothing);
          }
        }
        if (kMode == kWith) {
          float lo, hi;
          f2_unpack(nothing, lo, hi);
          if (!(lo + hi == 0.f)) *odd_ones = 1;
        }
        if (!kExact) sums_taken();
      }
    }
    __syncwarp();
    if (!rounds) break;
    {
      // The parts go to shared memory (the ring's: the tile's last MMA is done), [row of x][feature], and row r is joined by CTA r mod
      // splits (its own, where it has all of K), a warp a row, 16 reads on the way.  (Parts written to the CTA that joins them took 30 us where this takes 20, with 256 rows.)
      const int f = now.f, row_tile = now.r, t0 = row_tile * a.nt, n = idle ? 0 : min(a.nt, a.rows - t0);
      const int first = whole ? part : 0, joined = whole ? 1 : a.splits, mine = whole ? 0 : part;  // the parts of its rows, and which are its
      const HPlace place = kMode == kDown ? HPlace(sl, row_tile, f * per_tile, now.slots, lane * 4) : HPlace();
      float* parts = reinterpret_cast<float*>(smem);
      if (wid >= 4 && !idle) {
        const uint32_t from = lanes + (kExact ? a.sum_cols : acc_at() * a.acc_cols) + col0;
        for (int g = 0; g < cols; g += kGroup) {
          uint32_t r[kGroup];
          tmem_ld8(from + g, r);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < kGroup; ++j) parts[(col0 + g + j) * kFeat + m] = __uint_as_float(r[j]);
        }
        if (!kExact) {
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) give_acc();
          ++done;
        }
      }
      if (!ok) *gave_up = 1;
      __syncwarp();
      cluster_sync_all();
      uint32_t stop = 0;
      if (tid < size) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(stop) : "r"(at_rank(gave_up, tid)) : "memory");
      constexpr int kAtOnce = kMode == kDown ? 2 : 4, kParts = 4;  // rows and parts of a warp on the way
      const int apart = joined * kWarps;
      for (int r0 = mine + joined * wid; r0 < n; r0 += apart * kAtOnce) {
        float4 sum[kAtOnce];
        int row_slot[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          row_slot[i] = kMode == kDown ? __ldcg(sl.of_row + t0 + min(r0 + i * apart, n - 1)) : 0;
        }
        for (int p0 = 0; p0 < joined; p0 += kParts) {
          float4 x[kParts][kAtOnce];
#pragma unroll
          for (int p = 0; p < kParts; ++p) {
            if (p0 + p < joined) {
              const uint32_t from = at_rank(parts + lane * 4, (first + p0 + p) * kCtas + half);
#pragma unroll
              for (int i = 0; i < kAtOnce; ++i)
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                             : "=f"(x[p][i].x), "=f"(x[p][i].y), "=f"(x[p][i].z), "=f"(x[p][i].w)
                             : "r"(from + min(r0 + i * apart, n - 1) * kFeat * 4)
                             : "memory");
            }
          }
#pragma unroll
          for (int p = 0; p < kParts; ++p)
            if (p0 + p < joined) {
#pragma unroll
              for (int i = 0; i < kAtOnce; ++i) { sum[i].x += x[p][i].x; sum[i].y += x[p][i].y; sum[i].z += x[p][i].z; sum[i].w += x[p][i].w; }
            }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int r = r0 + i * apart;
          if (r < n) {
            if (kMode == kDown) {
              if (GF_CHECK((place.at == nullptr || place.slot < sl.most) && row_slot[i] < sl.most && r < a.nt, a.status, 603)) store_h(sl, place, r, row_slot[i], sum[i]);
            }
            else store_y4(a, t0 + r, f * kTileFeat + half * kFeat + lane * 4, sum[i]);
            if (kMode == kWith && !(finite(sum[i].x) && finite(sum[i].y) && finite(sum[i].z) && finite(sum[i].w))) *odd_ones = 1;
          }
        }
      }
      __syncwarp();
      cluster_sync_all();  // nobody leaves, or takes new stages to where its part was, while that is read
      fence_proxy_async_smem();  // (before the next round's copies to the ring)
      if (__syncthreads_or((int)stop)) break;
      if (whole) now.f += (a.splits - 1 - part) * f_step;
      advance(now);
    }
  }
  if (kMode == kWith) {
    __syncwarp();
    if (__any_sync(0xffffffffu, *odd_ones != 0)) {
      // (behind everything: a call in the loops above would cost them registers.  A round has one tile, and a warp of it two groups of rows at most: splits are two at least.)
      const int step = rounds ? a.splits * kWarps : 1;
      for (Tile t = start(); more(t); advance(t)) {
        const int t0 = t.r * a.nt, end = min(t0 + a.nt, a.rows), from = t0 + (rounds ? part + a.splits * wid : col0);
        const int groups = rounds ? 2 : cols / kGroup, feat = t.f * kTileFeat + half * kFeat + (rounds ? lane * 4 : m);
        if (rounds || wid >= 4) rework(a, t.r, (uint32_t)((1ull << groups) - 1ull), from, step, end, feat, rounds ? 4 : 1);
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (kTwo) cluster_sync_all();  // (neither leaves while the other's MMAs or arrivals may still come)
  tc_fence_after_sync();
  if (wid == 1) tmem_give<kTwo>(tmem, a.tmem_cols);
}

// The slots of a tile of x: the adapters that its rows name, ascending; one bit an adapter in shared memory, so that an adapter's slot is
// the number of bits below its own.
constexpr int kMaxWords = GF_MAX_ADAPTERS / 32;
struct SlotBits {
  uint32_t bits[kMaxWords];
  int before[kMaxWords];  // bits in the words before
  int count;
  __device__ int slot(int id) const { return id < 0 ? -1 : before[id >> 5] + __popc(bits[id >> 5] & ((1u << (id & 31)) - 1u)); }
};
// An adapter's number, -1 where it is none.
__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ adapter, int row, int num_adapters, int32_t* status) {
  const int id = adapter[row];
  if (id >= 0 && id < num_adapters) return id;
  if (id != -1) atomicCAS(status + kStatusReport, 0, (int)GF_ERR_INVALID_ARG);
  return -1;
}
// A projection without adapters has none to name: only the report of ids that do.
__global__ void __launch_bounds__(256) k_adapter_none(const int32_t* __restrict__ adapter, int rows, int32_t* status) {
  const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (row < rows) adapter_of(adapter, (int)row, 0, status);
}
// All threads of a CTA, at least n of them; returns the adapter of row t0 + (thread).
__device__ int find_slots(SlotBits& sb, const int32_t* __restrict__ adapter, int t0, int n, int num_adapters, int32_t* status) {
  const int tid = threadIdx.x, lane = tid & 31, words = (num_adapters + 31) / 32;
  const int id = tid < n ? adapter_of(adapter, t0 + tid, num_adapters, status) : -1;
  for (int i = tid; i < words; i += blockDim.x) sb.bits[i] = 0u;
  __syncthreads();
  if (id >= 0) atomicOr(&sb.bits[id >> 5], 1u << (id & 31));
  __syncthreads();
  if (tid < 32) {
    int sum = 0;
    for (int i0 = 0; i0 < words; i0 += 32) {
      const int here = i0 + lane < words ? __popc(sb.bits[i0 + lane]) : 0;
      int upto = here;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      if (i0 + lane < words) sb.before[i0 + lane] = sum + upto - here;
      sum += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) sb.count = sum;
  }
  __syncthreads();
  return id;
}
// The same threads write the tile's list.  (Rows of one adapter write the same.)
__device__ __forceinline__ void write_slots(const SlotBits& sb, const Slots& sl, int tile, int id, int32_t* status) {
  if (!GF_CHECK(sb.count <= sl.most && sb.slot(id) < sb.count, status, 604)) return;
  if (threadIdx.x == 0) sl.count[tile] = sb.count;
  if (id >= 0) sl.adapter[(int64_t)tile * sl.most + sb.slot(id)] = id;
}

__global__ void __launch_bounds__(256) k_adapter_slots(const int32_t* __restrict__ adapter, int rows, int nt, int num_adapters, Slots sl, int32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ SlotBits sb;
  const int t0 = blockIdx.x * nt, n = min(nt, rows - t0);
  const int id = find_slots(sb, adapter, t0, n, num_adapters, status);
  write_slots(sb, sl, blockIdx.x, id, status);
  if (threadIdx.x < n) sl.of_row[t0 + threadIdx.x] = sb.slot(id);
}

// A x for few rows, where the tiles' kernel would be all latency (slots 3 us, A x 15 to 20; this 7).  A CTA per row and 16 ranks: the warps
// share K, each lane 8 entries of x against 16 rows of A, all asked for at once; the lanes' sums are joined by halving the values that a
// lane holds.  fp32 throughout.  Bound: latency (the rows' adapters, A, the join), and for hundreds of rows L2, which reads A once per row.
constexpr int kRowThreads = 512, kRowWarps = kRowThreads / 32, kRowRanks = 16;
__global__ void __launch_bounds__(kRowThreads, 2) k_adapter_rows(const __nv_bfloat16* __restrict__ x, int64_t x_stride, int rows, int in_dim, int nt,
                                                                 const int32_t* __restrict__ adapter, int num_adapters, Slots sl,
                                                                 const __nv_bfloat16* __restrict__ a, int32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ SlotBits sb;
  __shared__ float sums[kRowWarps][kRowRanks], h[kRowRanks];
  const int t = blockIdx.x, tile = t / nt, t0 = tile * nt, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, r0 = blockIdx.y * kRowRanks;
  const int which = adapter_of(adapter, t, num_adapters, status), ranks = min(kRowRanks, sl.rank - r0);
  if (which >= 0) {
    const __nv_bfloat16* xr = x + (int64_t)t * x_stride;
    const __nv_bfloat16* ar = a + ((int64_t)which * sl.rank + r0) * in_dim;
    float v[kRowRanks];
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // (8 ranks at a time: registers)
      uint64_t acc[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) acc[r] = 0ull;
      if (half * 8 < ranks)  // (ranks are multiples of 8)
        for (int k = tid * 8; k < in_dim; k += kRowThreads * 8) {
          const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
          uint4 av[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) av[r] = __ldg(reinterpret_cast<const uint4*>(ar + (int64_t)(half * 8 + r) * in_dim + k));
          const uint64_t x0 = bf16x2_to_f2(xv.x), x1 = bf16x2_to_f2(xv.y), x2 = bf16x2_to_f2(xv.z), x3 = bf16x2_to_f2(xv.w);
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            acc[r] = f2_fma(bf16x2_to_f2(av[r].x), x0, acc[r]);
            acc[r] = f2_fma(bf16x2_to_f2(av[r].y), x1, acc[r]);
            acc[r] = f2_fma(bf16x2_to_f2(av[r].z), x2, acc[r]);
            acc[r] = f2_fma(bf16x2_to_f2(av[r].w), x3, acc[r]);
          }
        }
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        float lo, hi;
        f2_unpack(acc[r], lo, hi);
        v[half * 8 + r] = lo + hi;
      }
    }
    // sixteen sums over 32 lanes: each exchange halves the values held, the last adds the two that are left
#pragma unroll
    for (int half = 8; half > 0; half >>= 1) {
      const bool upper = (lane & half) != 0;
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const float keep = upper ? v[i + half] : v[i], give = upper ? v[i] : v[i + half];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, half);
      }
    }
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
    if (lane < kRowRanks) sums[wid][lane] = v[0];
  }
  const int id = find_slots(sb, adapter, t0, min(nt, rows - t0), num_adapters, status);
  if (t == t0 && r0 == 0) write_slots(sb, sl, tile, id, status);
  if (which >= 0 && tid < kRowRanks) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) sum += sums[w][tid];
    h[tid] = tid < ranks ? sum * (sl.scale != nullptr ? __ldg(sl.scale + which) : 1.f) : 0.f;
  }
  __syncthreads();
  // the row's pieces (8 ranks) of these 16 ranks, or of their padding, in all slots
  const int pieces = min(2, (sl.padded - r0) >> 3), slot = sb.slot(which);
  char* base = sl.h + (int64_t)tile * sl.most * sl.numbers * sl.block;
  for (int i = tid; i < sb.count * pieces; i += kRowThreads) {
    const int c = i % pieces, at = i / pieces;
    if (!GF_CHECK(at < sl.most && t - t0 < nt && r0 + (c + 1) * 8 <= sl.padded, status, 605)) break;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = at == slot ? h[c * 8 + j] : 0.f;
    for (int n = sl.numbers - 1; n >= 0; --n) {  // (the first number last, as in store_h)
      __align__(16) __nv_bfloat16 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = take_number(v[j]);
      *reinterpret_cast<uint4*>(base + (int64_t)(sl.numbers * at + n) * sl.block + ((t - t0) * sl.padded + r0 + c * 8) * 2) = *reinterpret_cast<uint4*>(p);
    }
  }
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeTiled)p;
  }();
  return f;
}

// bf16 [matrices, rows, cols], read as boxes of box_cols x box_rows of one matrix, swizzled over a row of the box; what lies outside
// reads as zero.
bool make_map(CUtensorMap* map, const void* base, int64_t matrices, int64_t rows, int64_t cols, int64_t stride, int box_cols, int box_rows) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const int rank = matrices > 0 ? 3 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)matrices}, strides[2] = {(cuuint64_t)stride * 2, (cuuint64_t)(rows * stride) * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
  const CUtensorMapSwizzle swizzle = box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : box_cols == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kHalfKb = 110;  // of shared memory, of which two CTAs share a multiprocessor
// Never launched: the occupancy calculation takes a kernel with tensor memory for one that has a multiprocessor to itself, though two of
// k_project's CTAs run side by side where they have room (4096 -> 6144 in 192 CTAs: 11 us, and 19 when registers allowed but one).
__global__ void __launch_bounds__(kThreads, 2) k_room() {}
// How many clusters of `size` CTAs the device has room for at once, with all of a multiprocessor's shared memory each or half of it.
// (Asked once: a GPC whose multiprocessors are no multiple of the size has some left over.)
int clusters_at_once(int size, bool half, int num_sms) {
  static int known[kMaxDevices][2][9];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  int& n = known[dev][half][size];
  if (n == 0) {
    static bool done[kMaxDevices];
    if (!ensure_dynamic_smem(k_room, 227 * 1024, done)) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(size * num_sms));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (half ? kHalfKb : 227) * 1024;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int got = 0;
    if (cudaOccupancyMaxActiveClusters(&got, k_room, &cfg) != cudaSuccess) {
      cudaGetLastError();
      got = 0;
    }
    n = got > 0 ? got : -1;
  }
  return n;
}

// How a launch shares out its tiles: CTAs and what they have.  Few tiles are shared by clusters of up to 8 CTAs, whose time is the stages
// of the multiprocessor that has most: the size with the fewest is taken, the smallest of those (a join costs 1 to 3 us), if all clusters
// find room at once.  Where four stages fit into half a multiprocessor's shared memory, two CTAs may share it.  (4096 -> 6144 for 64
// rows: 26 us with clusters of 1, 16.6 of 2, 15.7 of 4, which leave some multiprocessors with two CTAs.)
struct Shape {
  int ctas;
  size_t smem;
};
Shape shape_of(ProjectArgs& a, int64_t tiles, bool rounds, int num_sms) {
  const int steps = (a.in_dim + kStep - 1) / kStep, ctas = a.two ? 2 : 1;
  const uint32_t stage_bytes = kFeat * 128u + a.nt / ctas * 128u, extra = 1024 + 512;
  // (and only where tensor memory has room for two: CTAs of clusters that wait for each other must never wait for that)
  const int per_sm = 4 * stage_bytes + extra <= kHalfKb * 1024 && a.nt <= (a.y_fp32 ? 64 : 128) ? 2 : 1;
  const int room_for = num_sms / ctas;  // tiles at once
  a.splits = 1;
  int64_t best = (tiles + room_for - 1) / room_for * steps;
  for (int n = 2; n * ctas <= 8 && tiles * n <= (int64_t)per_sm * room_for && steps >= 4 * n; ++n) {
    const int64_t most = (tiles * n + room_for - 1) / room_for * ((steps + n - 1) / n);
    if (most < best - best / 16 && tiles <= clusters_at_once(n * ctas, per_sm == 2, num_sms)) {
      best = most;
      a.splits = n;
    }
  }
  // (where several turns of one CTA a multiprocessor are fewer than twice as many of two, the last is fuller: 64 rows of 4096 -> 128 000 176 us, 184 with
  // two; 100 000 features, where they are the same, 149 and 140)
  const bool even = 2 * ((tiles + 2 * num_sms - 1) / (2 * num_sms)) <= (tiles + num_sms - 1) / num_sms;
  const bool shared = per_sm == 2 && (a.splits > 1 || (tiles > num_sms && even));
  const uint32_t room = (shared ? kHalfKb : 227) * 1024 - extra;
  a.stages = (int)std::min<uint32_t>(12, room / stage_bytes);
  // With six and more, two share their barriers: the issuing thread is what bounds the kernel, and a commit costs it 100 cycles and a wait 65 where a
  // stage's MMAs cost 280.  (8192 rows: 332 us with a wait for each, 280 with a wait for two; 1 row 14.4 and 11.5.  Four stages in pairs leave too
  // few on the way: 707 us became 868 for 14336 -> 4096 where a CTA works by itself.)
  a.pair = a.stages >= 6 ? 2 : 1;
  a.stages -= a.stages % a.pair;
  const int64_t groups = a.splits > 1 ? tiles : std::min<int64_t>(tiles, shared ? 2 * room_for : room_for);
  return Shape{(int)(groups * a.splits * ctas), extra + std::max<uint32_t>(stage_bytes * a.stages, a.splits > 1 || rounds ? (uint32_t)a.nt * kFeat * 4u : 0u)};
}

struct Maps { CUtensorMap w, x, b, h; };
template <int kMode, int kExact, bool kTwo>
int launch_kind(const Maps& maps, ProjectArgs a, const Shape& shape, cudaStream_t st) {
  static bool done[kMaxDevices];
  if (!ensure_dynamic_smem(k_project<kMode, kExact, kTwo>, 227 * 1024, done)) return -1;
  // accumulators: one where a CTA has one tile of one chunk, or tensor memory holds no more beside the sums; the sums behind them
  const bool single = !kExact && (int64_t)a.feat_tiles * a.row_tiles <= shape.ctas / (a.splits * (kTwo ? 2 : 1));
  uint32_t cols = 32;
  while (cols < (uint32_t)a.nt) cols *= 2;
  a.accs = single || kExact == 8 ? 1 : 2;
  a.acc_cols = cols;
  a.sum_cols = a.accs * cols;
  a.tmem_cols = a.accs * cols + (kExact ? cols : 0);
  while (a.tmem_cols & (a.tmem_cols - 1)) a.tmem_cols += a.tmem_cols & -a.tmem_cols;  // (a power of two)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)shape.ctas);
  cfg.blockDim = dim3(kExact == 8 ? kWideThreads : kThreads);
  cfg.dynamicSmemBytes = shape.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (kTwo || a.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)(a.splits * (kTwo ? 2 : 1));
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (kMode != kPlain) {  // behind the kernel for the slots, or that for h, whose results only a tile's last stages need
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, k_project<kMode, kExact, kTwo>, maps.w, maps.x, maps.b, maps.h, a) == cudaSuccess ? 1 : -1;
}
template <int kMode>
int launch_main(const Maps& maps, const ProjectArgs& a, const Shape& shape, cudaStream_t st) {
  if constexpr (kMode != kDown)
    if (a.two) return a.y_fp32 ? launch_kind<kMode, 8, true>(maps, a, shape, st) : launch_kind<kMode, 0, true>(maps, a, shape, st);
  if (!a.y_fp32) return launch_kind<kMode, 0, false>(maps, a, shape, st);
  return a.nt <= 128 ? launch_kind<kMode, 4, false>(maps, a, shape, st) : launch_kind<kMode, 8, false>(maps, a, shape, st);
}

// Rows of x that one pass takes: more go in several, one behind the other, so that the scratch stays bounded.
constexpr int kPassRows = 16384;

// Rows of x in a tile.
constexpr int kRows = 256, kFewerRows = 128;
int padded_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }
void set_tiles(ProjectArgs& a, int nt) {
  a.nt = nt;
  a.two = nt == 256 && a.out_dim > kFeat;
  const int tile_feat = kFeat * (a.two ? 2 : 1);
  a.feat_tiles = (a.out_dim + tile_feat - 1) / tile_feat;
  a.row_tiles = (a.rows + nt - 1) / nt;
}
// 256 where there are as many, unless 128 give the multiprocessors a shorter way: a stage of 256 columns takes two of them 0.39 us (fp32: 0.54), one of
// 128 takes one 0.28 (0.31).  (4096 -> 6144: 300 rows 22.8 us with 128 and 27.7 with 256, 512 rows 39.2 and 28.2; 4096 -> 1328: 300 rows 12.1 and
// 16.3, 1294 rows 22.5 and 27.0, 2048 rows 38.5 and 29.6; in fp32 4096 -> 6144 for 1024 rows 65.8 and 73.2, 2048 rows 122.9 and 108.3.)
// Turns of A x beyond the first count too, 5 us (3.5) each beside their stages, as if every row named another adapter (7954 rows of 136 under 61
// adapters of rank 64: 219 us with 256, 304 with 128).
void choose_tiles(ProjectArgs& a, int num_adapters, int rank, int num_sms) {
  if (a.rows < kRows) return set_tiles(a, (a.rows + 15) / 16 * 16);
  const int steps = (a.in_dim + kStep - 1) / kStep;
  int64_t cost[2];
  for (int i = 0; i < 2; ++i) {
    ProjectArgs b = a;
    set_tiles(b, i ? kFewerRows : kRows);
    const int64_t tiles = (int64_t)b.feat_tiles * b.row_tiles, at_once = num_sms / (b.two ? 2 : 1);
    shape_of(b, tiles, false, num_sms);
    const int64_t turns = b.splits > 1 ? 1 : (tiles + at_once - 1) / at_once;
    const int64_t stage = i ? (a.y_fp32 ? 31 : 28) : (a.y_fp32 ? 54 : 39);
    cost[i] = turns * ((steps + b.splits - 1) / b.splits) * stage;
    if (num_adapters > 0) {
      const int per_tile = kFeat / padded_rank(rank), most = (std::min(b.nt, num_adapters) + per_tile - 1) / per_tile;
      cost[i] += ((int64_t)b.row_tiles * most - 1) / num_sms * (steps * stage + (i ? 350 : 500));
    }
  }
  set_tiles(a, cost[1] < cost[0] ? kFewerRows : kRows);
}
size_t align_to(size_t n, size_t a) { return (n + a - 1) / a * a; }

// Where the slots of a pass stand in the scratch, with tiles of nt rows; its size.
size_t place_slots(Slots* sl, char* scratch, int rows, int nt, int rank, int num_adapters, int numbers) {
  const int tiles = (rows + nt - 1) / nt, most = std::min(nt, num_adapters);
  const int padded = padded_rank(rank);
  const size_t ids = align_to((size_t)tiles * 4, 128), of_row = ids + align_to((size_t)tiles * most * 4, 128), h = of_row + align_to((size_t)rows * 4, 128);
  const size_t block = (size_t)nt * padded * 2;
  if (sl) *sl = Slots{(int32_t*)scratch, (int32_t*)(scratch + ids), (int32_t*)(scratch + of_row), nullptr, scratch + h, most, numbers, rank, padded, (uint32_t)block};
  return h + (size_t)tiles * most * numbers * block;
}

}  // namespace

// (a last pass of fewer rows needs no more than a whole one)
size_t project_scratch_bytes(int rows, int rank, int num_adapters) {
  rows = std::min(rows, kPassRows);
  if (rows < kRows) return place_slots(nullptr, nullptr, rows, (rows + 15) / 16 * 16, rank, num_adapters, 3);
  return std::max(place_slots(nullptr, nullptr, rows, kRows, rank, num_adapters, 3), place_slots(nullptr, nullptr, rows, kFewerRows, rank, num_adapters, 3));
}

static int launch_pass(const gf_projection_t& p, int rows, const void* x, int64_t x_stride, const int32_t* adapter, void* y, int64_t y_stride, int y_fp32,
                       void* scratch, int num_sms, int32_t* status, cudaStream_t st) {
  const bool with = adapter != nullptr && p.num_adapters > 0;
  ProjectArgs a = {};
  a.rows = rows;
  a.in_dim = p.in_dim;
  a.out_dim = p.out_dim;
  a.y = y;
  a.y_stride = y_stride;
  a.y_fp32 = y_fp32;
  a.status = status;
  a.w = (const __nv_bfloat16*)p.w_dev;
  a.x = (const __nv_bfloat16*)x;
  a.b = (const __nv_bfloat16*)p.b_dev;
  a.w_stride = p.w_stride;
  a.x_stride = x_stride;
  a.adapter = adapter;
  a.num_adapters = p.num_adapters;
  choose_tiles(a, with ? p.num_adapters : 0, p.rank, num_sms);
  a.y_vec = (y_stride & 3) == 0 && ((uintptr_t)y & (y_fp32 ? 15 : 7)) == 0;
  Maps maps = {};
  const int x_box = a.nt / (a.two ? 2 : 1);
  if (!make_map(&maps.w, p.w_dev, 0, p.out_dim, p.in_dim, p.w_stride, kStep, kFeat) || !make_map(&maps.x, x, 0, rows, p.in_dim, x_stride, kStep, x_box)) return -1;
  const Shape main_shape = shape_of(a, (int64_t)a.feat_tiles * a.row_tiles, false, num_sms);
  if (!with) return launch_main<kPlain>(maps, a, main_shape, st);
  place_slots(&a.slots, (char*)scratch, rows, a.nt, p.rank, p.num_adapters, y_fp32 ? 3 : 2);
  a.slots.scale = p.scale_dev;
  if (!make_map(&maps.b, p.b_dev, p.num_adapters, p.out_dim, p.rank, p.rank, a.slots.padded, kFeat) ||
      !make_map(&maps.h, a.slots.h, 0, (int64_t)a.row_tiles * a.slots.most * a.slots.numbers * a.nt, a.slots.padded, a.slots.padded, a.slots.padded, x_box))
    return -1;
  const int chunks = (a.slots.padded + kRowRanks - 1) / kRowRanks;
  if ((int64_t)rows * chunks <= 8 * num_sms) {
    k_adapter_rows<<<dim3((unsigned)rows, (unsigned)chunks), kRowThreads, 0, st>>>((const __nv_bfloat16*)x, x_stride, rows, p.in_dim, a.nt, adapter,
                                                                                    p.num_adapters, a.slots, (const __nv_bfloat16*)p.a_dev, status);
    if (cudaGetLastError() != cudaSuccess) return -1;
    return launch_main<kWith>(maps, a, main_shape, st) < 0 ? -1 : 2;
  }
  k_adapter_slots<<<(unsigned)a.row_tiles, 256, 0, st>>>(adapter, rows, a.nt, p.num_adapters, a.slots, status);
  if (cudaGetLastError() != cudaSuccess) return -1;
  // A x: as many tiles as there can be slots; those of none are passed over.  Shared out as if every tile of x had one.
  ProjectArgs d = a;
  Maps down = maps;
  if (!make_map(&down.w, p.a_dev, 0, (int64_t)p.num_adapters * p.rank, p.in_dim, p.in_dim, kStep, p.rank) ||
      (a.two && !make_map(&down.x, x, 0, rows, p.in_dim, x_stride, kStep, a.nt)))
    return -1;
  const int per_tile = kFeat / a.slots.padded;
  d.two = 0;
  d.feat_tiles = (a.slots.most + per_tile - 1) / per_tile;
  Shape shape = shape_of(d, (int64_t)a.row_tiles, true, num_sms);
  const int most_groups = std::max(1, num_sms * 3 / 4 / d.splits);
  int64_t down_groups = shape.ctas / d.splits;  // at most one per tile of x; more where multiprocessors are left
  if (down_groups == a.row_tiles) down_groups *= std::max<int64_t>(1, std::min<int64_t>(d.feat_tiles, most_groups / down_groups));
  shape.ctas = (int)down_groups * d.splits;
  if (launch_main<kDown>(down, d, shape, st) < 0) return -1;
  return launch_main<kWith>(maps, a, main_shape, st) < 0 ? -1 : 3;
}

int launch_project(const gf_projection_t& p, int rows, const void* x, int64_t x_stride, const int32_t* adapter, void* y, int64_t y_stride, int y_fp32,
                   void* scratch, int num_sms, int32_t* status, cudaStream_t st) {
  int launched = 0;
  if (adapter != nullptr && p.num_adapters == 0) {
    k_adapter_none<<<(unsigned)(((int64_t)rows + 255) / 256), 256, 0, st>>>(adapter, rows, status);
    if (cudaGetLastError() != cudaSuccess) return -1;
    ++launched;
    adapter = nullptr;
  }
  const int pass = adapter != nullptr && p.num_adapters > 0 ? kPassRows : 1 << 22;
  for (int64_t t = 0; t < rows; t += pass) {
    const int n = launch_pass(p, (int)std::min<int64_t>(pass, rows - t), (const char*)x + t * x_stride * 2, x_stride, adapter ? adapter + t : nullptr,
                              (char*)y + t * y_stride * (y_fp32 ? 4 : 2), y_stride, y_fp32, scratch, num_sms, status, st);
    if (n < 0) return -1;
    launched += n;
  }
  return launched;
}

}  // namespace gf
