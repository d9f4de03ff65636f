// Accumulated attention weights: how much of a decode batch's attention every resident token received.
//
//   w[kvh][slot(t)] (+)= sum over the requests r that share t's segment and the query heads h of KV head kvh
//                        of exp(scale q_rh . k_t - lse_rh)
//
// with lse from the decode call of the same step, so one pass over K is enough and no probability is ever
// stored.  It is a reduction over query rows for a fixed token, so a work unit is a block of tokens of one
// segment and KV head with ALL the rows that share it: every slot has one writer, which adds in a fixed
// order, and the result does not depend on scheduling (no atomics).  Of a 4-bit state the codes are
// multiplied, exact in bf16, and the token's (s, lo) enter outside of the product, in fp32:
//   s_t = sum over groups G of  s_tG (c . q_G)  +  (lo_tG + s_tG / 2) (sum of q_G)
//
// Two kernels, by how many query rows share a segment, beside each other on two streams:
//
// Up to kNarrowRows (k_weights_narrow): a stream of K, 64 tokens of it at a time copied into a warp's own piece of
// shared memory; the warp walks the rows eight at a time: S^T = K Q^T (mma.sync), exp2, sums per token in
// registers, and at the end a shuffle over the four lanes that share a token.  Nothing is shared between warps.
// 256 requests over 256 nodes in bf16: 416 MB of K in 73 us (5.7 TB/s), bound by HBM; with fewer keys per unit (4 bits: 168
// MB, half of the tiles so, 47 us) by the round trips of a unit (K, then queries, sums before), which twelve warps per
// SM, as many as K finds room for, do not hide.  Walking K once for 16 rows spilled and took 120 us instead of 94 in
// all; queries through 4-byte loads in K's natural order 102.
//
// More (k_weights_wide): tcgen05 MMAs with the tokens as rows make the reduction run along the columns of tensor
// memory: a thread owns a token, reads its scores 16 at a time and adds up 2^(scale s - lse), without a shuffle.
// Keys come as they lie in the pool (128-byte-swizzled, the operand layout) or are expanded from their codes, one
// accumulator per group.  2048 rows over 8192 tokens and 8 heads: 77 us in bf16, 100 in 4 bits; the exponentials
// alone, 16 per clock and SM, are 31.  Two warps per scheduler take 345 cycles for the 16 columns that need 256 of
// the exponential unit, and wait a quarter of the time for queries or a unit's end; units of 256 tokens, which fetch
// the queries half as often, or loads one step ahead changed nothing.
// One persistent CTA per SM, roles by warp, work in items of up to 64 rows of a unit of 128 tokens:
//   warp 19       resolves units (a fixed stride over all of them, 32 at a time) into a ring of eight
//   warps 14-17   keys: bulk copies, or the expansion of 4-bit codes, into three stages of 128 tokens
//   warps 8-13    query rows, gathered by request with asynchronous copies; every warp fills a slot of its own
//                 with each sixth item, and forms the columns' -lse (and sums of q, for a 4-bit unit)
//   warp 18       one thread issues the MMAs: 128 tokens x the rows of one item, or of two in neighbouring slots
//                 (what an MMA costs its issuing thread hardly depends on its columns)
//   warps 0-7     two groups of 128 threads take the items in turn and keep the tokens' sums; at the end
//                 of a unit group 1 hands its sums to group 0, which adds them to the array
// Every wait is bounded; a warp whose wait gave up leaves its role, and so do the others.
#include "kv4_device.cuh"
#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kNarrowThreads = 128;
constexpr int kThreads = 640;
constexpr int kBlock = 128;     // tokens of a unit
constexpr int kItemRows = 64;   // query rows of an item
constexpr int kKStages = 3, kSlots = 6, kUnits = 8, kBufs = 4;
constexpr int kBuckets = 1024;  // runs of segments whose unit counts are summed in shared memory

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

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t phase, const Params& p) { return mbar_wait(bar, phase & 1, p.status); }

// A unit of either kernel.
struct __align__(16) Unit {
  int32_t rows;  // query rows that share it; -1: no more units
  int32_t grp_begin, kvh, nv;
  int32_t slot0, tile, four, items;
};

// Where the segments' blocks of `block` tokens start: start[b] is the number of blocks before the b-th run of `per`
// segments, start[kBuckets] their total.  Executed by the whole CTA.
template <int kCtaThreads>
__device__ __forceinline__ void scan_segments(const Params& p, int32_t* start, int32_t* warp_tot, int S, int per, int block) {
  constexpr int kRun = (kBuckets + kCtaThreads - 1) / kCtaThreads;  // buckets a thread owns
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int cnt[kRun], local = 0;
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const int b = tid * kRun + i, s0 = b < kBuckets ? min(S, b * per) : S, s1 = min(S, s0 + per);
    cnt[i] = 0;
    for (int s = s0; s < s1; ++s) cnt[i] += (p.seg_len[s] + block - 1) / block;
    local += cnt[i];
  }
  int incl = local;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 31) warp_tot[warp] = incl;
  __syncthreads();
  int run = incl - local;
  for (int w = 0; w < warp; ++w) run += warp_tot[w];
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const int b = tid * kRun + i;
    if (b <= kBuckets) start[b] = run;
    run += cnt[i];
  }
  if (tid == kCtaThreads - 1 && kCtaThreads * kRun == kBuckets) start[kBuckets] = run;
}

// Unit u of all (block, KV head) pairs; rows 0 where there is nothing to do: past the end, not this kernel's
// (rows outside [least, most]), or a state kept as base + residual, which has no slots of its own.
__device__ __forceinline__ Unit resolve(const Params& p, const int32_t* start, int S, int per, int block, long long u, int least, int most) {
  Unit x{};
  if (u >= (long long)start[kBuckets] * p.num_kv_heads) return x;
  const int bi = (int)(u / p.num_kv_heads);
  int lo = 0, hi = kBuckets;  // the last bucket that starts at or before the block
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= bi) lo = mid; else hi = mid;
  }
  int seg = lo * per, at = start[lo];
  for (; seg < S - 1; ++seg) {
    const int c = (p.seg_len[seg] + block - 1) / block;
    if (bi < at + c) break;
    at += c;
  }
  const int tok0 = (bi - at) * block, gb = p.grp_ptr[seg];
  x.nv = min(block, p.seg_len[seg] - tok0);
  x.slot0 = p.seg_off[seg] + tok0;
  x.kvh = (int)(u % p.num_kv_heads);
  x.grp_begin = gb;
  x.rows = (p.grp_ptr[seg + 1] - gb) * p.gqa;
  x.items = (x.rows + kItemRows - 1) / kItemRows;
  const int tile = x.slot0 / kTile;
  x.four = tile >= p.kv4_tile0;
  x.tile = x.four ? GF_CLAMP(tile - p.kv4_tile0, p.cap4, p.status, 136) : GF_CLAMP(tile, p.cap16, p.status, 135);
  if (x.rows < least || x.rows > most || p.node_res[p.seg_node[seg]] >= 0) x.rows = 0;
  return x;
}

// ---- up to kNarrowRows rows: a warp each --------------------------------------------------------------------------

// B operands of eight query rows, for the order of the entries that 4-bit codes have (kv4_device.cuh) and bf16 keys are
// read in: entries 32 x + 8 l4 .. + 7 are MMAs 2 x and 2 x + 1, so that a lane takes 16 bytes at a time.
template <int D>
struct QueryRows {
  uint32_t f[D / 16][2];
  __device__ __forceinline__ void load(const __nv_bfloat16* row, bool ok, int l4) {
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      const uint4 v = ok ? reinterpret_cast<const uint4*>(row)[4 * x + l4] : make_uint4(0u, 0u, 0u, 0u);
      f[2 * x][0] = v.x;
      f[2 * x][1] = v.y;
      f[2 * x + 1][0] = v.z;
      f[2 * x + 1][1] = v.w;
    }
  }
};

// The token of a block of 16 that the MMA's row r (and r + 8, with token + 8) stands for.  For bf16 neighbouring rows are
// tokens whose swizzle differs in its highest bit, so that eight lanes read 16 bytes each from different banks.
template <bool k4>
__device__ __forceinline__ int token_of_row(int r) { return k4 ? r : (r >> 1) + 4 * (r & 1); }

// The scores of 16 tokens (block b of the unit's K in shared memory) and eight rows, in units of 1 / scale.
template <int D, bool k4>
__device__ __forceinline__ void block_scores(float (&s)[4], const unsigned char* k, int b, const QueryRows<D>& q,
                                             const float (&qsum)[D / kGroup4][2], int lane) {
  constexpr int NG = D / kGroup4;
  const int l4 = lane & 3, l8 = lane >> 2;
  s[0] = s[1] = s[2] = s[3] = 0.f;
  if (k4) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint4 c = reinterpret_cast<const uint4*>(k)[(b * NG + g) * 32 + lane];
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t a[4];
        kv4_expand(a, w[kk]);
        mma_bf16(acc, a, q.f[g * 4 + kk][0], q.f[g * 4 + kk][1]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t sl = reinterpret_cast<const uint32_t*>(k + kv4_code_bytes(D))[(b * 16 + l8 + 8 * h) * NG + g];
        const float sc = kv4_s(sl), z = fmaf(8.5f, sc, kv4_lo(sl));
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2) s[2 * h + c2] = fmaf(acc[2 * h + c2], sc, fmaf(qsum[g][c2], z, s[2 * h + c2]));
      }
    }
  } else {
    const uint32_t row = b * 16 + token_of_row<k4>(l8);
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      const uint32_t chunk = 4 * x + l4;
      const unsigned char* at = k + (chunk >> 3) * (kTile * 128u);
      const uint4 lo = *reinterpret_cast<const uint4*>(at + swz128(row, chunk & 7u)), hi = *reinterpret_cast<const uint4*>(at + swz128(row + 8, chunk & 7u));
      const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
      mma_bf16(s, a0, q.f[2 * x][0], q.f[2 * x][1]);
      mma_bf16(s, a1, q.f[2 * x + 1][0], q.f[2 * x + 1][1]);
    }
  }
}

// Adds the unit's rows to sum[b][h] (MMA rows l8 and l8 + 8 of block b, this lane's columns).  id and off: request and
// -lse in log2 units of rows lane and lane + 32 (-inf: no such row).  Eight rows share a walk over K; the first are asked
// for before K has come, the next before these are worked on.
template <int D, bool k4, typename Arrived>
__device__ __forceinline__ bool walk_rows(const Params& p, const unsigned char* k, const int (&id)[2], const float (&off)[2], int rows, int kvh,
                                          int lane, float (&sum)[4][2], Arrived&& arrived) {
  constexpr int NG = D / kGroup4;
  const int l4 = lane & 3, l8 = lane >> 2;
  auto load = [&](QueryRows<D>& q, int row0) {
    const int row = row0 + l8;
    const int req = __shfl_sync(0xffffffffu, row0 < 32 ? id[0] : id[1], row & 31);
    q.load(p.q + ((size_t)req * p.num_q_heads + kvh * p.gqa + (row & (p.gqa - 1))) * D, row < rows, l4);
  };
  QueryRows<D> q;
  auto walk = [&](int row0) {
    float o[2], qsum[NG][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) o[c] = __shfl_sync(0xffffffffu, row0 < 32 ? off[0] : off[1], (row0 + l4 * 2 + c) & 31);
    if (k4) {
#pragma unroll
      for (int x = 0; x < NG; ++x) {
        const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_bf16(acc, ones, q.f[x * 4 + kk][0], q.f[x * 4 + kk][1]);
        qsum[x][0] = acc[0];
        qsum[x][1] = acc[1];
      }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      float s[4];
      block_scores<D, k4>(s, k, b, q, qsum, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[b][e >> 1] += fast_exp2(fmaf(s[e], p.scale_log2, o[e & 1]));
    }
  };
  load(q, 0);
  if (!arrived()) return false;
#pragma unroll 1
  for (int row0 = 0;;) {
    const int left = rows - row0;
    QueryRows<D> next;
    if (left > 8) load(next, row0 + 8);
    walk(row0);
    if (left <= 8) return true;
    q = next;
    row0 += 8;
  }
}

template <int D>
struct __align__(128) NarrowSmem {
  unsigned char k[kNarrowThreads / 32][kTile * D * 2];  // a unit's K per warp
  uint64_t full[kNarrowThreads / 32];
  int32_t start[kBuckets + 1];
  int32_t warp_tot[kNarrowThreads / 32];
};

// A warp's units, one after the other; what hides its latencies are the other eleven warps of the SM.
template <int D>
__global__ void __launch_bounds__(kNarrowThreads, 3) k_weights_narrow(const Params p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  NarrowSmem<D>& sm = *reinterpret_cast<NarrowSmem<D>*>(smem);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) {
    mbar_init(&sm.full[warp], 1);
    mbar_fence_init();
  }
  chain_enter();
  if (!tables_usable(*p.hdr, p.slot_cap)) return;
  const int S = p.hdr->num_segments, per = (S + kBuckets - 1) / kBuckets, sh = __ffs(p.gqa) - 1;
  scan_segments<kNarrowThreads>(p, sm.start, sm.warp_tot, S, per, kTile);
  __syncthreads();
  const long long units = (long long)sm.start[kBuckets] * p.num_kv_heads;
  const long long stride = (long long)gridDim.x * (kNarrowThreads / 32);
  long long first = (long long)blockIdx.x * (kNarrowThreads / 32) + warp;
  Unit mine{};         // 32 units of this warp are resolved at a time, a lane each
  uint32_t have = 0;   // those that are still to come
  struct Next { int rows, kvh, nv, slot0, four, tile, id[2]; } nx;
  auto take = [&]() {  // the next unit's numbers and request ids
    nx.rows = 0;
    while (have == 0) {
      if (first >= units) return;
      mine = resolve(p, sm.start, S, per, kTile, first + lane * stride, 1, kNarrowRows);
      first += 32 * stride;
      have = __ballot_sync(0xffffffffu, mine.rows > 0);
    }
    const int from = __ffs(have) - 1;
    have &= have - 1;
    nx.rows = __shfl_sync(0xffffffffu, mine.rows, from);
    nx.kvh = __shfl_sync(0xffffffffu, mine.kvh, from);
    nx.nv = __shfl_sync(0xffffffffu, mine.nv, from);
    nx.slot0 = __shfl_sync(0xffffffffu, mine.slot0, from);
    nx.four = __shfl_sync(0xffffffffu, mine.four, from);
    nx.tile = __shfl_sync(0xffffffffu, mine.tile, from);
    const int gb = __shfl_sync(0xffffffffu, mine.grp_begin, from);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = lane + 32 * h;
      nx.id[h] = row < nx.rows ? GF_CLAMP(p.grp_req[GF_CLAMP(gb + (row >> sh), p.num_pairs, p.status, 137)], p.num_requests, p.status, 138) : 0;
    }
  };
  auto copy_keys = [&]() {  // of the next unit; its slot is free
    if (lane != 0 || nx.rows == 0) return;
    const uint32_t bytes = nx.four ? kv4_part_bytes(D) : kTile * D * 2u;
    const char* src = nx.four ? p.layer4 + (uint64_t)nx.kvh * p.head_stride4 + (uint64_t)nx.tile * kv4_tile_bytes(D)
                              : p.layer16 + (uint64_t)nx.kvh * p.head_stride16 + (uint64_t)nx.tile * p.tile_bytes16;
    mbar_arrive_expect_tx(&sm.full[warp], bytes);
    bulk_g2s(sm.k[warp], src, bytes, &sm.full[warp]);
  };
  take();
  copy_keys();
  for (int n = 0; nx.rows > 0; ++n) {
    const Next u = nx;
    float sum[4][2], off[2];
#pragma unroll
    for (int b = 0; b < 4; ++b) sum[b][0] = sum[b][1] = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = lane + 32 * h;
      off[h] = row < u.rows ? -1.4426950408889634f * p.lse[(size_t)u.id[h] * p.num_q_heads + u.kvh * p.gqa + (row & (p.gqa - 1))] : -INFINITY;
    }
    float* w = p.weights + (int64_t)u.kvh * p.slots + u.slot0;
    auto token = [&](int b, int h) { return b * 16 + (u.four ? lane >> 2 : token_of_row<false>(lane >> 2)) + 8 * h; };
    float old[4][2];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) old[b][h] = p.accumulate && (lane & 3) == 0 && token(b, h) < u.nv ? w[token(b, h)] : 0.f;
    take();
    auto arrived = [&] { return wait(&sm.full[warp], n, p); };
    const bool ok = u.four ? walk_rows<D, true>(p, sm.k[warp], u.id, off, u.rows, u.kvh, lane, sum, arrived)
                           : walk_rows<D, false>(p, sm.k[warp], u.id, off, u.rows, u.kvh, lane, sum, arrived);
    if (!ok) {
      if (lane == 0) mbar_drain(&sm.full[warp], n & 1, p.status);  // (after a wait that gave up)
      break;
    }
    __syncwarp();  // K has been read by every lane: the slot is free
    copy_keys();
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v = sum[b][h];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        const int t = token(b, h);
        if ((lane & 3) == 0 && t < u.nv) w[t] = old[b][h] + v;
      }
  }
}

// ---- more rows: a CTA with roles ------------------------------------------------------------------------------------

struct Smem {
  static constexpr uint32_t kStageBytes = 2 * 128 * 128;  // 128 tokens, two column blocks of 64 entries
  unsigned char k[kKStages][kStageBytes];
  unsigned char q[kSlots / 2][4][8192];  // slots 2 i and 2 i + 1: [column block][slot][64 rows][128 bytes]
  float4 scales[kUnits][kBlock];         // 4-bit units: s and lo + s / 2 of both groups per token
  float off[kSlots][kItemRows];          // -lse in log2 units, -inf for a row that does not exist
  float qsum[kSlots][2][kItemRows];
  Unit unit[kUnits];
  float handed[kBlock];                  // group 1's sums
  int32_t start[kBuckets + 1];           // units (per KV head) of the segments before the bucket
  int32_t warp_tot[kThreads / 32];
  uint32_t tmem_base;
  uint64_t unit_full[kUnits], unit_empty[kUnits], scales_full[kUnits];
  uint64_t k_full[kKStages], k_empty[kKStages];
  uint64_t q_full[kSlots], q_empty[kSlots];
  uint64_t s_full[kBufs], s_empty[kBufs];
  uint64_t handed_full, handed_empty, mmas_done;
};
constexpr int kUnitReaders = 8 + kSlots + 4 + 1;  // warps that read a unit's slot

// 16 bytes, of which the first `bytes` are read and the others become zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Where an item's scores stand in tensor memory: 64 columns, and as many 128 further for the second group of a 4-bit
// unit.  Two neighbouring items (an even one and the next) stand side by side.
__device__ __forceinline__ uint32_t item_columns(int item) { return ((item >> 1) & 1) * 256 + (item & 1) * 64; }

// Calls body(unit index, unit) for every unit of this CTA in order, from the ring; lane 0 of the calling warp gives
// the slot back.  False as soon as a wait or the body gave up.
template <typename F>
__device__ __forceinline__ bool for_units(Smem& sm, const Params& p, int lane, F&& body) {
  for (int n = 0;; ++n) {
    if (!wait(&sm.unit_full[n % kUnits], n / kUnits, p)) return false;
    const Unit u = sm.unit[n % kUnits];
    if (u.rows < 0) return true;
    if (!body(n, u)) return false;
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.unit_empty[n % kUnits]);
  }
}

// ---- warp 19: units ------------------------------------------------------------------------------------
__device__ __forceinline__ void schedule(Smem& sm, const Params& p, int per, int S, int lane) {
  const long long units = (long long)sm.start[kBuckets] * p.num_kv_heads;
  int n = 0;
  for (long long first = blockIdx.x; first < units; first += 32ll * gridDim.x) {
    const Unit x = resolve(p, sm.start, S, per, kBlock, first + (long long)lane * gridDim.x, kNarrowRows + 1, 0x7fffffff);
    for (uint32_t have = __ballot_sync(0xffffffffu, x.rows > 0); have != 0; have &= have - 1) {
      if (n >= kUnits && !wait(&sm.unit_empty[n % kUnits], n / kUnits - 1, p)) return;
      if (lane == __ffs(have) - 1) {
        sm.unit[n % kUnits] = x;
        mbar_arrive(&sm.unit_full[n % kUnits]);
      }
      __syncwarp();
      ++n;
    }
  }
  if (n >= kUnits && !wait(&sm.unit_empty[n % kUnits], n / kUnits - 1, p)) return;
  if (lane == 0) {
    sm.unit[n % kUnits].rows = -1;
    mbar_arrive(&sm.unit_full[n % kUnits]);
  }
}

// ---- warps 14-17: keys -----------------------------------------------------------------------------------
// Expands two blocks of 16 tokens (this warp's quarter of the stage) of a 4-bit part: codes as bf16 at their
// swizzled places, and the tokens' scales.
template <int D>
__device__ __forceinline__ void expand_keys(unsigned char* stage, float4* scales, const char* head, const Unit& u, int w, int lane) {
  constexpr int NG = D / kGroup4;
  const int l4 = lane & 3, l8 = lane >> 2;
  const char* tile = head + (uint64_t)(u.tile + (w >> 1)) * kv4_tile_bytes(D);
  if ((w >> 1) * kTile >= u.nv) return;  // the second tile does not exist
  uint4 c[2][NG];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int g = 0; g < NG; ++g) c[i][g] = reinterpret_cast<const uint4*>(tile)[(((w & 1) * 2 + i) * NG + g) * 32 + lane];
  const uint32_t* words = reinterpret_cast<const uint32_t*>(tile + kv4_code_bytes(D)) + ((w & 1) * 32 + lane) * NG;
  const uint32_t sl0 = words[0], sl1 = words[NG - 1];
  const float s0 = kv4_s(sl0), s1 = kv4_s(sl1);
  scales[w * 32 + lane] = make_float4(s0, fmaf(0.5f, s0, kv4_lo(sl0)), s1, fmaf(0.5f, s1, kv4_lo(sl1)));
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t word[4] = {c[i][g].x, c[i][g].y, c[i][g].z, c[i][g].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // token l8 + 8 h: nibbles h (entries e, e + 1) and h + 2 (e + 2, e + 3) of every word
        const uint32_t row = w * 32 + i * 16 + l8 + 8 * h;
        uint32_t x[8];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t r = ((word[kk] >> (4 * h + 8 * k)) & 0x000f000fu) | 0x43004300u;  // 128 + c
            asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x43004300u));
            x[2 * kk + k] = r;
          }
        unsigned char* block = stage + g * 16384;
        *reinterpret_cast<uint4*>(block + swz128(row, l4)) = make_uint4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint4*>(block + swz128(row, 4 + l4)) = make_uint4(x[4], x[5], x[6], x[7]);
      }
    }
}

template <int D>
__device__ __forceinline__ void load_keys(Smem& sm, const Params& p, int w, int lane) {
  constexpr int CB = D / 64;
  int issued = 0;  // units whose copies have been asked for
  const bool done = for_units(sm, p, lane, [&](int n, const Unit& u) {
    const int st = n % kKStages;
    if (n >= kKStages && !wait(&sm.k_empty[st], n / kKStages - 1, p)) return false;
    if (u.four) {
      expand_keys<D>(sm.k[st], sm.scales[n % kUnits], p.layer4 + (uint64_t)u.kvh * p.head_stride4, u, w, lane);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.k_full[st]);
    } else if (lane == 0) {
      if (w == 0) {
        const int nh = u.nv > kTile ? 2 : 1;  // 64-token pool tiles
        mbar_arrive_expect_tx(&sm.k_full[st], nh * CB * 8192);
        const char* src = p.layer16 + (uint64_t)u.kvh * p.head_stride16 + (uint64_t)u.tile * p.tile_bytes16;
        for (int h = 0; h < nh; ++h)
          for (int cb = 0; cb < CB; ++cb)
            bulk_g2s(sm.k[st] + cb * 16384 + h * 8192, src + (uint64_t)h * p.tile_bytes16 + cb * 8192, 8192, &sm.k_full[st]);
      } else {
        mbar_arrive(&sm.k_full[st]);
      }
    }
    issued = n + 1;
    if (lane == 0) mbar_arrive(&sm.scales_full[n % kUnits]);
    return true;
  });
  if (!done && w == 0 && lane == 0)  // (after a wait that gave up)
    for (int n = max(0, issued - kKStages); n < issued; ++n) mbar_drain(&sm.k_full[n % kKStages], (n / kKStages) & 1, p.status);
}

// ---- warps 8-13: query rows --------------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void load_queries(Smem& sm, const Params& p, int slot, int lane) {
  constexpr int CB = D / 64;
  const int sh = __ffs(p.gqa) - 1, chunk = lane & 7;
  unsigned char* tile = sm.q[slot >> 1][slot & 1];  // (the second column block 16384 bytes further)
  int item = 0;
  for_units(sm, p, lane, [&](int, const Unit& u) {
    const int end = item + u.items, head0 = u.kvh * p.gqa;
    for (int it = item + (slot + kSlots - item % kSlots) % kSlots; it < end; it += kSlots) {
      const int row0 = (it - item) * kItemRows, rows = min(kItemRows, u.rows - row0);
      auto request = [&](int row) {
        return row < rows ? GF_CLAMP(p.grp_req[GF_CLAMP(u.grp_begin + ((row0 + row) >> sh), p.num_pairs, p.status, 131)], p.num_requests, p.status, 132) : 0;
      };
      const int id[2] = {request(lane), request(lane + 32)};  // of rows lane and lane + 32
      if (it >= kSlots && !wait(&sm.q_empty[slot], it / kSlots - 1, p)) return false;
      const __nv_bfloat16* from = p.q + (size_t)head0 * D + chunk * 8;
      const uint32_t to = smem_u32(tile) + swz128(lane >> 3, chunk), to1 = smem_u32(tile) + swz128(4 + (lane >> 3), chunk);
#pragma unroll
      for (int k = 0; k < 16; ++k) {  // four rows; those that do not exist become zeros
        const int row = 4 * k + (lane >> 3);
        const int req = __shfl_sync(0xffffffffu, id[k >> 3], row & 31);
        const __nv_bfloat16* src = from + ((size_t)req * p.num_q_heads + (row & (p.gqa - 1))) * D;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) copy16((k & 1 ? to1 : to) + (k >> 1) * 1024 + cb * 16384, src + cb * 64, row < rows ? 16 : 0);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = lane + 32 * h;
        sm.off[slot][row] = row < rows ? -1.4426950408889634f * p.lse[(size_t)id[h] * p.num_q_heads + head0 + (row & (p.gqa - 1))] : -INFINITY;
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      if (u.four) {
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const int row = lane + 32 * h;
            uint64_t sum = 0;  // two sums, of the even and the odd entries
            if (row < rows) {
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const uint4 v = *reinterpret_cast<const uint4*>(tile + cb * 16384 + swz128(row, c));
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = f2_add(sum, f2_pack(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u)));
              }
            }
            float even, odd;
            f2_unpack(sum, even, odd);
            sm.qsum[slot][cb][row] = even + odd;
          }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full[slot]);
    }
    item = end;
    return true;
  });
}

// ---- warp 18: MMAs ---------------------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void issue_mmas(Smem& sm, const Params& p, int lane) {
  constexpr int CB = D / 64;
  const uint32_t tmem = sm.tmem_base;
  int item = 0;
  for_units(sm, p, lane, [&](int n, const Unit& u) {
    const int st = n % kKStages;
    if (!wait(&sm.k_full[st], n / kKStages, p)) return false;
    for (int i = 0; i < u.items;) {
      const int two = (item & 1) == 0 && i + 1 < u.items;  // this item and the next, whose slots lie side by side
      for (int k = 0; k <= two; ++k) {
        const int it = item + k;
        if (!wait(&sm.q_full[it % kSlots], it / kSlots, p)) return false;
        if (it >= kBufs && !wait(&sm.s_empty[it % kBufs], it / kBufs - 1, p)) return false;
      }
      tc_fence_after_sync();
      i += 1 + two;
      if (lane == 0) {
        const int slot = item % kSlots, rows = min(kItemRows * (1 + two), u.rows - (i - 1 - two) * kItemRows);
        const uint32_t idesc = tc_idesc_bf16(kBlock, (rows + 15) & ~15, false);
        const uint64_t kd = tc_smem_desc(smem_u32(sm.k[st]), 0, 1024);
        const uint64_t qd = tc_smem_desc(smem_u32(sm.q[slot >> 1][slot & 1]), 0, 1024);
        const uint32_t d = tmem + item_columns(item);
        if (u.four) {  // one accumulator per group
          umma_ss_kloop<1>(d, kd, qd, idesc);
          if (CB == 2) umma_ss_kloop<1>(d + 128, kd + 1024, qd + 1024, idesc);
        } else {
          umma_ss_kloop<CB>(d, kd, qd, idesc);
        }
        tc_commit(&sm.s_full[item % kBufs]);
        if (two) tc_commit(&sm.s_full[(item + 1) % kBufs]);
        if (i == u.items) tc_commit(&sm.k_empty[st]);
      }
      __syncwarp();
      item += 1 + two;
    }
    return true;
  });
  if (lane == 0) {  // (every MMA is waited for already, unless a wait gave up)
    tc_commit(&sm.mmas_done);
    mbar_drain(&sm.mmas_done, 0, p.status);
  }
}

// ---- warps 0-7: exponentials and sums --------------------------------------------------------------------------
struct TokenScales { uint64_t s[2], z[2]; };  // a 4-bit unit's: s and lo + s / 2 in log2 units, twice each, per group

__device__ __forceinline__ uint64_t pair_at(const float4& v, int h) { return h ? f2_pack(v.z, v.w) : f2_pack(v.x, v.y); }

// Columns c0 .. c0 + 15 of this thread's token: sum[0..3] += 2^(score - lse), four sums apart.
template <int D, bool kFour>
__device__ __forceinline__ void add_columns(uint64_t (&sum)[4], uint32_t tmem, const float* off, const float* q0, const float* q1,
                                            const TokenScales& t, uint64_t scale2) {
  constexpr bool kTwo = kFour && D == 128;
  uint32_t acc[16], acc1[16];
  tmem_ld16(tmem, acc);
  if (kTwo) tmem_ld16(tmem + 128, acc1);
  uint64_t x[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float4 o = reinterpret_cast<const float4*>(off)[k];
    x[2 * k] = pair_at(o, 0);
    x[2 * k + 1] = pair_at(o, 1);
    if (kFour) {
      const float4 a = reinterpret_cast<const float4*>(q0)[k];
      x[2 * k] = f2_fma(pair_at(a, 0), t.z[0], x[2 * k]);
      x[2 * k + 1] = f2_fma(pair_at(a, 1), t.z[0], x[2 * k + 1]);
    }
    if (kTwo) {
      const float4 b = reinterpret_cast<const float4*>(q1)[k];
      x[2 * k] = f2_fma(pair_at(b, 0), t.z[1], x[2 * k]);
      x[2 * k + 1] = f2_fma(pair_at(b, 1), t.z[1], x[2 * k + 1]);
    }
  }
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = f2_fma(f2_pack(__uint_as_float(acc[2 * i]), __uint_as_float(acc[2 * i + 1])), kFour ? t.s[0] : scale2, x[i]);
    if (kTwo) x[i] = f2_fma(f2_pack(__uint_as_float(acc1[2 * i]), __uint_as_float(acc1[2 * i + 1])), t.s[1], x[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float lo, hi;
    f2_unpack(x[i], lo, hi);
    sum[i & 3] = f2_add(sum[i & 3], f2_pack(fast_exp2(lo), fast_exp2(hi)));
  }
}

template <int D>
__device__ __forceinline__ void sum_weights(Smem& sm, const Params& p, int warp, int lane) {
  const int group = warp >> 2, token = (warp & 3) * 32 + lane;
  const uint32_t lanes = sm.tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
  const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2);
  int item = 0, handed = 0;
  for_units(sm, p, lane, [&](int n, const Unit& u) {
    TokenScales t{};
    if (u.four) {
      if (!wait(&sm.scales_full[n % kUnits], n / kUnits, p)) return false;
      const float4 x = sm.scales[n % kUnits][token];
      const float f = p.scale_log2;
      t.s[0] = f2_pack(x.x * f, x.x * f);
      t.z[0] = f2_pack(x.y * f, x.y * f);
      t.s[1] = f2_pack(x.z * f, x.z * f);
      t.z[1] = f2_pack(x.w * f, x.w * f);
    }
    uint64_t part[4] = {0, 0, 0, 0};  // pairs of +0
    const int end = item + u.items;
    for (int it = item + ((item & 1) != group); it < end; it += 2) {
      const int slot = it % kSlots, buf = it % kBufs;
      const int rows = min(kItemRows, u.rows - (it - item) * kItemRows);
      if (!wait(&sm.q_full[slot], it / kSlots, p)) return false;  // the columns' numbers
      if (!wait(&sm.s_full[buf], it / kBufs, p)) return false;
      tc_fence_after_sync();
      const uint32_t acc = lanes + item_columns(it);
      // (columns past the rows, up to a multiple of 16, weigh 2^-inf)
      if (u.four)
        for (int c0 = 0; c0 < rows; c0 += 16)
          add_columns<D, true>(part, acc + c0, &sm.off[slot][c0], &sm.qsum[slot][0][c0], &sm.qsum[slot][1][c0], t, scale2);
      else
        for (int c0 = 0; c0 < rows; c0 += 16) add_columns<D, false>(part, acc + c0, &sm.off[slot][c0], nullptr, nullptr, t, scale2);
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sm.s_empty[buf]);
        mbar_arrive(&sm.q_empty[slot]);
      }
    }
    item = end;
    float lo, hi;
    f2_unpack(f2_add(f2_add(part[0], part[1]), f2_add(part[2], part[3])), lo, hi);
    float sum = lo + hi;
    static_assert(kNarrowRows >= kItemRows, "a unit has two items or more, some of either group");
    if (group == 1) {  // hands its sums to group 0
      if (handed > 0 && !wait(&sm.handed_empty, handed - 1, p)) return false;
      sm.handed[token] = sum;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.handed_full);
      ++handed;
      return true;
    } else {
      if (!wait(&sm.handed_full, handed, p)) return false;
      sum += sm.handed[token];
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.handed_empty);
      ++handed;
    }
    if (token < u.nv) {
      float* w = p.weights + (int64_t)u.kvh * p.slots + u.slot0 + token;
      *w = p.accumulate ? *w + sum : sum;
    }
    return true;
  });
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) k_weights_wide(const Params p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Smem& sm = *reinterpret_cast<Smem*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(&sm.unit_full[i], 1);
      mbar_init(&sm.unit_empty[i], kUnitReaders);
      mbar_init(&sm.scales_full[i], 4);
    }
    for (int i = 0; i < kKStages; ++i) { mbar_init(&sm.k_full[i], 4); mbar_init(&sm.k_empty[i], 1); }
    for (int i = 0; i < kSlots; ++i) { mbar_init(&sm.q_full[i], 1); mbar_init(&sm.q_empty[i], 4); }
    for (int i = 0; i < kBufs; ++i) { mbar_init(&sm.s_full[i], 1); mbar_init(&sm.s_empty[i], 4); }
    mbar_init(&sm.handed_full, 4);
    mbar_init(&sm.handed_empty, 4);
    mbar_init(&sm.mmas_done, 1);
    mbar_fence_init();
  }
  chain_enter();
  if (!tables_usable(*p.hdr, p.slot_cap)) return;  // uniform over the launch
  if (warp == 18) tmem_alloc(&sm.tmem_base, 512);
  const int S = p.hdr->num_segments, per = (S + kBuckets - 1) / kBuckets;
  scan_segments<kThreads>(p, sm.start, sm.warp_tot, S, per, kBlock);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp < 8) sum_weights<D>(sm, p, warp, lane);
  else if (warp < 14) load_queries<D>(sm, p, warp - 8, lane);
  else if (warp < 18) load_keys<D>(sm, p, warp - 14, lane);
  else if (warp == 18) issue_mmas<D>(sm, p, lane);
  else schedule(sm, p, per, S, lane);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 18) tmem_dealloc(sm.tmem_base, 512);
}

}  // namespace

int launch_weights(const PoolGeom& pool16, const PoolGeom& pool4, const AttnShape& sh, const TablesDev& t, int layer, const void* q,
                   const float* lse, int accumulate, float* weights, int64_t slots, int most_rows, int32_t* status, bool chained,
                   cudaStream_t st, cudaStream_t side) {
  const bool any_wide = most_rows < 0 || most_rows > kNarrowRows;
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
  auto go = [&](auto wide, auto narrow, size_t narrow_smem, bool (&optin)[2][kMaxDevices]) {
    if (!ensure_dynamic_smem(wide, sizeof(Smem), optin[0]) || !ensure_dynamic_smem(narrow, narrow_smem, optin[1])) return false;
    if (any_wide && chained) launch_chained(wide, dim3((unsigned)t.num_sms), dim3(kThreads), sizeof(Smem), st, p);
    else if (any_wide) wide<<<t.num_sms, kThreads, sizeof(Smem), st>>>(p);
    const dim3 grid((unsigned)(3 * t.num_sms));
    if (side) narrow<<<grid, kNarrowThreads, narrow_smem, side>>>(p);
    else if (any_wide || chained) launch_chained(narrow, grid, dim3(kNarrowThreads), narrow_smem, st, p);
    else narrow<<<grid, kNarrowThreads, narrow_smem, st>>>(p);
    return true;
  };
  static bool optin[2][2][kMaxDevices] = {};
  if (!(sh.head_dim == 128 ? go(k_weights_wide<128>, k_weights_narrow<128>, sizeof(NarrowSmem<128>), optin[0])
                           : go(k_weights_wide<64>, k_weights_narrow<64>, sizeof(NarrowSmem<64>), optin[1])))
    return -1;
  return cudaGetLastError() == cudaSuccess ? 1 + any_wide : -1;
}

}  // namespace gf
