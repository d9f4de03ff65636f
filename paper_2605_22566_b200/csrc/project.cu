// A projection that all rows share, with a low-rank adapter of each row's own:
//   y[t] = W x[t] + scale_a B_a (A_a x[t]),  a the row's adapter.
//
// W x: tcgen05 MMAs with the output features as the MMA's rows (128 of W at a time, K-major) and up to 256 rows of x as its
// columns, so that one row and thousands go the same way; both operands come by TMA in stages of 64 entries of K, the sums stay in
// tensor memory in fp32.  Few rows leave few tiles: then a cluster of CTAs shares a tile, each with a part of K, and
// joins its parts through shared memory in a fixed order.
//
// The adapters are more entries of K.  For every adapter that rows of a tile of x name (a slot of the tile), h = scale_a A_a x is a
// [rows, rank] operand with zeros in the other rows, and B_a, [features, rank], stands beside W: the sums go on over the tile's
// slots, in the same pipeline, and nothing is left for the warps that take them out of tensor memory.  h is rounded to two bf16
// numbers, its nearest and the nearest of what is left (2^-17 of it), and multiplied twice.  k_adapter_down writes these operands in the layout
// of shared memory; only the copies behind a tile's last entry of W wait for it.
// (The same sums on the CUDA cores, while the MMAs ran, took 568 us for 8192 rows with adapters of rank 16 and 1143 of rank 64,
// where W x alone takes 295: their reads of B and h wait behind the copies' traffic.)
#include <cuda.h>

#include <algorithm>

#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kFeat = 128;        // output features of a tile
constexpr int kStep = 64;         // entries of K in a stage
constexpr int kThreads = 256;
constexpr int kGroup = 8;         // rows of x that are taken out of tensor memory together

// The slots of the tiles of x, in the caller's scratch.
struct Slots {
  int32_t* count;        // [row_tiles]
  int32_t* adapter;      // [row_tiles][most]
  char* h;               // [row_tiles][most][2][nt][padded rank], swizzled like a stage's operand
  int most;
  int rank, padded;      // padded: 16, 32 or 64
  uint32_t block;        // bytes of one [nt][padded]
};

struct ProjectArgs {
  int rows, in_dim, out_dim, nt;        // nt: rows of x in a tile
  int feat_tiles, row_tiles, stages;
  int splits;                           // CTAs that share a tile
  uint32_t tmem_cols, acc_cols;         // allocated; from one accumulator to the next
  Slots slots;
  void* y;
  int64_t y_stride;
  int y_fp32;
  int32_t* status;
};

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
               "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

__device__ __forceinline__ uint64_t bf16x2_to_f2(uint32_t v) { return f2_pack(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
               : "memory");
}

// Shared-memory matrix descriptor of a K-major operand whose rows are `row_bytes` (32, 64 or 128) long and swizzled over that many.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, int row_bytes) {
  const uint64_t kind = row_bytes == 128 ? 2 : row_bytes == 64 ? 4 : 6;
  return (tc_smem_desc(saddr, 0, 8 * row_bytes) & ~((uint64_t)7 << 61)) | kind << 61;
}
// Where the 16-byte piece c of row r of such an operand is.
__device__ __forceinline__ uint32_t operand_at(int r, int c, int row_bytes) {
  const int x = row_bytes == 128 ? r & 7 : row_bytes == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
  return (uint32_t)(r * row_bytes + ((c ^ x) << 4));
}

__device__ __forceinline__ void store_y(const ProjectArgs& a, int row, int feat, float v) {
  if (feat < a.out_dim && row >= 0 && row < a.rows) {
    const int64_t at = (int64_t)row * a.y_stride + feat;
    if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
    else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
  }
}

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared memory: the ring of stages (kFeat rows of W, then nt rows of x, 128 bytes each, 128-byte swizzle; a stage of the
// adapters holds one slot of rank 32, two of rank 16, or the first or second half of one of rank 64), which a cluster uses
// again for its parts of the sums; behind it the barriers.
template <bool kAdapters>
__global__ void __launch_bounds__(kThreads, 1) k_project(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
                                                         const __grid_constant__ CUtensorMap b_map, const __grid_constant__ ProjectArgs a) {
  extern __shared__ __align__(1024) char smem_raw[];
  char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t w_bytes = kFeat * 128u, x_bytes = (uint32_t)a.nt * 128u, stage_bytes = w_bytes + x_bytes;
  const uint32_t ring = max(stage_bytes * a.stages, a.splits > 1 ? (uint32_t)a.nt * kFeat * 4u : 0u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + ring);
  uint64_t* empty = full + a.stages;
  uint64_t* acc_full = empty + a.stages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* drained = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
  const int group = blockIdx.x / a.splits, groups = gridDim.x / a.splits, part = blockIdx.x - group * a.splits;
  const int tiles = a.feat_tiles * a.row_tiles;
  const int steps_all = (a.in_dim + kStep - 1) / kStep;
  const int step0 = (int)((int64_t)steps_all * part / a.splits), step1 = (int)((int64_t)steps_all * (part + 1) / a.splits);
  const Slots& sl = a.slots;
  const int h_row = sl.padded * 2;                       // bytes of a row of h, and of B's
  const uint32_t b_bytes = kFeat * (uint32_t)h_row;
  // the CTA's slots of a tile of x
  auto my_slots = [&](int row_tile, int& s0, int& s1) {
    const int n = *(volatile int32_t*)(sl.count + row_tile);
    s0 = n * part / a.splits;
    s1 = n * (part + 1) / a.splits;
  };
  if (tid == 0) {
    for (int i = 0; i < a.stages; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, 4); }
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (wid == 1) tmem_alloc(tmem_slot, a.tmem_cols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  if (wid == 0) {
    if (lane == 0) {
      int s = 0;
      int64_t issued = 0;
      uint32_t phase = 0;
      bool ok = true, waited = false;
      auto next = [&] { if (++s == a.stages) { s = 0; phase ^= 1u; } ++issued; };
      for (int tile = group; tile < tiles && ok; tile += groups) {
        const int f0 = (tile % a.feat_tiles) * kFeat, row_tile = tile / a.feat_tiles, t0 = row_tile * a.nt;
        int s0 = 0, s1 = 0;
        if (kAdapters && waited) my_slots(row_tile, s0, s1);  // (asked for here, used behind the loop)
        for (int k = step0; k < step1; ++k) {
          if (!(ok = mbar_wait(empty + s, phase ^ 1u, a.status))) break;
          mbar_arrive_expect_tx(full + s, stage_bytes);
          tma_load_2d(smem + s * stage_bytes, &w_map, k * kStep, f0, full + s);
          tma_load_2d(smem + s * stage_bytes + w_bytes, &x_map, k * kStep, t0, full + s);
          next();
        }
        if (kAdapters && ok) {
          if (!waited) {
            asm volatile("griddepcontrol.wait;" ::: "memory");  // the slots are the kernel's before this one
            waited = true;
            my_slots(row_tile, s0, s1);
          }
          const int32_t* which = sl.adapter + (int64_t)row_tile * sl.most;
          int ahead[2] = {s0 < s1 ? __ldcg(which + s0) : 0, s0 + 1 < s1 ? __ldcg(which + s0 + 1) : 0};  // of the next two slots
          const char* h = sl.h + (int64_t)row_tile * sl.most * 2 * sl.block;
          for (int i = s0; i < s1 && ok; ++i) {
            char* at = smem + s * stage_bytes;
            const int id = ahead[0], id2 = ahead[1];
            const int taken = h_row == 32 ? 2 : 1;
            ahead[0] = taken == 2 ? (i + 2 < s1 ? __ldcg(which + i + 2) : 0) : id2;
            ahead[1] = i + taken + 1 < s1 ? __ldcg(which + i + taken + 1) : 0;
            if (!(ok = mbar_wait(empty + s, phase ^ 1u, a.status))) break;
            if (h_row == 128) {
              for (int half = 0; half < 2 && ok; ++half) {
                at = smem + s * stage_bytes;
                if (half && !(ok = mbar_wait(empty + s, phase ^ 1u, a.status))) break;
                mbar_arrive_expect_tx(full + s, b_bytes + sl.block);
                tma_load_3d(at, &b_map, 0, f0, id, full + s);
                bulk_g2s(at + w_bytes, h + (int64_t)(2 * i + half) * sl.block, sl.block, full + s);
                next();
              }
            } else if (h_row == 64) {
              mbar_arrive_expect_tx(full + s, b_bytes + 2 * sl.block);
              tma_load_3d(at, &b_map, 0, f0, id, full + s);
              bulk_g2s(at + w_bytes, h + (int64_t)(2 * i) * sl.block, 2 * sl.block, full + s);
              next();
            } else {
              const int both = i + 1 < s1 ? 2 : 1;
              mbar_arrive_expect_tx(full + s, both * (b_bytes + 2 * sl.block));
              tma_load_3d(at, &b_map, 0, f0, id, full + s);
              if (both == 2) tma_load_3d(at + b_bytes, &b_map, 0, f0, id2, full + s);
              bulk_g2s(at + w_bytes, h + (int64_t)(2 * i) * sl.block, both * 2 * sl.block, full + s);
              i += both - 1;
              next();
            }
          }
        }
      }
      // nothing of its own is on the way when it leaves, also where it gave up
      for (int64_t i = issued > a.stages ? issued - a.stages : 0; i < issued; ++i)
        mbar_drain(full + i % a.stages, (uint32_t)(i / a.stages) & 1u, a.status);
    }
  } else if (wid == 1) {
    if (lane == 0) {
      const uint32_t idesc = tc_idesc_bf16(kFeat, a.nt, false);
      int s = 0, n = 0;
      uint32_t phase = 0;
      bool ok = true, waited = false;
      auto next = [&] {
        tc_commit(empty + s);
        if (++s == a.stages) { s = 0; phase ^= 1u; }
      };
      for (int tile = group; tile < tiles && ok; tile += groups, ++n) {
        const int buf = n & 1;
        int s0 = 0, s1 = 0;
        if (kAdapters && waited) my_slots(tile / a.feat_tiles, s0, s1);
        if (!(ok = mbar_wait(acc_empty + buf, ((n >> 1) & 1) ^ 1, a.status))) break;
        tc_fence_after_sync();
        const uint32_t d = tmem + buf * a.acc_cols;
        for (int k = step0; k < step1; ++k) {
          if (!(ok = mbar_wait(full + s, phase, a.status))) break;
          tc_fence_after_sync();
          const uint64_t wd = tc_smem_desc(smem_u32(smem + s * stage_bytes), 0, 1024);
          const uint64_t xd = tc_smem_desc(smem_u32(smem + s * stage_bytes + w_bytes), 0, 1024);
#pragma unroll
          for (int i = 0; i < kStep / 16; ++i) umma_ss(d, wd + 2 * i, xd + 2 * i, idesc, k > step0 || i > 0);
          next();
        }
        if (kAdapters && ok) {
          if (!waited) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
            my_slots(tile / a.feat_tiles, s0, s1);
          }
          // stages: two a slot of rank 64, one of rank 32, one for two of rank 16
          const int stages = h_row == 128 ? 2 * (s1 - s0) : h_row == 64 ? s1 - s0 : (s1 - s0 + 1) / 2;
          for (int i = 0; i < stages; ++i) {
            if (!(ok = mbar_wait(full + s, phase, a.status))) break;
            tc_fence_after_sync();
            const uint32_t at = smem_u32(smem + s * stage_bytes), ht = at + w_bytes;
            if (h_row == 128) {
              const uint64_t bd = operand_desc(at, 128), hd = operand_desc(ht, 128);
#pragma unroll
              for (int j = 0; j < 4; ++j) umma_ss(d, bd + 2 * j, hd + 2 * j, idesc, 1);
            } else if (h_row == 64) {
              const uint64_t bd = operand_desc(at, 64);
#pragma unroll
              for (int j = 0; j < 4; ++j) umma_ss(d, bd + 2 * (j & 1), operand_desc(ht + (j >> 1) * sl.block, 64) + 2 * (j & 1), idesc, 1);
            } else {
              const int both = s0 + 2 * i + 1 < s1 ? 4 : 2;
              for (int j = 0; j < both; ++j) umma_ss(d, operand_desc(at + (j >> 1) * b_bytes, 32), operand_desc(ht + j * sl.block, 32), idesc, 1);
            }
            next();
          }
        }
        tc_commit(acc_full + buf);
      }
      if (!ok) {  // (otherwise the tiles' own waits have seen the last of them)
        tc_commit(drained);
        mbar_drain(drained, 0, a.status);
      }
    }
  } else if (wid >= 4) {
    const int w = wid - 4;
    const uint32_t lanes = tmem + ((uint32_t)(w * 32) << 16);
    if (kAdapters) asm volatile("griddepcontrol.wait;" ::: "memory");  // (what is written here may be read by kernels before)
    int n = 0;
    for (int tile = group; tile < tiles; tile += groups, ++n) {
      const int feat = (tile % a.feat_tiles) * kFeat + w * 32 + lane, t0 = (tile / a.feat_tiles) * a.nt, buf = n & 1;
      if (!mbar_wait(acc_full + buf, (n >> 1) & 1, a.status)) break;
      tc_fence_after_sync();
      if (a.splits > 1) break;  // joined below
      for (int g = 0; g < a.nt && t0 + g < a.rows; g += kGroup) {
        uint32_t r[kGroup];
        tmem_ld8(lanes + buf * a.acc_cols + g, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < kGroup; ++j) store_y(a, t0 + g + j, feat, __uint_as_float(r[j]));
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(acc_empty + buf);
    }
  }
  __syncwarp();
  if (a.splits > 1) {
    __syncthreads();
    // One tile a cluster: the parts go to shared memory (the ring's: its last MMA is done), [row of x][feature], and each CTA adds
    // those of its share of the rows.
    const int f0 = (group % a.feat_tiles) * kFeat, t0 = (group / a.feat_tiles) * a.nt;
    float* parts = reinterpret_cast<float*>(smem);
    const int w = wid - 4;
    if (wid >= 4) {
      for (int g = 0; g < a.nt; g += kGroup) {
        uint32_t r[kGroup];
        tmem_ld8(tmem + ((uint32_t)(w * 32) << 16) + g, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < kGroup; ++j) parts[(g + j) * kFeat + w * 32 + lane] = __uint_as_float(r[j]);
      }
    }
    __syncthreads();
    cluster_sync_all();
    if (wid >= 4) {
      for (int g = part * kGroup; g < a.nt && t0 + g < a.rows; g += a.splits * kGroup) {
        float sum[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) sum[j] = 0.f;
        for (int p = 0; p < a.splits; ++p) {
          uint32_t from;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(smem_u32(parts + g * kFeat + w * 32 + lane)), "r"(p));
#pragma unroll
          for (int j = 0; j < kGroup; ++j) {
            float x;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(from + j * kFeat * 4) : "memory");
            sum[j] += x;
          }
        }
#pragma unroll
        for (int j = 0; j < kGroup; ++j) store_y(a, t0 + g + j, f0 + w * 32 + lane, sum[j]);
      }
    }
    __syncthreads();
    cluster_sync_all();  // nobody leaves while its part is read
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (wid == 1) tmem_dealloc(tmem, a.tmem_cols);
}

// ---- h -------------------------------------------------------------------------------------------------
// Both kernels below find a tile's slots by themselves: the adapters that its rows name, ascending, as bits in shared memory (one
// bit an adapter), so that an adapter's slot is the number of bits below its own.
constexpr int kMaxAdapters = GF_MAX_ADAPTERS;

struct TileSlots {
  uint32_t bits[kMaxAdapters / 32];
};

__device__ __forceinline__ int adapter_of(const int32_t* __restrict__ adapter, int row, int num_adapters, bool report, int32_t* status) {
  const int id = adapter[row];
  if (id >= 0 && id < num_adapters) return id;
  if (id != -1 && report) atomicCAS(status + kStatusReport, 0, (int)GF_ERR_INVALID_ARG);
  return -1;
}
// All threads of a CTA: the bits of rows t0 .. t0 + n.
__device__ void tile_slots(TileSlots& ts, const int32_t* __restrict__ adapter, int t0, int n, int num_adapters, int32_t* status) {
  for (int i = threadIdx.x; i < (num_adapters + 31) / 32; i += blockDim.x) ts.bits[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int id = adapter_of(adapter, t0 + i, num_adapters, true, status);
    if (id >= 0) atomicOr(&ts.bits[id >> 5], 1u << (id & 31));
  }
  __syncthreads();
}
// All lanes of a warp: how many slots come before the adapter `id` (num_adapters: how many there are).
__device__ __forceinline__ int slot_of(const TileSlots& ts, int id) {
  int n = 0;
  for (int i = threadIdx.x & 31; i <= id >> 5; i += 32) n += __popc(i < id >> 5 ? ts.bits[i] : id & 31 ? ts.bits[i] & ((1u << (id & 31)) - 1u) : 0u);
  return __reduce_add_sync(0xffffffffu, n);
}
// All threads of a CTA write the list of a tile's slots.
__device__ void write_slots(const TileSlots& ts, const Slots& sl, int row_tile, int num_adapters, int count) {
  if (threadIdx.x == 0) sl.count[row_tile] = count;
  const int lane = threadIdx.x & 31, words = (num_adapters + 31) / 32;
  for (int i = threadIdx.x >> 5; i < words; i += blockDim.x >> 5) {
    const int first = slot_of(ts, i * 32);
    const uint32_t w = ts.bits[i];
    if (w >> lane & 1u) sl.adapter[(int64_t)row_tile * sl.most + first + __popc(w & ((1u << lane) - 1u))] = i * 32 + lane;
  }
}
// One 16-byte piece (8 ranks, from h in shared memory) of a row's operand, of the first or second number.
__device__ __forceinline__ uint4 h_piece(const float* __restrict__ h, int half) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[j] = h[2 * i + j];
      const float first = __bfloat162float(__float2bfloat16_rn(v[j]));
      if (half) v[j] = fabsf(first) <= 3.3895e38f ? v[j] - first : 0.f;  // (nothing is left of an infinity, or a NaN)
    }
    w[i] = pack_bf16(v[0], v[1]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// A row's part of its tile's operands: h in its adapter's slot (-1: none), zeros in the others.  By `threads` threads, this the `who`-th.
__device__ void write_row(const Slots& sl, int row_tile, int row_in_tile, int count, int slot, const float* h, int who, int threads) {
  const int pieces = sl.padded >> 3, per_slot = 2 * pieces;
  char* base = sl.h + (int64_t)row_tile * sl.most * 2 * sl.block;
  for (int i = who; i < count * per_slot; i += threads) {
    const int s = i / per_slot, half = (i - s * per_slot) / pieces, c = i % pieces;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (s == slot && c * 8 < sl.rank) v = h_piece(h + c * 8, half);
    *reinterpret_cast<uint4*>(base + (int64_t)(2 * s + half) * sl.block + operand_at(row_in_tile, c, sl.padded * 2)) = v;
  }
}

// A CTA per row: the warps share K, each lane 8 entries of x against 16 rows of A at a time, all asked for at once; the lanes' sums
// are joined by halving the values that a lane holds.  fp32 throughout.  Bound: latency (a load of the row's adapter, one of A, and the
// join), and for hundreds of rows L2, which reads A once per row.
constexpr int kRowThreads = 512, kRowWarps = kRowThreads / 32;
__global__ void __launch_bounds__(kRowThreads) k_adapter_down_rows(const __nv_bfloat16* __restrict__ x, int64_t x_stride, int rows, int in_dim, int nt,
                                                                   const int32_t* __restrict__ adapter, int num_adapters, Slots sl,
                                                                   const __nv_bfloat16* __restrict__ a, const float* __restrict__ scale, int32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ TileSlots ts;
  __shared__ float sums[kRowWarps][64], h[64];
  const int t = blockIdx.x, tile = t / nt, t0 = tile * nt, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, rank = sl.rank;
  const int which = adapter_of(adapter, t, num_adapters, false, status);
  tile_slots(ts, adapter, t0, min(nt, rows - t0), num_adapters, status);
  const int count = slot_of(ts, num_adapters), slot = which < 0 ? -1 : slot_of(ts, which);
  if (t == t0) write_slots(ts, sl, tile, num_adapters, count);
  if (which >= 0) {
    const __nv_bfloat16* xr = x + (int64_t)t * x_stride;
    const __nv_bfloat16* ar = a + (int64_t)which * rank * in_dim;
    for (int r0 = 0; r0 < rank; r0 += 16) {
      uint64_t acc[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = 0ull;
      for (int k = (wid * 32 + lane) * 8; k < in_dim; k += kRowThreads * 8) {
        const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
        uint4 av[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) av[r] = r0 + r < rank ? __ldg(reinterpret_cast<const uint4*>(ar + (int64_t)(r0 + r) * in_dim + k)) : make_uint4(0u, 0u, 0u, 0u);
        const uint64_t x0 = bf16x2_to_f2(xv.x), x1 = bf16x2_to_f2(xv.y), x2 = bf16x2_to_f2(xv.z), x3 = bf16x2_to_f2(xv.w);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          acc[r] = f2_fma(bf16x2_to_f2(av[r].x), x0, acc[r]);
          acc[r] = f2_fma(bf16x2_to_f2(av[r].y), x1, acc[r]);
          acc[r] = f2_fma(bf16x2_to_f2(av[r].z), x2, acc[r]);
          acc[r] = f2_fma(bf16x2_to_f2(av[r].w), x3, acc[r]);
        }
      }
      float v[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float lo, hi;
        f2_unpack(acc[r], lo, hi);
        v[r] = lo + hi;
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
      if (lane < 16 && r0 + lane < rank) sums[wid][r0 + lane] = v[0];
    }
  }
  __syncthreads();
  if (which >= 0 && tid < rank) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) sum += sums[w][tid];
    h[tid] = sum * (scale != nullptr ? scale[which] : 1.f);
  }
  __syncthreads();
  write_row(sl, tile, t - t0, count, slot, h, tid, kRowThreads);
}

// Many rows.  A CTA has 32 rows that are next to each other in the order of their adapters within a tile (each CTA ranks its tile's
// rows by itself), so most have one adapter, or a few; for each of them the warps share K, 32 entries at a time, and multiply
// the CTA's rows by A (mma.sync, rows x rank, both operands straight from L2 in 16-byte pieces: K's order within a step does
// not matter as long as both have the same), and those of the adapter's rows are kept.  The warps' sums are added in a fixed
// order.  Bound: L2, which reads A once per 32 rows of one adapter.
constexpr int kDownThreads = 256, kDownWarps = kDownThreads / 32, kDownRows = 32;
template <int RT>  // 8-row pieces of A at most
__global__ void __launch_bounds__(kDownThreads) k_adapter_down(const __nv_bfloat16* __restrict__ x, int64_t x_stride, int rows, int in_dim, int nt,
                                                               const int32_t* __restrict__ adapter, int num_adapters, Slots sl,
                                                               const __nv_bfloat16* __restrict__ a, const float* __restrict__ scale, int32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int MT = kDownRows / 16;
  extern __shared__ float sums[];  // [kDownWarps][kDownRows][rank]
  __shared__ TileSlots ts;
  __shared__ int s_id[256], s_row[256], s_sorted[256];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, rank = sl.rank;
  const int chunks = (nt + kDownRows - 1) / kDownRows, tile = blockIdx.x / chunks, chunk = blockIdx.x - tile * chunks;
  const int t0 = tile * nt, n = min(nt, rows - t0), p0 = chunk * kDownRows;
  if (p0 >= n) return;
  const int id = tid < n ? adapter_of(adapter, t0 + tid, num_adapters, false, status) : 0x7fffffff;
  s_id[tid] = id;
  tile_slots(ts, adapter, t0, n, num_adapters, status);
  const int count = slot_of(ts, num_adapters);
  if (chunk == 0) write_slots(ts, sl, tile, num_adapters, count);
  if (tid < n) {
    int before = 0;
    for (int j = 0; j < n; ++j) before += s_id[j] < id || (s_id[j] == id && j < tid);
    s_row[before] = tid;
    s_sorted[before] = id;
  }
  __syncthreads();
  const int end = min(p0 + kDownRows, n), g = lane >> 2, q = lane & 3, pieces = rank >> 3;
  const __nv_bfloat16* xr[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) xr[i] = x + (int64_t)(t0 + s_row[min(p0 + i * 8 + g, end - 1)]) * x_stride + q * 8;
  for (int j0 = p0; j0 < end;) {
    const int which = s_sorted[j0];
    int j1 = j0 + 1;
    while (j1 < end && s_sorted[j1] == which) ++j1;
    if (which >= 0) {
      float acc[MT][RT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][r][i] = 0.f;
      const __nv_bfloat16* ar = a + ((int64_t)which * rank + g) * in_dim + q * 8;
#pragma unroll 2
      for (int k = wid * 32; k < in_dim; k += kDownWarps * 32) {
        const bool in = k + q * 8 < in_dim;
        uint4 xv[2 * MT], av[RT];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) xv[i] = in ? *reinterpret_cast<const uint4*>(xr[i] + k) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int r = 0; r < RT; ++r)
          av[r] = in && r < pieces ? __ldg(reinterpret_cast<const uint4*>(ar + (int64_t)r * 8 * in_dim + k)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t lo[4] = {xv[2 * m].x, xv[2 * m + 1].x, xv[2 * m].y, xv[2 * m + 1].y};
          const uint32_t hi[4] = {xv[2 * m].z, xv[2 * m + 1].z, xv[2 * m].w, xv[2 * m + 1].w};
#pragma unroll
          for (int r = 0; r < RT; ++r)
            if (r < pieces) {
              mma_bf16(acc[m][r], lo, av[r].x, av[r].y);
              mma_bf16(acc[m][r], hi, av[r].z, av[r].w);
            }
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int i = m * 16 + half * 8 + g;
          if (p0 + i >= j0 && p0 + i < j1) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
              if (r < pieces)
                *reinterpret_cast<float2*>(sums + ((size_t)wid * kDownRows + i) * rank + r * 8 + q * 2) = make_float2(acc[m][r][2 * half], acc[m][r][2 * half + 1]);
          }
        }
    }
    j0 = j1;
  }
  __syncthreads();
  for (int i = tid; i < (end - p0) * rank; i += kDownThreads) {
    const int which = s_sorted[p0 + i / rank];
    if (which < 0) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWarps; ++w) sum += sums[(size_t)w * kDownRows * rank + i];
    sums[i] = sum * (scale != nullptr ? scale[which] : 1.f);  // (the first warp's place, read by this thread alone)
  }
  __syncthreads();
  for (int j = p0 + wid; j < end; j += kDownWarps) {
    const int which = s_sorted[j], slot = which < 0 ? -1 : slot_of(ts, which);
    write_row(sl, tile, s_row[j], count, slot, sums + (j - p0) * rank, lane, 32);
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

template <bool kAdapters>
int launch_main(const CUtensorMap& w_map, const CUtensorMap& x_map, const CUtensorMap& b_map, const ProjectArgs& a, int ctas, size_t smem, cudaStream_t st) {
  static bool done[kMaxDevices];
  if (!ensure_dynamic_smem(k_project<kAdapters>, 227 * 1024, done)) return -1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (a.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)a.splits;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (kAdapters) {  // behind the kernel for h, whose results only a tile's last stages need
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, k_project<kAdapters>, w_map, x_map, b_map, a) == cudaSuccess ? 1 : -1;
}

template <int RT>
bool launch_down(const gf_projection_t& p, const ProjectArgs& a, const void* x, int64_t x_stride, const int32_t* adapter, cudaStream_t st) {
  static bool done[kMaxDevices];
  if (!ensure_dynamic_smem(k_adapter_down<RT>, kDownWarps * kDownRows * RT * 8 * 4, done)) return false;
  k_adapter_down<RT><<<(unsigned)(a.row_tiles * ((a.nt + kDownRows - 1) / kDownRows)), kDownThreads, (size_t)kDownWarps * kDownRows * p.rank * 4, st>>>(
      (const __nv_bfloat16*)x, x_stride, a.rows, p.in_dim, a.nt, adapter, p.num_adapters, a.slots, (const __nv_bfloat16*)p.a_dev, p.scale_dev, a.status);
  return cudaGetLastError() == cudaSuccess;
}

// Rows of x that one pass takes: more go in several, one behind the other, so that the scratch stays bounded.
constexpr int kPassRows = 16384;

int tile_rows(int rows) { return rows >= 256 ? 256 : (rows + 15) / 16 * 16; }
size_t align_to(size_t n, size_t a) { return (n + a - 1) / a * a; }

// Where the slots of a pass stand in the scratch; its size.
size_t place_slots(Slots* sl, char* scratch, int rows, int rank, int num_adapters) {
  const int nt = tile_rows(rows), tiles = (rows + nt - 1) / nt, most = std::min(nt, num_adapters);
  const int padded = rank <= 16 ? 16 : rank <= 32 ? 32 : 64;
  const size_t count = 0, ids = align_to((size_t)tiles * 4, 128), h = ids + align_to((size_t)tiles * most * 4, 128);
  const size_t block = (size_t)nt * padded * 2;
  if (sl) *sl = Slots{(int32_t*)(scratch + count), (int32_t*)(scratch + ids), scratch + h, most, rank, padded, (uint32_t)block};
  return h + (size_t)tiles * most * 2 * block;
}

}  // namespace

size_t project_scratch_bytes(int rows, int rank, int num_adapters) { return place_slots(nullptr, nullptr, std::min(rows, kPassRows), rank, num_adapters); }

static int launch_pass(const gf_projection_t& p, int rows, const void* x, int64_t x_stride, const int32_t* adapter, void* y, int64_t y_stride, int y_fp32,
                       void* scratch, int num_sms, int32_t* status, cudaStream_t st) {
  const bool with = adapter != nullptr && p.num_adapters > 0;
  ProjectArgs a = {};
  a.rows = rows;
  a.in_dim = p.in_dim;
  a.out_dim = p.out_dim;
  a.nt = tile_rows(rows);
  a.feat_tiles = (p.out_dim + kFeat - 1) / kFeat;
  a.row_tiles = (rows + a.nt - 1) / a.nt;
  a.y = y;
  a.y_stride = y_stride;
  a.y_fp32 = y_fp32;
  a.status = status;
  if (with) place_slots(&a.slots, (char*)scratch, rows, p.rank, p.num_adapters);
  const int64_t tiles = (int64_t)a.feat_tiles * a.row_tiles;
  const int steps = (p.in_dim + kStep - 1) / kStep;
  // Few tiles: clusters of 2, 4 or 8 share them (others do not fill the GPCs), two CTAs to a multiprocessor where the stages are
  // small enough for four of them in half its shared memory.
  const uint32_t stage_bytes = kFeat * 128u + a.nt * 128u, extra = 1024 + 512;
  const int per_sm = 4 * stage_bytes + extra <= 113 * 1024 ? 2 : 1;
  a.splits = 1;
  auto fit = [&](int splits) { return (int64_t)per_sm * num_sms * (splits <= 2 ? 8 : splits == 4 ? 7 : 6) / 8; };  // (a GPC's rest takes no cluster)
  while (a.splits < 8 && tiles * a.splits * 2 <= fit(a.splits * 2) && steps / (a.splits * 2) >= 4) a.splits *= 2;
  const bool shared = tiles * a.splits > num_sms && tiles * a.splits <= (int64_t)per_sm * num_sms;
  const uint32_t room = (shared ? 113 : 227) * 1024 - extra;
  a.stages = (int)std::min<uint32_t>(12, room / stage_bytes);
  const size_t smem = extra + std::max<uint32_t>(stage_bytes * a.stages, a.splits > 1 ? (uint32_t)a.nt * kFeat * 4u : 0u);
  const int64_t groups = a.splits > 1 || shared ? tiles : std::min<int64_t>(tiles, num_sms);
  const bool single = tiles <= groups;
  uint32_t cols = 32;
  while (cols < (uint32_t)a.nt) cols *= 2;
  a.acc_cols = single ? 0 : cols;
  a.tmem_cols = single ? cols : 2 * cols;
  CUtensorMap w_map, x_map, b_map = {};
  if (!make_map(&w_map, p.w_dev, 0, p.out_dim, p.in_dim, p.w_stride, kStep, kFeat) || !make_map(&x_map, x, 0, rows, p.in_dim, x_stride, kStep, a.nt) ||
      (with && !make_map(&b_map, p.b_dev, p.num_adapters, p.out_dim, p.rank, p.rank, a.slots.padded, kFeat)))
    return -1;
  int launched = 0;
  if (with) {
    if (rows <= 4 * num_sms) {
      k_adapter_down_rows<<<(unsigned)rows, kRowThreads, 0, st>>>((const __nv_bfloat16*)x, x_stride, rows, p.in_dim, a.nt, adapter, p.num_adapters, a.slots,
                                                                  (const __nv_bfloat16*)p.a_dev, p.scale_dev, status);
      if (cudaGetLastError() != cudaSuccess) return -1;
    } else if (!(p.rank <= 16 ? launch_down<2>(p, a, x, x_stride, adapter, st) : launch_down<8>(p, a, x, x_stride, adapter, st))) {
      return -1;
    }
    ++launched;
  }
  const int ctas = (int)(groups * a.splits);
  const int n = with ? launch_main<true>(w_map, x_map, b_map, a, ctas, smem, st) : launch_main<false>(w_map, x_map, b_map, a, ctas, smem, st);
  return n < 0 ? -1 : launched + n;
}

int launch_project(const gf_projection_t& p, int rows, const void* x, int64_t x_stride, const int32_t* adapter, void* y, int64_t y_stride, int y_fp32,
                   void* scratch, int num_sms, int32_t* status, cudaStream_t st) {
  int launched = 0;
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
