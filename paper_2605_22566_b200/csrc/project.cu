// A projection that all rows share, with a low-rank adapter of each row's own:
//   y[t] = W x[t] + scale_a B_a (A_a x[t]),  a the row's adapter.
//
// W x: tcgen05 MMAs with the output features as the MMA's rows (128 of W at a time, K-major) and up to 256 rows of x as its
// columns, so that one row and thousands go the same way; both operands come by TMA in stages of 64 entries of K, the sums stay in
// tensor memory in fp32.  Few rows leave few tiles: then a cluster of CTAs shares a tile, each with a part of K, and
// joins its parts through shared memory in a fixed order.
// The adapters: h[t] = A_a x[t] is computed first (k_adapter_down, fp32, its parts over K added in a fixed order), and the warps that
// take the sums out of tensor memory add B_a h[t] in fp32 before the one rounding to the output's type: an adapter's row of B
// belongs to a thread, as the output feature does.
#include <cuda.h>

#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kFeat = 128;        // output features of a tile
constexpr int kStep = 64;         // entries of K in a stage
constexpr int kThreads = 256;
constexpr int kGroup = 8;         // rows of x whose adapters are worked on together

struct ProjectArgs {
  int rows, in_dim, out_dim, nt;        // nt: rows of x in a tile
  int feat_tiles, row_tiles, stages;
  int splits;                           // CTAs that share a tile
  int lda_parts;                        // parts that h comes in
  int rank;
  uint32_t tmem_cols, acc_cols;         // allocated; from one accumulator to the next
  const int32_t* adapter;               // [rows], null: none
  int num_adapters;
  const __nv_bfloat16* b;               // [num_adapters, out_dim, rank]
  const float* h;                       // [parts, rows, rank]
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

// What a warp knows of the adapters of the eight rows it works on.  RB: 16-byte pieces (8 entries) of a row of B at most.
template <int RB>
struct Adapters {
  const ProjectArgs& a;
  float* stage;   // [kGroup][8 RB] of shared memory, the warp's own
  int current = -1;
  uint4 row[RB > 0 ? RB : 1];  // the thread's row of the current adapter's B

  __device__ Adapters(const ProjectArgs& args, float* s) : a(args), stage(s) {}

  // out[j] = B_a h[t0 + j] for the thread's output feature `feat`, rows t0 .. t0 + 7 of x.
  __device__ void group(int t0, int feat, float (&out)[kGroup]) {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) out[j] = 0.f;
    const int lane = threadIdx.x & 31, pieces = a.rank >> 3;
    int mine = -1;
    if (lane < kGroup && t0 + lane < a.rows) {
      mine = a.adapter[t0 + lane];
      if (mine < -1 || mine >= a.num_adapters) mine = -1;  // (k_adapter_down reports it)
    }
    if (__all_sync(0xffffffffu, mine < 0)) return;
    __syncwarp();
    for (int i = lane; i < kGroup * pieces * 2; i += 32) {
      const int j = i / (pieces * 2), c = i - j * (pieces * 2);
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t0 + j < a.rows)
        for (int p = 0; p < a.lda_parts; ++p) {
          const float4 x = *reinterpret_cast<const float4*>(a.h + ((int64_t)p * a.rows + t0 + j) * a.rank + c * 4);
          s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
      *reinterpret_cast<float4*>(stage + j * (RB * 8) + c * 4) = s;
    }
    __syncwarp();
    int which[kGroup];
#pragma unroll
    for (int j = 0; j < kGroup; ++j) which[j] = __shfl_sync(0xffffffffu, mine, j);
    bool same = true;
#pragma unroll
    for (int j = 1; j < kGroup; ++j) same = same && which[j] == which[0];
    const bool real = feat < a.out_dim;
    if (same) {
      if (which[0] != current) {
        current = which[0];
        const uint4* src = reinterpret_cast<const uint4*>(a.b + ((int64_t)current * a.out_dim + feat) * a.rank);
#pragma unroll
        for (int c = 0; c < RB; ++c) row[c] = real && c < pieces ? __ldg(src + c) : make_uint4(0u, 0u, 0u, 0u);
      }
      uint64_t acc[kGroup];
#pragma unroll
      for (int j = 0; j < kGroup; ++j) acc[j] = 0ull;
#pragma unroll
      for (int c = 0; c < RB; ++c) {
        if (c < pieces) {
          const uint64_t b0 = bf16x2_to_f2(row[c].x), b1 = bf16x2_to_f2(row[c].y), b2 = bf16x2_to_f2(row[c].z), b3 = bf16x2_to_f2(row[c].w);
#pragma unroll
          for (int j = 0; j < kGroup; ++j) {
            const ulonglong2 h0 = *reinterpret_cast<const ulonglong2*>(stage + j * (RB * 8) + c * 8);
            const ulonglong2 h1 = *reinterpret_cast<const ulonglong2*>(stage + j * (RB * 8) + c * 8 + 4);
            acc[j] = f2_fma(b0, h0.x, acc[j]);
            acc[j] = f2_fma(b1, h0.y, acc[j]);
            acc[j] = f2_fma(b2, h1.x, acc[j]);
            acc[j] = f2_fma(b3, h1.y, acc[j]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        float lo, hi;
        f2_unpack(acc[j], lo, hi);
        out[j] = lo + hi;
      }
    } else {
      for (int c = 0; c < pieces; ++c) {
        uint4 piece[kGroup];
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
          piece[j] = real && which[j] >= 0
                         ? __ldg(reinterpret_cast<const uint4*>(a.b + ((int64_t)which[j] * a.out_dim + feat) * a.rank) + c)
                         : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
          const ulonglong2 h0 = *reinterpret_cast<const ulonglong2*>(stage + j * (RB * 8) + c * 8);
          const ulonglong2 h1 = *reinterpret_cast<const ulonglong2*>(stage + j * (RB * 8) + c * 8 + 4);
          uint64_t acc = f2_fma(bf16x2_to_f2(piece[j].x), h0.x, 0ull);
          acc = f2_fma(bf16x2_to_f2(piece[j].y), h0.y, acc);
          acc = f2_fma(bf16x2_to_f2(piece[j].z), h1.x, acc);
          acc = f2_fma(bf16x2_to_f2(piece[j].w), h1.y, acc);
          float lo, hi;
          f2_unpack(acc, lo, hi);
          out[j] += lo + hi;
        }
      }
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (which[j] < 0) out[j] = 0.f;
    }
  }
};

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared memory: the ring of stages (kFeat rows of W, then nt rows of x, 128 bytes each, 128-byte swizzle), which a cluster uses
// again for its parts of the sums; behind it the warps' staging for h, then the barriers.
template <int RB>
__global__ void __launch_bounds__(kThreads, 1) k_project(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
                                                         const __grid_constant__ ProjectArgs a) {
  extern __shared__ __align__(1024) char smem_raw[];
  char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t w_bytes = kFeat * 128u, x_bytes = (uint32_t)a.nt * 128u, stage_bytes = w_bytes + x_bytes;
  const uint32_t ring = max(stage_bytes * a.stages, a.splits > 1 ? (uint32_t)a.nt * kFeat * 4u : 0u);
  float* h_stage = reinterpret_cast<float*>(smem + ring);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + ring + 4u * kGroup * RB * 8u * 4u);
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
      bool ok = true;
      for (int tile = group; tile < tiles && ok; tile += groups) {
        const int f0 = (tile % a.feat_tiles) * kFeat, t0 = (tile / a.feat_tiles) * a.nt;
        for (int k = step0; k < step1; ++k) {
          if (!(ok = mbar_wait(empty + s, phase ^ 1u, a.status))) break;
          mbar_arrive_expect_tx(full + s, stage_bytes);
          tma_load_2d(smem + s * stage_bytes, &w_map, k * kStep, f0, full + s);
          tma_load_2d(smem + s * stage_bytes + w_bytes, &x_map, k * kStep, t0, full + s);
          if (++s == a.stages) { s = 0; phase ^= 1u; }
          ++issued;
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
      bool ok = true;
      for (int tile = group; tile < tiles && ok; tile += groups, ++n) {
        const int buf = n & 1;
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
          tc_commit(empty + s);
          if (++s == a.stages) { s = 0; phase ^= 1u; }
        }
        tc_commit(acc_full + buf);
      }
      if (!ok) {  // (otherwise the tiles' own waits have seen the last of them)
        tc_commit(drained);
        mbar_drain(drained, 0, a.status);
      }
    }
  } else if (wid >= 4) {
    const int w = wid - 4, feat_in_tile = w * 32 + lane;
    Adapters<RB> adapters(a, h_stage + w * kGroup * RB * 8);
    if (RB > 0) asm volatile("griddepcontrol.wait;" ::: "memory");  // h is the kernel's before this one
    int n = 0;
    for (int tile = group; tile < tiles; tile += groups, ++n) {
      const int f0 = (tile % a.feat_tiles) * kFeat, t0 = (tile / a.feat_tiles) * a.nt, buf = n & 1;
      const int feat = f0 + feat_in_tile;
      adapters.current = -1;  // (the row that it holds is another feature's)
      if (!mbar_wait(acc_full + buf, (n >> 1) & 1, a.status)) break;
      tc_fence_after_sync();
      const uint32_t d = tmem + ((uint32_t)(w * 32) << 16) + buf * a.acc_cols;
      if (a.splits > 1) break;  // joined below
      for (int g = 0; g < a.nt; g += kGroup) {
        if (t0 + g >= a.rows) break;
        uint32_t r[8];
        tmem_ld8(d + g, r);
        float add[kGroup];
        if (RB > 0) adapters.group(t0 + g, feat, add);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
          const float v = __uint_as_float(r[j]) + (RB > 0 ? add[j] : 0.f);
          if (feat < a.out_dim && t0 + g + j < a.rows) {
            const int64_t at = (int64_t)(t0 + g + j) * a.y_stride + feat;
            if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
            else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
          }
        }
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
    if (wid >= 4) {
      const int w = wid - 4;
      for (int g = 0; g < a.nt; g += kGroup) {
        uint32_t r[8];
        tmem_ld8(tmem + ((uint32_t)(w * 32) << 16) + g, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < kGroup; ++j) parts[(g + j) * kFeat + w * 32 + lane] = __uint_as_float(r[j]);
      }
      tc_fence_before_sync();
    }
    __syncthreads();
    cluster_sync_all();
    if (wid >= 4) {
      const int w = wid - 4, feat = f0 + w * 32 + lane;
      Adapters<RB> adapters(a, h_stage + w * kGroup * RB * 8);
      for (int g = part * kGroup; g < a.nt; g += a.splits * kGroup) {
        if (t0 + g >= a.rows) break;
        float sum[kGroup], add[kGroup];
        if (RB > 0) adapters.group(t0 + g, feat, add);
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
        for (int j = 0; j < kGroup; ++j)
          if (feat < a.out_dim && t0 + g + j < a.rows) {
            const float v = sum[j] + (RB > 0 ? add[j] : 0.f);
            const int64_t at = (int64_t)(t0 + g + j) * a.y_stride + feat;
            if (a.y_fp32) static_cast<float*>(a.y)[at] = v;
            else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
          }
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

// h[part][t] = scale_a A_a x[t] over the part's entries of K; a warp per (row, part).  fp32 products and sums; the lanes' sums are
// joined so that each of the warp's results takes one round of exchanges less than the one before.
__global__ void __launch_bounds__(256) k_adapter_down(const __nv_bfloat16* __restrict__ x, int64_t x_stride, int rows, int in_dim, int parts,
                                                      int part_len, const int32_t* __restrict__ adapter, int num_adapters, int rank,
                                                      const __nv_bfloat16* __restrict__ a, const float* __restrict__ scale,
                                                      float* __restrict__ h, int32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= (int64_t)rows * parts) return;
  const int t = (int)(unit / parts), part = (int)(unit - (int64_t)t * parts);
  const int which = adapter[t];
  if (which < 0 || which >= num_adapters) {
    if (which != -1 && lane == 0) atomicCAS(status + kStatusReport, 0, (int)GF_ERR_INVALID_ARG);
    return;  // (its h is not read)
  }
  const int k0 = part * part_len, k1 = min(in_dim, k0 + part_len);
  const float f = scale != nullptr ? scale[which] : 1.f;
  const __nv_bfloat16* xr = x + (int64_t)t * x_stride;
  const __nv_bfloat16* ar = a + (int64_t)which * rank * in_dim;
  for (int r0 = 0; r0 < rank; r0 += 8) {
    uint64_t acc[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) acc[r] = 0ull;
    for (int k = k0 + lane * 8; k < k1; k += 256) {
      const uint4 xv = *reinterpret_cast<const uint4*>(xr + k);
      const uint64_t x0 = bf16x2_to_f2(xv.x), x1 = bf16x2_to_f2(xv.y), x2 = bf16x2_to_f2(xv.z), x3 = bf16x2_to_f2(xv.w);
      uint4 av[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) av[r] = __ldg(reinterpret_cast<const uint4*>(ar + (int64_t)(r0 + r) * in_dim + k));
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        acc[r] = f2_fma(bf16x2_to_f2(av[r].x), x0, acc[r]);
        acc[r] = f2_fma(bf16x2_to_f2(av[r].y), x1, acc[r]);
        acc[r] = f2_fma(bf16x2_to_f2(av[r].z), x2, acc[r]);
        acc[r] = f2_fma(bf16x2_to_f2(av[r].w), x3, acc[r]);
      }
    }
    float v[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      float lo, hi;
      f2_unpack(acc[r], lo, hi);
      v[r] = lo + hi;
    }
    // eight sums over 32 lanes: halve the values held three times, then two rounds for the one that is left
#pragma unroll
    for (int half = 4; half > 0; half >>= 1) {
      const bool upper = (lane & half) != 0;
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const float keep = upper ? v[i + half] : v[i], give = upper ? v[i] : v[i + half];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, half);
      }
    }
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 8);
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
    if (lane < 8) h[((int64_t)part * rows + t) * rank + r0 + lane] = v[0] * f;
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

// [rows, cols] of bf16, read as boxes of 64 columns x box_rows; what lies outside reads as zero.
bool make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {(cuuint32_t)kStep, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int RB>
int launch_main(const CUtensorMap& w_map, const CUtensorMap& x_map, const ProjectArgs& a, int ctas, size_t smem, cudaStream_t st) {
  static bool done[kMaxDevices];
  if (!ensure_dynamic_smem(k_project<RB>, 227 * 1024, done)) return -1;
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
  if (RB > 0) {  // behind k_adapter_down, whose results only the last part of a tile needs
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, k_project<RB>, w_map, x_map, a) == cudaSuccess ? 1 : -1;
}

}  // namespace

int project_parts(int in_dim) { return (in_dim + 1023) / 1024; }

int launch_project(const gf_projection_t& p, int rows, const void* x, int64_t x_stride, const int32_t* adapter, void* y, int64_t y_stride, int y_fp32,
                   float* scratch, int num_sms, int32_t* status, cudaStream_t st) {
  const bool with = adapter != nullptr && p.num_adapters > 0;
  ProjectArgs a = {};
  a.rows = rows;
  a.in_dim = p.in_dim;
  a.out_dim = p.out_dim;
  a.nt = rows >= 256 ? 256 : (rows + 15) / 16 * 16;
  a.feat_tiles = (p.out_dim + kFeat - 1) / kFeat;
  a.row_tiles = (rows + a.nt - 1) / a.nt;
  a.rank = with ? p.rank : 0;
  a.lda_parts = project_parts(p.in_dim);
  a.adapter = adapter;
  a.num_adapters = p.num_adapters;
  a.b = (const __nv_bfloat16*)p.b_dev;
  a.h = scratch;
  a.y = y;
  a.y_stride = y_stride;
  a.y_fp32 = y_fp32;
  a.status = status;
  const int64_t tiles = (int64_t)a.feat_tiles * a.row_tiles;
  const int steps = (p.in_dim + kStep - 1) / kStep;
  a.splits = 1;
  while (a.splits < 8 && tiles * a.splits * 2 <= num_sms && steps / (a.splits * 2) >= 4) a.splits *= 2;
  const int rb = with ? (p.rank <= 16 ? 2 : 8) : 0;
  const uint32_t stage_bytes = kFeat * 128u + a.nt * 128u, extra = 1024 + 4 * kGroup * rb * 32 + 512;
  a.stages = (int)std::min<uint32_t>(8, (227 * 1024 - extra) / stage_bytes);
  const size_t smem = extra + std::max<uint32_t>(stage_bytes * a.stages, a.splits > 1 ? (uint32_t)a.nt * kFeat * 4u : 0u);
  const int64_t groups = a.splits > 1 ? tiles : std::min<int64_t>(tiles, num_sms);
  a.acc_cols = 32;
  while (a.acc_cols < (uint32_t)a.nt) a.acc_cols *= 2;
  a.tmem_cols = a.acc_cols * (tiles > groups ? 2 : 1);
  if (tiles <= groups) a.acc_cols = 0;
  CUtensorMap w_map, x_map;
  if (!make_map(&w_map, p.w_dev, p.out_dim, p.in_dim, p.w_stride, kFeat) || !make_map(&x_map, x, rows, p.in_dim, x_stride, a.nt)) return -1;
  int launched = 0;
  if (with) {
    const int64_t units = (int64_t)rows * a.lda_parts;
    k_adapter_down<<<(unsigned)((units + 7) / 8), 256, 0, st>>>((const __nv_bfloat16*)x, x_stride, rows, p.in_dim, a.lda_parts, 1024, adapter,
                                                               p.num_adapters, p.rank, (const __nv_bfloat16*)p.a_dev, p.scale_dev, scratch, status);
    if (cudaGetLastError() != cudaSuccess) return -1;
    ++launched;
  }
  const int ctas = (int)(groups * a.splits);
  const int n = rb == 0 ? launch_main<0>(w_map, x_map, a, ctas, smem, st) : rb == 2 ? launch_main<2>(w_map, x_map, a, ctas, smem, st)
                                                                                   : launch_main<8>(w_map, x_map, a, ctas, smem, st);
  return n < 0 ? -1 : launched + n;
}

}  // namespace gf
