// K2 over node states held in 4 bits: the decode kernel for the chunks that lie in the 4-bit pool.
//
// Same units, partials and merge as decode.cu: for a chunk of one node's segment and up to 16 of the query
// rows that share it, S^T = K Q^T (tokens are the MMA's rows), an online softmax with shuffles across the
// token lanes, O^T += V^T P^T.  What differs is the operand: the MMAs multiply the codes themselves (c - 8,
// exact in bf16), and a token's (s, lo) enter outside of them, in fp32:
//   S_t = sum over groups G of  s_tG (q_G . (c - 8))  +  (lo_tG + 8.5 s_tG) (sum of q_G)
//   O   = sum over tokens of  (p_t s_tG) (c - 8)  +  sum of  p_t (lo_tG + 8.5 s_tG)
// so the scores carry no rounding but fp32's; p s is rounded to bf16 for the second product, as P is in the
// bf16 kernel (the sum of p and the second term are not).
//
// No shared memory and no barriers: the layout (kv4_device.cuh) gives every lane its MMA operands as 16-byte
// pieces of the tile, so a warp reads them straight from global memory into registers, and every warp is
// on its own: it takes a unit (from a counter, longest segments first), walks its tiles and writes the
// partial.
#include "kv4_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 128;

struct Params {
  const char* pool_layer;
  uint64_t head_stride;
  int32_t tile_base;  // index of the 4-bit pool's first tile among all tiles
  const Item* items;
  const int32_t* list;  // last entry; entry i is list[-i] = 4 * item + row group
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

template <int D>
struct Warp4 {
  static constexpr int NG = D / kGroup4, KS = D / 16;
  uint32_t qf[2][KS][2];
  float qsum[2][NG][2];  // sum of a query row's entries per group, for this thread's two columns
  float o[KS][2][4];
  float oz[2][NG][2];    // sum over tokens of p (lo + 8.5 s), this thread's tokens
  float m_run[2][2], l_run[2][2];

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int c = 0; c < 2; ++c) { m_run[j][c] = -INFINITY; l_run[j][c] = 0.f; }
#pragma unroll
      for (int g = 0; g < NG; ++g) oz[j][g][0] = oz[j][g][1] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_bf16(acc, ones, qf[j][g * 4 + kk][0], qf[j][g * 4 + kk][1]);
        qsum[j][g][0] = acc[0];
        qsum[j][g][1] = acc[1];
      }
    }
  }

  // One tile: tokens 0..nv-1 of the 64 at `tile`.  NT: 8-row halves of the row group in use.
  template <int NT, bool kMask>
  __device__ __forceinline__ void step(const char* tile, int nv, float scale_log2, int lane) {
    constexpr uint32_t kPart = kv4_part_bytes(D), kCodes = kv4_code_bytes(D);
    const int l8 = lane >> 2;
    const int nb = kMask ? (nv + 15) >> 4 : 4;  // blocks of 16 tokens that hold any
    const uint4* kc = reinterpret_cast<const uint4*>(tile) + lane;
    const uint4* vc = reinterpret_cast<const uint4*>(tile + kPart) + lane;
    const uint32_t* ks = reinterpret_cast<const uint32_t*>(tile + kCodes);
    const uint32_t* vs = reinterpret_cast<const uint32_t*>(tile + kPart + kCodes);
    float s[4][NT][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (kMask && b >= nb) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][j][e] = -INFINITY;
        continue;
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[b][j][e] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint4 c4 = kc[(b * NG + g) * 32];
        const uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
        float acc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t a[4];
          kv4_expand(a, w[kk]);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_bf16(acc[j], a, qf[j][g * 4 + kk][0], qf[j][g * 4 + kk][1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // tokens l8 and l8 + 8
          const uint32_t sl = ks[(b * 16 + l8 + 8 * h) * NG + g];
          const float sc = kv4_s(sl), z = fmaf(8.5f, sc, kv4_lo(sl));
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              s[b][j][2 * h + c] = fmaf(acc[j][2 * h + c], sc, fmaf(qsum[j][g][c], z, s[b][j][2 * h + c]));
        }
      }
    }
    float mx[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) { mx[j][0] = -INFINITY; mx[j][1] = -INFINITY; }
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool on = !kMask || b * 16 + l8 + 8 * (e >> 1) < nv;
          s[b][j][e] = on ? s[b][j][e] * scale_log2 : -INFINITY;
          mx[j][e & 1] = fmaxf(mx[j][e & 1], s[b][j][e]);
        }
    bool grew = false;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v = mx[j][c];
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
        mx[j][c] = fmaxf(v, m_run[j][c]);
        grew |= mx[j][c] > m_run[j][c];
      }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float r[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          r[c] = (mx[j][c] == -INFINITY) ? 0.f : fast_exp2(m_run[j][c] - mx[j][c]);
          l_run[j][c] *= r[c];
          m_run[j][c] = mx[j][c];
#pragma unroll
          for (int g = 0; g < NG; ++g) oz[j][g][c] *= r[c];
        }
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][j][e] *= r[e & 1];
      }
    }
    float ref[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) ref[j][c] = (m_run[j][c] == -INFINITY) ? 0.f : m_run[j][c];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (kMask && b >= nb) continue;
      float p[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[j][e] = fast_exp2(s[b][j][e] - ref[j][e & 1]);
          l_run[j][e & 1] += p[j][e];
        }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float sc[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t sl = vs[(b * 16 + l8 + 8 * h) * NG + g];
          sc[h] = kv4_s(sl);
          const float z = fmaf(8.5f, sc[h], kv4_lo(sl));
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) oz[j][g][c] = fmaf(p[j][2 * h + c], z, oz[j][g][c]);
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h)  // P^T as the B operand: k = token, n = row
            pb[j][h] = movmatrix_trans(pack_bf16(p[j][2 * h] * sc[h], p[j][2 * h + 1] * sc[h]));
        const uint4 c4 = vc[(b * NG + g) * 32];
        const uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t a[4];
          kv4_expand(a, w[kk]);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_bf16(o[g * 4 + kk][j], a, pb[j][0], pb[j][1]);
        }
      }
    }
  }

  // Adds up what the token lanes hold apart: the row sums and the second term of O.
  __device__ __forceinline__ void finish_sums() {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          l_run[j][c] += __shfl_xor_sync(0xffffffffu, l_run[j][c], d);
#pragma unroll
          for (int g = 0; g < NG; ++g) oz[j][g][c] += __shfl_xor_sync(0xffffffffu, oz[j][g][c], d);
        }
      }
  }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2) k_decode4(const Params p) {
  constexpr int NG = D / kGroup4;
  chain_enter();
  const int lane = threadIdx.x & 31, l4 = lane & 3, l8 = lane >> 2, g = p.gqa;
  const int num_units = tables_usable(*p.hdr, p.slot_cap) ? p.hdr->kv4_list_n * p.num_kv_heads : 0;
  Warp4<D> wa;
  while (true) {
    int u = 0;
    if (lane == 0) u = atomicAdd(&p.counters[0], 1);
    u = __shfl_sync(0xffffffffu, u, 0);
    if (u >= num_units) break;
    const int entry = p.list[-(long long)(u / p.num_kv_heads)], kvh = u % p.num_kv_heads;
    const Item it = p.items[GF_CLAMP(entry >> 2, p.slot_cap, p.status, 121)];
    const int row0 = (entry & 3) * 16;
    const int rows_here = min(16, it.grp_count * g - row0);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = j * 8 + l8;
      const bool ok = row < rows_here;
      int req = ok ? p.grp_req[GF_CLAMP(it.grp_begin + (row0 + row) / g, p.num_pairs, p.status, 122)] : 0;
      req = GF_CLAMP(req, p.num_requests, p.status, 123);
      const uint4* qrow = reinterpret_cast<const uint4*>(p.q + ((size_t)req * p.num_q_heads + kvh * g + (row0 + row) % g) * D);
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {  // entries 32 x + 8 l4 .. + 7: MMAs 2 x and 2 x + 1
        const uint4 v = ok ? qrow[4 * x + l4] : make_uint4(0u, 0u, 0u, 0u);
        wa.qf[j][2 * x][0] = v.x;
        wa.qf[j][2 * x][1] = v.y;
        wa.qf[j][2 * x + 1][0] = v.z;
        wa.qf[j][2 * x + 1][1] = v.w;
      }
    }
    wa.init();
    const char* base = p.pool_layer + (uint64_t)kvh * p.head_stride;
    const int ntile = (it.tok_count + kTile - 1) / kTile;
    for (int t = 0; t < ntile; ++t) {
      const int nv = it.tok_count - t * kTile;
      const char* tile = base + (uint64_t)GF_CLAMP(it.tile0 - p.tile_base + t, p.cap_tiles, p.status, 124) * kv4_tile_bytes(D);
      if (rows_here <= 8) {
        if (nv >= kTile) wa.template step<1, false>(tile, kTile, p.scale_log2, lane);
        else wa.template step<1, true>(tile, nv, p.scale_log2, lane);
      } else {
        if (nv >= kTile) wa.template step<2, false>(tile, kTile, p.scale_log2, lane);
        else wa.template step<2, true>(tile, nv, p.scale_log2, lane);
      }
    }
    wa.finish_sums();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = j * 8 + l4 * 2 + c;
        if (row < rows_here && GF_CHECK(it.part_base + (row0 + row) / g < p.slot_cap, p.status, 125)) {
          const int srow = row0 + row;
          const size_t ph = (size_t)(it.part_base + srow / g) * p.num_q_heads + kvh * g + srow % g;
          float4* po = reinterpret_cast<float4*>(p.part_o + ph * D);
#pragma unroll
          for (int gr = 0; gr < NG; ++gr) {  // entries 8 l8 .. + 7 of the group
            const float z = wa.oz[j][gr][c];
            po[gr * 16 + l8 * 2] = make_float4(wa.o[gr * 4][j][c] + z, wa.o[gr * 4][j][2 + c] + z,
                                               wa.o[gr * 4 + 1][j][c] + z, wa.o[gr * 4 + 1][j][2 + c] + z);
            po[gr * 16 + l8 * 2 + 1] = make_float4(wa.o[gr * 4 + 2][j][c] + z, wa.o[gr * 4 + 2][j][2 + c] + z,
                                                   wa.o[gr * 4 + 3][j][c] + z, wa.o[gr * 4 + 3][j][2 + c] + z);
          }
          if (l8 == 0) *reinterpret_cast<float2*>(p.part_ml + ph * 2) = make_float2(wa.m_run[j][c], wa.l_run[j][c]);
        }
      }
  }
  // the last CTA to run out of work re-arms the counters for the next launch
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&p.counters[1], 1) == (int)gridDim.x - 1) {
      p.counters[0] = 0;
      p.counters[1] = 0;
    }
  }
}

}  // namespace

int launch_decode4(const PoolGeom& pool, const AttnShape& sh, const TablesDev& t, int num_units, int layer, const void* q,
                   int32_t* status, bool chained, cudaStream_t st) {
  if (num_units == 0) return 0;
  Params p;
  p.pool_layer = pool.base + (uint64_t)layer * pool.layer_stride;
  p.head_stride = pool.head_stride;
  p.tile_base = t.kv4_tile0;
  p.items = t.items;
  p.list = t.wide_list + t.slot_cap - 1;
  p.grp_req = t.grp_req;
  p.q = (const __nv_bfloat16*)q;
  p.part_o = t.part_o;
  p.part_ml = t.part_ml;
  p.status = status;
  p.counters = status + kStatusKv4Queue;
  p.hdr = t.hdr;
  p.slot_cap = t.slot_cap;
  p.num_q_heads = sh.num_q_heads;
  p.num_kv_heads = sh.num_kv_heads;
  p.gqa = sh.num_q_heads / sh.num_kv_heads;
  p.scale_log2 = sh.scale_log2;
  p.cap_tiles = (int32_t)pool.cap_tiles;
  p.num_pairs = t.num_pairs_in;
  p.num_requests = t.num_requests;
  const long long warps = num_units < 0 ? (1ll << 40) : (long long)num_units * sh.num_kv_heads;
  const long long blocks = (warps + kThreads / 32 - 1) / (kThreads / 32), most = 2ll * t.num_sms;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  auto go = [&](auto kernel) {
    if (chained) launch_chained(kernel, grid, dim3(kThreads), 0, st, p);
    else kernel<<<grid, dim3(kThreads), 0, st>>>(p);  // behind a join with another stream
  };
  if (sh.head_dim == 128) go(k_decode4<128>);
  else go(k_decode4<64>);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace gf
