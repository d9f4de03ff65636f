// K2 over node states held in 4 bits: the decode kernel for the chunks that lie in the 4-bit pool.
//
// Same units, partials and merge as decode.cu: for a chunk of one node's segment and up to 16 of the query
// rows that share it, S^T = K Q^T (tokens are the MMA's rows), an online softmax with shuffles across the
// token lanes, O^T += V^T P^T.  What differs is the operand: the MMAs multiply the codes themselves, and a
// token's (s, lo) enter outside of them, in fp32:
//   S_t = sum over groups G of  s_tG (q_G . c)  +  (lo_tG + s_tG / 2) (sum of q_G)
//   O   = sum over tokens of  (p_t s_tG) c  +  sum of  p_t (lo_tG + s_tG / 2)
// What bounds it is the number of instructions that turn codes into operands.  A code in the low bits of an
// fp16 pattern is the subnormal number c 2^-24, and one nibble up 16 c 2^-24: both exact MMA operands, so
// eight codes take one shift and four ANDs, and the powers of two go into the scales.  Queries are fp16 times
// a power of two per row (all eight bits of every entry down to 2^-31 of the row's largest), p s is fp16 times
// one power of two per row and group, chosen with the softmax's reference; scores, sums, O and the terms without
// codes are fp32.
// What that rounding of p s costs: the codes that it multiplies are 0..15, not centred, which makes it count 2.2 times
// as much as with c - 8 (over 2000 tokens of normal values 4.8e-4 of the output instead of 2.2e-4; p in bf16, as the
// kernel for bf16 states has it, 1.5e-3; the output's own rounding to bf16 1.6e-3).  Centred operands would take 128 more
// instructions per tile.
//
// Every warp is on its own: it takes units (an item's 16 query rows, or what is left of them) from a counter,
// longest segments first, streams their tiles through a ring of its own in shared memory (bulk copies,
// completion counted in bytes on mbarriers; the layout of kv4_device.cuh makes every operand load a
// conflict-free 16 bytes per lane) and writes the partial.  The next unit is claimed while the current one
// streams, a step of the claim (counter, list, item) per tile, so that none of its round trips is waited for.
// 256 requests over 256 nodes, all in 4 bits, 133 us with the merge: 101 us for the groups of 9..16 rows, the others
// (47 alone) mostly beside them on a second stream.
// One kernel that takes 16 rows for all was slower: 154 us for that call then against 137, 41 against 36 for one request
// over 57 000 tokens, 499 against 464 for 1024 requests.
// The schedulers issue in 43 to 46 % of their cycles, with 8 and 11 warps per SM and a third of a warp's time in waits
// for results of fixed latency: registers, that is warps, are what is short.  Unpacking takes 320 of the 1100 (8 rows)
// or 1300 (16) instructions of a tile.
// Units of up to 8 rows use one column block of the MMA and run twelve warps to an SM, the others eight: what 168 and
// 255 registers per thread allow.  Chunks shared by 64 rows and more go to decode4_wide.cu where those fill the GPU.
#include <stddef.h>

#include "kv4_device.cuh"
#include "tc_device.cuh"

namespace gf {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
struct Params {
  const char* pool_layer;
  uint64_t head_stride;
  int32_t tile_base;  // index of the 4-bit pool's first tile among all tiles
  const Item* items;
  const int32_t* list;  // the handle's unit lists (see TablesDev::wide_list)
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

// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four A registers from one word of codes: fp16 pairs c 2^-24 (registers 0 and 2) and 16 c 2^-24 (1 and 3).
__device__ __forceinline__ void expand_f16(uint32_t (&a)[4], uint32_t w) {
  const uint32_t v = w >> 8;
  a[0] = w & 0x000f000fu;
  a[1] = w & 0x00f000f0u;
  a[2] = v & 0x000f000fu;
  a[3] = v & 0x00f000f0u;
}
// The state of one unit: 8 NT query rows over its tokens, a tile at a time.  Token rows 8..15 of a block come out of
// the first product 16 times too large (registers 1 and 3 hold them), odd entries of O out of the second.
template <int D, int NT>
struct Warp4 {
  static constexpr int NG = D / kGroup4, KS = D / 16;
  uint32_t qf[NT][KS][2];
  // fp32 pairs are this thread's two columns (query rows); arithmetic on them is packed
  uint64_t qsum[NT][NG];  // sum of a query row's entries per group
  uint64_t scale[NT];     // softmax scale in log2 units over the power of two that the row was multiplied by
  uint64_t bias[NT];      // 0, or -inf for a row that does not exist (its p are 0)
  float o[KS][NT][4];     // O^T in units of 2^-24 / f and 2^-20 / f
  uint64_t oz[NT][NG];    // sum over tokens of p (lo + s / 2), this thread's tokens
  uint64_t nref[NT], l_run[NT];  // the softmax's reference (negative), the sum of p
  uint64_t f[NT][NG];     // powers of two that the second product's p s are multiplied by (0: no such row)

  // Queries in fp16: a row is multiplied by the power of two that brings its largest entry to 2^14..2^15,
  // which keeps all eight bits of every entry down to 2^-31 of the largest.
  __device__ __forceinline__ void load_queries(const Params& p, int grp_begin, int row0, int kvh, int rows, int lane) {
    const int l4 = lane & 3, l8 = lane >> 2, g = p.gqa;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int row = j * 8 + l8;
      const bool ok = row < rows;
      int req = ok ? p.grp_req[GF_CLAMP(grp_begin + (row0 + row) / g, p.num_pairs, p.status, 122)] : 0;
      req = GF_CLAMP(req, p.num_requests, p.status, 123);
      const uint4* qrow = reinterpret_cast<const uint4*>(p.q + ((size_t)req * p.num_q_heads + kvh * g + (row0 + row) % g) * D);
      uint4 v[D / 32];
#pragma unroll
      for (int x = 0; x < D / 32; ++x) v[x] = ok ? qrow[4 * x + l4] : make_uint4(0u, 0u, 0u, 0u);
      float big = 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          big = fmaxf(big, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      const float mul = pow2_to(big, 14);
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {  // entries 32 x + 8 l4 .. + 7: MMAs 2 x and 2 x + 1
        const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          qf[j][2 * x + (i >> 1)][i & 1] = pack_f16(__uint_as_float(w[i] << 16) * mul, __uint_as_float(w[i] & 0xffff0000u) * mul);
      }
      // this thread's columns are the rows of the lanes 8 l4 and 8 l4 + 4
      float sc[2], none[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        sc[c] = p.scale_log2 * pow2_inverse(__shfl_sync(0xffffffffu, mul, 8 * l4 + 4 * c));
        none[c] = j * 8 + 2 * l4 + c < rows ? 0.f : -INFINITY;
      }
      scale[j] = f2_pack(sc[0], sc[1]);
      bias[j] = f2_pack(none[0], none[1]);
    }
  }

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float b0, b1;
      f2_unpack(bias[j], b0, b1);
      nref[j] = f2_pack(b0 == 0.f ? INFINITY : 0.f, b1 == 0.f ? INFINITY : 0.f);
      l_run[j] = 0;
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        oz[j][g] = 0;
        f[j][g] = f2_pack(b0 == 0.f ? 1.f : 0.f, b1 == 0.f ? 1.f : 0.f);
        const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_f16(acc, ones, qf[j][g * 4 + kk][0], qf[j][g * 4 + kk][1]);
        qsum[j][g] = f2_pack(acc[0], acc[1]);
      }
    }
  }

  // The (s, lo) words of this thread's tokens of block b: l8 and l8 + 8.
  static __device__ __forceinline__ void load_words(uint32_t (&sl)[2][NG], const char* part, int b, int lane) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(part + kv4_code_bytes(D)) + (b * 16 + (lane >> 2) + 8 * h) * NG;
      if (NG == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(w);
        sl[h][0] = v.x;
        sl[h][NG - 1] = v.y;
      } else {
        sl[h][0] = *w;
      }
    }
  }

  // The tile's scores in log2 units: x[b][j][h] of token 16 b + l8 + 8 h.
  __device__ __forceinline__ void scores(uint64_t (&x)[4][NT][2], const char* part, int nv, int lane) const {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint32_t sl[2][NG];
      load_words(sl, part, b, lane);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint4 c4 = reinterpret_cast<const uint4*>(part)[(b * NG + g) * 32 + lane];
        const uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
        float acc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t a[4];
          expand_f16(a, w[kk]);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_f16(acc[j], a, qf[j][g * 4 + kk][0], qf[j][g * 4 + kk][1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sc = kv4_s(sl[h][g]), z = fmaf(0.5f, sc, kv4_lo(sl[h][g])), su = sc * (h ? kUnit1 : kUnit0);
          const uint64_t z2 = f2_pack(z, z), su2 = f2_pack(su, su);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const uint64_t zq = f2_fma(qsum[j][g], z2, g ? x[b][j][h] : 0);
            x[b][j][h] = f2_fma(f2_pack(acc[j][2 * h], acc[j][2 * h + 1]), su2, zq);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[b][j][h] = f2_fma(x[b][j][h], scale[j], bias[j]);
    }
    if (nv < kTile) {  // the last tile: tokens past the end
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (b * 16 + (lane >> 2) + 8 * h >= nv) x[b][j][h] = f2_pack(-INFINITY, -INFINITY);
    }
  }

  // Column maxima of a tile's scores (this thread's tokens).
  static __device__ __forceinline__ void column_max(const uint64_t (&x)[4][NT][2], int j, float (&m)[2]) {
    f2_unpack(x[0][j][0], m[0], m[1]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      float a, b;
      f2_unpack(x[i >> 1][j][i & 1], a, b);
      m[0] = fmaxf(m[0], a);
      m[1] = fmaxf(m[1], b);
    }
  }

  // Adds the tile to (O, l).  Any reference of the softmax is exact as long as p, l and O share it: it moves only
  // when a score outgrew it by more than 2^8.  The second product's p s are fp16 times a power of two f per row and
  // group, chosen whenever the reference moves so that the row's largest p s so far stands at 2^2 or above (a move may
  // count what came before it half as large as it is); an s with which p s could pass fp16's range, or the first
  // one that is not 0, makes it move too.  Rounding changes a token's p s by 2^-11 of it at most, or by 2^-27 of the
  // row's largest p s, and what it adds to O by as much of p s c.
  __device__ __forceinline__ void accumulate(const uint64_t (&x)[4][NT][2], const char* part, int lane) {
    bool move = false;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float m[2], n[2];
      column_max(x, j, m);
      f2_unpack(nref[j], n[0], n[1]);
      move |= m[0] + n[0] > 8.f || m[1] + n[1] > 8.f;
    }
    {
      uint32_t m[NG];  // the largest s in the low half (not negative: its bits order as it does)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        uint32_t sl[2][NG];
        load_words(sl, part, b, lane);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if (b == 0) m[g] = sl[0][g];
          else asm("max.u16x2 %0, %0, %1;" : "+r"(m[g]) : "r"(sl[0][g]));
          asm("max.u16x2 %0, %0, %1;" : "+r"(m[g]) : "r"(sl[1][g]));
        }
      }
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float a, b;
          f2_unpack(f[j][g], a, b);
          move |= kv4_s(m[g]) * fmaxf(a, b) > 128.f;
        }
    }
    if (__any_sync(0xffffffffu, move)) move_reference(x, part, lane);
    asm volatile("" ::: "memory");  // (the words are read again below instead of being kept in registers)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint32_t sl[2][NG];
      load_words(sl, part, b, lane);
      uint64_t pr[NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float lo, hi;
          f2_unpack(f2_add(x[b][j][h], nref[j]), lo, hi);
          pr[j][h] = f2_pack(fast_exp2(lo), fast_exp2(hi));
          l_run[j] = f2_add(l_run[j], pr[j][h]);
        }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        uint32_t pb[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sc = kv4_s(sl[h][g]), z = fmaf(0.5f, sc, kv4_lo(sl[h][g]));
          const uint64_t z2 = f2_pack(z, z), s2 = f2_pack(sc, sc);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            oz[j][g] = f2_fma(pr[j][h], z2, oz[j][g]);
            // P^T as the B operand: k = token, n = row
            float lo, hi;
            f2_unpack(f2_mul(f2_mul(pr[j][h], f[j][g]), s2), lo, hi);
            pb[j][h] = movmatrix_trans(pack_f16(lo, hi));
          }
        }
        const uint4 c4 = reinterpret_cast<const uint4*>(part)[(b * NG + g) * 32 + lane];
        const uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          uint32_t a[4];
          expand_f16(a, w[kk]);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_f16(o[g * 4 + kk][j], a, pb[j][0], pb[j][1]);
        }
      }
    }
  }

  __device__ __forceinline__ void move_reference(const uint64_t (&x)[4][NT][2], const char* part, int lane) {
    float r[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float m[2], n[2], l[2];
      column_max(x, j, m);
      f2_unpack(nref[j], n[0], n[1]);
      f2_unpack(l_run[j], l[0], l[1]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        m[c] = fmaxf(m[c], -n[c]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) m[c] = fmaxf(m[c], __shfl_xor_sync(0xffffffffu, m[c], d));
        r[j][c] = fast_exp2(-n[c] - m[c]);  // 0 for the unit's first tile
      }
      nref[j] = f2_pack(-m[0], -m[1]);
      l_run[j] = f2_pack(l[0] * r[j][0], l[1] * r[j][1]);
    }
    float big[NT][NG][2];  // the largest p s of the tile, by row and group
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint32_t sl[2][NG];
      load_words(sl, part, b, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float pr[2];
          f2_unpack(f2_add(x[b][j][h], nref[j]), pr[0], pr[1]);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            pr[c] = fast_exp2(pr[c]);
#pragma unroll
            for (int g = 0; g < NG; ++g) big[j][g][c] = fmaxf(b + h ? big[j][g][c] : 0.f, pr[c] * kv4_s(sl[h][g]));
          }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float old[2], ratio[2];
        f2_unpack(f[j][g], old[0], old[1]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float& m = big[j][g][c];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
          const float inv = pow2_inverse(old[c]);  // 4 inv: half the largest p s before, or more
          const float fn = old[c] > 0.f ? pow2_to(fmaxf(4.f * inv * r[j][c], m), 2) : 0.f;
          ratio[c] = fn * r[j][c] * inv;  // (in this order: fn / f may leave fp32's range)
          old[c] = fn;
        }
        f[j][g] = f2_pack(old[0], old[1]);
        oz[j][g] = f2_mul(oz[j][g], f2_pack(r[j][0], r[j][1]));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[g * 4 + kk][j][e] *= ratio[e & 1];
      }
  }

  // Adds up what the token lanes hold apart: the row sums and the second term of O.
  __device__ __forceinline__ void finish_sums() {
    auto total = [](uint64_t v) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) v = f2_add(v, __shfl_xor_sync(0xffffffffu, v, d));
      return v;
    };
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      l_run[j] = total(l_run[j]);
#pragma unroll
      for (int g = 0; g < NG; ++g) oz[j][g] = total(oz[j][g]);
    }
  }
};

// Registers -> fp32 partial of the unit's rows row0 .. row0 + rows - 1.
template <int D, int NT>
__device__ __forceinline__ void write_partial(const Params& p, Warp4<D, NT>& wa, int part_base, int row0, int kvh, int rows, int lane) {
  constexpr int NG = D / kGroup4;
  wa.finish_sums();
  const int l4 = lane & 3, l8 = lane >> 2, g = p.gqa;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = j * 8 + l4 * 2 + c;
      if (row < rows && GF_CHECK(part_base + (row0 + row) / g < p.slot_cap, p.status, 125)) {
        const int srow = row0 + row;
        const size_t ph = (size_t)(part_base + srow / g) * p.num_q_heads + kvh * g + srow % g;
        float4* po = reinterpret_cast<float4*>(p.part_o + ph * D);
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {  // entries 8 l8 .. + 7 of the group
          float zz[2];
          f2_unpack(wa.oz[j][gr], zz[0], zz[1]);
          const float z = zz[c];
          float ff[2];
          f2_unpack(wa.f[j][gr], ff[0], ff[1]);
          const float inv = pow2_inverse(ff[c]);
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = fmaf(wa.o[gr * 4 + (i >> 1)][j][2 * (i & 1) + c] * inv, (i & 1) ? kUnit1 : kUnit0, z);
          po[gr * 16 + l8 * 2] = make_float4(v[0], v[1], v[2], v[3]);
          po[gr * 16 + l8 * 2 + 1] = make_float4(v[4], v[5], v[6], v[7]);
        }
        float n[2], l[2];
        f2_unpack(wa.nref[j], n[0], n[1]);
        f2_unpack(wa.l_run[j], l[0], l[1]);
        if (l8 == 0) *reinterpret_cast<float2*>(p.part_ml + ph * 2) = make_float2(-n[c], l[c]);
      }
    }
}

// A unit in progress: what is needed when its first tile is consumed.
struct __align__(16) Unit {
  int32_t grp_begin, rows, part_base, tok_count;
  int32_t kvh, row0, pad0, pad1;
};

// The claims of one warp (every lane calls).  The claimed item lies in the lanes, a word each, until it is taken.
struct Claims {
  const int32_t* list;  // 4 * item + 16-row group of unit u: list[dir * (u / num_kv_heads)]
  int dir, num_units, claimants;
  int state = 0;  // 0 ask the counter, 1 read the list, 2 read the item, 3 ready, 4 no more
  int u = 0, index = 0, word = 0;
  // the first claim needs no counter: claimant i starts with unit i, and the counter counts from the last of those
  __device__ __forceinline__ void first(int i) { u = i; state = 1; }
  __device__ __forceinline__ void step(const Params& p, int lane) {
    if (state == 0) {
      if (lane == 0) u = atomicAdd(&p.counters[0], 1) + claimants;
      state = 1;
    } else if (state == 1) {
      u = __shfl_sync(0xffffffffu, u, 0);
      if (u >= num_units) {
        state = 4;
      } else {
        index = list[(long long)dir * (u / p.num_kv_heads)];
        state = 2;
      }
    } else if (state == 2) {
      word = reinterpret_cast<const int32_t*>(p.items + GF_CLAMP(index >> 2, p.slot_cap, p.status, 121))[lane & 7];
      state = 3;
    }
  }
  __device__ __forceinline__ int item_word(int i) const { return __shfl_sync(0xffffffffu, word, i); }  // in the order of Item
  __device__ __forceinline__ Unit unit(const Params& p) const {
    static_assert(sizeof(Item) == 32 && offsetof(Item, tok_count) == 8 && offsetof(Item, grp_begin) == 12 && offsetof(Item, grp_count) == 16 &&
                  offsetof(Item, part_base) == 20 && offsetof(Item, tile0) == 24, "the words that are taken below");
    Unit x{};
    x.tok_count = item_word(2);
    x.grp_begin = item_word(3);
    x.row0 = (index & 3) * 16;
    x.rows = min(16, item_word(4) * p.gqa - x.row0);
    x.part_base = item_word(5);
    x.kvh = u % p.num_kv_heads;
    return x;
  }
  __device__ __forceinline__ const char* tiles(const Params& p, uint32_t tile_bytes) const {
    return p.pool_layer + (uint64_t)(u % p.num_kv_heads) * p.head_stride +
           (uint64_t)GF_CLAMP(item_word(6) - p.tile_base, p.cap_tiles, p.status, 124) * tile_bytes;
  }
};

// CTAs of four warps per SM (four CTAs at 128 registers spill: 213 us instead of 194 for 256 requests), and tiles in
// flight or in use per warp.
template <int NT> constexpr int kCtas4 = NT == 1 ? 3 : 2;
constexpr int kTiles4 = 2;

template <int D, int NT>
struct __align__(16) WarpSmem {
  unsigned char tile[kTiles4][kv4_tile_bytes(D)];
  Unit unit[4];
  uint64_t full[kTiles4];
};

// One warp's stream of its units' tiles, one after the other.
template <int D, int NT>
struct TileStream {
  const Params& p;
  WarpSmem<D, NT>& ws;
  const int lane;
  Claims& claims;
  int issued = 0;             // tiles issued
  int issue_units = 0;        // units whose issue has begun
  int left = 0;               // tiles of the current one not issued yet
  const char* src = nullptr;  // the next tile

  // A step of the next claim, if it is not complete.
  __device__ __forceinline__ void claim() {
    if (claims.state < 3) claims.step(p, lane);
  }
  // Issues the next tile; its slot must be free.
  __device__ __forceinline__ void issue() {
    if (left == 0) {
      while (claims.state < 3) claims.step(p, lane);
      if (claims.state == 4) return;
      const Unit u = claims.unit(p);
      src = claims.tiles(p, kv4_tile_bytes(D));
      if (lane == 0) ws.unit[issue_units & 3] = u;
      ++issue_units;
      left = (u.tok_count + kTile - 1) / kTile;
      claims.state = 0;
    }
    if (lane == 0) {
      const int slot = issued % kTiles4;
      mbar_arrive_expect_tx(&ws.full[slot], kv4_tile_bytes(D));
      bulk_g2s(ws.tile[slot], src, kv4_tile_bytes(D), &ws.full[slot]);
    }
    src += kv4_tile_bytes(D);
    --left;
    ++issued;
  }
  __device__ __forceinline__ bool wait(int n) { return mbar_wait(&ws.full[n % kTiles4], (n / kTiles4) & 1, p.status); }
  __device__ __forceinline__ const char* tile(int n) const { return reinterpret_cast<const char*>(ws.tile[n % kTiles4]); }
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, kCtas4<NT>) k_decode4(const Params p) {
  extern __shared__ __align__(128) unsigned char smem[];
  const int lane = threadIdx.x & 31;
  WarpSmem<D, NT>& ws = reinterpret_cast<WarpSmem<D, NT>*>(smem)[threadIdx.x >> 5];
  if (lane == 0) {
    for (int i = 0; i < kTiles4; ++i) mbar_init(&ws.full[i], 1);
    mbar_fence_init();
  }
  __syncwarp();
  chain_enter();
  const bool usable = tables_usable(*p.hdr, p.slot_cap);
  Claims claims{NT == 1 ? p.list + p.slot_cap - 1 : p.list + p.hdr->kv4_rows16_first, NT == 1 ? -1 : 1,
                usable ? (NT == 1 ? p.hdr->kv4_rows8 : p.hdr->kv4_rows16) * p.num_kv_heads : 0, (int)gridDim.x * kWarps};
  claims.first((int)blockIdx.x * kWarps + (threadIdx.x >> 5));
  TileStream<D, NT> ts{p, ws, lane, claims};
  for (int i = 0; i < kTiles4; ++i) ts.issue();
  int tile = 0;
  bool ok = true;
  for (int n = 0; ok && tile < ts.issued; ++n) {
    __syncwarp();
    const Unit it = ws.unit[n & 3];
    Warp4<D, NT> wa;
    wa.load_queries(p, it.grp_begin, it.row0, it.kvh, it.rows, lane);
    wa.init();
    for (int left = it.tok_count; left > 0; left -= kTile, ++tile) {
      uint64_t x[4][NT][2];
      if (!(ok = ts.wait(tile))) break;
      ts.claim();
      wa.scores(x, ts.tile(tile), left, lane);
      ts.claim();
      wa.accumulate(x, ts.tile(tile) + kv4_part_bytes(D), lane);
      __syncwarp();
      ts.issue();
    }
    if (!ok) break;
    write_partial(p, wa, it.part_base, it.row0, it.kvh, it.rows, lane);
  }
  for (; tile < ts.issued; ++tile)  // (after a wait that gave up)
    if (lane == 0) mbar_drain(&ws.full[tile % kTiles4], (tile / kTiles4) & 1, p.status);
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

int launch_decode4(const PoolGeom& pool, const AttnShape& sh, const TablesDev& t, int rows, int units, int layer, const void* q,
                   int32_t* status, bool chained, cudaStream_t st) {
  if (units == 0) return 0;
  Params p;
  p.pool_layer = pool.base + (uint64_t)layer * pool.layer_stride;
  p.head_stride = pool.head_stride;
  p.tile_base = t.kv4_tile0;
  p.items = t.items;
  p.list = t.wide_list;
  p.grp_req = t.grp_req;
  p.q = (const __nv_bfloat16*)q;
  p.part_o = t.part_o;
  p.part_ml = t.part_ml;
  p.status = status;
  p.counters = status + (rows == 8 ? kStatusKv4Queue8 : kStatusKv4Queue);
  p.hdr = t.hdr;
  p.slot_cap = t.slot_cap;
  p.num_q_heads = sh.num_q_heads;
  p.num_kv_heads = sh.num_kv_heads;
  p.gqa = sh.num_q_heads / sh.num_kv_heads;
  p.scale_log2 = sh.scale_log2;
  p.cap_tiles = (int32_t)pool.cap_tiles;
  p.num_pairs = t.num_pairs_in;
  p.num_requests = t.num_requests;
  auto go = [&](auto kernel, size_t smem, int per_sm, bool (&optin)[kMaxDevices]) {
    if (!ensure_dynamic_smem(kernel, smem, optin)) return false;
    const long long warps = units < 0 ? (1ll << 40) : (long long)units * sh.num_kv_heads;
    const long long blocks = (warps + kWarps - 1) / kWarps, most = (long long)per_sm * t.num_sms;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (chained) launch_chained(kernel, grid, dim3(kThreads), smem, st, p);
    else kernel<<<grid, dim3(kThreads), smem, st>>>(p);  // behind an event of another stream
    return true;
  };
  static bool optin[4][kMaxDevices] = {};
  bool ok;
  if (sh.head_dim == 128)
    ok = rows == 8 ? go(k_decode4<128, 1>, kWarps * sizeof(WarpSmem<128, 1>), kCtas4<1>, optin[1])
                   : go(k_decode4<128, 2>, kWarps * sizeof(WarpSmem<128, 2>), kCtas4<2>, optin[0]);
  else
    ok = rows == 8 ? go(k_decode4<64, 1>, kWarps * sizeof(WarpSmem<64, 1>), kCtas4<1>, optin[3])
                   : go(k_decode4<64, 2>, kWarps * sizeof(WarpSmem<64, 2>), kCtas4<2>, optin[2]);
  return ok && cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace gf
