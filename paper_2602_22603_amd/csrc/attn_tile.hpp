// attn_tile.hpp - the 64-key block tile of the attention kernels that run many
// query rows against the paged cache on the matrix cores (gfx950, wave64): the
// chunk kernel (extend_kernels.hip), where it is described, and the drafted
// trees' kernel (draft_kernels.hip).
// Internal to libsq; to be included inside one .hip file, which is compiled
// without honouring NaN operands.
#pragma once

#include <hip/hip_bf16.h>

#include "extend_args.hpp"
#include "fp8.hpp"

namespace sq {
namespace {

constexpr int BK = kExtKeys;
constexpr float kNegInf = -__builtin_huge_valf();
// Two waves per SIMD (up to 256 registers each): the eight waves of the one
// 256-row workgroup a CU holds, or of two with 128 rows.
constexpr int kExtWavesPerEu = 2;

typedef __bf16 bf16x2_t __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef __bf16 bf16x8_t __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef float f32x4_t __attribute__((__vector_size__(4 * sizeof(float))));

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline float max_xrow16(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_xrow32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_xrow16(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float sum_xrow32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));

// bf16 round-to-nearest-even of two floats, packed low | high << 16 (one
// v_cvt_pk_bf16_f32).
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, bf16x2v_t));
}

// p less the low or the high half of a packed pair of bf16 values: the dot
// product with (-1, 0) or (0, -1) plus p, one instruction in place of
// unpacking the half and subtracting.  Exact either way: p's bf16 rounding
// is within a factor of two of p.  The factors come from registers (as a
// constant the compiler turns (-1, 0) into the inline constant -1.0, which
// this instruction reads as (0, -1)).
__device__ inline uint32_t minus_one(int half) {
  uint32_t x = half ? 0xbf800000u : 0xbf80u;
  asm("" : "+s"(x));
  return x;
}
__device__ inline float residue(uint32_t pair, uint32_t minus_one_at, float p) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair),
                                         __builtin_bit_cast(bf16x2_t, minus_one_at), p, false);
}

template <int D, int W> struct ExtLayout {
  static constexpr int CH = D / 8;             // 16-byte chunks per K row
  static constexpr int KROWS = 1024 / (2 * D); // K rows one wave-wide DMA writes
  static constexpr int K_ELEMS = BK * D;       // bf16 per K buffer
  static constexpr int V_ELEMS = D * BK;       // bf16 per V^T buffer
  static constexpr int NK = K_ELEMS * 2 / 1024 / W; // K DMAs per wave per block
  static constexpr int NV = V_ELEMS * 2 / 1024 / W; // V DMAs per wave per block
  static constexpr int KPP = kPage / KROWS; // K copy instructions that fill a page
  static constexpr int VPP = kPage * D * 2 / 1024; // and V^T ones
  static constexpr int NP = NK > KPP ? NK / KPP : 1; // pages a wave's copies cover
  // block buffers of a bf16 store: three, or two where two workgroups are to
  // share a CU's LDS (an 8-bit store, whose next block passes through
  // registers, uses two whatever the tile; the third then takes no LDS)
  static constexpr int NB = D == 128 && W < 8 ? 2 : 3;
  static_assert(KPP == VPP && (NK % KPP == 0 || KPP % NK == 0), "a wave copies whole pages or a part of one");
};

// LDS layouts.  A 16-byte LDS read (ds_read_b128) is served 16 lanes at a
// time from 64 four-byte banks, the 16 being lanes 0-3, 12-15, 20-23 and
// 24-27, or 4-11, 16-19 and 28-31, of each half-wave (measured on gfx950 with
// the bank-conflict counter), so it is conflict-free when the chunks of each
// such set are distinct modulo 16.
//   K: one row of D channels per key; an operand read has lane (n, kg) read
//      logical chunk 4 kc + kg of row tile_key(t, n) = 32a + 8(n >> 2) + 4h
//      + (n & 3), so chunks are XOR-swizzled within the row.  With 256-byte
//      rows the key (n & 3) + 4 (n >> 2) = n gives kg ^ n, distinct in each
//      set.  With 128-byte rows two rows share the banks, the row's parity
//      choosing the half, and bit 1 of n & 3 and of n >> 2 separate the rest
//      (within a set kg tells n >> 2 = 0, 3 from 1, 2).
//   V^T: the block's four pages one after another, each as the pool holds
//      it (D rows of 16 keys, 32 bytes), so a page is copied as it lies.  A
//      P.V operand read has lane (n, kg) read keys 8 (4 c2 + kg) .. +7 of row
//      d = 16 dt + n: page 2 c2 + kg / 2, chunk 2 d + kg % 2 of it, distinct
//      in each set.
template <int D> __device__ inline int k_phys(int row, int c) {
  if constexpr (D == 128) return c ^ ((row & 3) + 4 * ((row >> 3) & 3));
  else return c ^ ((row & 2) + 4 * ((row >> 4) & 1));
}
// Element offset, in a V^T block buffer, of keys 8 j .. 8 j + 7 of row d.
template <int D> __device__ inline int v_off(int d, int j) {
  return (j >> 1) * (D * kPage) + d * kPage + 8 * (j & 1);
}

// The block key held by A row r of S^T tile t (0..3): tiles 2c and 2c + 1
// cover the 32-key chunk c, row 4 kg + i of tile 2c + h being key
// 32 c + 8 kg + 4 h + i.
__device__ inline int tile_key(int t, int r) {
  return 32 * (t >> 1) + 8 * (r >> 2) + 4 * (t & 1) + (r & 3);
}

typedef __attribute__((address_space(3))) void lds_void;

// s_waitcnt immediate that waits until at most N vector memory operations
// are outstanding and leaves the other counters alone (gfx9 encoding:
// vmcnt in bits 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8).
template <int N> constexpr int kVmcntKeep = (N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8);

// A workgroup barrier for LDS written by ordinary stores: this wave's LDS
// stores complete, then the barrier.  __syncthreads() (and a fence on LDS
// alone) also waits for every vector memory operation in flight, the block
// copies into the other buffers included, since they too write LDS.  The
// memory clobber keeps the compiler from moving memory accesses across it.
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The bits from d on, of 64 keys.
__device__ inline uint64_t ones_from(int d) { return d <= 0 ? ~0ull : d >= 64 ? 0ull : ~0ull << d; }
// This lane's 16 keys of a block's 64 (bit per key): bit 4 tt + i is key
// tile_key(tt, 4 kg + i) = 32 (tt >> 1) + 8 kg + 4 (tt & 1) + i.
__device__ inline int lane_bits(uint64_t w, int kg) {
  return (int)((w >> (8 * kg)) & 0xff) | (int)((w >> (32 + 8 * kg)) & 0xff) << 8;
}

// Page ids of block blk (4 pages; ids past the sequence's list repeat its
// last page: every key there is at or past L, so its score is masked and its
// V zeroed before use).  The index is uniform, so these are scalar loads,
// issued a block ahead of their use.
// (Read through the constant address space: scalar loads, which the
// scalar-load counter tracks.  As vector loads, each wait for them would
// also wait for the block copies in flight, which count on the same
// in-order vector counter.)
typedef const int32_t __attribute__((address_space(4))) *ext_sptr_t;
// PG: a sequence's pages (pt, n_pages, page_stride).
template <class PG> __device__ inline void block_ids(int32_t (&ids)[4], const PG &a, int blk) {
#pragma unroll
  for (int i = 0; i < 4; ++i) ids[i] = ((ext_sptr_t)a.pt)[min(blk * (BK / kPage) + i, a.n_pages - 1)];
}

// ids[q] for a q that may differ per lane, without branches.
__device__ inline int32_t pick4(const int32_t (&ids)[4], int q) {
  const int32_t lo = (q & 1) ? ids[1] : ids[0];
  const int32_t hi = (q & 1) ? ids[3] : ids[2];
  return (q & 2) ? hi : lo;
}

// A buffer resource over one page of a pool (the 16-byte loads below are
// relative to it).
__device__ inline __amdgpu_buffer_rsrc_t ext_page(const void *page, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(page), (short)0, bytes, 0x00020000);
}

// Global -> LDS (direct) for one block: each wave copies NP whole pages of the
// block, or a part of one, K rows and V^T alike, so one page address (formed by
// the scalar unit from the page id) serves all copy instructions of a page and
// the lanes add offsets that do not change from block to block.
// AUX: the loads' cache policy (2: non-temporal, for keys that are read once).
template <int D, int W, int AUX = 0, class PG>
__device__ inline void ext_dma(uint16_t *sk, uint16_t *sv, const PG &a,
                               const uint16_t *kbase, const uint16_t *vbase,
                               const int32_t (&ids)[4], int wave, int lane) {
  using Lt = ExtLayout<D, W>;
  constexpr int kPageBytes = kPage * D * 2;
  constexpr int IPP = Lt::KPP, PER = Lt::NK / Lt::NP; // instructions per page; this wave's of each
#pragma unroll
  for (int pg = 0; pg < Lt::NP; ++pg) {
    const int64_t off = (int64_t)pick4(ids, (wave * Lt::NK + pg * PER) / IPP) * a.page_stride;
    const __amdgpu_buffer_rsrc_t kr = ext_page(kbase + off, kPageBytes);
    const __amdgpu_buffer_rsrc_t vr = ext_page(vbase + off, kPageBytes);
#pragma unroll
    for (int u = pg * PER; u < (pg + 1) * PER; ++u) {
      const int ins = wave * Lt::NK + u;
      const int row = ins * Lt::KROWS + lane / Lt::CH;
      const int c = k_phys<D>(row, lane % Lt::CH); // the swizzle is an involution
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void *)(sk + ins * 512), 16,
                                               ((row % kPage) * D + 8 * c) * 2, 0, 0, AUX);
    }
#pragma unroll
    for (int u = pg * PER; u < (pg + 1) * PER; ++u) {
      const int ins = wave * Lt::NV + u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void *)(sv + ins * 512), 16,
                                               ((ins % IPP) * 512 + lane * 8) * 2, 0, 0, AUX);
    }
  }
}

// An 8-bit store: the same block through registers.  ext_load8 loads the 8
// codes each lane's DMA would have copied as 8 bf16 values (half the bytes);
// ext_store8 converts them and writes the bf16 tile exactly where the DMA
// writes it, so the compute is unchanged.
template <int D, int W, int N, class PG>
__device__ inline void ext_load8(uint2 (&kr)[N], uint2 (&vr)[N],
                                 const PG &a, const uint8_t *kbase, const uint8_t *vbase,
                                 const int32_t (&ids)[4], int wave, int lane) {
  using Lt = ExtLayout<D, W>;
#pragma unroll
  for (int u = 0; u < Lt::NK; ++u) {
    const int ins = wave * Lt::NK + u;
    const int row = ins * Lt::KROWS + lane / Lt::CH;
    const int c = k_phys<D>(row, lane % Lt::CH);
    const int p = ins / Lt::KPP;
    kr[u] = *reinterpret_cast<const uint2 *>(kbase + (int64_t)pick4(ids, p) * a.page_stride +
                                             (row % kPage) * D + 8 * c);
  }
  constexpr int IPP = kPage * D * 2 / 1024; // bf16 copy instructions per page
#pragma unroll
  for (int u = 0; u < Lt::NV; ++u) {
    const int ins = wave * Lt::NV + u;
    vr[u] = *reinterpret_cast<const uint2 *>(vbase + (int64_t)pick4(ids, ins / IPP) * a.page_stride +
                                             (ins % IPP) * 512 + lane * 8);
  }
}
template <int D, int W, int N>
__device__ inline void ext_store8(uint16_t *sk, uint16_t *sv, const uint2 (&kr)[N],
                                  const uint2 (&vr)[N], int wave, int lane) {
  using Lt = ExtLayout<D, W>;
#pragma unroll
  for (int u = 0; u < Lt::NK; ++u) {
    const uint2 lo = e4m3x4_to_bf16(kr[u].x), hi = e4m3x4_to_bf16(kr[u].y);
    *reinterpret_cast<uint4 *>(sk + (wave * Lt::NK + u) * 512 + lane * 8) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
#pragma unroll
  for (int u = 0; u < Lt::NV; ++u) {
    const uint2 lo = e4m3x4_to_bf16(vr[u].x), hi = e4m3x4_to_bf16(vr[u].y);
    *reinterpret_cast<uint4 *>(sv + (wave * Lt::NV + u) * 512 + lane * 8) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
}

// Zero V^T entries of keys at or past L in the block's buffer (the last
// block only), so that 0 * v stays 0 whatever the pool holds there.
template <int D, int W>
__device__ inline void ext_zero_tail(uint16_t *sv, int blk, int L, int tid) {
  for (int q = tid; q < D * 8; q += 64 * W) {
    const int d = q >> 3, j = q & 7;
    const int k0 = blk * BK + 8 * j;
    if (k0 + 8 <= L) continue;
    uint4 *p = reinterpret_cast<uint4 *>(sv + v_off<D>(d, j));
    uint4 x = *p;
    uint32_t m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      m[e] = (k0 + 2 * e < L ? 0xffffu : 0u) | (k0 + 2 * e + 1 < L ? 0xffff0000u : 0u);
    x.x &= m[0];
    x.y &= m[1];
    x.z &= m[2];
    x.w &= m[3];
    *p = x;
  }
}

// Softmax state of one lane: two query columns (rows of the attention).  m
// is the reference in log2 units: the weights of a half block (32 keys) are
// taken as 2^(s - m) against the m in hand, and only when some lane's sum of
// them reaches kBig (or the row has no reference yet) does the wave raise m
// to the half block's maximum, rescale O^T and l, and take the weights
// again.  A weight below 2^64 leaves fp32 room for l and acc over any key
// count, and out = acc / l does not depend on m.
constexpr float kBig = 0x1p64f;

// One 64-key block against this wave's 32 query columns.  need_mask: some
// column does not see every key of the block; only then is the per-key test
// made.  Column cg sees keys first[cg] .. lim[cg] of those whose bit is set in
// lm (bit 4 tt + i = this lane's key tile_key(tt, 4 kg + i); a deferred
// eviction clears bits), or, with BITS, the keys whose bit is set in lim[cg].
// after_scores() runs once the score MFMAs are issued: the caller's scalar
// loads go there, since while one is in flight (scalar loads return out of
// order on the counter they share with LDS reads) an MFMA could only wait
// for all 16 K reads at once instead of for its own.
template <int D, bool BITS = false, typename F>
__device__ __attribute__((always_inline)) inline void ext_block(const uint16_t *sk, const uint16_t *sv, int b, int n, int kg,
                                 float c, bool need_mask, const bf16x8_t (&qf)[2][D / 32],
                                 const int (&first)[2], const int (&lim)[2], uint32_t lm,
                                 f32x4_t (&acc)[D / 16][2], float (&m_run)[2], float (&l_run)[2],
                                 F &&after_scores) {
  constexpr int NKC = D / 32;
  constexpr int NDT = D / 16;
  f32x4_t st[4][2];
#pragma unroll
  for (int tt = 0; tt < 4; ++tt)
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) st[tt][cg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // all the block's K fragments are read first (their LDS latency then
  // overlaps), k chunks outermost: the 8 accumulators of a block are 8
  // independent chains, so consecutive MFMAs never wait on each other's result
  bf16x8_t ka[NKC][4];
#pragma unroll
  for (int kc = 0; kc < NKC; ++kc)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const int row = tile_key(tt, n);
      ka[kc][tt] = __builtin_bit_cast(
          bf16x8_t, *reinterpret_cast<const uint4 *>(sk + row * D + 8 * k_phys<D>(row, 4 * kc + kg)));
    }
  __builtin_amdgcn_sched_barrier(0); // (the compiler would move each read back next to its use)
#pragma unroll
  for (int kc = 0; kc < NKC; ++kc)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int cg = 0; cg < 2; ++cg)
        st[tt][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[kc][tt], qf[cg][kc], st[tt][cg], 0, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
  after_scores();
  if (need_mask) {
#pragma unroll
    for (int cg = 0; cg < 2; ++cg)
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (BITS) {
            if (!((lim[cg] >> (4 * tt + i)) & 1)) st[tt][cg][i] = kNegInf;
          } else {
            const int key = b * BK + tile_key(tt, 4 * kg + i);
            if (key > lim[cg] || key < first[cg] || !((lm >> (4 * tt + i)) & 1)) st[tt][cg][i] = kNegInf;
          }
        }
  }
  const uint32_t m1l = minus_one(0), m1h = minus_one(1);
  float nm[2];
#pragma unroll
  for (int cg = 0; cg < 2; ++cg) nm[cg] = m_run[cg] == kNegInf ? 0.f : -m_run[cg];
#pragma unroll
  for (int c2 = 0; c2 < 2; ++c2) {
    bf16x8_t phi[2], plo[2];
    float psum[2];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int cg = 0; cg < 2; ++cg) {
        uint32_t h[4], l[4];
        psum[cg] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tt = 2 * c2 + (e >> 1);
          const float p0 = exp2_fast(fmaf(st[tt][cg][2 * (e & 1)], c, nm[cg]));
          const float p1 = exp2_fast(fmaf(st[tt][cg][2 * (e & 1) + 1], c, nm[cg]));
          h[e] = pack_bf16(p0, p1);
          l[e] = pack_bf16(residue(h[e], m1l, p0), residue(h[e], m1h, p1));
          psum[cg] += p0 + p1;
        }
        phi[cg] = __builtin_bit_cast(bf16x8_t, make_uint4(h[0], h[1], h[2], h[3]));
        plo[cg] = __builtin_bit_cast(bf16x8_t, make_uint4(l[0], l[1], l[2], l[3]));
      }
    };
    weights();
    const bool ok = m_run[0] != kNegInf && m_run[1] != kNegInf && psum[0] < kBig && psum[1] < kBig;
    if (!__all(ok)) { // (wave-uniform) raise the references to this half block's maxima
      float alpha[2];
#pragma unroll
      for (int cg = 0; cg < 2; ++cg) {
        float mx = kNegInf;
#pragma unroll
        for (int tt = 2 * c2; tt < 2 * c2 + 2; ++tt)
          mx = fmaxf(mx, fmaxf(fmaxf(st[tt][cg][0], st[tt][cg][1]), fmaxf(st[tt][cg][2], st[tt][cg][3])));
        mx = max_xrow16(mx);
        mx = max_xrow32(mx) * c; // scale > 0: the max commutes with it
        const float m_new = fmaxf(m_run[cg], mx);
        alpha[cg] = m_new == m_run[cg] ? 1.f : exp2_fast(m_run[cg] - m_new); // 0 from -inf
        m_run[cg] = m_new;
        nm[cg] = m_new == kNegInf ? 0.f : -m_new;
        l_run[cg] *= alpha[cg];
      }
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int cg = 0; cg < 2; ++cg) acc[dt][cg] *= alpha[cg];
      weights();
    }
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) l_run[cg] += psum[cg];
    // all hi products, then all lo: the two MFMAs into one accumulator are
    // 2 * NDT instructions apart
    bf16x8_t va[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) {
      const int d = 16 * dt + n;
      va[dt] = __builtin_bit_cast(
          bf16x8_t, *reinterpret_cast<const uint4 *>(sv + v_off<D>(d, 4 * c2 + kg)));
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int cg = 0; cg < 2; ++cg)
        acc[dt][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[dt], phi[cg], acc[dt][cg], 0, 0, 0);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int cg = 0; cg < 2; ++cg)
        acc[dt][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[dt], plo[cg], acc[dt][cg], 0, 0, 0);
  }
}

} // namespace
} // namespace sq
