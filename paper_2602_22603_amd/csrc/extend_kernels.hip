// extend_kernels.hip - causal attention of a chunk of appended tokens over the
// paged, possibly compacted, KV cache, for gfx950 (CDNA4, wave64).
//
// Algorithm 1 grows the main thread's context by whole chunks (Phase 3: the
// turn's reasoning, then the tool output).  Each appended token attends to
// every cached key up to and including itself: the compacted prefix left by
// Phase 1's eviction and the chunk's earlier tokens.  Unlike decode this is a
// dense contraction (256 query rows share every K/V tile), so it runs on the
// matrix cores:
//
//   workgroup = 8 waves (one workgroup per CU, two waves per SIMD), 256
//               query rows = (256 / G tokens) x (G query heads of one KV
//               head); each wave owns 32 rows as two MFMA column groups of
//               16.  Chunks whose rows would leave much of such a tile to
//               padding run 4 or 2 waves per workgroup, two workgroups per
//               CU (77 tokens x 4 heads over 60.5K keys: 127 us with three
//               128-row tiles, 152 with two of 256).
//   K/V       = blocks of 64 keys (4 pages), copied global -> LDS by the
//               gfx950 direct-to-LDS buffer loads (16 bytes a lane) into
//               three buffers: blocks b + 1 and b + 2 are in flight while
//               block b is computed, and no registers hold staging data (two
//               buffers, one block in flight, for the narrow tiles of 128
//               channels, so that two workgroups fit the CU's LDS).  K
//               rows have their 16-byte chunks XOR-swizzled and V^T keeps
//               the pool's page layout, so that the MFMA operand reads below
//               are free of bank conflicts.
//   S^T       = K . Q^T      v_mfma_f32_16x16x32_bf16 (A = K rows from LDS,
//                            B = Q^T held in registers for the whole pass)
//   O^T      += V^T . P^T    v_mfma_f32_16x16x32_bf16 over 32 keys at once.
//               The A rows of the S^T tiles are chosen so that lane group kg
//               ends up holding the scores of keys 8kg .. 8kg+7 of each 32-key
//               chunk: exactly the k slots of its P^T operand and, in the
//               page-transposed V pool, one contiguous 16-byte piece of V^T.
//               P never moves between lanes.  P is split into bf16 hi + lo
//               halves (two MFMAs) so the weights keep ~16 bits.
//   softmax   online, per query row, in log2 units (one v_exp_f32 per score)
//               against a running reference that is raised only when the
//               weights of a half block could grow too large (see kBig); a
//               raise takes the half block's row maximum across the four
//               lane groups by permlane swaps.
//
// Work order: workgroup w takes KV head w % Hkv (consecutive workgroups land
// on different XCDs, so each XCD's L2 serves one head's K/V) and query block
// (n_qblocks - 1 - w / Hkv): the blocks that see the most keys start first.
#include "attn_tile.hpp"

namespace sq {
namespace {


// FIRST: a windowed call whose queries also see the sequence's first tokens.  A
// query block's list of key blocks then has the first tokens' blocks in front,
// and a column's keys are two ranges, tested as one word of 64 bits.
template <int D, int G, int W, bool KV8 = false, bool FIRST = false>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(kExtWavesPerEu, kExtWavesPerEu))) void
k_extend(ExtendArgs a) {
  using Lt = ExtLayout<D, W>;
  constexpr int NKC = D / 32; // k chunks of S^T = K . Q^T
  constexpr int NDT = D / 16; // 16-channel tiles of O^T
  constexpr int ROWS = 32 * W;
  constexpr int TQ = ROWS / G;
  constexpr int NB = Lt::NB;
  // Three block buffers: block b is read from buffer b % 3 while the copies
  // of blocks b + 1 and b + 2 land in the other two.  They are separate LDS
  // objects and the block loop below is unrolled by three, so every LDS
  // read names its buffer at compile time: the compiler then knows that the
  // copies in flight cannot alias it and does not wait for them.
  // With two buffers block b + 1 alone is in flight.
  __shared__ __attribute__((aligned(16))) uint16_t sk0[Lt::K_ELEMS], sk1[Lt::K_ELEMS], sk2[NB > 2 ? Lt::K_ELEMS : 8];
  __shared__ __attribute__((aligned(16))) uint16_t sv0[Lt::V_ELEMS], sv1[Lt::V_ELEMS], sv2[NB > 2 ? Lt::V_ELEMS : 8];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6); // uniform: the DMA destination is M0
  const int n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.x % a.hkv;
  const int rest = blockIdx.x / a.hkv;
  const int sp = rest % a.n_split; // key-range split
  const int qb = a.n_qblocks - 1 - rest / a.n_split;
  const int j0 = qb * TQ;
  const int base = a.L - a.n; // logical index of new token 0

  // this lane's two query columns (rows of the attention)
  bf16x8_t qf[2][NKC];
  int lim[2], first[2], jrow[2], hrow[2];
  bool live[2];
#pragma unroll
  for (int cg = 0; cg < 2; ++cg) {
    const int col = 32 * wave + 16 * cg + n;
    jrow[cg] = j0 + col / G;
    hrow[cg] = g * G + col % G;
    live[cg] = jrow[cg] < a.n;
    lim[cg] = live[cg] ? base + jrow[cg] : a.L - 1;
    first[cg] = a.window > 0 ? lim[cg] - a.window + 1 : 0; // may be negative
    const uint16_t *qp = a.q + ((int64_t)jrow[cg] * a.hq + hrow[cg]) * D + 8 * kg;
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc) {
      const uint4 w = live[cg] ? *reinterpret_cast<const uint4 *>(qp + 32 * kc)
                               : make_uint4(0, 0, 0, 0);
      qf[cg][kc] = __builtin_bit_cast(bf16x8_t, w);
    }
  }
  const int kend = min(a.L, base + j0 + TQ); // keys this query block needs: [kbeg, kend)
  const int kbeg = a.window > 0 ? max(0, base + j0 - a.window + 1) : 0;
  // this workgroup's blocks [b_lo, b_hi), by place in the query block's list
  // where that has two parts
  const int nf = FIRST ? min((a.first + BK - 1) / BK, kbeg / BK) : 0, skip = FIRST ? kbeg / BK - nf : 0;
  const int b_lo = (FIRST ? 0 : kbeg / BK) + sp * a.split_blocks;
  const int b_hi = min((kend + BK - 1) / BK - skip, b_lo + a.split_blocks);
  auto at = [&](int i) __attribute__((always_inline)) { return !FIRST || i < nf ? i : i + skip; };
  const int mask_from = base + j0;           // keys above this need the causal test
  // keys below this are outside the window of the block's last token
  const int mask_below = a.window > 0 ? min(a.L - 1, base + j0 + TQ - 1) - a.window + 1 : 0;

  f32x4_t acc[NDT][2];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) acc[dt][cg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run[2] = {kNegInf, kNegInf}, l_run[2] = {0.f, 0.f};

  const uint16_t *kbase = a.k + (int64_t)g * a.head_stride;
  const uint16_t *vbase = a.v + (int64_t)g * a.head_stride;
  const uint8_t *kbase8 = reinterpret_cast<const uint8_t *>(a.k) + (int64_t)g * a.head_stride;
  const uint8_t *vbase8 = reinterpret_cast<const uint8_t *>(a.v) + (int64_t)g * a.head_stride;
  uint2 kr[Lt::NK], vr[Lt::NV]; // an 8-bit store's next block, in flight
  int32_t ids[4];
  // Copies run NB - 1 blocks ahead (one for an 8-bit store, whose next block
  // passes through registers): ids holds the page ids of the next block to
  // be fetched.  The copies of the NB - 1 blocks past b_hi are issued too (of
  // the last page, block_ids clamps) into buffers that no block reads: with
  // a copy issued at the top of every block, the copies in flight at each
  // block's top are the same on every path, which the compiler can follow,
  // and it adds no wait of its own before the LDS reads.
  if (b_lo < b_hi) {
    block_ids(ids, a, at(b_lo));
    if constexpr (KV8) {
      ext_load8<D, W>(kr, vr, a, kbase8, vbase8, ids, wave, lane);
      ext_store8<D, W>(sk0, sv0, kr, vr, wave, lane);
    } else {
      ext_dma<D, W>(sk0, sv0, a, kbase, vbase, ids, wave, lane);
      // the query loads, issued before this copy, have landed (said here, on
      // the only way into the loop, so that the compiler knows it)
      __builtin_amdgcn_s_waitcnt(kVmcntKeep<Lt::NK + Lt::NV>);
      if constexpr (NB > 2) {
        block_ids(ids, a, at(b_lo + 1));
        ext_dma<D, W>(sk1, sv1, a, kbase, vbase, ids, wave, lane);
      }
    }
    block_ids(ids, a, at(KV8 || NB == 2 ? b_lo + 1 : b_lo + 2));
    // block b from buffers c; buffers n1 and n2 are those of blocks b + 1 and
    // b + 2 (with two buffers, and for an 8-bit store, n2 is c)
    auto block = [&](int pb, uint16_t *ck, uint16_t *cv, uint16_t *n1k, uint16_t *n1v,
                     uint16_t *n2k, uint16_t *n2v) __attribute__((always_inline)) {
      const int b = at(pb);
      // keep bits of this lane's 16 keys of the block (deferred evictions)
      uint32_t lm = 0xffffu;
      bool masked_here = false;
      if (a.masked) {
        const ext_sptr_t mr = (ext_sptr_t)a.mask_row;
        const int p0 = b * (BK / kPage), last = a.n_pages - 1;
        const uint32_t m0 = mr[min(p0, last)], m1 = mr[min(p0 + 1, last)];
        const uint32_t m2 = mr[min(p0 + 2, last)], m3 = mr[min(p0 + 3, last)];
        masked_here = (m0 & m1 & m2 & m3) != 0xffffu;
        if (masked_here) {
          // bit 4 tt + i is key tile_key(tt, 4 kg + i) = 32 (tt >> 1) + 8 kg
          // + 4 (tt & 1) + i: page 2 (tt >> 1) + (kg >> 1), slot 8 (kg & 1)
          // + 4 (tt & 1) + i, so tiles 0, 1 take 8 consecutive slots of page
          // kg >> 1 and tiles 2, 3 the same slots of page 2 + (kg >> 1)
          const int sh = 8 * (kg & 1);
          const uint32_t lo = (kg >> 1) ? m1 : m0, hi = (kg >> 1) ? m3 : m2;
          lm = ((lo >> sh) & 0xffu) | (((hi >> sh) & 0xffu) << 8);
        }
      }
      // block b has landed (every wave's copies; with three buffers those of
      // block b + 1, issued later, may still be in flight) and every wave is
      // done with block b - 1, whose buffer the next copy overwrites
      __builtin_amdgcn_s_waitcnt(KV8 ? 0 : kVmcntKeep<NB == 2 ? 0 : Lt::NK + Lt::NV>);
      lds_barrier();
      if ((b + 1) * BK > a.L) {
        ext_zero_tail<D, W>(cv, b, a.L, tid);
        lds_barrier();
      }
      if constexpr (KV8) {
        if (pb + 1 < b_hi) ext_load8<D, W>(kr, vr, a, kbase8, vbase8, ids, wave, lane); // stored after this block
      } else {
        if constexpr (NB > 2) ext_dma<D, W>(n2k, n2v, a, kbase, vbase, ids, wave, lane);
        else ext_dma<D, W>(n1k, n1v, a, kbase, vbase, ids, wave, lane);
      }
      auto next_ids = [&]() __attribute__((always_inline)) {
        if constexpr (KV8) {
          if (pb + 1 < b_hi) block_ids(ids, a, at(pb + 2));
        } else {
          block_ids(ids, a, at(pb + NB));
        }
      };
      const bool late = b * BK + BK - 1 > mask_from;
      if constexpr (FIRST) {
        const bool need = late || (b * BK < mask_below && b * BK + BK > a.first);
        const uint64_t early = ~ones_from(a.first - b * BK);
        int seen[2];
#pragma unroll
        for (int cg = 0; cg < 2; ++cg)
          seen[cg] = lane_bits(~ones_from(lim[cg] + 1 - b * BK) & (ones_from(first[cg] - b * BK) | early), kg);
        ext_block<D, true>(ck, cv, b, n, kg, a.scale_log2, need, qf, first, seen, lm, acc, m_run, l_run, next_ids);
      } else {
        ext_block<D>(ck, cv, b, n, kg, a.scale_log2, late || b * BK < mask_below || masked_here, qf, first, lim, lm,
                     acc, m_run, l_run, next_ids);
      }
      if constexpr (KV8) { // a buffer every wave left by the top of this block
        if (pb + 1 < b_hi) ext_store8<D, W>(n1k, n1v, kr, vr, wave, lane);
      }
    };
    if constexpr (KV8) {
      for (int b = b_lo; b < b_hi; b += 2) {
        block(b, sk0, sv0, sk1, sv1, sk0, sv0);
        if (b + 1 < b_hi) block(b + 1, sk1, sv1, sk0, sv0, sk1, sv1);
      }
    } else if constexpr (NB == 2) {
      int b = b_lo;
      for (; b + 1 < b_hi; b += 2) {
        block(b, sk0, sv0, sk1, sv1, sk0, sv0);
        block(b + 1, sk1, sv1, sk0, sv0, sk1, sv1);
      }
      if (b < b_hi) block(b, sk0, sv0, sk1, sv1, sk0, sv0);
      __builtin_amdgcn_s_waitcnt(0); // no copy lands in LDS after the workgroup ends
    } else {
      // whole turns of the three buffers, then the rest: the loop's back
      // edge leaves every block of a turn behind it
      int b = b_lo;
      for (; b + 2 < b_hi; b += 3) {
        block(b, sk0, sv0, sk1, sv1, sk2, sv2);
        block(b + 1, sk1, sv1, sk2, sv2, sk0, sv0);
        block(b + 2, sk2, sv2, sk0, sv0, sk1, sv1);
      }
      if (b < b_hi) block(b, sk0, sv0, sk1, sv1, sk2, sv2);
      if (b + 1 < b_hi) block(b + 1, sk1, sv1, sk2, sv2, sk0, sv0);
      __builtin_amdgcn_s_waitcnt(0); // no copy lands in LDS after the workgroup ends
    }
  }

  if (a.n_split > 1) {
    // partial rows (a split may see no key of some rows: m = -inf, l = 0)
    const int64_t slot = ((int64_t)qb * a.hkv + g) * a.n_split + sp;
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) {
      float l = sum_xrow16(l_run[cg]);
      l = sum_xrow32(l);
      if (!live[cg]) continue;
      const int64_t row = slot * ROWS + 32 * wave + 16 * cg + n;
      if (kg == 0) {
        a.part_m[row] = m_run[cg];
        a.part_l[row] = l;
      }
      float *pp = a.part_acc + row * D + 4 * kg;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
        *reinterpret_cast<float4 *>(pp + 16 * dt) =
            make_float4(acc[dt][cg][0], acc[dt][cg][1], acc[dt][cg][2], acc[dt][cg][3]);
    }
    return;
  }
#pragma unroll
  for (int cg = 0; cg < 2; ++cg) {
    float l = sum_xrow16(l_run[cg]);
    l = sum_xrow32(l);
    if (!live[cg]) continue;
    float sc = 1.f;
    if (a.sinks) { // one more term of the sum, no value: rescale both to the larger maximum
      const float sk_l2 = a.sinks[hrow[cg]] * a.sink_scale;
      const float big = fmaxf(m_run[cg], sk_l2);
      sc = exp2_fast(m_run[cg] - big);
      l = fmaf(l, sc, exp2_fast(sk_l2 - big));
    }
    const float inv = sc / l * a.out_scale;
    float *op = a.out + ((int64_t)jrow[cg] * a.hq + hrow[cg]) * D + 4 * kg;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
      *reinterpret_cast<float4 *>(op + 16 * dt) =
          make_float4(acc[dt][cg][0] * inv, acc[dt][cg][1] * inv, acc[dt][cg][2] * inv,
                      acc[dt][cg][3] * inv);
  }
}

// Merge of the split key range: one wave per (new token j, query head h),
// lanes over channels.  Its partials are row (j % tq) * G + h % G of the
// n_split slots of (query block j / TQ, KV head h / G):
//   M = max m_s;  out = sum 2^(m_s - M) acc_s / sum 2^(m_s - M) l_s.
template <int D, int G>
__global__ __launch_bounds__(256) void k_extend_merge(ExtendArgs a) {
  constexpr int DPT = D / 64;
  const int tq = a.rows / G;
  constexpr int U = 8;
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); // (j, h) row
  if (r >= (int64_t)a.n * a.hq) return;
  const int j = (int)(r / a.hq), h = (int)(r % a.hq);
  const int g = h / G;
  const int64_t slot0 = ((int64_t)(j / tq) * a.hkv + g) * a.n_split;
  const int col = (j % tq) * G + h % G;
  const int S = a.n_split;
  float mine = kNegInf, lmine = 0.f;
  if (lane < S) {
    mine = a.part_m[(slot0 + lane) * a.rows + col];
    lmine = a.part_l[(slot0 + lane) * a.rows + col];
  }
  float big = mine;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor(big, o));
  const float sink = a.sinks ? a.sinks[h] * a.sink_scale : kNegInf;
  big = fmaxf(big, sink);
  const float w = (lane < S && big != kNegInf) ? exp2_fast(mine - big) : 0.f;
  float den = w * lmine;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o);
  if (a.sinks) den += exp2_fast(sink - big); // the sink's term, no value
  float num[DPT];
#pragma unroll
  for (int q = 0; q < DPT; ++q) num[q] = 0.f;
  for (int s0 = 0; s0 < S; s0 += U) {
    float x[U][DPT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int sidx = min(s0 + u, S - 1);
      const float *p = a.part_acc + ((slot0 + sidx) * a.rows + col) * D + lane * DPT;
#pragma unroll
      for (int q = 0; q < DPT; ++q) x[u][q] = p[q];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float wu = s0 + u < S ? __shfl(w, s0 + u) : 0.f;
#pragma unroll
      for (int q = 0; q < DPT; ++q) num[q] = fmaf(wu, x[u][q], num[q]);
    }
  }
  float *op = a.out + r * D + lane * DPT;
#pragma unroll
  for (int q = 0; q < DPT; ++q) op[q] = num[q] / den * a.out_scale;
}

template <int D, int G, int W, bool KV8> void extend_start(dim3 grid, dim3 block, const ExtendArgs &a, hipStream_t s) {
  if (a.first > 0) hipLaunchKernelGGL((k_extend<D, G, W, KV8, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_extend<D, G, W, KV8>), grid, block, 0, s, a);
}
template <int D, int W, bool KV8> hipError_t extend_dispatch(int group, const ExtendArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_qblocks * (unsigned)a.hkv * (unsigned)a.n_split), block(64 * W);
  switch (group) {
  case 1: extend_start<D, 1, W, KV8>(grid, block, a, s); break;
  case 2: extend_start<D, 2, W, KV8>(grid, block, a, s); break;
  case 4: extend_start<D, 4, W, KV8>(grid, block, a, s); break;
  case 8: extend_start<D, 8, W, KV8>(grid, block, a, s); break;
  default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
template <int D, bool KV8> hipError_t extend_dispatch_rows(int group, const ExtendArgs &a, hipStream_t s) {
  switch (a.rows) {
  case 256: return extend_dispatch<D, 8, KV8>(group, a, s);
  case 128: return extend_dispatch<D, 4, KV8>(group, a, s);
  case 64:
    if constexpr (D == 128) return extend_dispatch<D, 2, KV8>(group, a, s);
    return hipErrorInvalidValue; // (64 channels: 64 rows measured no faster than 128)
  default: return hipErrorInvalidValue;
  }
}

} // namespace

template <int D> hipError_t extend_merge_dispatch(int group, const ExtendArgs &a, hipStream_t s) {
  const int64_t rows = (int64_t)a.n * a.hq;
  const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
  switch (group) {
  case 1: hipLaunchKernelGGL((k_extend_merge<D, 1>), grid, block, 0, s, a); break;
  case 2: hipLaunchKernelGGL((k_extend_merge<D, 2>), grid, block, 0, s, a); break;
  case 4: hipLaunchKernelGGL((k_extend_merge<D, 4>), grid, block, 0, s, a); break;
  case 8: hipLaunchKernelGGL((k_extend_merge<D, 8>), grid, block, 0, s, a); break;
  default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_extend_merge(int d, int group, const ExtendArgs &a, hipStream_t s) {
  if (a.n <= 0 || a.n_split <= 1) return hipSuccess;
  if (d == 128) return extend_merge_dispatch<128>(group, a, s);
  if (d == 64) return extend_merge_dispatch<64>(group, a, s);
  return hipErrorInvalidValue;
}

hipError_t launch_extend(int d, int group, const ExtendArgs &a, hipStream_t s) {
  if (a.n <= 0) return hipSuccess;
  if (d == 128) return a.kv8 ? extend_dispatch_rows<128, true>(group, a, s) : extend_dispatch_rows<128, false>(group, a, s);
  if (d == 64) return a.kv8 ? extend_dispatch_rows<64, true>(group, a, s) : extend_dispatch_rows<64, false>(group, a, s);
  return hipErrorInvalidValue;
}

} // namespace sq
