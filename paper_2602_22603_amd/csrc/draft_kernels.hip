// draft_kernels.hip - attention of trees of drafted tokens over the paged,
// possibly compacted, KV cache, for gfx950 (CDNA4, wave64).
//
// To verify drafted tokens a model runs all nodes of a tree in one pass: node i
// of a sequence sees the sequence's cache and, of the draft, its own ancestors
// and itself,
//   out_i = sum_t softmax_t(scale q_i . k_t) v_t   over those t.
// Every K and V row is read once for all of a sequence's nodes, so a pass costs
// what a decode step of the sequence costs until the nodes' products outweigh
// the read: 4 D Hq flops a (node, key) pair, half as much again for weights of
// 16 bits, against 4 D Hkv bytes a key, a balance at about 128 query rows (nodes
// x heads of a KV head) on MI355X.
//
// The tile is the chunk kernel's (attn_tile.hpp, extend_kernels.hip): 32 query
// rows a wave, blocks of 64 keys through LDS.  The work of a launch is laid out
// by the host as pieces, runs of key blocks of one (tile of nodes, KV head),
// dealt out evenly to one round of workgroups whatever the sequences' lengths;
// a row that one workgroup takes whole goes straight to the output, the others
// leave partial rows that k_draft_merge joins.  Which nodes a node sees is one
// 64-bit word, shifted to the block's keys; a block of the cache alone needs no
// test.
#include "attn_tile.hpp"
#include "draft_args.hpp"

namespace sq {
namespace {

// The pages of one sequence.
struct SeqPages {
  const int32_t *pt;
  int32_t n_pages;
  int64_t page_stride;
};

template <int D, int W, bool KV8>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(kExtWavesPerEu, kExtWavesPerEu))) void
k_draft(DraftArgs a) {
  using Lt = ExtLayout<D, W>;
  constexpr int NKC = D / 32;
  constexpr int NDT = D / 16;
  constexpr int ROWS = 32 * W;
  constexpr int NB = Lt::NB;
  // block buffers as separate LDS objects, the block loop unrolled over them:
  // see k_extend
  __shared__ __attribute__((aligned(16))) uint16_t sk0[Lt::K_ELEMS], sk1[Lt::K_ELEMS], sk2[NB > 2 ? Lt::K_ELEMS : 8];
  __shared__ __attribute__((aligned(16))) uint16_t sv0[Lt::V_ELEMS], sv1[Lt::V_ELEMS], sv2[NB > 2 ? Lt::V_ELEMS : 8];
  // what the tile's nodes see (read for the few blocks that need a test; in
  // registers it made the 256-row kernel spill)
  __shared__ uint64_t s_anc[kMaxDraft];
  __shared__ int32_t s_lo[kMaxDraft];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, kg = lane >> 4;
  const int plan = a.windowed;
  const DraftSplit &sp = a.blob->split[plan];
  const int p_end = ((ext_sptr_t)sp.piece0)[blockIdx.x + 1];
  for (int p = ((ext_sptr_t)sp.piece0)[blockIdx.x]; p < p_end; ++p) {
    const ext_sptr_t pc = (ext_sptr_t)&sp.pieces[p];
    const int row = pc[0], b_lo = pc[1], b_hi = pc[2], slot = pc[3];
    const int g = row % a.hkv;
    const ext_sptr_t tl = (ext_sptr_t)&a.blob->tiles[row / a.hkv];
    const int pt_row = tl[0], base = tl[1], n_draft = tl[2], n_pages = tl[3], node0 = tl[4], n_nodes = tl[5];
    const int masked = tl[6];
    const int nf = tl[8 + plan], skip = tl[10 + plan], lo_max = tl[12 + plan];
    const int L = base + n_draft;
    const SeqPages pg{a.pt + (int64_t)pt_row * a.max_pages, n_pages, a.page_stride};
    const ext_sptr_t mask_row = (ext_sptr_t)(a.mask + (int64_t)pt_row * a.max_pages);
    // the block at place i of the row's list
    auto at = [&](int i) { return i < nf ? i : i + skip; };

    // every wave has left the piece before (its LDS is written next)
    lds_barrier();
    if (tid < n_nodes) {
      s_anc[tid] = a.blob->nodes[node0 + tid].anc[plan];
      s_lo[tid] = a.blob->nodes[node0 + tid].lo;
    }
    // this lane's two query columns (rows of the attention)
    bf16x8_t qf[2][NKC];
    auto node_of = [&](int cg) { return (32 * wave + 16 * cg + n) >> a.lg; }; // in the tile
    auto head_of = [&](int cg) { return (g << a.lg) + ((32 * wave + 16 * cg + n) & ((1 << a.lg) - 1)); };
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) {
      const bool live = node_of(cg) < n_nodes;
      const uint16_t *qp = a.q + ((int64_t)(node0 + node_of(cg)) * a.hq + head_of(cg)) * D + 8 * kg;
#pragma unroll
      for (int kc = 0; kc < NKC; ++kc)
        qf[cg][kc] = __builtin_bit_cast(bf16x8_t, live ? *reinterpret_cast<const uint4 *>(qp + 32 * kc)
                                                       : make_uint4(0, 0, 0, 0));
    }
    const bool wave_live = ((32 * wave) >> a.lg) < n_nodes;

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
    uint2 kr[Lt::NK], vr[Lt::NV];
    int32_t ids[4];
    block_ids(ids, pg, at(b_lo));
    if constexpr (KV8) {
      ext_load8<D, W>(kr, vr, pg, kbase8, vbase8, ids, wave, lane);
      ext_store8<D, W>(sk0, sv0, kr, vr, wave, lane);
    } else {
      ext_dma<D, W>(sk0, sv0, pg, kbase, vbase, ids, wave, lane);
      __builtin_amdgcn_s_waitcnt(kVmcntKeep<Lt::NK + Lt::NV>); // the query loads have landed
      if constexpr (NB > 2) {
        block_ids(ids, pg, at(b_lo + 1));
        ext_dma<D, W>(sk1, sv1, pg, kbase, vbase, ids, wave, lane);
      }
    }
    block_ids(ids, pg, at(KV8 || NB == 2 ? b_lo + 1 : b_lo + 2));
    auto block = [&](int i, uint16_t *ck, uint16_t *cv, uint16_t *n1k, uint16_t *n1v, uint16_t *n2k,
                     uint16_t *n2v) __attribute__((always_inline)) {
      const int k0 = at(i) * BK; // the block's first key
      // keep bits of the block's keys (deferred evictions)
      uint64_t keep = ~0ull;
      if (masked) {
        const int p0 = k0 / kPage, last = n_pages - 1;
        const uint32_t m0 = mask_row[min(p0, last)], m1 = mask_row[min(p0 + 1, last)];
        const uint32_t m2 = mask_row[min(p0 + 2, last)], m3 = mask_row[min(p0 + 3, last)];
        keep = (uint64_t)(m0 | m1 << 16) | (uint64_t)(m2 | m3 << 16) << 32;
      }
      const bool tail = k0 + BK > base;
      const bool need = tail || (plan && k0 < lo_max && k0 + BK > a.first) || keep != ~0ull;
      __builtin_amdgcn_s_waitcnt(KV8 ? 0 : kVmcntKeep<NB == 2 ? 0 : Lt::NK + Lt::NV>);
      lds_barrier();
      if (k0 + BK > L) {
        ext_zero_tail<D, W>(cv, k0 / BK, L, tid);
        lds_barrier();
      }
      if constexpr (KV8) {
        if (i + 1 < b_hi) ext_load8<D, W>(kr, vr, pg, kbase8, vbase8, ids, wave, lane);
      } else {
        if constexpr (NB > 2) ext_dma<D, W>(n2k, n2v, pg, kbase, vbase, ids, wave, lane);
        else ext_dma<D, W>(n1k, n1v, pg, kbase, vbase, ids, wave, lane);
      }
      int seen[2] = {0, 0};
      if (need) {
        const uint64_t cache = ~ones_from(base - k0); // keys of the cache
        const uint64_t early = ~ones_from(a.first - k0);
        const int off = base - k0; // place of node 0
#pragma unroll
        for (int cg = 0; cg < 2; ++cg) {
          // a row past the nodes sees every key, so that it never has to look
          // for a first one
          const int i = node_of(cg);
          const uint64_t anc = i < n_nodes ? s_anc[i] : ~0ull >> (64 - n_draft);
          uint64_t w = cache;
          if (plan && i < n_nodes) w &= ones_from(s_lo[i] - k0) | early;
          if (off > -64 && off < 64) w |= off >= 0 ? anc << off : anc >> -off;
          w &= keep;
          seen[cg] = lane_bits(w, kg);
        }
      }
      auto next_ids = [&]() __attribute__((always_inline)) {
        if constexpr (KV8) {
          if (i + 1 < b_hi) block_ids(ids, pg, at(i + 2));
        } else {
          block_ids(ids, pg, at(i + NB));
        }
      };
      const int none[2] = {0, 0};
      if (wave_live) ext_block<D, true>(ck, cv, 0, n, kg, a.scale_log2, need, qf, none, seen, 0, acc, m_run, l_run, next_ids);
      else next_ids();
      if constexpr (KV8) {
        if (i + 1 < b_hi) ext_store8<D, W>(n1k, n1v, kr, vr, wave, lane);
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
      __builtin_amdgcn_s_waitcnt(0);
    } else {
      int b = b_lo;
      for (; b + 2 < b_hi; b += 3) {
        block(b, sk0, sv0, sk1, sv1, sk2, sv2);
        block(b + 1, sk1, sv1, sk2, sv2, sk0, sv0);
        block(b + 2, sk2, sv2, sk0, sv0, sk1, sv1);
      }
      if (b < b_hi) block(b, sk0, sv0, sk1, sv1, sk2, sv2);
      if (b + 1 < b_hi) block(b + 1, sk1, sv1, sk2, sv2, sk0, sv0);
      __builtin_amdgcn_s_waitcnt(0);
    }

#pragma unroll
    for (int cg = 0; cg < 2; ++cg) {
      float l = sum_xrow16(l_run[cg]);
      l = sum_xrow32(l);
      if (node_of(cg) >= n_nodes) continue;
      if (slot >= 0) { // a part of the row's keys
        const int64_t r = (int64_t)slot * ROWS + 32 * wave + 16 * cg + n;
        if (kg == 0) {
          a.part_m[r] = m_run[cg];
          a.part_l[r] = l;
        }
        float *pp = a.part_acc + r * D + 4 * kg;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
          *reinterpret_cast<float4 *>(pp + 16 * dt) =
              make_float4(acc[dt][cg][0], acc[dt][cg][1], acc[dt][cg][2], acc[dt][cg][3]);
        continue;
      }
      float sc = 1.f;
      if (a.sinks) { // one more term of the sum, no value
        const float sk_l2 = a.sinks[head_of(cg)] * a.sink_scale;
        const float big = fmaxf(m_run[cg], sk_l2);
        sc = exp2_fast(m_run[cg] - big);
        l = fmaf(l, sc, exp2_fast(sk_l2 - big));
      }
      const float inv = sc / l * a.out_scale;
      float *op = a.out + ((int64_t)(node0 + node_of(cg)) * a.hq + head_of(cg)) * D + 4 * kg;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
        *reinterpret_cast<float4 *>(op + 16 * dt) = make_float4(acc[dt][cg][0] * inv, acc[dt][cg][1] * inv,
                                                                acc[dt][cg][2] * inv, acc[dt][cg][3] * inv);
    }
  }
}

// The rows whose keys were split: M = max m_s, out = sum 2^(m_s - M) acc_s / sum
// 2^(m_s - M) l_s.  A workgroup of NW waves takes one (node, head), each wave a
// share of its partial slots, lanes over channels.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void k_draft_merge(DraftArgs a) {
  constexpr int DPT = D / 64;
  constexpr int U = 8;
  __shared__ float s_m[NW], s_l[NW], s_acc[NW][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i = blockIdx.x / a.hq, h = blockIdx.x % a.hq;
  const int tile = a.blob->nodes[i].tile;
  const int g = h >> a.lg;
  const DraftMerge mr = a.blob->split[a.windowed].merge[tile * a.hkv + g];
  if (mr.n == 0) return;
  const int col = ((i - a.blob->tiles[tile].node0) << a.lg) + (h & ((1 << a.lg) - 1));
  float big = kNegInf, den = 0.f, num[DPT];
#pragma unroll
  for (int q = 0; q < DPT; ++q) num[q] = 0.f;
  for (int s0 = wave * U; s0 < mr.n; s0 += NW * U) {
    float x[U][DPT], m[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = (int64_t)(mr.slot0 + min(s0 + u, mr.n - 1)) * a.rows + col;
      m[u] = s0 + u < mr.n ? a.part_m[r] : kNegInf;
      l[u] = a.part_l[r];
#pragma unroll
      for (int q = 0; q < DPT; ++q) x[u][q] = a.part_acc[r * D + lane * DPT + q];
    }
    float top = big;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, m[u]);
    if (top == kNegInf) continue;
    const float sc = exp2_fast(big - top);
    den *= sc;
#pragma unroll
    for (int q = 0; q < DPT; ++q) num[q] *= sc;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = exp2_fast(m[u] - top);
      den = fmaf(w, l[u], den);
#pragma unroll
      for (int q = 0; q < DPT; ++q) num[q] = fmaf(w, x[u][q], num[q]);
    }
    big = top;
  }
  if (NW > 1) {
    if (lane == 0) {
      s_m[wave] = big;
      s_l[wave] = den;
    }
#pragma unroll
    for (int q = 0; q < DPT; ++q) s_acc[wave][lane * DPT + q] = num[q];
    __syncthreads();
    if (wave != 0) return;
    float top = kNegInf;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[w]);
    den = 0.f;
#pragma unroll
    for (int q = 0; q < DPT; ++q) num[q] = 0.f;
    big = top;
    if (top != kNegInf) {
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float sc = exp2_fast(s_m[w] - top);
        den = fmaf(sc, s_l[w], den);
#pragma unroll
        for (int q = 0; q < DPT; ++q) num[q] = fmaf(sc, s_acc[w][lane * DPT + q], num[q]);
      }
    }
  }
  float sc = 1.f;
  if (a.sinks) {
    const float sink = a.sinks[h] * a.sink_scale, top = fmaxf(big, sink);
    sc = exp2_fast(big - top);
    den = fmaf(den, sc, exp2_fast(sink - top));
  }
  sc = sc / den * a.out_scale; // (a node sees itself, so there is always a term)
  float *op = a.out + ((int64_t)i * a.hq + h) * D + lane * DPT;
#pragma unroll
  for (int q = 0; q < DPT; ++q) op[q] = num[q] * sc;
}

template <int D, int W> hipError_t draft_dispatch(const DraftArgs &a, hipStream_t s) {
  if (a.kv8) hipLaunchKernelGGL((k_draft<D, W, true>), dim3(a.n_wg), dim3(64 * W), 0, s, a);
  else hipLaunchKernelGGL((k_draft<D, W, false>), dim3(a.n_wg), dim3(64 * W), 0, s, a);
  return hipGetLastError();
}
template <int D> hipError_t draft_dispatch_rows(const DraftArgs &a, hipStream_t s) {
  switch (a.rows) {
  case 256: return draft_dispatch<D, 8>(a, s);
  case 128: return draft_dispatch<D, 4>(a, s);
  case 64: return draft_dispatch<D, 2>(a, s);
  default: return hipErrorInvalidValue;
  }
}
template <int D> hipError_t draft_merge_dispatch(const DraftArgs &a, hipStream_t s) {
  const dim3 grid(a.total * a.hq);
  // few rows: more waves for each, since they may be split over the whole chip
  if ((int64_t)a.total * a.hq <= 2048) hipLaunchKernelGGL((k_draft_merge<D, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_draft_merge<D, 1>), grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

} // namespace

hipError_t launch_draft(int d, const DraftArgs &a, hipStream_t s) {
  if (d == 128) return draft_dispatch_rows<128>(a, s);
  if (d == 64) return draft_dispatch_rows<64>(a, s);
  return hipErrorInvalidValue;
}

hipError_t launch_draft_merge(int d, const DraftArgs &a, hipStream_t s) {
  if (d == 128) return draft_merge_dispatch<128>(a, s);
  if (d == 64) return draft_merge_dispatch<64>(a, s);
  return hipErrorInvalidValue;
}

} // namespace sq
