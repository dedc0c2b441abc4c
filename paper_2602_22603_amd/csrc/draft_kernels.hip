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
//
// Measured, one layer of 32 + 8 heads of 128 channels: 16 nodes over 8 x 128K tokens
// 631 us, 6.8 TB/s of K and V (HBM); 64 over 60547 tokens 98-100 us, 640 TFLOP/s
// useful (matrix and vector work one after the other; 16-bit weights take half as
// many products again); 5 over 2048 tokens 8.6 us and the merge 3.5 (a chain of
// reads).
//
// A weight is held as two bf16 halves, 16 bits, since the products take bf16: an
// output is 2e-6 to 3e-6 off float64 in the 2-norm, where fp32 weights would be 3e-7
// (a short cache) to 4e-6 (128K tokens) off and one half 1e-3; a third part would
// cost another product of every weight and value.
#include "attn_tile.hpp"
#include "draft_args.hpp"
#include "page_frags.hpp"

namespace sq {
namespace {

// A piece, by scalar loads.
struct PieceRef {
  int32_t g, row, base, n, n_pages, node0, n_nodes, masked, nf, skip, lo_max, b_lo, b_hi, slot, next;
  __device__ PieceRef(const DraftPiece &p) {
    const ext_sptr_t x = (ext_sptr_t)&p;
    g = x[0], row = x[1], base = x[2], n = x[3], n_pages = x[4], node0 = x[5], n_nodes = x[6], masked = x[7];
    nf = x[8], skip = x[9], lo_max = x[10], b_lo = x[11], b_hi = x[12], slot = x[13], next = x[14];
  }
};

// Whether a launch was laid out for this plan: the rows of its tiles and the nodes
// of q and out.  (A captured one may be replayed while another draft is open: its
// partial rows would lie past the workspace, its nodes past q and out.)
__device__ inline bool fits(const DraftArgs &a, const DraftSplit &sp) {
  const ext_sptr_t x = (ext_sptr_t)&sp.n_used;
  return (int)blockIdx.x < x[0] && x[1] == a.rows && x[2] == a.total;
}

// The pages of one sequence.
struct SeqPages {
  const int32_t *pt;
  int32_t n_pages;
  int64_t page_stride;
};

// ---------------------------------------------------------------------------
// The streaming form, for an 8-bit store and few rows: K and V go straight from
// the pools to matrix-core operands in registers, with no LDS and no barrier
// between a wave and its pages (the tiled form would pass the codes through
// registers, LDS and a barrier: 4 nodes over 4 x 128K tokens 298 us, 211 so).  A
// workgroup of 4 waves takes RG groups of 16 CG query rows against a piece's
// keys; the 4 / RG waves of a row group take contiguous shares of the keys and
// join their states in LDS at the end.  A step is a chunk of 32 keys (two
// pages): S^T of page h (16 keys) lands with keys 4 kg + i in lane group kg,
// which are slots (kg, 4 h + i) of the P^T operand, and the two pages' V^T
// fragments side by side are the same slots of the V^T operand, so one
// 16x16x32 product takes both pages.  PF chunks of K and V are in flight per
// wave: chunk c + PF's K is loaded as soon as chunk c's scores are taken, its V
// after the products.
template <int WR> struct StreamLds {
  float (*m)[WR], (*l)[WR]; // by wave: its rows' maxima and sums
  uint64_t *anc;            // what the tile's nodes see
  int32_t *lo;
};
// The waves' accumulators: rows of D + 4 floats,
template <int D, int WR> struct PaddedRows {
  float *base;
  __device__ float *at(int wave, int row, int d) const { return base + (wave * WR + row) * (D + 4) + d; }
};
// or in four buffers of a tile, D floats a row, chunk c of row r at c ^ r.
template <int D> struct SwizzledRows {
  float *a0, *a1, *a2, *a3;
  __device__ float *at(int wave, int row, int d) const {
    float *p = wave == 0 ? a0 : wave == 1 ? a1 : wave == 2 ? a2 : a3;
    return p + row * D + (((d >> 2) ^ row) & (D / 4 - 1)) * 4;
  }
};

template <int D, int CG, int RG, class Rows>
__device__ inline void stream_piece(const DraftArgs &a, const PieceRef &pc, const StreamLds<16 * CG> &lds,
                                    const Rows &states) {
  constexpr int NKC = D / 32, NDT = D / 16, KG = 4 / RG, PF = 2;
  constexpr int WR = 16 * CG;        // rows of a wave
  constexpr int kPageBytes = kPage * D;
  constexpr bool NT = RG == 1;       // read by one wave: past the caches
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, kg = lane >> 4;
  const int rg = wave % RG, kpart = wave / RG;
  const int plan = a.windowed;
  const int g = pc.g, base = pc.base, n_draft = pc.n, n_pages = pc.n_pages, node0 = pc.node0;
  const int n_nodes = pc.n_nodes;
  const int masked = pc.masked, nf = pc.nf, skip = pc.skip, lo_max = pc.lo_max, b_lo = pc.b_lo, b_hi = pc.b_hi;
  const int slot = pc.slot, pt_row = pc.row;
  const int L = base + n_draft;
  const ext_sptr_t pt = (ext_sptr_t)(a.pt + (int64_t)pt_row * a.max_pages);
  const ext_sptr_t mask_row = (ext_sptr_t)(a.mask + (int64_t)pt_row * a.max_pages);
  const char *khead = reinterpret_cast<const char *>(a.k) + (int64_t)g * a.head_stride;
  const char *vhead = reinterpret_cast<const char *>(a.v) + (int64_t)g * a.head_stride;
  const int koff = n * D + 16 * kg, voff = (16 * kg + n) * kPage;

  __syncthreads(); // the piece before is done with the LDS
  if (tid < n_nodes) {
    lds.anc[tid] = a.blob->nodes[node0 + tid].anc[plan];
    lds.lo[tid] = a.blob->nodes[node0 + tid].lo;
  }
  __syncthreads();
  const int rows = n_nodes << a.lg;
  auto node_of = [&](int cg) { return (WR * rg + 16 * cg + n) >> a.lg; }; // in the tile
  auto head_of = [&](int cg) { return (g << a.lg) + ((WR * rg + 16 * cg + n) & ((1 << a.lg) - 1)); };
  bf16x8_t qf[CG][NKC];
#pragma unroll
  for (int cg = 0; cg < CG; ++cg) {
    const bool live = node_of(cg) < n_nodes;
    const uint16_t *qp = a.q + ((int64_t)(node0 + node_of(cg)) * a.hq + head_of(cg)) * D;
#pragma unroll
    for (int kc = 0; kc < NKC; ++kc) {
      const int c0 = 16 * kg + 64 * (kc >> 1) + 8 * (kc & 1); // the channels that the K fragments hold
      qf[cg][kc] = __builtin_bit_cast(bf16x8_t, live ? *reinterpret_cast<const uint4 *>(qp + c0)
                                                     : make_uint4(0, 0, 0, 0));
    }
  }
  f32x4_t acc[NDT][CG];
  float m_run[CG], l_run[CG];
#pragma unroll
  for (int cg = 0; cg < CG; ++cg) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) acc[dt][cg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m_run[cg] = kNegInf;
    l_run[cg] = 0.f;
  }

  // this wave's chunks [c_lo, c_hi) of the piece's; the last block may end in
  // its first chunk
  auto key_of = [&](int c) {
    const int i = b_lo + (c >> 1);
    return (i < nf ? i : i + skip) * BK + 32 * (c & 1);
  };
  int total = 2 * (b_hi - b_lo);
  if (key_of(total - 1) >= L) --total;
  const int c_lo = WR * rg < rows ? total * kpart / KG : 0; // a row group without rows: nothing
  const int c_hi = WR * rg < rows ? total * (kpart + 1) / KG : 0;
  KFrag8<D> kf[PF][2];
  VFrag8<D> vf[PF][2];
  int nid[PF][2]; // page ids of the chunks to be loaded next
  auto ids_of = [&](int c, int (&id)[2]) {
    const int p0 = key_of(min(c, max(c_hi - 1, 0))) / kPage;
    id[0] = pt[min(p0, n_pages - 1)];
    id[1] = pt[min(p0 + 1, n_pages - 1)];
  };
  auto rsrc = [&](const char *head, int id, bool want) {
    return page_rsrc(head + (int64_t)(want ? id : 0) * kPageBytes, want, kPageBytes);
  };
  if (c_lo < c_hi) {
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      ids_of(c_lo + u, nid[u]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load_k<D, NT>(kf[u][h], rsrc(khead, nid[u][h], c_lo + u < c_hi), koff);
        load_v<D, NT>(vf[u][h], rsrc(vhead, nid[u][h], c_lo + u < c_hi), voff);
      }
    }
#pragma unroll
    for (int u = 0; u < PF; ++u) ids_of(c_lo + PF + u, nid[u]);
  }
  const uint32_t m1l = minus_one(0), m1h = minus_one(1);
  for (int c0 = c_lo; c0 < c_hi; c0 += PF) {
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      const int c = c0 + u;
      const int k0 = key_of(c);
      const bool in = c < c_hi; // a chunk past the share: zeros, and no key seen
      f32x4_t st[2][CG];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const KFrag<D> kb = to_bf16(kf[u][h]);
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) st[h][cg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < NKC; ++kc)
#pragma unroll
          for (int cg = 0; cg < CG; ++cg)
            st[h][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kb.k[kc]), qf[cg][kc],
                                                                st[h][cg], 0, 0, 0);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) load_k<D, NT>(kf[u][h], rsrc(khead, nid[u][h], c + PF < c_hi), koff);
      // keep bits of the chunk's keys (deferred evictions)
      uint32_t keep = ~0u;
      if (masked) {
        const int p0 = k0 / kPage, last = n_pages - 1;
        keep = (uint32_t)mask_row[min(p0, last)] | (uint32_t)mask_row[min(p0 + 1, last)] << 16;
      }
      if (!in || k0 + 32 > base || (plan && k0 < lo_max && k0 + 32 > a.first) || keep != ~0u) {
        const uint64_t cache = ~ones_from(base - k0), early = ~ones_from(a.first - k0);
        const int off = base - k0; // place of node 0
        int here = n, part = kg; // (their own copies: nothing of this is to be held through the loop)
        asm("" : "+v"(here), "+v"(part));
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) {
          // a row past the nodes sees every key, so that it never has to look
          // for a first one
          const int i = (WR * rg + 16 * cg + here) >> a.lg;
          const uint64_t anc = i < n_nodes ? lds.anc[i] : ~0ull >> (64 - n_draft);
          uint64_t w = cache;
          if (plan && i < n_nodes) w &= ones_from(lds.lo[i] - k0) | early;
          if (off > -64 && off < 64) w |= off >= 0 ? anc << off : anc >> -off;
          const uint32_t w32 = in ? (uint32_t)w & keep : 0u;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!((w32 >> (16 * h + 4 * part + e)) & 1)) st[h][cg][e] = kNegInf;
        }
      }
      bf16x8_t phi[CG], plo[CG];
      float psum[CG];
      for (bool raised = false;; raised = true) {
        bool ok = true;
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) {
          const float nm = m_run[cg] == kNegInf ? 0.f : -m_run[cg];
          uint32_t hi[4], lw[4];
          psum[cg] = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p0 = exp2_fast(fmaf(st[e >> 1][cg][2 * (e & 1)], a.scale_log2, nm));
            const float p1 = exp2_fast(fmaf(st[e >> 1][cg][2 * (e & 1) + 1], a.scale_log2, nm));
            hi[e] = pack_bf16(p0, p1);
            lw[e] = pack_bf16(residue(hi[e], m1l, p0), residue(hi[e], m1h, p1));
            psum[cg] += p0 + p1;
          }
          phi[cg] = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
          plo[cg] = __builtin_bit_cast(bf16x8_t, make_uint4(lw[0], lw[1], lw[2], lw[3]));
          ok = ok && m_run[cg] != kNegInf && psum[cg] < kBig;
        }
        if (raised || __all(ok)) break;
        // raise the references to this chunk's maxima and take the weights again
        float alpha[CG];
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) {
          float mx = fmaxf(fmaxf(fmaxf(st[0][cg][0], st[0][cg][1]), fmaxf(st[0][cg][2], st[0][cg][3])),
                           fmaxf(fmaxf(st[1][cg][0], st[1][cg][1]), fmaxf(st[1][cg][2], st[1][cg][3])));
          mx = max_xrow16(mx);
          mx = max_xrow32(mx) * a.scale_log2;
          const float m_new = fmaxf(m_run[cg], mx);
          alpha[cg] = m_new == m_run[cg] ? 1.f : exp2_fast(m_run[cg] - m_new); // 0 from -inf
          m_run[cg] = m_new;
          l_run[cg] *= alpha[cg];
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int cg = 0; cg < CG; ++cg) acc[dt][cg] *= alpha[cg];
      }
#pragma unroll
      for (int cg = 0; cg < CG; ++cg) l_run[cg] += psum[cg];
      const VFrag<D> v0 = to_bf16(vf[u][0]), v1 = to_bf16(vf[u][1]);
      uint4 va[NDT];
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) va[dt] = make_uint4(v0.v[dt].x, v0.v[dt].y, v1.v[dt].x, v1.v[dt].y);
      if (k0 + 32 > L) { // slots that hold no token may hold anything: keep 0 * v finite
        uint32_t m[4];
        int part = kg;
        asm("" : "+v"(part));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = k0 + 16 * (e >> 1) + 4 * part + 2 * (e & 1);
          m[e] = (k < L ? 0xffffu : 0u) | (k + 1 < L ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
          va[dt] = make_uint4(va[dt].x & m[0], va[dt].y & m[1], va[dt].z & m[2], va[dt].w & m[3]);
      }
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int cg = 0; cg < CG; ++cg)
          acc[dt][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, va[dt]), phi[cg],
                                                                acc[dt][cg], 0, 0, 0);
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int cg = 0; cg < CG; ++cg)
          acc[dt][cg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, va[dt]), plo[cg],
                                                                acc[dt][cg], 0, 0, 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) load_v<D, NT>(vf[u][h], rsrc(vhead, nid[u][h], c + PF < c_hi), voff);
    }
#pragma unroll
    for (int u = 0; u < PF; ++u) ids_of(c0 + 2 * PF + u, nid[u]);
  }

  // The rows' states: of the row group's waves, joined (M = max m, out = sum
  // 2^(m - M) acc), or this wave's own.
  auto finish = [&](int r, float l, float m, float *sc) { // row r of the tile to the output
    *sc = 1.f;
    if (a.sinks) { // one more term of the sum, no value
      const float sk_l2 = a.sinks[(g << a.lg) + (r & ((1 << a.lg) - 1))] * a.sink_scale;
      const float big = fmaxf(m, sk_l2);
      *sc = exp2_fast(m - big);
      l = fmaf(l, *sc, exp2_fast(sk_l2 - big));
    }
    *sc = *sc / l * a.out_scale;
    return a.out + ((int64_t)(node0 + (r >> a.lg)) * a.hq + (g << a.lg) + (r & ((1 << a.lg) - 1))) * D;
  };
  int tx = tid; // read again, so that no address below is held through the loop
  asm("" : "+v"(tx));
  const int en = tx & 15, ek = (tx >> 4) & 3;
#pragma unroll
  for (int cg = 0; cg < CG; ++cg) {
    float l = sum_xrow16(l_run[cg]);
    l = sum_xrow32(l);
    if (ek == 0) {
      lds.m[wave][16 * cg + en] = m_run[cg];
      lds.l[wave][16 * cg + en] = l;
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
      *reinterpret_cast<float4 *>(states.at(wave, 16 * cg + en, 16 * dt + 4 * ek)) =
          make_float4(acc[dt][cg][0], acc[dt][cg][1], acc[dt][cg][2], acc[dt][cg][3]);
  }
  __syncthreads();
  for (int e = tx * 4; e < rows * D; e += 1024) {
    const int r = e / D, d = e % D, rw = r % WR, w0 = r / WR;
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int q = 0; q < KG; ++q) m = fmaxf(m, lds.m[w0 + RG * q][rw]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < KG; ++q) {
      const int w = w0 + RG * q;
      const float sc = m == kNegInf ? 0.f : exp2_fast(lds.m[w][rw] - m);
      l = fmaf(sc, lds.l[w][rw], l);
      const float4 x = *reinterpret_cast<const float4 *>(states.at(w, rw, d));
      o.x = fmaf(sc, x.x, o.x);
      o.y = fmaf(sc, x.y, o.y);
      o.z = fmaf(sc, x.z, o.z);
      o.w = fmaf(sc, x.w, o.w);
    }
    if (slot >= 0) {
      const int64_t pr = slot + r;
      if (d == 0) {
        a.part_m[pr] = m;
        a.part_l[pr] = l;
      }
      *reinterpret_cast<float4 *>(a.part_acc + pr * D + d) = o;
    } else {
      float sc;
      float *op = finish(r, l, m, &sc);
      *reinterpret_cast<float4 *>(op + d) = make_float4(o.x * sc, o.y * sc, o.z * sc, o.w * sc);
    }
  }
}

template <int D, int CG, int RG>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void
k_draft_stream(DraftArgs a) {
  constexpr int WR = 16 * CG;
  __shared__ float s_m[4][WR], s_l[4][WR];
  __shared__ __attribute__((aligned(16))) float s_acc[4 * WR * (D + 4)];
  __shared__ uint64_t s_anc[kMaxDraft];
  __shared__ int32_t s_lo[kMaxDraft];
  const DraftSplit &sp = a.blob->split[a.windowed];
  if (!fits(a, sp)) return;
  int next = blockIdx.x;
  while (next >= 0) {
    const PieceRef pc(sp.pieces[next]);
    next = pc.next;
    if (pc.b_lo >= pc.b_hi) continue; // (a workgroup without work)
    stream_piece<D, CG, RG>(a, pc, StreamLds<WR>{s_m, s_l, s_anc, s_lo}, PaddedRows<D, WR>{s_acc});
  }
}

// ---------------------------------------------------------------------------
// NT: each key is read by one workgroup, past the caches (64 query rows over 4 x
// 128K tokens: 372 us with temporal copies, 328 so).
template <int D, int W, bool KV8, bool NT>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(kExtWavesPerEu, kExtWavesPerEu))) void
k_draft(DraftArgs a) {
  using Lt = ExtLayout<D, W>;
  constexpr int NKC = D / 32;
  constexpr int NDT = D / 16;
  constexpr int NB = Lt::NB;
  constexpr int AUX = NT ? 2 : 0;
  // block buffers as separate LDS objects, the block loop unrolled over them:
  // see k_extend
  __shared__ __attribute__((aligned(16))) uint16_t sk0[Lt::K_ELEMS], sk1[Lt::K_ELEMS], sk2[NB > 2 ? Lt::K_ELEMS : 8];
  __shared__ __attribute__((aligned(16))) uint16_t sv0[Lt::V_ELEMS], sv1[Lt::V_ELEMS], sv2[NB > 2 ? Lt::V_ELEMS : 8];
  // what the tile's nodes see (read for the few blocks that need a test; in
  // registers it made the 256-row kernel spill)
  __shared__ uint64_t s_anc[kMaxDraft];
  __shared__ int32_t s_lo[kMaxDraft];
  constexpr bool kSmall = KV8 && W == 4; // tiles of up to 64 rows in the streaming form
  __shared__ float s_m[kSmall ? 4 : 1][32], s_l[kSmall ? 4 : 1][32];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, kg = lane >> 4;
  const int plan = a.windowed;
  const DraftSplit &sp = a.blob->split[plan];
  if (!fits(a, sp)) return;
  int next = blockIdx.x;
  while (next >= 0) {
    const PieceRef pc(sp.pieces[next]);
    const int g = pc.g, base = pc.base, n_draft = pc.n, n_pages = pc.n_pages, node0 = pc.node0;
    const int n_nodes = pc.n_nodes;
    const int masked = pc.masked, nf = pc.nf, skip = pc.skip, lo_max = pc.lo_max, b_lo = pc.b_lo, b_hi = pc.b_hi;
    const int slot = pc.slot, pt_row = pc.row;
    next = pc.next;
    if (b_lo >= b_hi) continue; // (a workgroup without work)
    if constexpr (kSmall) { // (12 mixed trees 298 us without, 172 with)
      static_assert(Lt::K_ELEMS * 2 >= 32 * D * 4 && Lt::V_ELEMS * 2 >= 32 * D * 4, "a wave's accumulator in each");
      const StreamLds<32> lds{s_m, s_l, s_anc, s_lo};
      const SwizzledRows<D> states{reinterpret_cast<float *>(sk0), reinterpret_cast<float *>(sk1),
                                   reinterpret_cast<float *>(sv0), reinterpret_cast<float *>(sv1)};
      const int rows = n_nodes << a.lg;
      if (rows <= 32) stream_piece<D, 2, 1>(a, pc, lds, states);
      else if (rows <= 64) stream_piece<D, 2, 2>(a, pc, lds, states);
      if (rows <= 64) continue;
    }
    const int L = base + n_draft;
    const SeqPages pg{a.pt + (int64_t)pt_row * a.max_pages, n_pages, kPage * D};
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
      ext_dma<D, W, AUX>(sk0, sv0, pg, kbase, vbase, ids, wave, lane);
      __builtin_amdgcn_s_waitcnt(kVmcntKeep<Lt::NK + Lt::NV>); // the query loads have landed
      if constexpr (NB > 2) {
        block_ids(ids, pg, at(b_lo + 1));
        ext_dma<D, W, AUX>(sk1, sv1, pg, kbase, vbase, ids, wave, lane);
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
        if constexpr (NB > 2) ext_dma<D, W, AUX>(n2k, n2v, pg, kbase, vbase, ids, wave, lane);
        else ext_dma<D, W, AUX>(n1k, n1v, pg, kbase, vbase, ids, wave, lane);
      }
      int seen[2] = {0, 0};
      if (need) {
        const uint64_t cache = ~ones_from(base - k0); // keys of the cache
        const uint64_t early = ~ones_from(a.first - k0);
        const int off = base - k0; // place of node 0
        int here = n; // (its own copy: nothing of this is to be held through the loop)
        asm("" : "+v"(here));
#pragma unroll
        for (int cg = 0; cg < 2; ++cg) {
          // a row past the nodes sees every key, so that it never has to look
          // for a first one
          const int i = (32 * wave + 16 * cg + here) >> a.lg;
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
      if (wave_live)
        ext_block<D, true>(ck, cv, 0, n, kg, a.scale_log2, need, qf, none, seen, 0, acc, m_run, l_run, next_ids);
      else
        next_ids();
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

    int tx = lane; // read again, so that no address below is held through the loop
    asm("" : "+v"(tx));
    const int n = tx & 15, kg = tx >> 4;
#pragma unroll
    for (int cg = 0; cg < 2; ++cg) {
      float l = sum_xrow16(l_run[cg]);
      l = sum_xrow32(l);
      const int r0 = 32 * wave + 16 * cg + n, nd = r0 >> a.lg, head = (g << a.lg) + (r0 & ((1 << a.lg) - 1));
      if (nd >= n_nodes) continue;
      if (slot >= 0) { // a part of the row's keys
        const int64_t r = slot + r0;
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
        const float sk_l2 = a.sinks[head] * a.sink_scale;
        const float big = fmaxf(m_run[cg], sk_l2);
        sc = exp2_fast(m_run[cg] - big);
        l = fmaf(l, sc, exp2_fast(sk_l2 - big));
      }
      const float inv = sc / l * a.out_scale;
      float *op = a.out + ((int64_t)(node0 + nd) * a.hq + head) * D + 4 * kg;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
        *reinterpret_cast<float4 *>(op + 16 * dt) = make_float4(acc[dt][cg][0] * inv, acc[dt][cg][1] * inv,
                                                                acc[dt][cg][2] * inv, acc[dt][cg][3] * inv);
    }
  }
}

// The rows whose keys were split: M = max m_s, out = sum 2^(m_s - M) acc_s / sum
// 2^(m_s - M) l_s.  D / 4 lanes take a (node, head)'s slots, four channels each, a
// workgroup 1024 / D of them; or, SHARED, all of a workgroup's lane groups take
// shares of one row's slots, for few rows whose keys were split over the chip.
// Bound by the partial rows it reads (64 nodes over 60547 tokens: 34 MB, 7.5 us)
// and, below some MB, by a chain of four loads (3.5 us).  With a wave to a row, 13760
// rows of 64 channels took 6.9 us, 5.8 so.
template <int D, bool SHARED>
__global__ __launch_bounds__(256) void k_draft_merge(DraftArgs a) {
  constexpr int L = D / 4, GROUPS = 256 / L, SH = SHARED ? GROUPS : 1;
  constexpr int U = SHARED ? 4 : 8;
  __shared__ float s_m[GROUPS], s_l[GROUPS];
  __shared__ __attribute__((aligned(16))) float s_acc[SHARED ? GROUPS : 1][D];
  const int lane = threadIdx.x % L, group = threadIdx.x / L, share = SHARED ? group : 0;
  const int r = SHARED ? blockIdx.x : blockIdx.x * GROUPS + group;
  const bool live = r < a.total * a.hq;
  const int i = live ? r / a.hq : 0, h = live ? r % a.hq : 0;
  const int tile = a.blob->nodes[i].tile, in_tile = a.blob->nodes[i].in_tile;
  const int g = h >> a.lg;
  const DraftSplit &sp = a.blob->split[a.windowed];
  const ext_sptr_t plan = (ext_sptr_t)&sp.n_used;
  const bool fit = plan[1] == a.rows && plan[2] == a.total;
  const DraftMerge mr = sp.merge[tile * a.hkv + g]; // (of another draft's plan at worst)
  if (!live || !fit || mr.n == 0) return; // (SHARED: the whole workgroup)
  const int col = (in_tile << a.lg) + (h & ((1 << a.lg) - 1));
  float big = kNegInf, den = 0.f;
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
  auto scale = [](float4 x, float w) { return make_float4(x.x * w, x.y * w, x.z * w, x.w * w); };
  auto add = [](float4 s, float4 x, float w) {
    return make_float4(fmaf(w, x.x, s.x), fmaf(w, x.y, s.y), fmaf(w, x.z, s.z), fmaf(w, x.w, s.w));
  };
  for (int s0 = share * U; s0 < mr.n; s0 += SH * U) {
    float4 x[U];
    float m[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = mr.row0 + (int64_t)min(s0 + u, mr.n - 1) * a.rows + col;
      m[u] = s0 + u < mr.n ? a.part_m[at] : kNegInf;
      l[u] = a.part_l[at];
      x[u] = reinterpret_cast<const float4 *>(a.part_acc + at * D)[lane];
    }
    float top = big;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, m[u]);
    if (top == kNegInf) continue;
    const float sc = exp2_fast(big - top);
    den *= sc;
    num = scale(num, sc);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = exp2_fast(m[u] - top);
      den = fmaf(w, l[u], den);
      num = add(num, x[u], w);
    }
    big = top;
  }
  if constexpr (SHARED) {
    if (lane == 0) {
      s_m[group] = big;
      s_l[group] = den;
    }
    reinterpret_cast<float4 *>(s_acc[group])[lane] = num;
    __syncthreads();
    if (group != 0) return;
    float top = kNegInf;
#pragma unroll
    for (int w = 0; w < GROUPS; ++w) top = fmaxf(top, s_m[w]);
    den = 0.f;
    num = make_float4(0.f, 0.f, 0.f, 0.f);
    big = top;
    if (top != kNegInf) {
#pragma unroll
      for (int w = 0; w < GROUPS; ++w) {
        const float sc = exp2_fast(s_m[w] - top);
        den = fmaf(sc, s_l[w], den);
        num = add(num, reinterpret_cast<const float4 *>(s_acc[w])[lane], sc);
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
  reinterpret_cast<float4 *>(a.out + ((int64_t)i * a.hq + h) * D)[lane] = scale(num, sc);
}

template <int D, int W> hipError_t tile_dispatch(const DraftArgs &a, hipStream_t s) {
  const dim3 grid(a.n_wg), block(64 * W);
  if constexpr (W > 2) {
    if (a.kv8) hipLaunchKernelGGL((k_draft<D, W, true, false>), grid, block, 0, s, a);
    else if (a.shared) hipLaunchKernelGGL((k_draft<D, W, false, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_draft<D, W, false, true>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((k_draft<D, W, false, true>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}
template <int D, int CG, int RG> hipError_t stream_dispatch(const DraftArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((k_draft_stream<D, CG, RG>), dim3(a.n_wg), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int D> hipError_t draft_dispatch(const DraftArgs &a, hipStream_t s) {
  switch (a.rows) {
  case 256: return tile_dispatch<D, 8>(a, s);
  case 128: return tile_dispatch<D, 4>(a, s);
  case 64: return a.kv8 ? stream_dispatch<D, 2, 2>(a, s) : tile_dispatch<D, 2>(a, s);
  case 32: return a.kv8 ? stream_dispatch<D, 2, 1>(a, s) : hipErrorInvalidValue;
  case 16: return a.kv8 ? stream_dispatch<D, 1, 1>(a, s) : hipErrorInvalidValue;
  default: return hipErrorInvalidValue;
  }
}
template <int D> hipError_t draft_merge_dispatch(const DraftArgs &a, hipStream_t s) {
  const int64_t rows = (int64_t)a.total * a.hq;
  constexpr int per_wg = 1024 / D;
  if (rows <= 2048) hipLaunchKernelGGL((k_draft_merge<D, true>), dim3(rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_draft_merge<D, false>), dim3((rows + per_wg - 1) / per_wg), dim3(256), 0, s, a);
  return hipGetLastError();
}

} // namespace

hipError_t launch_draft(int d, const DraftArgs &a, hipStream_t s) {
  if (d == 128) return draft_dispatch<128>(a, s);
  if (d == 64) return draft_dispatch<64>(a, s);
  return hipErrorInvalidValue;
}

hipError_t launch_draft_merge(int d, const DraftArgs &a, hipStream_t s) {
  if (d == 128) return draft_merge_dispatch<128>(a, s);
  if (d == 64) return draft_merge_dispatch<64>(a, s);
  return hipErrorInvalidValue;
}

} // namespace sq
