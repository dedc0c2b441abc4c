// draft_plan.hpp - how the host lays out the attention of drafted trees: query rows
// per tile, what each node sees, and the tiles' key blocks dealt out to workgroups
// (the plan that draft_kernels.hip runs).  No GPU call in here.
// Internal to libsq.
#pragma once

#include <algorithm>
#include <cstdint>
#include <vector>

#include "draft_args.hpp"

namespace sq {

struct DraftModel {
  int hkv, G, D, cus; // KV heads, query heads of each, channels; compute units
  bool kv8;
};

// Depths of a tree's nodes; false for a parent that is no earlier node or -1.
inline bool tree_depths(const int32_t *parents, int32_t n, int32_t *depth) {
  for (int32_t i = 0; i < n; ++i) {
    if (parents[i] < -1 || parents[i] >= i) return false;
    depth[i] = parents[i] < 0 ? 0 : depth[parents[i]] + 1;
  }
  return true;
}

// How a draft's work is cut: query rows per workgroup, and workgroups of a launch
// (one round: two waves a SIMD, fewer where the LDS says so).  It follows from
// the counts alone, so that a captured layer replays for later drafts of the same
// counts.  A wave takes 32 rows, so the tile is the smallest that holds the
// largest tree's rows (nodes x heads of a KV head; more than 256 take several
// tiles), unless trees of both sides of 128 rows meet: small ones would leave most
// of an eight-wave workgroup idle, and a block takes it about as long with one
// wave at work as with eight.  Those run tiles of 128, the large trees several
// (12 trees of 5 to 61 nodes over 3K to 61K tokens of an 8-bit store: 303 us in
// tiles of 256, 246 in tiles of 128, 291 with a launch for each size of tree; 172
// now that an 8-bit store's tiles of up to 64 rows are streamed inside that launch
// and the runs are weighed as below).  For the same reason trees whose rows
// end in a small tile run tiles of 128 in an 8-bit store, by the measured times of a
// block: 60 for a full 256-row tile, 56 for a part, kBlock8 for 128 rows and less (8
// x 22673 tokens, 40 nodes 230 us in tiles of 256, 203 in tiles of 128, 64 nodes
// 257 and 275; a bf16 store 223 and 260, 271 and 280).
constexpr int kBlock8[5] = {0, 12, 18, 30, 32}; // 8-bit store, 128-row tiles, by waves at work
struct DraftShape {
  int32_t rows = 0, n_wg = 0, shared = 0;
};
inline DraftShape draft_shape(const DraftModel &s, const int32_t *counts, int32_t batch) {
  int32_t most = 0, least = INT32_MAX, by128 = 0, by256 = 0;
  for (int b = 0; b < batch; ++b) {
    const int32_t r = counts[b] * s.G;
    most = std::max(most, r);
    least = std::min(least, r);
    by128 += r / 128 * kBlock8[4] + kBlock8[(r % 128 + 31) / 32];
    by256 += r / 256 * 60 + (r % 256 ? 56 : 0);
  }
  DraftShape d;
  d.rows = most <= 64 ? 64 : least > 128 && !(s.kv8 && by128 < by256) ? 256 : 128;
  if (s.kv8 && most <= 64) d.rows = most <= 16 ? 16 : most <= 32 ? 32 : 64;
  d.shared = most > d.rows;
  const int per_cu = d.rows == 256 ? 1 : d.rows == 64 && s.D == 64 && !s.kv8 ? 3 : 2;
  d.n_wg = std::min<int32_t>(s.cus * per_cu, kDraftWgs);
  return d;
}

// The tiles of a draft, by the list of key blocks of one plan.
struct DraftTile {
  DraftPiece as; // every field but KV head, blocks, slot and next
  int64_t blocks;
};
// One sequence of a draft: n nodes behind `base` tokens, the first of them node tok0
// of all.
struct DraftEntry {
  int32_t row, n_pages;
  int64_t base;
  int32_t n, tok0, masked;
  const int32_t *parents, *depth; // its own nodes'
};
// Its nodes' words and its tiles, for the plan of every key and that of the window;
// returns the first key from a window's start on.
inline int64_t draft_entry(const DraftEntry &e, int32_t window, int32_t first, const DraftShape &shape, int G,
                           DraftNode *all, std::vector<DraftTile> *tiles) {
  const int64_t L = e.base + e.n, blocks = (L + kExtKeys - 1) / kExtKeys;
  DraftNode *nodes = all + e.tok0;
  for (int32_t i = 0; i < e.n; ++i) {
    DraftNode &nd = nodes[i];
    nd.anc[0] = (e.parents[i] < 0 ? 0 : nodes[e.parents[i]].anc[0]) | 1ull << i;
    nd.anc[1] = nd.anc[0];
    nd.lo = 0;
    if (window > 0) {
      const int64_t lo = e.base + e.depth[i] - window + 1; // first index of the window
      for (int32_t j = 0; j < i; ++j) {
        const int64_t at = e.base + e.depth[j];
        if (at < lo && at >= first) nd.anc[1] &= ~(1ull << j);
      }
      nd.lo = (int32_t)std::min(e.base, std::max<int64_t>(0, lo));
    }
  }
  int64_t lo_seq = L;
  const int32_t per_tile = shape.rows / G;
  for (int32_t i0 = 0; i0 < e.n; i0 += per_tile) {
    DraftTile t{};
    t.as.row = e.row;
    t.as.base = (int32_t)e.base;
    t.as.n = e.n;
    t.as.n_pages = e.n_pages;
    t.as.node0 = e.tok0 + i0;
    t.as.n_nodes = std::min<int32_t>(per_tile, e.n - i0);
    t.as.masked = e.masked;
    t.blocks = blocks;
    int32_t lo_min = INT32_MAX, lo_max = 0;
    for (int32_t i = 0; i < t.as.n_nodes; ++i) {
      DraftNode &nd = nodes[i0 + i];
      nd.tile = (int32_t)tiles[0].size();
      nd.in_tile = i;
      lo_min = std::min(lo_min, nd.lo);
      lo_max = std::max(lo_max, nd.lo);
    }
    tiles[0].push_back(t);
    // windowed: the first tokens' blocks, then those from the window's start
    const int32_t from = lo_min / kExtKeys;
    t.as.nf = std::min<int32_t>((int32_t)(((int64_t)first + kExtKeys - 1) / kExtKeys), from);
    t.as.skip = from - t.as.nf;
    t.as.lo_max = lo_max;
    t.blocks = blocks - t.as.skip;
    tiles[1].push_back(t);
    lo_seq = std::min<int64_t>(lo_seq, lo_min);
  }
  return lo_seq;
}

// The tiles' blocks (for every KV head) dealt out to the workgroups in runs of
// equal time: a block of a 128-row tile takes 20 with one wave at work, 23 with
// four (with 26 the mixed batches below took 1.5% longer); in an 8-bit store 12 and
// 18 where it is streamed (up to 32 and 64 rows), 30 and 32 where not; others about
// the same whatever the rows.  The start of a row takes a block, three of a full
// round of 128-row tiles (a piece more costs a workgroup 4 us at 64 channels, 8 at
// 128, timed by their clocks).
//
// Of such a round's two workgroups on a CU the first one's waves are older and
// issue first: with equal shares they ended at 130 us, the others at 164 (8-bit, 32
// nodes over 8 x 22673 tokens; 64 channels, 16 nodes: 86 and 113).  So the first
// get a fifth more and the others a fifth less: the 12 trees above 180 -> 172 us, 16
// windowed trees of 64 channels 54 -> 50.  128 channels of bf16 wait for HBM and end
// together (12 such trees 232 us so, 236 with a tenth), and so do tiles of up to 64
// rows (16 nodes over 8 x 22673 tokens 125 and 142).  Only for a full round: of
// fewer workgroups the index does not say which share a CU.  (That it says so of a
// full one is how the dispatcher hands workgroups out here; nothing but time
// depends on it.)
constexpr int64_t kEarly = 200; // of 1000
// A workgroup takes three blocks at least, one (of a 256-row tile two) while there
// is a CU for each: 12 nodes over 1000 tokens 20.3 us with three, 15.7 with one;
// past a workgroup a CU, 30 over 4 x 1500 tokens 27 with three, 33 with one.
constexpr int64_t kMinRun = 3;
inline int32_t draft_split(const std::vector<DraftTile> &tiles, const DraftModel &s, const DraftShape &shape,
                           DraftSplit *out) {
  const int hkv = s.hkv, G = s.G, D = s.D, cus = s.cus;
  const bool kv8 = s.kv8;
  auto weight = [&](const DraftTile &t) -> int64_t {
    const int waves = (t.as.n_nodes * G + 31) / 32;
    return shape.rows != 128 ? 20 : kv8 ? kBlock8[waves] : 20 + waves - 1;
  };
  int64_t blocks = 0;
  for (const DraftTile &t : tiles) blocks += t.blocks * hkv;
  // a workgroup leaves two partial tiles at most, and all together one each and
  // one for every row
  const int64_t most = (int64_t)kMaxItems * kRows / shape.rows;
  const int64_t fit = std::max(most / 2, most - (int64_t)tiles.size() * hkv);
  const int64_t runs = std::max(blocks / kMinRun, std::min<int64_t>(cus, blocks / (shape.rows == 256 ? 2 : 1)));
  const int64_t n = std::max<int64_t>(1, std::min<int64_t>({shape.n_wg, fit, runs}));
  const bool pairs = shape.rows == 128 && n == 2 * cus;
  const int64_t start = pairs ? 60 : 20; // of a row
  int64_t total = 0;
  for (const DraftTile &t : tiles) total += (t.blocks * weight(t) + start) * hkv;
  int32_t extra = (int32_t)n, slots = 0; // pieces behind the workgroups' first ones
  int64_t w = 0, at = 0;                 // the workgroup at `at`, and its last piece
  int32_t last = -1;
  const int64_t skew = pairs && (kv8 || D == 64) ? kEarly : 0;
  auto end_of = [&](int64_t x) {
    const int64_t early = std::min<int64_t>(x + 1, cus), late = x + 1 - early;
    return (early * (1000 + skew) + late * (1000 - skew)) * total / (1000 * n);
  };
  for (int64_t i = 0; i < n; ++i) {
    out->pieces[i] = DraftPiece{};
    out->pieces[i].next = -1; // (without blocks, unless it gets some below)
  }
  std::vector<int32_t> mine; // the row's pieces
  for (size_t t = 0; t < tiles.size(); ++t) {
    const int64_t wt = weight(tiles[t]), nb = tiles[t].blocks;
    for (int g = 0; g < hkv; ++g) {
      const int64_t stop = at + nb * wt + start;
      mine.clear();
      for (int64_t b = 0; b < nb;) {
        while (w + 1 < n && end_of(w) <= at) ++w, last = -1;
        const int64_t x = end_of(w);
        int64_t e = nb;
        if (x < stop && w + 1 < n) e = std::min(nb, std::max(b, (x - (stop - nb * wt - start) + wt / 2) / wt));
        if (e > b) {
          const int32_t p = last < 0 ? (int32_t)w : extra++;
          if (last >= 0) out->pieces[last].next = p;
          out->pieces[p] = tiles[t].as;
          out->pieces[p].g = g;
          out->pieces[p].b_lo = (int32_t)b;
          out->pieces[p].b_hi = (int32_t)e;
          out->pieces[p].slot = -1;
          out->pieces[p].next = -1;
          mine.push_back(p);
          last = p;
          b = e;
        }
        at = std::min(stop, x);
        if (b < nb) ++w, last = -1;
      }
      at = stop;
      const int32_t cnt = (int32_t)mine.size();
      out->merge[t * hkv + g] = {slots * shape.rows, cnt > 1 ? cnt : 0};
      if (cnt > 1)
        for (int32_t p : mine) out->pieces[p].slot = slots++ * shape.rows;
    }
  }
  out->n_used = (int32_t)n;
  out->rows = shape.rows;
  out->total = tiles.back().as.node0 + tiles.back().as.n_nodes;
  return extra;
}

} // namespace sq
