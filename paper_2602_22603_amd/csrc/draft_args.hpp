// draft_args.hpp - plan, kernel arguments and launchers of the attention of
// drafted tokens (draft_kernels.hip).
// Internal to libsq.
#pragma once

#include "extend_args.hpp"
#include "open_args.hpp"

#include <cstddef>

namespace sq {

// What a node sees: of the draft the nodes of anc (bit i: node i), of the cache
// the tokens from lo on and, in the windowed plan, the first tokens.
struct DraftNode {
  uint64_t anc[2]; // full plan, windowed plan
  int32_t lo;      // windowed plan
  int32_t tile;    // its tile, and its place in it
  int32_t in_tile;
  int32_t pad;
};
// A tile is up to rows / G nodes of one sequence with the G query heads of a KV
// head; a row of the plan is (tile, KV head).  Its keys are a list of blocks of
// 64: of a windowed plan the blocks of the first tokens, then (from place nf on)
// those from the window's start, `skip` blocks later.  A piece is a run of one
// row's blocks, for one workgroup: with all that the workgroup has to know, so
// that it starts after one load.  Workgroup w's first piece is piece w.
struct DraftPiece {
  int32_t g;          // KV head
  int32_t row;        // page-table row
  int32_t base;       // tokens in front of the draft
  int32_t n;          // nodes of the sequence
  int32_t n_pages;
  int32_t node0;      // first node of the tile, among all
  int32_t n_nodes;    // nodes of the tile
  int32_t masked;     // the sequence has slots masked by deferred evictions
  int32_t nf, skip;
  int32_t lo_max;     // where the last node's window starts
  int32_t b_lo, b_hi; // places in the list
  int32_t slot;       // first partial row of a part of the blocks, or -1: to the output
  int32_t next;       // the workgroup's next piece, or -1
  int32_t pad;
};
// The partial rows of a row's n pieces, one tile's rows apart (n = 0: written by
// its one piece).
struct DraftMerge {
  int32_t row0, n;
};

constexpr int kDraftRows = 4096; // (tile, KV head) rows
constexpr int kDraftWgs = 1024;  // workgroups of a launch
// A captured launch has its tile and its number of nodes from the draft it was
// captured with; where the plan's are others it does nothing.
struct DraftSplit {
  int32_t n_used;                // workgroups that have work (0: no such plan)
  int32_t rows, total;           // query rows of a tile, nodes in all
  int32_t pad;
  DraftMerge merge[kDraftRows];
  DraftPiece pieces[kDraftRows + kDraftWgs];
};
// The blob in device memory (and, pinned, on the host), uploaded in the parts
// that are used.
struct OpenBlob {
  OpenPlan plan;
  int32_t ids[kOpenMaxUnits];
  int32_t depth[kMaxBatch * kMaxDraft];
  DraftNode nodes[kMaxBatch * kMaxDraft];
  DraftSplit split[2]; // every key; a window
};
static_assert(sizeof(OpenPlan) % 16 == 0 && offsetof(OpenBlob, ids) % 16 == 0 && offsetof(OpenBlob, depth) % 16 == 0 &&
                  offsetof(OpenBlob, nodes) % 16 == 0 && offsetof(OpenBlob, split) % 16 == 0 &&
                  sizeof(DraftSplit) % 16 == 0 && offsetof(DraftSplit, merge) % 16 == 0 &&
                  offsetof(DraftSplit, pieces) % 16 == 0,
              "uploaded as 16-byte units");

struct DraftArgs {
  const uint16_t *q; // bf16 [total][Hq][D]
  const uint16_t *k; // K pool of the layer
  const uint16_t *v;
  float *out;        // fp32 [total][Hq][D]
  const int32_t *pt;
  const int32_t *mask;
  int64_t head_stride;
  int32_t max_pages;
  int32_t hq, hkv;
  int32_t lg;        // log2 of G
  int32_t total;     // nodes
  float scale_log2;
  const float *sinks;
  float sink_scale;
  float out_scale;
  float *part_m, *part_l, *part_acc; // [partial rows], acc [partial rows][D]
  const OpenBlob *blob;
  int32_t windowed;  // which plan
  int32_t first;     // first tokens beside the window
  int32_t rows;      // query rows per workgroup: 256, 128 or 64 (8-bit stores also 32 or 16)
  int32_t n_wg;
  int32_t shared;    // a sequence may have several tiles, which read the same keys
  int32_t kv8;
};
static_assert(sizeof(DraftArgs) < 4096, "draft kernel arguments too large");

hipError_t launch_draft(int d, const DraftArgs &a, hipStream_t s);
hipError_t launch_draft_merge(int d, const DraftArgs &a, hipStream_t s);

} // namespace sq
