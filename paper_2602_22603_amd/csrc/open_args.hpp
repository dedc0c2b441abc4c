// open_args.hpp - kernel arguments and launchers of tokens whose slots are taken
// before their K and V exist (open_kernels.hip): opening the slots, normed and
// rotated queries and keys, and keeping a drafted path.
// Internal to libsq.
#pragma once

#include "sq_common.hpp"

namespace sq {

constexpr int kMaxDraft = 64;        // drafted tokens of one sequence (one bit each in a 64-bit word)
constexpr int kOpenMaxUnits = 20480; // (entry, page) units of one opening

// The open tokens, by entry (sequence).  Entry e's tokens are tok0[e] ..
// tok0[e] + n[e] - 1 of the caller's rows and logical indices base[e] .. of its
// sequence.  Its pages are the units unit0[e] .. unit0[e + 1] - 1; there are as
// many as n[e] tokens touch from the worst first slot, so that launches depend
// on the counts alone, and a unit past the last page has page id -1.
struct OpenPlan {
  int32_t batch, total, n_units, pad;
  int32_t base[kMaxBatch];
  int32_t n[kMaxBatch];
  int32_t tok0[kMaxBatch];
  int32_t unit0[kMaxBatch + 4]; // [batch] = n_units
};
inline int32_t open_units(int64_t n) { return (int32_t)((n + 14) / kPage + 1); }

// Opens the slots: copies the segments (16-byte units) of the pinned blob to
// the device blob, writes the plan there, and for every unit its page-table
// entry and its tokens' positions pos0[e] + depth (depth: the token's place in
// the entry, or, drafted, what the pinned array says).
constexpr int kOpenSegs = 12;
struct OpenArgs {
  const char *src; // pinned
  char *dst;       // device, the same layout; the plan lies at offset 0
  int32_t n_segs, n16;             // segments, 16-byte units in all
  int32_t seg_off[kOpenSegs];      // byte offsets
  int32_t seg_n16[kOpenSegs];
  const int32_t *ids;              // pinned: page id of every unit
  const int32_t *depth;            // pinned: [total], or null
  int32_t *pt;
  int32_t *pos;
  int32_t max_pages;
  int32_t row[kMaxBatch];          // page-table row
  int32_t pos0[kMaxBatch];
  OpenPlan plan;
};
static_assert(sizeof(OpenArgs) < 4096, "open arguments too large");

// One layer's queries and keys, normed and rotated.  Stored form (plan not
// null): K and V of the open tokens into their slots.  Plain form: K to k_out.
struct QkArgs {
  const uint16_t *q, *k, *v;           // bf16 rows of [heads][D]
  int64_t q_stride, k_stride, v_stride; // elements from token to token
  uint16_t *q_out, *k_out;             // bf16 [n][heads][D]
  const int32_t *pos;                  // plain: [n]; stored: the position pool
  const float *inv_freq;               // [rot / 2], or null: no rotation
  const float *q_weight, *k_weight;    // [D], or null: no norm
  float eps, mscale;
  int32_t rot, interleaved;
  int32_t n, hq, hkv;
  int32_t its;                         // head iterations of one workgroup
  int32_t blocks;                      // workgroups of one unit
  const OpenPlan *plan;
  const int32_t *ids;                  // page id of every unit
  uint16_t *k_pool, *v_pool;           // the layer's
  int64_t page_stride, head_stride;
  float inv_k, inv_v;                  // 8-bit store: 1 / K and 1 / V scale
  int32_t kv8;
  int32_t n_units;
};

// Keeping a path of drafted nodes: token j of entry e's path (bit j-th set of
// mask[e]) moves to slot base + j, in every layer and head, and takes position
// pos0 + j.
struct AcceptArgs {
  int32_t n;
  int32_t max_pages;
  const int32_t *pt;
  uint64_t mask[kMaxBatch];
  int32_t row[kMaxBatch];
  int32_t base[kMaxBatch];
  int32_t pos0[kMaxBatch];
};
static_assert(sizeof(AcceptArgs) + sizeof(Pools) < 4096, "accept arguments too large");

hipError_t launch_open(const OpenArgs &a, hipStream_t s);
hipError_t launch_qk(int d, const QkArgs &a, hipStream_t s);
hipError_t launch_accept(const Pools &p, const AcceptArgs &a, hipStream_t s);

} // namespace sq
