// The host's batch plan and argument checks, shared by the files that
// implement the C ABI's handles.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <string>
#include <vector>

#include "../../include/rosa.h"
#include "rosa_internal.h"

namespace rosa {

struct Plan {
  std::vector<int32_t> order;        // plan position -> caller index
  std::vector<int32_t> tok_off;      // by plan position
  std::vector<int32_t> steps;        // by plan position: Euler steps this call runs
  std::vector<int32_t> m_k;          // per step
  std::vector<int32_t> n_active;     // per step
  std::vector<float> taus;
  std::vector<int32_t> tau_idx;      // [max_K][n]
  // Attention work: set 0 serves joint (or, alternating, cross-attention)
  // layers, set 1 the self-attention layers of the alternating layout.  The
  // device holds set 0's items then set 1's (likewise groups); launch orders
  // index the whole item array; partial slots are numbered across both sets.
  struct AttnSet {
    std::vector<AttnItem> items;
    std::vector<AttnGroup> groups;
    std::vector<int32_t> items_upto;   // items of plan requests [0, r]
    std::vector<int32_t> groups_upto;
    int item_base = 0, group_base = 0;
  };
  AttnSet sets[2];
  int n_sets = 1;
  int slots = 0;
  int M0 = 0, Kmax = 0;
  // Lanes: disjoint request sets run as independent sub-batches on their own
  // streams.  Lane l owns plan positions [req_lo, req_hi) and stacked rows
  // [row_lo, row_hi); at step k its active requests and rows are the prefixes
  // n_act[k] and m[k] of those ranges (each lane is sorted by K descending).
  struct Lane {
    int req_lo = 0, req_hi = 0, row_lo = 0, row_hi = 0;
    std::vector<int32_t> n_act, m;
    // Per attention set and step: offset of the attention launch order in
    // attn_lists, and the launch's block count.
    std::vector<int32_t> list_at[2], list_blocks[2];
  };
  std::vector<Lane> lanes;
  // Attention launch orders, one per distinct set of active requests of a
  // lane: the persistent blocks' item lists (item index per entry, -1: an
  // idle block) and each entry's link to its block's next entry.
  std::vector<int32_t> attn_lists, attn_next;
};

// Address ranges of a call: whether a written one overlaps any other.
struct Range { uintptr_t lo, hi; bool written; };
inline bool clash(std::vector<Range> &r) {
  std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.lo < b.lo; });
  uintptr_t any = 0, written = 0;              // ends of the ranges so far
  for (const Range &x : r) {
    if (x.lo == x.hi) continue;
    if (x.lo < written || (x.written && x.lo < any)) return true;
    any = std::max(any, x.hi);
    if (x.written) written = std::max(written, x.hi);
  }
  return false;
}
inline void add_range(std::vector<Range> &r, const void *p, size_t bytes, bool written) {
  if (p && bytes) r.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written});
}
// Masses of a request set over caches of cache_bytes(request) bytes: usable, and apart from each other and from
// the caches (requests may share caches, but each token's mass is one block's to write).
template <typename Bytes>
const char *masses_unusable(const rosa_request *reqs, int n, float *const *mass, size_t rows, Bytes cache_bytes) {
  std::vector<Range> ranges;
  for (int i = 0; i < n; ++i) {
    if (reqs[i].prefix_len <= 0) continue;
    if (!mass[i] || (uintptr_t)mass[i] & 3) return "a request's masses are NULL or not 4-byte aligned";
    add_range(ranges, reqs[i].prefix_k, cache_bytes(reqs[i]), false);
    add_range(ranges, reqs[i].prefix_v, cache_bytes(reqs[i]), false);
    add_range(ranges, mass[i], rows * reqs[i].prefix_len * 4, true);
  }
  return clash(ranges) ? "a request's masses overlap another array of the call" : nullptr;
}

rosa_status check_config(const rosa_model_config *c);
rosa_status check_capacity(const rosa_capacity *c);
Dims make_dims(const rosa_model_config *c);
// Attention set of a layer: 0 for joint layers and the alternating layout's
// cross-attention (even) layers, 1 for its self-attention (odd) layers.
int attn_set_of(const rosa_model_config *cfg, int layer);
// Validation of a request set (all-or-nothing) and the batch plan.
rosa_status build_plan(const rosa_model_config *cfg, const rosa_capacity *cap, const rosa_request *reqs, int n,
                       bool sort_by_steps, bool allow_split, int lanes_wanted, Plan &p, std::string &err,
                       int max_steps_call = INT32_MAX, int max_slots = -1);

}  // namespace rosa
