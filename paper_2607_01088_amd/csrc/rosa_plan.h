// The host's batch plan and argument checks, shared by the files that
// implement the C ABI's handles.
#pragma once

#include <stdint.h>

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
