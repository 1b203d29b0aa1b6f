// The host handle of a cache, shared by the host files of the library.
#pragma once

#include <vector>

#include "mkv_decoding.h"

namespace mkv {

enum Phase { PH_CREATED, PH_PROMPT, PH_READY, PH_APPENDED, PH_SELECTED, PH_ATTENDED };

constexpr int kProfKinds = 5;

}  // namespace mkv

struct mkv_cache {
  mkv::Shape sh{};
  std::vector<mkv_config> cfg;
  std::vector<mkv::SeqDesc> hs;  // absolute device pointers
  std::vector<mkv::SeqGroup> groups;
  char *arena = nullptr;
  mkv::Dev dv{};
  mkv::Phase phase = mkv::PH_CREATED;
  int steps = 0;
  bool any_h2o = false, any_rocket = false, h2o_done = false, snap_done = false;
  int topk_max = 0;
  int h2o_rows = 0, rocket_rows = 0;
  mkv::TreePlan tree_plans[MKV_TREE_MAX_NODES + 1] = {};  // by number of nodes; rows 0: not worked out yet
  // profiling
  bool evict_pending = false;  // H2O: the last eviction call's victims await the next decode append
  int prof_mask = 0;  // bit k: launches of kind k are timed
  int prof_cap = 0;
  std::vector<hipEvent_t> ev[mkv::kProfKinds][2];
  int prof_n[mkv::kProfKinds] = {};
};
