// Launchers of the operators around a decode step (rotary positions, drafted trees, beams), defined in
// k_rope.hip, k_tree.hip, k_beam.hip and k_reorder.hip.  All enqueue on `st`.
#pragma once

#include <vector>

#include "mkv_internal.h"

namespace mkv {

// ---- rotary positions (mkv_rope) ------------------------------------------------------------------
struct RopeArgs {
  const float *inv_freq;
  const int32_t *pos;
  mkv_rope_set sets[MKV_ROPE_MAX_SETS];
  int32_t n_rows, d, rot, n_sets, inverse, pairs_layout;
  int32_t n_heads;                   // of all sets
  int32_t ends[MKV_ROPE_MAX_AXES];  // first pair behind each axis's section (INT32_MAX for unused axes)
};
hipError_t launch_rope(const RopeArgs &a, hipStream_t st);

// ---- beam selection (mkv_beam_select) ---------------------------------------------------------------
struct BeamArgs {
  const void *logits;
  const float *scores;
  const uint8_t *finished;
  int32_t *token, *parent;
  float *score_out;
  void *workspace;
  int64_t row_stride;
  int32_t n_batch, n_beams, vocab, n_select, pad_token;
  bool half;
};
constexpr int kScanThreads = 512;
struct BeamPartial {  // of a chunk of one beam's logits
  double sum;         // sum of 2^((x - max) log2 e)
  float max;
  int32_t pad;
};
struct BeamCandidate {
  float logit;
  int32_t token;  // -1: none
};
// Logits per thread of a scan workgroup: 16 where that still leaves one for every CU, else 4.
inline int beam_values(int n_rows, int vocab) {
  return (int64_t)n_rows * ((vocab - 1) / (16 * kScanThreads) + 1) >= kCus ? 16 : 4;
}
inline int beam_chunks(int n_rows, int vocab) { return (vocab - 1) / (kScanThreads * beam_values(n_rows, vocab)) + 1; }
inline size_t beam_workspace(int n_batch, int n_beams, int vocab, int n_select) {
  const int rows = n_batch * n_beams;
  return (size_t)rows * beam_chunks(rows, vocab) * (sizeof(BeamPartial) + n_select * sizeof(BeamCandidate));
}
hipError_t launch_beam_select(const BeamArgs &a, hipStream_t st);

// ---- beam states (mkv_cache_reorder) ----------------------------------------------------------------
// tail_bytes: the most bytes of a kv head's rows that decode steps can have written.
hipError_t launch_reorder(const Dev &dv, const Shape &sh, const int32_t *parent, int width, size_t tail_bytes,
                          hipStream_t st);

// ---- drafted trees (mkv_tree_attention, mkv_tree_accept) --------------------------------------------
struct TreeArgs {
  const uint16_t *q, *k, *v;
  const uint64_t *mask;
  const int32_t *n_valid;
  uint16_t *out;
  float *workspace;
  int32_t n_nodes;
};
constexpr int kTreeTile = 64;  // tokens of a tile (a uniform 4-bit key block)
// Rows and splits of one call.
struct TreePlan {
  int rows;        // query rows (node, head of the group) of a workgroup
  int row_blocks;  // per (sequence, kv head)
  int chunk;       // cached tokens per split, by capacity (a multiple of 64)
  int max_splits;  // of one sequence
  int splits;      // of all sequences
  int slots;       // places for them in the workspace
  size_t bytes;    // workspace
};
TreePlan tree_plan(const Shape &sh, const std::vector<SeqDesc> &seqs, int n_nodes);
hipError_t launch_tree_attention(const Dev &dv, const Shape &sh, const TreePlan &plan, const TreeArgs &a, hipStream_t st);
hipError_t launch_tree_accept(const Dev &dv, const Shape &sh, const uint16_t *k, const uint16_t *v, int n_nodes,
                              const int32_t *path, const int32_t *n_path, int max_path, int32_t *counts, hipStream_t st);

}  // namespace mkv
