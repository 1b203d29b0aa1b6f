// Host side of the operators around a decode step: rotary positions, drafted trees, beams.  Argument
// checks and launches; see include/mkv.h for the contract.
#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "mkv.h"
#include "mkv_decoding.h"
#include "mkv_handle.h"

using namespace mkv;

namespace mkv {

TreePlan tree_plan(const Shape &sh, const std::vector<SeqDesc> &seqs, int n_nodes) {
  TreePlan p{};
  const int rows = n_nodes * sh.G;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  p.row_blocks = (rows + p.rows - 1) / p.rows;
  int longest = 0, quantized = 0;
  int64_t tiles = 0;
  for (const SeqDesc &d : seqs) {
    longest = std::max(longest, d.cap);
    quantized += d.method != FP16;
    tiles += (d.cap + kTreeTile - 1) / kTreeTile + 1;
  }
  auto splits_for = [&](int chunk) {
    int64_t n = 0;
    for (const SeqDesc &d : seqs) n += (d.cap + chunk - 1) / chunk;
    return n;
  };
  // the smallest split, by capacity, with at most `target` workgroups
  auto chunk_for = [&](int64_t target) {
    auto count = [&](int chunk) { return splits_for(chunk) * sh.Hkv * p.row_blocks; };
    int lo = 1, hi = std::max(1, (longest + kTreeTile - 1) / kTreeTile);  // tiles
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (count(mid * kTreeTile) <= target) hi = mid;
      else lo = mid + 1;
    }
    return lo * kTreeTile;
  };
  // All workgroups are resident at once.  Where a CU has few tiles to go through, one workgroup each is
  // best: every further split writes its rows' partial outputs, which the merge reads again (2 sequences of
  // 4000 fp16 tokens, 16 nodes: 20.8 us against 23.4 with two a CU).  Over many tiles two, of 32 rows at most
  // three, hide each other's waits.  With one, two and three a CU, 8 sequences of 8192 tokens: KVQuant at 4
  // bits 71.9, 49.4 and 42.8 us at 4 nodes (16 rows), 78.3, 53.6 and 46.9 at 8 (32 rows), 84.4, 59.8 and
  // 76.8 at 16; uniform 4-bit at 8 nodes 58.9, 42.3 and 40.5; fp16, which waits for memory alone, 53.4, 49.3
  // and 53.0.  More than fit at once are slower at every size measured.  The limits lie where the two met:
  // quantized tiles, with more to wait for, gain from a second workgroup earlier.
  // Without any split the merge's launch goes too, and one a CU holds out twice as long (32 sequences, fp16,
  // 1000 tokens: 25.8, 28.6 and 29.2 us at 4 nodes, 32.8, 36.6 and 43.1 at 16; KVQuant at 4 bits, 600 tokens,
  // 16 nodes: 33.0, 34.7 and 43.0), but for quantized tiles under few rows, where decoding is most of the
  // work and further splits add little to merge (600 tokens: 27.3, 25.5 and 23.7 at 4 nodes, 29.7, 28.3 and
  // 27.0 at 8).
  p.chunk = chunk_for(kCus);
  double few = quantized ? 6 : 12;
  if (p.chunk >= longest && (!quantized || p.rows >= 64)) few *= 2;
  if ((double)tiles * sh.Hkv * p.row_blocks > few * kCus) p.chunk = chunk_for((p.rows <= 32 ? 3 : 2) * kCus);
  p.max_splits = (longest + p.chunk - 1) / p.chunk;
  p.splits = (int)splits_for(p.chunk);
  const SeqDesc &last = seqs.back();
  p.slots = (int)((last.row0 + (int64_t)(seqs.size() - 1) * (sh.max_new + 3)) / p.chunk + (int64_t)seqs.size() - 1 +
                  (last.cap + p.chunk - 1) / p.chunk);
  p.bytes = p.max_splits == 1 ? 0 : sizeof(float) * (size_t)p.slots * sh.Hkv * p.row_blocks * p.rows * (sh.D + 2);
  return p;
}

}  // namespace mkv

namespace {

mkv_status fail(mkv_status s, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return report_error(s, buf);
}

mkv_status check_hip(hipError_t e, const char *what) {
  return e == hipSuccess ? MKV_OK : fail(MKV_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// Between steps: after prefill, or after a decode step that is complete.
mkv_status check_idle(const mkv_cache *c, const char *what) {
  if (c->phase == PH_READY || (c->phase == PH_ATTENDED && !c->any_h2o)) return MKV_OK;
  return fail(MKV_ESTATE, "%s must follow prefill or a completed decode step", what);
}

mkv_status check_tree(const mkv_cache *c, int n_nodes, const char *what) {
  if (!c) return fail(MKV_EINVAL, "cache is NULL");
  if (n_nodes < 1 || n_nodes > MKV_TREE_MAX_NODES)
    return fail(MKV_EINVAL, "n_nodes must be 1..%d (got %d)", MKV_TREE_MAX_NODES, n_nodes);
  if (c->any_h2o || c->any_rocket)
    return fail(MKV_EUNSUPPORTED, "%s needs FP16, UQ and KVQ sequences only (an H2O or ROCKET sequence is present)", what);
  return MKV_OK;
}

// A call's rows and splits, which the cache's layout settles: worked out once per number of nodes.
const TreePlan &plan_of(mkv_cache *c, int n_nodes) {
  TreePlan &p = c->tree_plans[n_nodes];
  if (p.rows == 0) p = tree_plan(c->sh, c->hs, n_nodes);
  return p;
}

mkv_status check_workspace(const void *p, size_t bytes, size_t need) {
  if (need == 0) return MKV_OK;
  if (!p) return fail(MKV_EINVAL, "workspace is NULL, %zu bytes are needed", need);
  if (((uintptr_t)p & 255) != 0) return fail(MKV_EINVAL, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(MKV_ENOMEM, "workspace has %zu bytes, %zu are needed", bytes, need);
  return MKV_OK;
}

mkv_status check_beam_sizes(int n_batch, int n_beams, int vocab, int n_select) {
  if (n_batch < 0) return fail(MKV_EINVAL, "n_batch must be >= 0");
  if (n_beams < 1 || n_beams > MKV_BEAM_MAX) return fail(MKV_EINVAL, "n_beams must be 1..%d", MKV_BEAM_MAX);
  if (vocab < 1 || vocab > (1 << 30)) return fail(MKV_EINVAL, "vocab must be 1..2^30");
  if (n_select < 1 || n_select > std::min(2 * MKV_BEAM_MAX, vocab))
    return fail(MKV_EINVAL, "n_select must be 1..min(%d, vocab)", 2 * MKV_BEAM_MAX);
  // a launch takes under 2^32 threads: one workgroup per chunk of a row, one per request
  const int64_t rows = (int64_t)n_batch * n_beams;
  if (n_batch >= 1 << 22 || rows >= 1 << 23 || rows * beam_chunks((int)rows, vocab) >= 1 << 23)
    return fail(MKV_EINVAL, "too many rows: n_batch must be below 2^22 and n_batch * n_beams * (chunks of a row) below 2^23");
  return MKV_OK;
}

}  // namespace

extern "C" {

mkv_status mkv_rope(const mkv_rope_spec *spec, const float *inv_freq, const int32_t *pos, int32_t n_rows,
                    const mkv_rope_set *sets, int32_t n_sets, int32_t inverse, void *stream) {
  if (!spec || !inv_freq || !pos || !sets) return fail(MKV_EINVAL, "spec, inv_freq, pos and sets must be non-NULL");
  const int d = spec->head_dim, rot = spec->rotary_dim;
  if (d < 2 || d > 1024 || d % 2 != 0) return fail(MKV_EINVAL, "head_dim must be even, 2..1024 (got %d)", d);
  if (rot < 2 || rot > d || rot % 2 != 0) return fail(MKV_EINVAL, "rotary_dim must be even, 2..head_dim (got %d)", rot);
  if (spec->n_axes < 1 || spec->n_axes > MKV_ROPE_MAX_AXES)
    return fail(MKV_EINVAL, "n_axes must be 1..%d (got %d)", MKV_ROPE_MAX_AXES, spec->n_axes);
  if (spec->layout != MKV_ROPE_HALVES && spec->layout != MKV_ROPE_PAIRS) return fail(MKV_EINVAL, "unknown layout %d", spec->layout);
  if (n_rows < 0) return fail(MKV_EINVAL, "n_rows must be >= 0");
  if (n_sets < 1 || n_sets > MKV_ROPE_MAX_SETS) return fail(MKV_EINVAL, "n_sets must be 1..%d (got %d)", MKV_ROPE_MAX_SETS, n_sets);
  RopeArgs a{};
  int64_t pairs = 0;
  for (int x = 0; x < MKV_ROPE_MAX_AXES; ++x) {
    if (x < spec->n_axes) {
      if (spec->sections[x] < 0) return fail(MKV_EINVAL, "sections must be >= 0");
      pairs += spec->sections[x];
    }
    // the last axis takes what is left, so no pair is past it
    a.ends[x] = x + 1 < spec->n_axes ? (int32_t)std::min<int64_t>(pairs, INT32_MAX) : INT32_MAX;
  }
  if (pairs != rot / 2) return fail(MKV_EINVAL, "sections sum to %lld pairs, rotary_dim has %d", (long long)pairs, rot / 2);
  int64_t heads = 0;
  for (int i = 0; i < n_sets; ++i) {
    const mkv_rope_set &t = sets[i];
    if (!t.x || !t.y) return fail(MKV_EINVAL, "set %d: x and y must be non-NULL", i);
    if (t.n_heads < 1 || t.n_heads > MKV_ROPE_MAX_HEADS)
      return fail(MKV_EINVAL, "set %d: n_heads must be 1..%d", i, MKV_ROPE_MAX_HEADS);
    const int64_t row = (int64_t)t.n_heads * d;
    if (t.x_stride < row || t.y_stride < row) return fail(MKV_EINVAL, "set %d: a row stride is below n_heads * head_dim", i);
    if (t.x == t.y && t.x_stride != t.y_stride) return fail(MKV_EINVAL, "set %d: in place needs equal strides", i);
    a.sets[i] = t;
    heads += t.n_heads;
  }
  if (n_rows == 0) return MKV_OK;
  a.inv_freq = inv_freq;
  a.pos = pos;
  a.n_rows = n_rows;
  a.d = d;
  a.rot = rot;
  a.n_sets = n_sets;
  a.inverse = inverse != 0;
  a.pairs_layout = spec->layout == MKV_ROPE_PAIRS;
  a.n_heads = (int32_t)heads;
  return check_hip(launch_rope(a, static_cast<hipStream_t>(stream)), "rope");
}

mkv_status mkv_tree_workspace(mkv_cache *c, int32_t n_nodes, size_t *bytes) {
  if (!bytes) return fail(MKV_EINVAL, "bytes is NULL");
  const mkv_status st = check_tree(c, n_nodes, "mkv_tree_workspace");
  if (st != MKV_OK) return st;
  *bytes = plan_of(c, n_nodes).bytes;
  return MKV_OK;
}

mkv_status mkv_tree_attention(mkv_cache *c, const uint16_t *q, const uint16_t *k, const uint16_t *v, const uint64_t *mask,
                              const int32_t *n_valid, int32_t n_nodes, uint16_t *out, void *workspace,
                              size_t workspace_bytes, void *stream) {
  mkv_status st = check_tree(c, n_nodes, "mkv_tree_attention");
  if (st != MKV_OK) return st;
  if (!q || !k || !v || !mask || !out) return fail(MKV_EINVAL, "q, k, v, mask and out must be non-NULL");
  if ((st = check_idle(c, "mkv_tree_attention")) != MKV_OK) return st;
  const TreePlan &plan = plan_of(c, n_nodes);
  if ((st = check_workspace(workspace, workspace_bytes, plan.bytes)) != MKV_OK) return st;
  const TreeArgs a{q, k, v, mask, n_valid, out, static_cast<float *>(workspace), n_nodes};
  return check_hip(launch_tree_attention(c->dv, c->sh, plan, a, static_cast<hipStream_t>(stream)), "tree attention");
}

mkv_status mkv_tree_accept(mkv_cache *c, const uint16_t *k, const uint16_t *v, int32_t n_nodes, const int32_t *path,
                           const int32_t *n_path, int32_t max_path, int32_t *counts, void *stream) {
  mkv_status st = check_tree(c, n_nodes, "mkv_tree_accept");
  if (st != MKV_OK) return st;
  if (!k || !v || !path || !n_path) return fail(MKV_EINVAL, "k, v, path and n_path must be non-NULL");
  if (max_path < 1) return fail(MKV_EINVAL, "max_path must be >= 1");
  if ((st = check_idle(c, "mkv_tree_accept")) != MKV_OK) return st;
  return check_hip(launch_tree_accept(c->dv, c->sh, k, v, n_nodes, path, n_path, max_path, counts,
                                      static_cast<hipStream_t>(stream)),
                   "tree accept");
}

mkv_status mkv_beam_workspace(int32_t n_batch, int32_t n_beams, int32_t vocab, int32_t n_select, size_t *bytes) {
  if (!bytes) return fail(MKV_EINVAL, "bytes is NULL");
  const mkv_status st = check_beam_sizes(n_batch, n_beams, vocab, n_select);
  if (st != MKV_OK) return st;
  *bytes = n_batch > 0 ? beam_workspace(n_batch, n_beams, vocab, n_select) : 0;
  return MKV_OK;
}

mkv_status mkv_beam_select(const void *logits, int32_t dtype, int64_t row_stride, int32_t n_batch, int32_t n_beams,
                           int32_t vocab, const float *scores, const uint8_t *finished, int32_t pad_token,
                           int32_t n_select, int32_t *token, int32_t *parent, float *score_out, void *workspace,
                           size_t workspace_bytes, void *stream) {
  mkv_status st = check_beam_sizes(n_batch, n_beams, vocab, n_select);
  if (st != MKV_OK) return st;
  if (dtype != MKV_F32 && dtype != MKV_F16) return fail(MKV_EINVAL, "logits are MKV_F32 or MKV_F16 (got %d)", dtype);
  if (row_stride < vocab) return fail(MKV_EINVAL, "row_stride is below vocab");
  if (pad_token < 0 || pad_token >= vocab) return fail(MKV_EINVAL, "pad_token must be 0..vocab-1");
  if (n_batch == 0) return MKV_OK;
  if (!logits || !scores || !token || !parent || !score_out)
    return fail(MKV_EINVAL, "logits, scores, token, parent and score_out must be non-NULL");
  if ((st = check_workspace(workspace, workspace_bytes, beam_workspace(n_batch, n_beams, vocab, n_select))) != MKV_OK) return st;
  const BeamArgs a{logits, scores, finished, token, parent, score_out, workspace, row_stride,
                   n_batch, n_beams, vocab, n_select, pad_token, dtype == MKV_F16};
  return check_hip(launch_beam_select(a, static_cast<hipStream_t>(stream)), "beam select");
}

mkv_status mkv_cache_reorder(mkv_cache *c, const int32_t *parent, int32_t width, void *stream) {
  if (!c) return fail(MKV_EINVAL, "cache is NULL");
  if (!parent) return fail(MKV_EINVAL, "parent is NULL");
  if (width < 1 || width > MKV_BEAM_MAX) return fail(MKV_EINVAL, "width must be 1..%d (got %d)", MKV_BEAM_MAX, width);
  if (c->sh.S % width != 0) return fail(MKV_EINVAL, "%d sequences are no groups of %d beams", c->sh.S, width);
  size_t tail = 0;
  for (int s = 0; s < c->sh.S; ++s) {
    // beams are alike in all sizes of their layout, which follow from these
    const SeqDesc &a = c->hs[s], &b = c->hs[s - s % width];
    const mkv_config &x = c->cfg[s], &y = c->cfg[s - s % width];
    bool same = a.method == b.method && a.n0 == b.n0;
    if (same && a.method == KVQ) same = x.bits == y.bits && x.outlier_bp == y.outlier_bp;
    if (same && a.method == H2O) same = x.budget_pct == y.budget_pct;
    if (same && a.method == ROCKET) same = a.T == b.T && a.topk == b.topk && a.window == b.window && a.pool == b.pool && a.nch == b.nch;
    if (!same) return fail(MKV_EINVAL, "seq %d differs from its group's first beam in configuration or prompt length", s);
    const size_t rows = a.method == H2O ? a.cap : c->sh.max_new;
    const size_t row = a.method == UQ || a.method == KVQ ? a.rowbytes : (size_t)c->sh.D * 2;
    tail = std::max(tail, rows * row);
  }
  const mkv_status st = check_idle(c, "mkv_cache_reorder");
  if (st != MKV_OK || width == 1) return st;
  return check_hip(launch_reorder(c->dv, c->sh, parent, width, tail, static_cast<hipStream_t>(stream)), "cache reorder");
}

}  // extern "C"
