// Host-side checks of the operators around a decode step that need no GPU, built with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code (the kernel launchers are stubbed out, so nothing reaches a
// device): every refusal, the work that an empty call leaves out, and the places of the tree attention's
// partial results, which have to lie apart and within the workspace.  Exit status 0 when every check holds.
#include <climits>
#include <cstdio>
#include <cstring>
#include <set>
#include <vector>

#include "mkv.h"
#include "mkv_decoding.h"
#include "mkv_handle.h"

static int launches = 0;

namespace mkv {
mkv_status report_error(mkv_status s, const char *) { return s; }
hipError_t launch_rope(const RopeArgs &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_beam_select(const BeamArgs &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_reorder(const Dev &, const Shape &, const int32_t *, int, size_t, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_tree_attention(const Dev &, const Shape &, const TreePlan &, const TreeArgs &, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_tree_accept(const Dev &, const Shape &, const uint16_t *, const uint16_t *, int, const int32_t *, const int32_t *, int, int32_t *, hipStream_t) { ++launches; return hipSuccess; }
}  // namespace mkv

static int failures = 0;
#define CHECK(c)                                                  \
  do {                                                            \
    if (!(c)) {                                                   \
      std::printf("FAILED line %d: %s\n", __LINE__, #c);          \
      ++failures;                                                 \
    }                                                             \
  } while (0)

using namespace mkv;

// Pointers that are never read here.
static uint16_t *const H = reinterpret_cast<uint16_t *>(0x1000);
static int32_t *const I = reinterpret_cast<int32_t *>(0x1000);
static float *const F = reinterpret_cast<float *>(0x1000);
static uint64_t *const M = reinterpret_cast<uint64_t *>(0x1000);

static mkv_cache cache(const std::vector<int> &methods, const std::vector<int> &prompts, int max_new, int hkv = 2, int g = 4, int d = 128) {
  mkv_cache c;
  const int S = (int)methods.size();
  c.sh = Shape{S, hkv * g, hkv, d, g, max_new};
  c.cfg.resize(S);
  int row0 = 0;
  for (int s = 0; s < S; ++s) {
    std::memset(&c.cfg[s], 0, sizeof c.cfg[s]);
    SeqDesc q{};
    q.method = c.cfg[s].method = methods[s];
    q.n0 = prompts[s];
    q.row0 = row0;
    row0 += q.n0;
    q.cap = q.method == FP16 ? q.n0 + max_new : (q.n0 + max_new + 3) & ~3;
    c.any_h2o |= q.method == H2O;
    c.any_rocket |= q.method == ROCKET;
    c.hs.push_back(q);
  }
  c.phase = PH_READY;
  return c;
}

static void check_rope() {
  mkv_rope_spec ok{128, 64, 2, {20, 12, 0, 0}, MKV_ROPE_HALVES};
  mkv_rope_set set[2] = {{H, H + 64, 512, 256, 2}, {H, H, 128, 128, 1}};
  auto run = [&](const mkv_rope_spec &s, int rows = 3, int sets = 2) { return mkv_rope(&s, F, I, rows, set, sets, 0, nullptr); };
  launches = 0;
  CHECK(run(ok) == MKV_OK && launches == 1);
  CHECK(run(ok, 0) == MKV_OK && launches == 1);
  CHECK(run(ok, -1) == MKV_EINVAL && run(ok, 3, 0) == MKV_EINVAL && run(ok, 3, MKV_ROPE_MAX_SETS + 1) == MKV_EINVAL);
  CHECK(mkv_rope(nullptr, F, I, 1, set, 1, 0, nullptr) == MKV_EINVAL && mkv_rope(&ok, nullptr, I, 1, set, 1, 0, nullptr) == MKV_EINVAL);
  CHECK(mkv_rope(&ok, F, nullptr, 1, set, 1, 0, nullptr) == MKV_EINVAL && mkv_rope(&ok, F, I, 1, nullptr, 1, 0, nullptr) == MKV_EINVAL);
  for (const mkv_rope_spec &bad : std::vector<mkv_rope_spec>{{127, 64, 2, {20, 12}, 0}, {128, 63, 2, {20, 12}, 0}, {128, 130, 2, {33, 32}, 0},
                                                              {128, 64, 0, {32}, 0}, {128, 64, 5, {20, 12}, 0}, {128, 64, 2, {20, 13}, 0},
                                                              {128, 64, 2, {33, -1}, 0}, {128, 64, 2, {INT_MAX, 12}, 0}, {128, 64, 2, {20, 12}, 2},
                                                              {1026, 64, 2, {20, 12}, 0}, {128, 0, 1, {0}, 0}})
    CHECK(run(bad) == MKV_EINVAL);
  const mkv_rope_set good = set[0];
  for (const mkv_rope_set &bad : std::vector<mkv_rope_set>{{nullptr, H, 512, 256, 2}, {H, nullptr, 512, 256, 2}, {H, H + 64, 255, 256, 2},
                                                            {H, H + 64, 512, 255, 2}, {H, H + 64, 512, 256, 0}, {H, H, 512, 256, 2}}) {
    set[0] = bad;
    CHECK(run(ok) == MKV_EINVAL);
  }
  set[0] = good;
  CHECK(launches == 1);
}

static void check_beam() {
  size_t need = 0;
  CHECK(mkv_beam_workspace(2, 4, 1000, 8, &need) == MKV_OK && need > 0);
  void *ws = reinterpret_cast<void *>(0x10000);
  auto run = [&](int b, int w, int v, int k, int pad = 0, int64_t stride = -1, int dtype = MKV_F32, void *p = nullptr, size_t bytes = ~size_t(0), const float *logits = F) {
    return mkv_beam_select(logits, dtype, stride < 0 ? v : stride, b, w, v, F, nullptr, pad, k, I, I, F, p ? p : ws, bytes, nullptr);
  };
  launches = 0;
  CHECK(run(2, 4, 1000, 8) == MKV_OK && launches == 1);
  CHECK(run(0, 4, 1000, 8) == MKV_OK && launches == 1);
  CHECK(run(-1, 4, 1000, 8) == MKV_EINVAL && run(2, 0, 1000, 8) == MKV_EINVAL && run(2, MKV_BEAM_MAX + 1, 1000, 8) == MKV_EINVAL);
  CHECK(run(2, 4, 0, 1) == MKV_EINVAL && run(2, 4, (1 << 30) + 1, 1) == MKV_EINVAL && run(2, 4, 7, 8) == MKV_EINVAL);
  CHECK(run(2, 4, 1000, 0) == MKV_EINVAL && run(2, 4, 1000, 2 * MKV_BEAM_MAX + 1) == MKV_EINVAL);
  CHECK(run(2, 4, 1000, 8, -1) == MKV_EINVAL && run(2, 4, 1000, 8, 1000) == MKV_EINVAL && run(2, 4, 1000, 8, 0, 999) == MKV_EINVAL);
  CHECK(run(2, 4, 1000, 8, 0, 1000, 2) == MKV_EINVAL && run(2, 4, 1000, 8, 0, 1000, 0, nullptr, need - 1) == MKV_ENOMEM);
  CHECK(run(2, 4, 1000, 8, 0, 1000, 0, reinterpret_cast<void *>(0x10008)) == MKV_EINVAL);
  CHECK(run(2, 4, 1000, 8, 0, 1000, 0, nullptr, need, nullptr) == MKV_EINVAL);
  CHECK(run(1 << 27, 32, 1000, 8) == MKV_EINVAL);  // more rows than an int counts
  CHECK(mkv_beam_workspace(2, 4, 1000, 8, nullptr) == MKV_EINVAL && launches == 1);
  // no launch of 2^32 threads: requests, rows, chunks of rows
  CHECK(mkv_beam_workspace((1 << 22) - 1, 1, 32, 8, &need) == MKV_OK);
  CHECK(mkv_beam_workspace(1 << 22, 1, 32, 8, &need) == MKV_EINVAL);
  CHECK(mkv_beam_workspace((1 << 18) - 1, 32, 8192, 8, &need) == MKV_OK);
  CHECK(mkv_beam_workspace(1 << 18, 32, 8192, 8, &need) == MKV_EINVAL);
  CHECK(mkv_beam_workspace((1 << 18) - 1, 32, 8193, 8, &need) == MKV_EINVAL);
  CHECK(mkv_beam_workspace(INT32_MAX, 32, 32, 8, &need) == MKV_EINVAL);
}

static void check_cache_calls() {
  mkv_cache c = cache({FP16, KVQ, UQ, FP16}, {4000, 100, 70, 1}, 9);
  size_t need = 0;
  CHECK(mkv_tree_workspace(&c, 8, &need) == MKV_OK && need > 0);
  void *ws = reinterpret_cast<void *>(0x10000);
  auto tree = [&](mkv_cache *p, int n, void *w, size_t bytes, const uint16_t *q = H) {
    return mkv_tree_attention(p, q, H, H, M, nullptr, n, H, w, bytes, nullptr);
  };
  auto accept = [&](mkv_cache *p, int n, int m, const int32_t *path = I) { return mkv_tree_accept(p, H, H, n, path, I, m, nullptr, nullptr); };
  launches = 0;
  CHECK(tree(&c, 8, ws, need) == MKV_OK && accept(&c, 8, 3) == MKV_OK && launches == 2);
  CHECK(tree(nullptr, 8, ws, need) == MKV_EINVAL && tree(&c, 0, ws, need) == MKV_EINVAL && tree(&c, 65, ws, need) == MKV_EINVAL);
  CHECK(tree(&c, 8, nullptr, need) == MKV_EINVAL && tree(&c, 8, ws, need - 1) == MKV_ENOMEM);
  CHECK(tree(&c, 8, reinterpret_cast<void *>(0x10010), need) == MKV_EINVAL && tree(&c, 8, ws, need, nullptr) == MKV_EINVAL);
  CHECK(mkv_tree_workspace(&c, 8, nullptr) == MKV_EINVAL && mkv_tree_workspace(nullptr, 8, &need) == MKV_EINVAL);
  CHECK(accept(nullptr, 8, 3) == MKV_EINVAL && accept(&c, 8, 0) == MKV_EINVAL && accept(&c, 0, 3) == MKV_EINVAL && accept(&c, 8, 3, nullptr) == MKV_EINVAL);
  for (Phase p : {PH_CREATED, PH_PROMPT, PH_APPENDED, PH_SELECTED}) {
    c.phase = p;
    CHECK(tree(&c, 8, ws, need) == MKV_ESTATE && accept(&c, 8, 3) == MKV_ESTATE && mkv_cache_reorder(&c, I, 1, nullptr) == MKV_ESTATE);
  }
  c.phase = PH_ATTENDED;
  CHECK(tree(&c, 8, ws, need) == MKV_OK && launches == 3);
  for (int m : {H2O, ROCKET}) {
    mkv_cache e = cache({FP16, m}, {100, 100}, 4);
    CHECK(tree(&e, 4, ws, 1 << 20) == MKV_EUNSUPPORTED && accept(&e, 4, 1) == MKV_EUNSUPPORTED && mkv_tree_workspace(&e, 4, &need) == MKV_EUNSUPPORTED);
    CHECK(mkv_cache_reorder(&e, I, 2, nullptr) == MKV_EINVAL);
  }
  // H2O: not between the attention and its eviction
  mkv_cache e = cache({H2O, H2O}, {100, 100}, 4);
  e.phase = PH_ATTENDED;
  CHECK(mkv_cache_reorder(&e, I, 2, nullptr) == MKV_ESTATE);
  e.phase = PH_READY;
  CHECK(mkv_cache_reorder(&e, I, 2, nullptr) == MKV_OK && launches == 4);
  CHECK(mkv_cache_reorder(&e, I, 1, nullptr) == MKV_OK && launches == 4);
  CHECK(mkv_cache_reorder(&e, I, 0, nullptr) == MKV_EINVAL && mkv_cache_reorder(&e, I, 3, nullptr) == MKV_EINVAL);
  CHECK(mkv_cache_reorder(&e, nullptr, 2, nullptr) == MKV_EINVAL && mkv_cache_reorder(nullptr, I, 2, nullptr) == MKV_EINVAL);
  e.cfg[1].budget_pct = 7;
  CHECK(mkv_cache_reorder(&e, I, 2, nullptr) == MKV_EINVAL);
  mkv_cache f = cache({FP16, FP16, FP16, FP16}, {100, 100, 90, 91}, 4);
  CHECK(mkv_cache_reorder(&f, I, 2, nullptr) == MKV_EINVAL && mkv_cache_reorder(&f, I, 1, nullptr) == MKV_OK);
  mkv_cache g = cache({KVQ, KVQ}, {100, 100}, 4);
  g.cfg[0].bits = 3;
  g.cfg[1].bits = 4;
  CHECK(mkv_cache_reorder(&g, I, 2, nullptr) == MKV_EINVAL && launches == 4);
}

// The slots of a plan, as the kernels compute them.
static void check_plan(const std::vector<int> &methods, const std::vector<int> &prompts, int max_new, int n, int hkv, int g, int d) {
  const mkv_cache c = cache(methods, prompts, max_new, hkv, g, d);
  const TreePlan p = tree_plan(c.sh, c.hs, n);
  CHECK(p.chunk % kTreeTile == 0 && p.chunk > 0);
  CHECK(p.rows * p.row_blocks >= n * g && p.rows * (p.row_blocks - 1) < n * g);
  std::set<int64_t> used;
  int most = 0, all = 0;
  for (int s = 0; s < c.sh.S; ++s) {
    const SeqDesc &q = c.hs[s];
    const int splits = (q.cap + p.chunk - 1) / p.chunk;
    most = std::max(most, splits);
    const int64_t first = (q.row0 + (int64_t)s * (max_new + 3)) / p.chunk + s;
    for (int i = 0; i < splits; ++i) {
      CHECK(used.insert(first + i).second);
      CHECK(first + i >= 0 && first + i < p.slots);
    }
    // every tile and the drafted one in exactly one of the splits in use, however many tokens there are
    for (int m : {1, 63, 64, 65, q.cap / 2 + 1, q.cap}) {
      if (m < 1 || m > q.cap) continue;
      const int tiles = (m + kTreeTile - 1) / kTreeTile + 1, in_use = std::min(splits, tiles), each = tiles / splits, more = tiles % splits;
      int next = 0;
      for (int i = 0; i < splits; ++i) {
        const int begin = i * each + std::min(i, more), end = begin + each + (i < more);
        CHECK(begin == next && (end > begin) == (i < in_use));
        next = end;
      }
      CHECK(next == tiles);
    }
    all += splits;
  }
  CHECK(all == p.splits);
  CHECK(most == p.max_splits);
  CHECK(p.max_splits == 1 ? p.bytes == 0 : p.bytes == sizeof(float) * (size_t)p.slots * hkv * p.row_blocks * p.rows * (d + 2));
}

static void check_plans() {
  unsigned r = 12345;
  auto rnd = [&](int n) { r = r * 1664525u + 1013904223u; return (int)((r >> 8) % (unsigned)n); };
  for (int round = 0; round < 300; ++round) {
    std::vector<int> methods, prompts;
    const int S = 1 + rnd(round % 7 == 0 ? 200 : 9), most = 1 + rnd(round % 5 == 0 ? 60000 : 3000);
    for (int s = 0; s < S; ++s) {
      methods.push_back(rnd(3));
      prompts.push_back(1 + rnd(most));
    }
    check_plan(methods, prompts, rnd(300), 1 + rnd(MKV_TREE_MAX_NODES), 1 << rnd(4), 1 << rnd(4), rnd(2) ? 64 : 128);
  }
}

int main() {
  check_rope();
  check_beam();
  check_cache_calls();
  check_plans();
  std::printf("ok (%d failures)\n", failures);
  return failures != 0;
}
