// Beam states: every beam of a group takes the state another one had, in place.
//
// What decode steps change of a (sequence, kv head) is a handful of byte ranges (the rows past the prompt,
// their codes, scales and outliers; everything an eviction can touch for H2O).  Any of a group's beams may
// be the source of any others while it is overwritten itself, so a column of bytes belongs to one thread
// for the whole group: it loads the column of every moved beam's parent, then stores them all.  No
// scratch, one read and one write a moved byte; bound by that traffic, or by round trips where tails
// are short.  Where a launch has several workgroups per (group, kv head) the counts, which all of them
// read, are copied by a launch behind it.
#include <algorithm>

#include "kernels_common.h"
#include "mkv_decoding.h"

namespace mkv {

namespace {

constexpr int kSmallThreads = 512, kLargeThreads = 256;
constexpr int kMaxRegions = 7;
constexpr size_t kSmallTail = 16;  // rows of a tail that one workgroup moves, in units of 4 KiB

// The beams of one group and kv head that take another one's state, in order, and the state words of that
// parent that the ranges follow from.
struct Moves {
  int n;
  int beam[MKV_BEAM_MAX], parent[MKV_BEAM_MAX];
  int count[MKV_BEAM_MAX];
  int fill[MKV_BEAM_MAX];  // KVQ: entries of the key-outlier pool
  int sel[MKV_BEAM_MAX];   // ROCKET: selected tokens
};

// Fill in the moves (every thread of the workgroup calls this).  Thread 8 b + w also returns word w of the
// state that beam b takes, for store_state.
MKV_DEV int32_t read_moves(Moves &mv, const int32_t *parent, const int32_t *state, int g, int h, int width, int Hkv) {
  static_assert(ST_WORDS == 8, "eight threads a beam");
  __shared__ int s_parent[64], s_words[MKV_BEAM_MAX][ST_WORDS];
  const int tid = threadIdx.x, b = tid / ST_WORDS, w = tid % ST_WORDS;
  int32_t word = 0;
  if (b < width) {
    int p = parent[g * width + b];
    if (p < 0 || p >= width) p = b;
    word = state[((int64_t)(g * width + p) * Hkv + h) * ST_WORDS + w];
    if (w == 0) s_parent[b] = p;
    s_words[b][w] = word;
  }
  __syncthreads();
  if (tid < 64) {
    const int p = tid < width ? s_parent[tid] : tid;
    const uint64_t moved = __ballot(p != tid);
    const int j = __popcll(moved & ((1ull << tid) - 1));
    if (p != tid) {
      mv.beam[j] = tid;
      mv.parent[j] = p;
      mv.count[j] = s_words[tid][ST_COUNT];
      mv.fill[j] = s_words[tid][ST_KOUT_FILL];
      mv.sel[j] = s_words[tid][ST_SEL_COUNT];
    }
    if (tid == 0) mv.n = __popcll(moved);
  }
  __syncthreads();
  return word;
}
MKV_DEV void store_state(int32_t word, int32_t *state, int g, int h, int width, int Hkv) {
  const int b = threadIdx.x / ST_WORDS, w = threadIdx.x % ST_WORDS;
  if (b < width) state[((int64_t)(g * width + b) * Hkv + h) * ST_WORDS + w] = word;
}
static_assert(MKV_BEAM_MAX * 8 <= kLargeThreads, "a thread per state word");

// One unit (at byte `at` of a region, `col` of its row) for all moves: every load, then every store where
// the column lies before that move's end.  Loads need no such test: the regions of a group are alike, and
// from() gives the last one's place for moves past it.
template <int W, typename T, typename From, typename To, typename End>
MKV_DEV void move_unit(char *base, int n, int64_t at, int64_t col, From from, To to, End end) {
  T v[W];
#pragma unroll
  for (int j = 0; j < W; ++j) v[j] = gld(reinterpret_cast<const T *>(base + from(j) + at));
#pragma unroll
  for (int j = 0; j < W; ++j)
    if (j < n && col < end(j)) gst(reinterpret_cast<T *>(base + to(j) + at), v[j]);
}

// visit(field, bytes per kv head, unit, begin, end(j), rows, pitch) for every region of d's method that
// decode steps change; end(j): of move j, by its parent's counts.
template <typename Visit>
MKV_DEV void for_regions(const SeqDesc &d, const Moves &mv, int h, int D, Visit visit) {
  const std::integral_constant<int, 16> wide{};
  const std::integral_constant<int, 4> word{};
  const int n0 = d.n0;
  const int64_t row = (int64_t)D * 2;
  auto tokens = [&](int64_t bytes) { return [&mv, bytes](int b) { return mv.count[b] * bytes; }; };
  switch (d.method) {
    case FP16:
      visit(&SeqDesc::k, d.cap * row, wide, n0 * row, tokens(row), 1, 0);
      visit(&SeqDesc::v, d.cap * row, wide, n0 * row, tokens(row), 1, 0);
      break;
    case UQ: {
      const int64_t code = d.rowbytes, vm = (int64_t)(D / 64) * 8, km = (int64_t)D * 8;
      visit(&SeqDesc::kc, d.cap * code, wide, (n0 & -64) * code, [&](int b) { return (mv.count[b] & -64) * code; }, 1, 0);
      visit(&SeqDesc::kmeta, d.nblk * km, wide, n0 / 64 * km, [&](int b) { return mv.count[b] / 64 * km; }, 1, 0);
      visit(&SeqDesc::kres, 64 * row, wide, 0, [&](int) { return 64 * row; }, 1, 0);
      // value codes lie in 4-token blocks
      visit(&SeqDesc::vc, d.cap * code, wide, (n0 & -4) * code, [&](int b) { return ((mv.count[b] + 3) & -4) * code; }, 1, 0);
      visit(&SeqDesc::vmeta, d.cap * vm, wide, n0 * vm, tokens(vm), 1, 0);
      break;
    }
    case KVQ: {
      const int64_t code = d.rowbytes, cap = d.cap;
      visit(&SeqDesc::kc, cap * code, wide, n0 * code, tokens(code), 1, 0);
      visit(&SeqDesc::vc, cap * code, wide, (n0 & -4) * code, [&](int b) { return ((mv.count[b] + 3) & -4) * code; }, 1, 0);
      visit(&SeqDesc::vmeta, cap * 4, wide, n0 * (int64_t)4, tokens(4), 1, 0);
      visit(&SeqDesc::vout, cap * 4 * d.nov_slots, wide, n0 * (int64_t)4, tokens(4), d.nov_slots, cap * 4);
      visit(&SeqDesc::vdel, cap * 4 * d.nov_slots, wide, n0 * (int64_t)4, tokens(4), d.nov_slots, cap * 4);
      // the outliers of the tokens past the prompt (whose CSR word, alike in all beams, says where they
      // begin)
      visit(&SeqDesc::krow, (cap + 1) * 4, word, (n0 + 1) * (int64_t)4, [&](int b) { return (mv.count[b] + 1) * (int64_t)4; }, 1, 0);
      const uint32_t first = gld(reinterpret_cast<const uint32_t *>(d.krow) + h * (cap + 1) + n0);
      visit(&SeqDesc::kout, (int64_t)d.pool_cap * 4, wide, (int64_t)first * 4, [&](int b) { return mv.fill[b] * (int64_t)4; }, 1, 0);
      break;
    }
    case H2O:
      // any slot may have been evicted and filled again
      visit(&SeqDesc::k, d.cap * row, wide, 0, tokens(row), 1, 0);
      visit(&SeqDesc::v, d.cap * row, wide, 0, tokens(row), 1, 0);
      visit(&SeqDesc::pos, (int64_t)d.cap * 4, word, 0, tokens(4), 1, 0);
      visit(&SeqDesc::score, (int64_t)d.cap * 4, word, 0, tokens(4), 1, 0);
      visit(&SeqDesc::vbest, (int64_t)d.vparts * 16, wide, 0, [&](int) { return (int64_t)d.vparts * 16; }, 1, 0);
      break;
    case ROCKET: {
      const int64_t kept = min(d.T, n0);
      visit(&SeqDesc::k, d.cap * row, wide, kept * row, tokens(row), 1, 0);
      visit(&SeqDesc::v, d.cap * row, wide, kept * row, tokens(row), 1, 0);
      visit(&SeqDesc::kcm, (int64_t)d.cstride * row, wide, kept * 2, tokens(2), D, (int64_t)d.cstride * 2);
      visit(&SeqDesc::pos, (int64_t)d.cap * 4, word, kept * 4, tokens(4), 1, 0);
      // the last step's selection and channels, which exports report
      visit(&SeqDesc::sel, stride_sel(d) * 4, word, 0, [&](int b) { return mv.sel[b] * (int64_t)4; }, 1, 0);
      visit(&SeqDesc::aux1, (int64_t)D * 4, word, 0, [&](int) { return (int64_t)d.nch * 4; }, 1, 0);
      break;
    }
    default:
      break;
  }
}

template <int UNIT>
struct UnitType {
  typedef u32x4 type;
};
template <>
struct UnitType<4> {
  typedef uint32_t type;
};

// What of a region moves where one workgroup moves all of a pair: bytes [begin, end[j]) of each of `rows`
// rows `pitch` bytes apart, in units of 16 bytes or of 4.  The sequences of a group lie at one distance
// from each other (seq_pitch), having one layout.
struct Region {
  char *base;
  int64_t seq_pitch, begin, pitch;
  int cols, rows, unit, first;  // cols: units of a row that some beam takes; first: units before it
  int64_t end[MKV_BEAM_MAX];
};

// One workgroup per (group, kv head): all regions in one sweep, so that their loads overlap (region after
// region a tail of 160 tokens under KVQuant takes 16 us, most of it one round trip a region), then the
// state.
template <int W>
__global__ __launch_bounds__(kSmallThreads) void k_reorder_small(const SeqDesc *__restrict__ seqs, int32_t *state,
                                                                 const int32_t *__restrict__ parent, int width, int Hkv,
                                                                 int D) {
  __shared__ Moves mv;
  __shared__ Region regions[kMaxRegions];
  __shared__ int s_total;
  const int g = blockIdx.x / Hkv, h = blockIdx.x % Hkv, tid = threadIdx.x;
  const SeqDesc *sq = seqs + (int64_t)g * width;
  const SeqDesc &d = sq[0];  // sizes are alike within the group
  const int32_t word = read_moves(mv, parent, state, g, h, width, Hkv);
  const int moves = mv.n;
  if (moves == 0) return;
  int n = 0;
  for_regions(d, mv, h, D, [&](uint64_t SeqDesc::*f, int64_t per_head, auto unit, int64_t begin, auto end, int rows, int64_t pitch) {
    Region &rg = regions[n++];
    if (tid < moves) rg.end[tid] = end(tid);
    if (tid == 0) {
      rg.base = reinterpret_cast<char *>(d.*f) + h * per_head;
      rg.seq_pitch = (int64_t)(sq[1].*f - d.*f);
      rg.begin = begin & -(int64_t)unit.value;
      rg.pitch = pitch;
      rg.rows = rows;
      rg.unit = unit.value;
    }
  });
  __syncthreads();
  if (tid < 64) {
    int cols = 0, units = 0;
    if (tid < n) {
      const Region &rg = regions[tid];
      int64_t longest = 0;
      for (int j = 0; j < moves; ++j) longest = max(longest, rg.end[j]);
      cols = longest > rg.begin ? (int)((longest - rg.begin + rg.unit - 1) / rg.unit) : 0;
      units = cols * rg.rows;
    }
    const int upto = wave_incl_scan(units);
    if (tid < n) {
      regions[tid].cols = cols;
      regions[tid].first = upto - units;
      if (tid == n - 1) s_total = upto;
    }
  }
  __syncthreads();
  const int total = s_total;
  for (int i = tid; i < total; i += kSmallThreads) {
    int r = 0;
    while (r + 1 < n && i >= regions[r + 1].first) ++r;
    const Region &rg = regions[r];
    const int u = i - rg.first, line = rg.rows == 1 ? 0 : u / rg.cols;
    const int64_t col = rg.begin + (int64_t)(u - line * rg.cols) * rg.unit, at = line * rg.pitch + col;
    auto from = [&](int j) { return mv.parent[min(j, moves - 1)] * rg.seq_pitch; };
    auto to = [&](int j) { return mv.beam[j] * rg.seq_pitch; };
    auto end = [&](int j) { return rg.end[j]; };
    if (rg.unit == 16) move_unit<W, u32x4>(rg.base, moves, at, col, from, to, end);
    else move_unit<W, uint32_t>(rg.base, moves, at, col, from, to, end);
  }
  store_state(word, state, g, h, width, Hkv);  // (every thread has read its word)
}

// Long tails: one (group, kv head) per blockIdx.x, the units of each region over blockIdx.y; the state by the
// launch behind.
template <int W>
__global__ __launch_bounds__(kLargeThreads) void k_reorder_large(const SeqDesc *__restrict__ seqs, const int32_t *state,
                                                                 const int32_t *__restrict__ parent, int width, int Hkv,
                                                                 int D) {
  __shared__ Moves mv;
  const int g = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  const SeqDesc *sq = seqs + (int64_t)g * width;
  const SeqDesc &d = sq[0];
  read_moves(mv, parent, state, g, h, width, Hkv);
  const int n = __builtin_amdgcn_readfirstlane(mv.n);
  if (n == 0) return;
  int from[W], to[W];  // (uniform: in scalar registers)
#pragma unroll
  for (int j = 0; j < W; ++j) {
    from[j] = __builtin_amdgcn_readfirstlane(mv.parent[min(j, n - 1)]);
    to[j] = __builtin_amdgcn_readfirstlane(mv.beam[min(j, n - 1)]);
  }
  for_regions(d, mv, h, D, [&](uint64_t SeqDesc::*f, int64_t per_head, auto unit, int64_t begin, auto end, int rows, int64_t pitch) {
    constexpr int U = decltype(unit)::value;
    begin &= -(int64_t)U;
    int64_t ends[W], longest = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int64_t e = end(min(j, n - 1));
      ends[j] = (int64_t)__builtin_amdgcn_readfirstlane((int)(e >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)e);
      longest = max(longest, ends[j]);
    }
    const int64_t cols = longest > begin ? (longest - begin + U - 1) / U : 0;
    char *base = reinterpret_cast<char *>(d.*f) + h * per_head;
    const int64_t seq_pitch = (int64_t)(sq[1].*f - d.*f);
    for (int64_t i = (int64_t)blockIdx.y * kLargeThreads + threadIdx.x; i < cols * rows; i += (int64_t)gridDim.y * kLargeThreads) {
      const int64_t line = rows == 1 ? 0 : i / cols, col = begin + (i - line * cols) * U;
      move_unit<W, typename UnitType<U>::type>(
          base, n, line * pitch + col, col, [&](int j) { return from[j] * seq_pitch; },
          [&](int j) { return to[j] * seq_pitch; }, [&](int j) { return ends[j]; });
    }
  });
}

__global__ __launch_bounds__(kLargeThreads) void k_reorder_state(int32_t *state, const int32_t *__restrict__ parent,
                                                                 int width, int Hkv) {
  __shared__ Moves mv;
  const int g = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  const int32_t word = read_moves(mv, parent, state, g, h, width, Hkv);  // (barriers behind every read)
  if (mv.n > 0) store_state(word, state, g, h, width, Hkv);
}

}  // namespace

hipError_t launch_reorder(const Dev &dv, const Shape &sh, const int32_t *parent, int width, size_t tail_bytes,
                          hipStream_t st) {
  const int pairs = sh.S / width * sh.Hkv;
  // several workgroups a pair, and the launch behind them, where a pair's rows are long
  const size_t most = tail_bytes / (16 * kLargeThreads);
  auto pick = [&](auto two, auto four, auto eight, auto sixteen, auto all) {
    return width <= 2 ? two : width <= 4 ? four : width <= 8 ? eight : width <= 16 ? sixteen : all;
  };
  if (most < kSmallTail) {
    hipLaunchKernelGGL(pick(k_reorder_small<2>, k_reorder_small<4>, k_reorder_small<8>, k_reorder_small<16>, k_reorder_small<32>),
                       dim3(pairs), dim3(kSmallThreads), 0, st, dv.seqs, dv.state, parent, width, sh.Hkv, sh.D);
    return hipGetLastError();
  }
  const dim3 grid(pairs, (unsigned)std::min<size_t>(most, std::max(1, 8 * kCus / pairs)));
  hipLaunchKernelGGL(pick(k_reorder_large<2>, k_reorder_large<4>, k_reorder_large<8>, k_reorder_large<16>, k_reorder_large<32>),
                     grid, dim3(kLargeThreads), 0, st, dv.seqs, dv.state, parent, width, sh.Hkv, sh.D);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_reorder_state, dim3(pairs), dim3(kLargeThreads), 0, st, dv.state, parent, width, sh.Hkv);
  return hipGetLastError();
}

}  // namespace mkv
