// Beam states: every beam of a group takes the state another one had, in place.
//
// What decode steps change of a (sequence, kv head) is a handful of byte ranges (the rows past the prompt,
// their codes, scales and outliers; everything an eviction can touch for H2O).  Any of a group's beams may
// be the source of any others while it is overwritten itself, so a column of bytes belongs to one thread
// for the whole group: it loads the column of every moved beam's parent, then stores them all.  No
// scratch, one read and one write a moved byte; bound by that traffic.  Where a launch has several
// workgroups per (group, kv head) the counts, which all of them read, are copied by a launch behind it.
#include <algorithm>

#include "kernels_common.h"
#include "mkv_decoding.h"

namespace mkv {

namespace {

constexpr int kReorderThreads = 256;

// The beams of one group and kv head: whose state each takes (itself: it stays), and the state words of
// that parent that the ranges follow from.
struct Moves {
  int parent[MKV_BEAM_MAX];
  int count[MKV_BEAM_MAX];
  int fill[MKV_BEAM_MAX];  // KVQ: entries of the key-outlier pool
  int sel[MKV_BEAM_MAX];   // ROCKET: selected tokens
  int any;
};

MKV_DEV void read_moves(Moves &mv, const int32_t *parent, const int32_t *state, int g, int h, int width, int Hkv) {
  if (threadIdx.x == 0) mv.any = 0;
  __syncthreads();
  const int b = threadIdx.x;
  if (b < width) {
    int p = parent[g * width + b];
    if (p < 0 || p >= width) p = b;
    const int32_t *st = state + ((int64_t)(g * width + p) * Hkv + h) * ST_WORDS;
    mv.parent[b] = p;
    mv.count[b] = st[ST_COUNT];
    mv.fill[b] = st[ST_KOUT_FILL];
    mv.sel[b] = st[ST_SEL_COUNT];
    if (p != b) atomicOr(&mv.any, 1);
  }
  __syncthreads();
}

// Copy, of a region with `rows` rows of `pitch` bytes, the bytes [begin, end(beam)) of each row: units of
// T, columns spread over the workgroups of the (group, kv head).  base(b): beam b's region.
template <int W, typename T, typename Base, typename End>
MKV_DEV void move_range(const Moves &mv, int width, int part, int parts, int rows, int64_t pitch, int64_t begin,
                        Base base, End end) {
  constexpr int U = sizeof(T);
  begin &= -(int64_t)U;
  int64_t longest = 0;
  for (int b = 0; b < width; ++b)
    if (mv.parent[b] != b) longest = max(longest, (int64_t)end(b));
  const int64_t cols = longest > begin ? (longest - begin + U - 1) / U : 0;
  for (int64_t i = (int64_t)part * kReorderThreads + threadIdx.x; i < cols * rows; i += (int64_t)parts * kReorderThreads) {
    const int64_t r = rows == 1 ? 0 : i / cols, c = begin + (rows == 1 ? i : i % cols) * U, at = r * pitch + c;
    T v[W];
#pragma unroll
    for (int b = 0; b < W; ++b)
      if (b < width && mv.parent[b] != b && c < end(b)) v[b] = gld(reinterpret_cast<const T *>(base(mv.parent[b]) + at));
#pragma unroll
    for (int b = 0; b < W; ++b)
      if (b < width && mv.parent[b] != b && c < end(b)) gst(reinterpret_cast<T *>(base(b) + at), v[b]);
  }
}

MKV_DEV void move_state(const Moves &mv, int32_t *state, int g, int h, int width, int Hkv) {
  // the words of one column by one thread, as above
  if (threadIdx.x >= ST_WORDS) return;
  int32_t v[MKV_BEAM_MAX];
#pragma unroll
  for (int b = 0; b < MKV_BEAM_MAX; ++b)
    if (b < width) v[b] = state[((int64_t)(g * width + mv.parent[b]) * Hkv + h) * ST_WORDS + threadIdx.x];
#pragma unroll
  for (int b = 0; b < MKV_BEAM_MAX; ++b)
    if (b < width) state[((int64_t)(g * width + b) * Hkv + h) * ST_WORDS + threadIdx.x] = v[b];
}

// One (group, kv head) per blockIdx.y, its columns over blockIdx.x.
template <int W>
__global__ __launch_bounds__(kReorderThreads) void k_reorder(const SeqDesc *__restrict__ seqs, int32_t *state,
                                                             const int32_t *__restrict__ parent, int width, int Hkv,
                                                             int D) {
  __shared__ Moves mv;
  const int g = blockIdx.x / Hkv, h = blockIdx.x % Hkv, part = blockIdx.y, parts = gridDim.y;
  read_moves(mv, parent, state, g, h, width, Hkv);
  if (!mv.any) return;
  const SeqDesc *sq = seqs + (int64_t)g * width;
  const SeqDesc &d = sq[0];  // sizes are alike within the group
  const int n0 = d.n0;
  auto field = [&](uint64_t SeqDesc::*f, int64_t stride) {  // beam -> its kv head's part of a region
    return [=](int b) { return reinterpret_cast<char *>(sq[b].*f) + h * stride; };
  };
  auto wide = [&](auto base, int64_t begin, auto end) { move_range<W, u32x4>(mv, width, part, parts, 1, 0, begin, base, end); };
  auto words = [&](auto base, int64_t begin, auto end) { move_range<W, uint32_t>(mv, width, part, parts, 1, 0, begin, base, end); };
  const int64_t row = (int64_t)D * 2;
  switch (d.method) {
    case FP16: {
      auto end = [&](int b) { return mv.count[b] * row; };
      wide(field(&SeqDesc::k, d.cap * row), n0 * row, end);
      wide(field(&SeqDesc::v, d.cap * row), n0 * row, end);
      break;
    }
    case UQ: {
      const int64_t code = d.rowbytes, vm = (int64_t)(D / 64) * 8, km = (int64_t)D * 8;
      wide(field(&SeqDesc::kc, d.cap * code), (n0 & -64) * code, [&](int b) { return (mv.count[b] & -64) * code; });
      wide(field(&SeqDesc::kmeta, d.nblk * km), n0 / 64 * km, [&](int b) { return mv.count[b] / 64 * km; });
      wide(field(&SeqDesc::kres, 64 * row), 0, [&](int) { return 64 * row; });
      // value codes lie in 4-token blocks
      wide(field(&SeqDesc::vc, d.cap * code), (n0 & -4) * code, [&](int b) { return ((mv.count[b] + 3) & -4) * code; });
      wide(field(&SeqDesc::vmeta, d.cap * vm), n0 * vm, [&](int b) { return mv.count[b] * vm; });
      break;
    }
    case KVQ: {
      const int64_t code = d.rowbytes, cap = d.cap;
      wide(field(&SeqDesc::kc, cap * code), n0 * code, [&](int b) { return mv.count[b] * code; });
      wide(field(&SeqDesc::vc, cap * code), (n0 & -4) * code, [&](int b) { return ((mv.count[b] + 3) & -4) * code; });
      auto tokens = [&](int b) { return mv.count[b] * (int64_t)4; };
      wide(field(&SeqDesc::vmeta, cap * 4), n0 * (int64_t)4, tokens);
      auto slots = [&](uint64_t SeqDesc::*f) {
        move_range<W, u32x4>(mv, width, part, parts, d.nov_slots, cap * 4, n0 * (int64_t)4,
                             field(f, cap * 4 * d.nov_slots), tokens);
      };
      slots(&SeqDesc::vout);
      slots(&SeqDesc::vdel);
      // the outliers of the tokens past the prompt (whose CSR word, alike in all beams, says where they
      // begin)
      words(field(&SeqDesc::krow, (cap + 1) * 4), (n0 + 1) * (int64_t)4, [&](int b) { return (mv.count[b] + 1) * (int64_t)4; });
      const uint32_t first = gld(reinterpret_cast<const uint32_t *>(d.krow) + h * (cap + 1) + n0);
      wide(field(&SeqDesc::kout, (int64_t)d.pool_cap * 4), (int64_t)first * 4, [&](int b) { return mv.fill[b] * (int64_t)4; });
      break;
    }
    case H2O: {
      // any slot may have been evicted and filled again
      auto rows = [&](int b) { return mv.count[b] * row; };
      auto tokens = [&](int b) { return mv.count[b] * (int64_t)4; };
      wide(field(&SeqDesc::k, d.cap * row), 0, rows);
      wide(field(&SeqDesc::v, d.cap * row), 0, rows);
      words(field(&SeqDesc::pos, (int64_t)d.cap * 4), 0, tokens);
      words(field(&SeqDesc::score, (int64_t)d.cap * 4), 0, tokens);
      wide(field(&SeqDesc::vbest, (int64_t)d.vparts * 16), 0, [&](int) { return (int64_t)d.vparts * 16; });
      break;
    }
    case ROCKET: {
      const int64_t kept = min(d.T, n0);
      auto rows = [&](int b) { return mv.count[b] * row; };
      wide(field(&SeqDesc::k, d.cap * row), kept * row, rows);
      wide(field(&SeqDesc::v, d.cap * row), kept * row, rows);
      move_range<W, u32x4>(mv, width, part, parts, D, (int64_t)d.cstride * 2, kept * 2,
                           field(&SeqDesc::kcm, (int64_t)d.cstride * row), [&](int b) { return mv.count[b] * (int64_t)2; });
      words(field(&SeqDesc::pos, (int64_t)d.cap * 4), kept * 4, [&](int b) { return mv.count[b] * (int64_t)4; });
      // the last step's selection and channels, which exports report
      words(field(&SeqDesc::sel, stride_sel(d) * 4), 0, [&](int b) { return mv.sel[b] * (int64_t)4; });
      words(field(&SeqDesc::aux1, (int64_t)D * 4), 0, [&](int) { return (int64_t)d.nch * 4; });
      break;
    }
    default:
      break;
  }
  if (parts > 1) return;
  __syncthreads();
  move_state(mv, state, g, h, width, Hkv);
}

__global__ __launch_bounds__(64) void k_reorder_state(int32_t *state, const int32_t *__restrict__ parent, int width,
                                                      int Hkv) {
  __shared__ Moves mv;
  const int g = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  read_moves(mv, parent, state, g, h, width, Hkv);
  if (mv.any) move_state(mv, state, g, h, width, Hkv);
}

}  // namespace

hipError_t launch_reorder(const Dev &dv, const Shape &sh, const int32_t *parent, int width, size_t tail_bytes,
                          hipStream_t st) {
  const int pairs = sh.S / width * sh.Hkv;
  // a second workgroup of a pair pays for the second launch only where a pair's rows are long
  const size_t most = tail_bytes / (16 * kReorderThreads);
  const int parts = most < 8 ? 1 : (int)std::min<size_t>(most, std::max(1, 8 * kCus / pairs));
  const dim3 grid(pairs, parts);
  auto kernel = width <= 2 ? k_reorder<2> : width <= 4 ? k_reorder<4> : width <= 8 ? k_reorder<8> : width <= 16 ? k_reorder<16> : k_reorder<32>;
  hipLaunchKernelGGL(kernel, grid, dim3(kReorderThreads), 0, st, dv.seqs, dv.state, parent, width, sh.Hkv, sh.D);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  hipLaunchKernelGGL(k_reorder_state, dim3(pairs), dim3(64), 0, st, dv.state, parent, width, sh.Hkv);
  return hipGetLastError();
}

}  // namespace mkv
