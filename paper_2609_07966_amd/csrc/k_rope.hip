// Rotary positions: every frequency pair of a row's heads turned by its position's angle.
//
// A pair (a, b) becomes (a cos t - b sin t, b cos t + a sin t), t = pos * inv_freq.  The rows are read
// once and written once; nothing else is large, so the kernel is bound by that traffic (8192 rows of 40
// heads of 128, each pass on other rows: 168 MB in 37 us a pass, 4.5 TB/s, where a large copy reaches 4.9; 64
// rows: 3.6 us).  A thread takes VEC pairs at one place of `heads` heads of one row: their angles are the
// same for all heads, so each sine and cosine serves all of them.  The angle is formed in turns in float64 (a position past 2^16
// times an fp32 frequency has no bits left for its fraction in float32), its whole turns removed, and
// the rest goes to the hardware sine and cosine, which take turns (error below 2^-20, the fp16 result's
// half step is 2^-11 of its size).
#include <algorithm>

#include "kernels_common.h"
#include "mkv_decoding.h"

namespace mkv {

namespace {

constexpr int kRopeThreads = 256;

// 16 bytes to a caller's fp16 tensor, aligned to its elements only (see gld16h)
MKV_DEV void gst16h(uint16_t *p, const uint4 &u) {
  typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
  u32x4h v;
  v[0] = u.x;
  v[1] = u.y;
  v[2] = u.z;
  v[3] = u.w;
  *(MKV_GLOBAL u32x4h *)p = v;
}

MKV_DEV uint4 pack8(const float *f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f2h_bits(f[2 * i]) | (uint32_t)f2h_bits(f[2 * i + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int VEC>
MKV_DEV void load(const uint16_t *p, float *f) {
  if constexpr (VEC == 8) unpack8(gld16h(p), f);
  else f[0] = h2f(gld(p));
}
template <int VEC>
MKV_DEV void store(uint16_t *p, const float *f) {
  if constexpr (VEC == 8) gst16h(p, pack8(f));
  else gst(p, f2h_bits(f[0]));
}

constexpr int64_t kMaxBlocks = 1 << 23;  // of a launch: it takes under 2^32 threads along an axis

// A row's work is NC = pairs / VEC places (and, where values behind rotary_dim have to be copied, those
// places too) times `slots` head slots; slot i takes heads i, i + slots, ...  A block holds whole rows,
// or a part of one.
template <int VEC, bool PAIRS>
__global__ __launch_bounds__(kRopeThreads) void k_rope(RopeArgs a, int places, int slots, int rows_per_block,
                                                       int64_t first_row) {
  const int units = places * slots;
  const int local = blockIdx.y * kRopeThreads + threadIdx.x;
  const int r = local / units, u = local % units;
  const int64_t row = first_row + (int64_t)blockIdx.x * rows_per_block + r;
  if (r >= rows_per_block || row >= a.n_rows) return;
  const int place = u % places, slot = u / places, half = a.rot / 2, nc = half / VEC;
  float c[VEC], s[VEC];
  if (place < nc) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int pair = place * VEC + i;
      int axis = 0;
#pragma unroll
      for (int x = 0; x + 1 < MKV_ROPE_MAX_AXES; ++x) axis += pair >= a.ends[x] ? 1 : 0;
      const double turns = (double)gld(a.pos + (int64_t)axis * a.n_rows + row) * (double)gld(a.inv_freq + pair) *
                           0.15915494309189533577;  // 1 / (2 pi)
      const float t = (float)(turns - rint(turns));
      c[i] = __builtin_amdgcn_cosf(t);
      s[i] = a.inverse ? -__builtin_amdgcn_sinf(t) : __builtin_amdgcn_sinf(t);
    }
  }
  for (int h = slot; h < a.n_heads; h += slots) {
    int j = h, n = 0;
    while (j >= a.sets[n].n_heads) j -= a.sets[n++].n_heads;  // the head's set
    const uint16_t *x = a.sets[n].x + row * a.sets[n].x_stride + (int64_t)j * a.d;
    uint16_t *y = a.sets[n].y + row * a.sets[n].y_stride + (int64_t)j * a.d;
    if (place >= nc) {  // behind rotary_dim: copied
      const int at = a.rot + (place - nc) * 2 * VEC;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (VEC == 8) gst16h(y + at + 8 * i, gld16h(x + at + 8 * i));
        else gst(y + at + i, gld(x + at + i));
      }
      continue;
    }
    if constexpr (PAIRS) {
      float v[2 * VEC], o[2 * VEC];
      const int at = 2 * place * VEC;
      load<VEC>(x + at, v);
      load<VEC>(x + at + VEC, v + VEC);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        o[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * s[i];
        o[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * s[i];
      }
      store<VEC>(y + at, o);
      store<VEC>(y + at + VEC, o + VEC);
    } else {
      float v[VEC], w[VEC], p[VEC], q[VEC];
      const int at = place * VEC;
      load<VEC>(x + at, v);
      load<VEC>(x + half + at, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        p[i] = v[i] * c[i] - w[i] * s[i];
        q[i] = w[i] * c[i] + v[i] * s[i];
      }
      store<VEC>(y + at, p);
      store<VEC>(y + half + at, q);
    }
  }
}

template <int VEC>
hipError_t rope_impl(const RopeArgs &a, bool copy_tail, hipStream_t st) {
  const int places = a.rot / 2 / VEC + (copy_tail ? (a.d - a.rot) / (2 * VEC) : 0);
  // heads per thread: enough threads to fill the card first, then fewer sines
  constexpr int64_t kFull = (int64_t)kCus * 2048;
  const int64_t all = (int64_t)a.n_rows * a.n_heads * places;
  const int per = (int)std::min<int64_t>(8, std::max<int64_t>(1, all / kFull));
  const int slots = (a.n_heads + per - 1) / per, units = places * slots;
  const int rows_per_block = std::max(1, kRopeThreads / units);
  const int64_t blocks = (a.n_rows + (int64_t)rows_per_block - 1) / rows_per_block;
  auto kernel = a.pairs_layout ? k_rope<VEC, true> : k_rope<VEC, false>;
  for (int64_t first = 0; first < blocks; first += kMaxBlocks) {
    const dim3 grid((unsigned)std::min(kMaxBlocks, blocks - first), (unsigned)((units + kRopeThreads - 1) / kRopeThreads));
    hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), 0, st, a, places, slots, rows_per_block, first * rows_per_block);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, hipStream_t st) {
  bool copy_tail = false;
  for (int i = 0; i < a.n_sets; ++i) copy_tail |= a.rot < a.d && a.sets[i].x != a.sets[i].y;
  // 16-byte pieces where the head splits into them
  if (a.rot % 16 == 0 && a.d % 16 == 0) return rope_impl<8>(a, copy_tail, st);
  return rope_impl<1>(a, copy_tail, st);
}

}  // namespace mkv
