// Beam selection: the best continuations of every request's beams.
//
// A continuation (w, t) scores scores[w] + logit(w, t) - lse(w).  Within a beam that order is the
// logits' own (but for scores that are equal though the logits are not, see take_ties), so one pass over the
// logits is enough: each workgroup takes a chunk of one beam's vocabulary into registers and writes the
// chunk's best n_select logits, its maximum and its sum of exponentials; a second, small launch has every
// request's candidates compared by their full scores in float64 (two beams' scores lie closer than float32 tells apart once in some thousand selections).
// Bound by reading the logits once (128 rows of 128000 float32: 65 MB in 18 us, 3.6 TB/s), small calls by the
// two launches' latency (4 rows of 32001: 5 and 6 us).
//
// Choosing the best K of a workgroup's values: the maxima over its 64 groups of lanes are 64 values, and the
// K-th largest of these (K <= 64) is not above the K-th largest of all.  Only the values that reach it are
// collected (about K of random ones), as unique 64-bit keys (order-preserving bits of the value, then the
// lower index first), and ranked against each other.  Where they do not fit the list (values in ascending
// order, or constant), the best ones are taken one after another.
#include <algorithm>

#include "kernels_common.h"
#include "mkv_decoding.h"

namespace mkv {

namespace {

constexpr int kScanWaves = kScanThreads / 64, kMergeThreads = 1024, kMergeWaves = kMergeThreads / 64;
constexpr int kBeamGroups = 64;  // groups of lanes in either workgroup: of 8, of 16
constexpr int kListCap = 2048;
static_assert(2 * MKV_BEAM_MAX <= kBeamGroups && kScanThreads / 8 == kBeamGroups && kMergeThreads / 16 == kBeamGroups,
              "the K-th largest group maximum is taken by one wave");

typedef unsigned long long u64;

// Largest value over each group of N lanes (8 or 16), in all its lanes.
template <int CTRL>
MKV_DEV uint32_t dpp_u32(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false); }
template <int N>
MKV_DEV uint32_t group_max(uint32_t x) {
  x = max(x, dpp_u32<0xB1>(x));
  x = max(x, dpp_u32<0x4E>(x));
  x = max(x, dpp_u32<0x141>(x));
  return N == 16 ? max(x, dpp_u32<0x140>(x)) : x;
}
MKV_DEV u64 group8_max(u64 x) {
  auto step = [&](auto ctrl) {
    constexpr int C = decltype(ctrl)::value;
    const u64 y = ((u64)dpp_u32<C>((uint32_t)(x >> 32)) << 32) | dpp_u32<C>((uint32_t)x);
    x = y > x ? y : x;
  };
  step(std::integral_constant<int, 0xB1>{});
  step(std::integral_constant<int, 0x4E>{});
  step(std::integral_constant<int, 0x141>{});
  return x;
}

// The K-th largest of the 64 values in `s` (16-byte aligned), for one whole wave.
MKV_DEV uint32_t kth_of_64(const uint32_t *s, int k) {
  const int lane = threadIdx.x & 63;
  const uint32_t mine = s[lane];
  int above = 0, reach = 0;  // values over this one; values not under it
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    const uint4 o = *reinterpret_cast<const uint4 *>(s + i);
    above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
    reach += (o.x >= mine) + (o.y >= mine) + (o.z >= mine) + (o.w >= mine);
  }
  return s[__builtin_ctzll(__ballot(above < k && reach >= k))];
}

struct PickLds {
  __attribute__((aligned(16))) uint32_t group[kBeamGroups];
  u64 group64[kBeamGroups];  // where the list overflows
  uint32_t tau;
  int n;
};

// The keys of a chunk's values: high word the value's order, low word the lower index first; 0: no value.
MKV_DEV u64 chunk_key(float x, int index) { return ((u64)float_key(x) << 32) | (uint32_t)~index; }

// One workgroup per (chunk, row): E values a thread, in pieces of 4 contiguous ones.
template <typename T, int E>
__global__ __launch_bounds__(kScanThreads) void k_beam_scan(const T *__restrict__ logits, int64_t row_stride, int vocab,
                                                            int k, int n_chunks, BeamPartial *__restrict__ parts,
                                                            BeamCandidate *__restrict__ cands) {
  __shared__ PickLds L;
  __shared__ u64 s_list[kListCap];
  __shared__ float s_max[kScanWaves];
  __shared__ double s_sum[kScanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x % n_chunks;
  const int64_t row = blockIdx.x / n_chunks;
  const T *p = logits + row * row_stride;
  const int base = chunk * kScanThreads * E;
  float x[E];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    const int at = base + (i * kScanThreads + tid) * 4;
    float *f = x + 4 * i;
    if (at + 4 <= vocab) {
      if constexpr (sizeof(T) == 4) {
        const uint4 u = gld16w(reinterpret_cast<const uint32_t *>(p) + at);
        f[0] = __builtin_bit_cast(float, u.x);
        f[1] = __builtin_bit_cast(float, u.y);
        f[2] = __builtin_bit_cast(float, u.z);
        f[3] = __builtin_bit_cast(float, u.w);
      } else {
        typedef uint32_t u32x2h __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2h u = *(const MKV_GLOBAL u32x2h *)(p + at);
        f[0] = h2f(u[0]);
        f[1] = h2f(u[0] >> 16);
        f[2] = h2f(u[1]);
        f[3] = h2f(u[1] >> 16);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j] = -INFINITY;
        if (at + j < vocab) {
          if constexpr (sizeof(T) == 4) f[j] = gld(p + at + j);
          else f[j] = h2f(gld(p + at + j));
        }
      }
    }
  }
  float mx = -INFINITY;
  auto key_of = [&](int i, float v) { return chunk_key(v, base + ((i >> 2) * kScanThreads + tid) * 4 + (i & 3)); };
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if (!(x[i] > -INFINITY)) x[i] = -INFINITY;  // NaN
    mx = fmaxf(mx, x[i]);
  }
  const uint32_t gm = group_max<8>(float_key(mx));
  if ((lane & 7) == 0) L.group[tid >> 3] = gm;
  const float wm = wave_max(mx);
  if (lane == 0) s_max[wave] = wm;
  if (tid == 0) L.n = 0;
  __syncthreads();
  float M = s_max[0];
#pragma unroll
  for (int w = 1; w < kScanWaves; ++w) M = fmaxf(M, s_max[w]);
  if (wave == 0) {
    const uint32_t t = kth_of_64(L.group, k);
    if (lane == 0) L.tau = t;
  }
  // the sum of exponentials: float32 over a thread's values, float64 over the threads
  float sum = 0.f;
  if (M != -INFINITY) {
#pragma unroll
    for (int i = 0; i < E; ++i) sum += fexp2((x[i] - M) * kLog2e);
  }
  double ds = sum;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) ds += __shfl_xor(ds, m);
  if (lane == 0) s_sum[wave] = ds;
  __syncthreads();
  const uint32_t tau = max(L.tau, float_key(-INFINITY) + 1u);
  if (float_key(mx) >= tau) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (float_key(x[i]) < tau) continue;
      const int at = atomicAdd(&L.n, 1);
      if (at < kListCap) s_list[at] = key_of(i, x[i]);
    }
  }
  __syncthreads();
  const int n = L.n;
  BeamCandidate *out = cands + (row * n_chunks + chunk) * k;
  if (n <= kListCap) {
    for (int i = tid; i < n; i += kScanThreads) {
      const u64 mine = s_list[i];
      int above = 0;
      for (int j = 0; j < n; ++j) above += s_list[j] > mine ? 1 : 0;
      if (above < k) {
        const int token = (int)~(uint32_t)mine;
        const uint32_t o = (uint32_t)(mine >> 32);
        out[above] = {__builtin_bit_cast(float, (o & 0x80000000u) ? o ^ 0x80000000u : ~o), token};
      }
    }
    if (tid < k && tid >= n) out[tid] = {-INFINITY, -1};
  } else {
    // one after another: the largest key below the last one
    u64 last = ~0ull;
    for (int r = 0; r < k; ++r) {
      u64 top = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const u64 key = x[i] == -INFINITY ? 0 : key_of(i, x[i]);
        top = key < last && key > top ? key : top;
      }
      const u64 g = group8_max(top);
      __syncthreads();
      if ((lane & 7) == 0) L.group64[tid >> 3] = g;
      __syncthreads();
      u64 all = 0;
      for (int i = 0; i < kBeamGroups; ++i) all = L.group64[i] > all ? L.group64[i] : all;
      last = all;  // (n > kListCap >= k values are there)
      if (tid == 0) {
        const uint32_t o = (uint32_t)(all >> 32);
        out[r] = {__builtin_bit_cast(float, (o & 0x80000000u) ? o ^ 0x80000000u : ~o), (int)~(uint32_t)all};
      }
    }
  }
  if (tid == 0) {
    double total = 0.0;
    for (int w = 0; w < kScanWaves; ++w) total += s_sum[w];
    parts[row * n_chunks + chunk] = {total, M, 0};
  }
}

// A candidate's place in the order of a request: score (order-preserving bits), then the lower index.
struct Rank {
  u64 score, index;  // score 0: not above -infinity
};
MKV_DEV bool above(const Rank &a, const Rank &b) { return a.score > b.score || (a.score == b.score && a.index < b.index); }
MKV_DEV u64 double_key(double x) {
  if (!(x > -INFINITY)) return 0;
  x += 0.0;  // -0 is +0
  const u64 u = __builtin_bit_cast(u64, x);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
MKV_DEV double key_double(u64 k) { return __builtin_bit_cast(double, k >> 63 ? k ^ 0x8000000000000000ull : ~k); }

MKV_DEV Rank row_best(Rank x) {
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) {
    const Rank y = {(u64)__shfl_xor((long long)x.score, m), (u64)__shfl_xor((long long)x.index, m)};
    if (above(y, x)) x = y;
  }
  return x;
}

// Where the K-th score is shared by continuations that no chunk listed, which one is taken is the lower index's,
// not the larger logit's: scores of 64 bits so far from 0 that a logit changes nothing (dead beams given
// the lowest finite score), or logits that small.  A chunk can hide such a one only if the last it listed ties
// too: its logits are gone through again, in the order of the indexes, with what the other chunks listed
// (16 of 8 beams of 128000, a finished one and seven dead: 38 us, where 25 are usual).
// For the whole workgroup; `need` outputs, which exist, go to write(i, rank) for i < need.
template <typename CandOf, typename Write>
MKV_DEV void take_ties(const BeamArgs &a, u64 score, int need, int n_chunks, int chunk, const double *s_base, const int *s_done,
                       int *s_counts, CandOf cand_of, Write write) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.n_select, b = blockIdx.x;
  const uint64_t below = (1ull << lane) - 1;
  int got = 0;
  for (int w = 0; w < a.n_beams && got < need; ++w) {
    const double base = s_base[w];
    const u64 index = (u64)w * a.vocab;
    if (s_done[w]) {
      if (double_key(base) == score) {
        if (tid == 0) write(got, Rank{score, index + a.pad_token});
        ++got;
      }
      continue;
    }
    auto ties = [&](double logit) { return double_key(base + logit) == score; };
    for (int c = 0; c < n_chunks && got < need; ++c) {
      const int first = (w * n_chunks + c) * K;
      const BeamCandidate top = cand_of(first), last = cand_of(first + K - 1);
      if (top.token < 0 || double_key(base + (double)top.logit) < score) continue;
      if (last.token >= 0 && ties((double)last.logit)) {
        const int end = min(a.vocab, (c + 1) * chunk);
        for (int t0 = c * chunk; t0 < end && got < need; t0 += kMergeThreads) {
          const int t = t0 + tid;
          const int64_t at = ((int64_t)b * a.n_beams + w) * a.row_stride + t;
          bool hit = false;
          if (t < end)
            hit = ties(a.half ? h2f(gld(static_cast<const uint16_t *>(a.logits) + at)) : gld(static_cast<const float *>(a.logits) + at));
          const uint64_t hits = __ballot(hit);
          if (lane == 0) s_counts[wave] = __popcll(hits);
          __syncthreads();
          int before = 0, all = 0;
          for (int i = 0; i < kMergeWaves; ++i) {
            before += i < wave ? s_counts[i] : 0;
            all += s_counts[i];
          }
          const int place = got + before + __popcll(hits & below);
          if (hit && place < need) write(place, Rank{score, index + t});
          got += all;
          __syncthreads();
        }
      } else {  // (at most 64 listed, best first: every wave looks at them, the first one writes)
        const BeamCandidate mine = cand_of(first + min(lane, K - 1));
        const bool hit = lane < K && mine.token >= 0 && ties((double)mine.logit);
        uint64_t rest = __ballot(hit);
        const int all = __popcll(rest);
        int place = got;
        for (; rest; rest &= rest - 1) place += __shfl(mine.token, __builtin_ctzll(rest)) < mine.token ? 1 : 0;
        if (wave == 0 && hit && place < need) write(place, Rank{score, index + mine.token});
        got += all;
      }
    }
  }
}

// One workgroup per request.
__global__ __launch_bounds__(kMergeThreads) void k_beam_merge(BeamArgs a, const BeamPartial *__restrict__ parts,
                                                             const BeamCandidate *__restrict__ cands, int n_chunks,
                                                             int chunk) {
  __shared__ double s_base[MKV_BEAM_MAX];  // scores[w] - lse(w); a finished beam: scores[w]
  __shared__ int s_done[MKV_BEAM_MAX];
  __shared__ Rank s_group[kBeamGroups];
  __shared__ Rank s_list[kListCap / 2];
  __shared__ __attribute__((aligned(16))) uint32_t s_group32[kBeamGroups];
  __shared__ uint32_t s_tau;
  __shared__ int s_n;
  __shared__ u64 s_edge;  // the best score that a chunk listed last: it may have more of that one
  __shared__ int s_over;  // outputs above it
  __shared__ int s_counts[kMergeWaves];
  constexpr int kCap = kListCap / 2, kAhead = 2;
  static_assert(kCap <= kMergeThreads, "a thread for every one listed");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, W = a.n_beams, K = a.n_select;
  const int per = n_chunks * K, total = W * per;
  auto cand_of = [&](int i) { return cands[(int64_t)b * total + i]; };
  // (the thread's first candidates are on their way while the beams' sums are put together)
  BeamCandidate mine[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) mine[u] = cand_of(min(tid + u * kMergeThreads, total - 1));
  const int lists = W * n_chunks;
  const BeamCandidate final = cand_of(min(tid, lists - 1) * K + K - 1);
  auto rank = [&](int i, const BeamCandidate &c) {
    const int w = i / per;
    if (s_done[w])
      return i % per == 0 ? Rank{double_key(s_base[w]), (u64)w * a.vocab + a.pad_token} : Rank{0, ~0ull};
    if (c.token < 0) return Rank{0, ~0ull};
    return Rank{double_key(s_base[w] + (double)c.logit), (u64)w * a.vocab + c.token};
  };
  if (tid == 0) {
    s_n = s_over = 0;
    s_edge = 0;
  }
  for (int w = wave; w < W; w += kMergeWaves) {
    const int64_t row = (int64_t)b * W + w;
    float m = -INFINITY;
    for (int c = lane; c < n_chunks; c += 64) m = fmaxf(m, parts[row * n_chunks + c].max);
    m = wave_max(m);
    double sum = 0.0;
    for (int c = lane; c < n_chunks; c += 64) {
      const BeamPartial p = parts[row * n_chunks + c];
      if (p.max != -INFINITY) sum += p.sum * exp((double)p.max - (double)m);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) {
      const int done = a.finished && a.finished[row] ? 1 : 0;
      s_done[w] = done;
      s_base[w] = (double)a.scores[row] - (done ? 0.0 : (double)m + log(sum));
    }
  }
  __syncthreads();
  // candidate i: beam i / per, the i % per-th of its chunks' candidates
  auto rank_of = [&](int i) { return rank(i, cand_of(i)); };
  Rank best = {0, ~0ull}, ahead[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int i = tid + u * kMergeThreads;
    ahead[u] = i < total ? rank(i, mine[u]) : Rank{0, ~0ull};
    if (above(ahead[u], best)) best = ahead[u];
  }
  for (int i = tid + kAhead * kMergeThreads; i < total; i += kMergeThreads) {
    const Rank r = rank_of(i);
    if (above(r, best)) best = r;
  }
  u64 edge = 0;
  for (int l = tid; l < lists; l += kMergeThreads) {
    const BeamCandidate c = l == tid ? final : cand_of(l * K + K - 1);
    const int w = l / n_chunks;
    if (!s_done[w] && c.token >= 0) edge = max(edge, double_key(s_base[w] + (double)c.logit));
  }
  edge = group8_max(edge);
  if ((lane & 7) == 0 && edge != 0) atomicMax(&s_edge, edge);
  // the K-th best group by the upper half of its score
  const uint32_t gm = group_max<16>((uint32_t)(best.score >> 32));
  if ((lane & 15) == 0) s_group32[tid >> 4] = gm;
  __syncthreads();
  if (wave == 0) {
    const uint32_t t = kth_of_64(s_group32, K);
    if (lane == 0) s_tau = t;
  }
  __syncthreads();
  const uint32_t tau = s_tau;
  const u64 last_listed = s_edge;
  auto collect = [&](const Rank &r) {
    if (r.score == 0 || (uint32_t)(r.score >> 32) < tau) return;
    if (r.score > last_listed) atomicAdd(&s_over, 1);
    const int at = atomicAdd(&s_n, 1);
    if (at < kCap) s_list[at] = r;
  };
  if ((uint32_t)(best.score >> 32) >= tau) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) collect(ahead[u]);
    for (int i = tid + kAhead * kMergeThreads; i < total; i += kMergeThreads) collect(rank_of(i));
  }
  __syncthreads();
  const int n = s_n;
  auto write = [&](int at, const Rank &r) {
    const int64_t o = (int64_t)b * K + at;
    a.token[o] = r.score ? (int)(r.index % a.vocab) : a.pad_token;
    a.parent[o] = r.score ? (int)(r.index / a.vocab) : 0;
    a.score_out[o] = r.score ? (float)key_double(r.score) : -INFINITY;
  };
  // (no chunk's last score is above the K-th: with fewer than K above it, it is the K-th)
  const int over = last_listed != 0 && s_over < K ? s_over : K;
  if (n <= kCap) {
    if (tid < n) {
      const Rank mine = s_list[tid];
      int before = 0;
      for (int j = 0; j < n; ++j) before += above(s_list[j], mine) ? 1 : 0;
      if (before < over) write(before, mine);
    }
    if (tid < over && tid >= n) write(tid, Rank{0, 0});
  } else {
    Rank last = {~0ull, 0};
    for (int r = 0; r < over; ++r) {
      Rank top = {0, ~0ull};
      for (int i = tid; i < total; i += kMergeThreads) {
        const Rank c = rank_of(i);
        if (above(last, c) && above(c, top)) top = c;
      }
      top = row_best(top);
      __syncthreads();
      if ((lane & 15) == 0) s_group[tid >> 4] = top;
      __syncthreads();
      Rank all = s_group[0];
      for (int i = 1; i < kBeamGroups; ++i)
        if (above(s_group[i], all)) all = s_group[i];
      last = all;
      if (tid == 0) write(r, all);
    }
  }
  if (over < K)
    take_ties(a, last_listed, K - over, n_chunks, chunk, s_base, s_done, s_counts, cand_of, [&](int i, const Rank &r) { write(over + i, r); });
}

template <typename T>
hipError_t beam_impl(const BeamArgs &a, hipStream_t st) {
  const int rows = a.n_batch * a.n_beams, chunks = beam_chunks(rows, a.vocab);
  BeamPartial *parts = static_cast<BeamPartial *>(a.workspace);
  BeamCandidate *cands = reinterpret_cast<BeamCandidate *>(parts + (int64_t)rows * chunks);
  auto kernel = beam_values(rows, a.vocab) == 16 ? k_beam_scan<T, 16> : k_beam_scan<T, 4>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)rows * chunks)), dim3(kScanThreads), 0, st,
                     static_cast<const T *>(a.logits), a.row_stride, a.vocab, a.n_select, chunks, parts, cands);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_beam_merge, dim3(a.n_batch), dim3(kMergeThreads), 0, st, a, parts, cands, chunks,
                     kScanThreads * beam_values(rows, a.vocab));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_beam_select(const BeamArgs &a, hipStream_t st) {
  return a.half ? beam_impl<uint16_t>(a, st) : beam_impl<float>(a, st);
}

}  // namespace mkv
