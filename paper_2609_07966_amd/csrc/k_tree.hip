// Drafted trees: attention of several drafted tokens per sequence over its cache and over each other, and
// the append of those that are accepted.
//
// Attention.  The query rows of a (sequence, kv head) are its nodes' query heads, N G of them; all
// attend to the same cached tokens, so their logits and outputs are matrix products.  A workgroup takes
// R rows and a range of 64-token tiles; the last range ends with one more tile, the tree's own keys and
// values under the nodes' masks.  A tile is brought into LDS as fp16 rows, whatever the method it is
// stored under (each code is dequantized once per workgroup and serves all its rows; outliers replace
// their values there), keys as [token][channel], values as [channel][token], which are the two products'
// operands:
//   S^T = K Q^T (tokens x rows),  O^T = V^T P^T (channels x rows)
// with v_mfma_f32_16x16x32_f16.  S^T's result layout (tokens 4 (lane / 16) + i, row lane % 16) is P^T's
// operand layout up to the order of the tokens, which the value reads follow, so probabilities stay in
// their lanes.  One pass: running maximum and sum per row in float32; ranges are merged by their
// maxima, waves through LDS and splits by a second launch.
//
// Roundings to fp16: dequantized keys and values (at most half a step, 2^-11 of the value; fp16 rows and
// outliers are exact), uniform middles and steps before they are put together (as much; a step below 2^-14 to
// 2^-25, of which a code takes up to 8), and probabilities, which are formed 2^kLift times too large (2^15 at
// most, with the reference 2^kLazy behind), so that fp16 holds them to half a step down to 2^-27 of the largest
// and a long tail of small ones is not lost.  Everything summed is float32.  Nothing finite becomes infinite on
// the way: uniform groups at fp16's end round towards 0, KVQuant values are held times a power of two that takes
// their codebook to 1 (values near 0 lose as many bits as it goes past that), and results that are means of
// finite values are held to 65504.  Against 64 bits the outputs of quantized caches are 3e-4 to 1.1e-3 off
// (2-norm), of fp16 ones 2.2e-4, of which their own rounding is 2.1e-4.  (Most of it is the keys' rounding; keys
// in two fp16 parts would need half as many products again, and a second key tile in the LDS.)
//
// What bounds it (8 sequences of 8192 tokens, 32 query and 8 kv heads of 128): few rows, the cache's bytes
// (fp16, 1 to 16 nodes: 5.3 to 5.0 TB/s; the quantized tiles cost more than their bytes, in conversion and
// table lookups: uniform 4-bit 2.4 TB/s, vector operations 60 % of the time; KVQuant at 4 bits 1.9, the LDS
// half of the time); many, the matrix units, the exponentials and the LDS one after
// another, two waves a SIMD being too few to overlap them (64 nodes: 590 to 650 TFLOP/s, where a large fp16
// product of the library reaches 1330).

#include <algorithm>

#include "append_dev.h"
#include "mkv_decoding.h"

namespace mkv {

namespace {

constexpr int kTreeThreads = 256;
constexpr int kTile = kTreeTile;
constexpr float kLazy = 2.f;   // the reference of a row's softmax moves when a logit passes it by this (log2)
constexpr float kLift = 13.f;  // probabilities are formed 2^kLift times too large: at most 2^15 in fp16

typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));

MKV_DEV f4v mfma32(h8v a, h8v b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
MKV_DEV f4v mfma16(h4v a, h4v b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }
MKV_DEV uint32_t pk_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
MKV_DEV uint32_t pk_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
MKV_DEV uint32_t pk_f16(float lo, float hi) { return __builtin_bit_cast(uint32_t, h2v{(_Float16)lo, (_Float16)hi}); }
MKV_DEV uint16_t f2h_toward_0(float x) {
  return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, 0.f));
}
constexpr uint32_t kOnePair = 0x3C003C00u;
MKV_DEV uint32_t pk_mul(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2v, a) * __builtin_bit_cast(h2v, b));
}
MKV_DEV uint32_t pk_fma(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(h2v, a), __builtin_bit_cast(h2v, b),
                                                                __builtin_bit_cast(h2v, c)));
}
// the 4-bit nibbles k and k + 4 of w (k < 4), each less 8, as a packed pair of exact fp16 integers: set
// into the mantissa of 1024 (or, 4 bits up, of 64), which is then taken off with the 8
MKV_DEV uint32_t nib_pair(uint32_t w, int k) {
  const uint32_t x = k >= 2 ? w >> 8 : w;
  const bool up = k & 1;
  const uint32_t y = (x & (up ? 0x00F000F0u : 0x000F000Fu)) | (up ? 0x54005400u : 0x64006400u);
  const _Float16 base = up ? (_Float16)72.0f : (_Float16)1032.0f;
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2v, y) - h2v{base, base});
}

// A tile in LDS.  Value rows hold 16 blocks of 4 tokens, block b of channel c at b ^ vswz(c): the writers
// (16 channel groups at one block) and the readers (16 channels at one block) both spread over all banks.
template <int D>
struct Tile {
  static constexpr int KS = D + 8;  // key row stride (halves)
  uint16_t k[kTile * KS];
  uint16_t v[D * kTile];
};
MKV_DEV int vswz(int ch) { return (ch ^ (ch >> 3)) & 15; }
// Byte offset of block b of channel 16 m + lr, given that of m = 0: the swizzle of the channel is that of lr
// with 2 m xored in, so a read costs one xor (and its 2048 m goes into the instruction).
MKV_DEV uint32_t v_offset(uint32_t of_lr, int m) { return (of_lr ^ (16 * m & 127)) + 2 * kTile * 16 * m; }
template <int D>
MKV_DEV uint16_t *v_at(Tile<D> &t, int ch, int block) { return t.v + ch * kTile + 4 * (block ^ vswz(ch)); }
template <int D>
MKV_DEV void put_v(Tile<D> &t, int ch, int block, uint32_t t01, uint32_t t23) {
  *reinterpret_cast<uint2 *>(v_at(t, ch, block)) = make_uint2(t01, t23);
}
template <int D>
MKV_DEV void put_k8(Tile<D> &t, int token, int ch, const uint32_t *w) {
  *reinterpret_cast<uint4 *>(t.k + token * Tile<D>::KS + ch) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- tile loaders: fetch(tile, raw, carry) reads a tile's data into registers, kDepth tiles ahead of
// put(tile, raw, lds), which writes it as fp16 rows; fix(tile, raw, lds) (kFix, after a barrier) writes what
// replaces some of them.  Tokens at or past `n` get value rows of zero (their probabilities are 0, and 0 x
// anything must stay 0).  A quantized tile is a quarter of the bytes of fp16 rows, so more of them have to
// be on their way to cover the memory's latency.

// fp16 rows `stride` elements apart: a cache's, or the drafted ones
template <int D>
struct RowsLoader {
  static constexpr bool kFix = false;
  static constexpr int kDepth = 1;
  static constexpr int NK = D / 32, VPL = D / 16;  // key pieces, value channels per thread
  struct Carry {};
  const uint16_t *K, *V;
  int64_t stride;
  int n;
  struct Raw {
    uint4 k[NK];
    uint32_t v[4][VPL / 2];
  };
  MKV_DEV void start(int, Carry &) const {}
  MKV_DEV void put_tables() const {}
  MKV_DEV void fetch(int tile, Raw &r, Carry &) const {
    const int tid = threadIdx.x, last = n - 1;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int t = min(tile * kTile + tid / (D / 8) + i * (2048 / D), last);
      r.k[i] = gld16h(K + t * stride + 8 * (tid % (D / 8)));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = min(tile * kTile + 4 * (tid >> 4) + j, last);
      const uint16_t *p = V + t * stride + VPL * (tid & 15);
      if constexpr (VPL == 8) {
        const uint4 u = gld16h(p);
        r.v[j][0] = u.x;
        r.v[j][1] = u.y;
        r.v[j][2] = u.z;
        r.v[j][3] = u.w;
      } else {
        typedef uint32_t u32x2h __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2h u = *(const MKV_GLOBAL u32x2h *)p;
        r.v[j][0] = u[0];
        r.v[j][1] = u[1];
      }
    }
  }
  MKV_DEV void put(int tile, const Raw &r, Tile<D> &t) const {
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const uint32_t w[4] = {r.k[i].x, r.k[i].y, r.k[i].z, r.k[i].w};
      put_k8(t, tid / (D / 8) + i * (2048 / D), 8 * (tid % (D / 8)), w);
    }
    const int b = tid >> 4, left = n - (tile * kTile + 4 * b);
    const bool whole = (tile + 1) * kTile <= n;
#pragma unroll
    for (int i = 0; i < VPL / 2; ++i) {
      uint32_t x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = whole || j < left ? r.v[j][i] : 0u;
      const int ch = VPL * (tid & 15) + 2 * i;
      put_v(t, ch, b, pk_lo(x[0], x[1]), pk_lo(x[2], x[3]));
      put_v(t, ch + 1, b, pk_hi(x[0], x[1]), pk_hi(x[2], x[3]));
    }
  }
};

// Uniform 4-bit: a tile is one 64-token key block, the last one of an incomplete block fp16 rows.  A
// value is (min + 8 step) + (code - 8) step, one fused operation a pair in fp16: taken from the middle of
// the group's range, the step's rounding weighs as much as the value's own (from its minimum, codes of 7
// or 8 times the step would carry 2.5 times that into values near 0).  A tile's middles and steps are read
// and converted once, a thread per channel and per token group, one tile ahead of its codes, and put
// into LDS in the order of the code pairs.
template <int D>
struct UqLoader {
  static constexpr bool kFix = false;
  // (8 x 8192 tokens: within 3 % of one tile ahead at 1 to 64 nodes, either way.  The registers that it
  // takes lead the compiler to KVQuant tiles that are 5 % faster at 128 rows, in the same kernel.)
  static constexpr int kDepth = 2;
  static constexpr int NK = D / 32, NGRP = D / 64, NW = D / 32;
  const uint8_t *kc, *vc;
  const float *kmeta, *vmeta;
  const uint16_t *kres;
  int first_tile;
  uint16_t *meta;  // LDS: two buffers of key middles, key steps [D] and value middles, value steps [NGRP][64]
  int n;
  struct Carry {};
  struct Raw {
    uint32_t k[NK], v[NW];
    float mn, st;  // of the next tile: key channel tid, or value group (tid - D)
  };
  MKV_DEV void fetch_meta(int tile, float &mn, float &st) const {
    const int tid = threadIdx.x;
    mn = st = 0.f;
    const float *p = nullptr;
    if (tid < D) {
      if ((tile + 1) * kTile <= n) p = kmeta + ((int64_t)tile * D + tid) * 2;
    } else if (tid < 2 * D && tile * kTile + (tid - D) / NGRP < n) {
      p = vmeta + ((int64_t)tile * kTile * NGRP + tid - D) * 2;
    }
    if (p) {
      const f2v x = gld(reinterpret_cast<const f2v *>(p));
      mn = x[0];
      st = x[1];
    }
  }
  MKV_DEV void put_meta(int tile, float mn, float st) const {
    const int tid = threadIdx.x;
    if (tid >= 2 * D) return;
    uint16_t *buf = meta + (tile & 1) * 4 * D;
    int at;
    if (tid < D) {
      at = (tid & ~7) + 2 * (tid & 3) + ((tid >> 2) & 1);  // channels (0, 4), (1, 5), (2, 6), (3, 7) of 8
    } else {
      const int e = tid - D;
      at = 2 * D + (e % NGRP) * kTile + e / NGRP;
    }
    // (where the range may end within a rounding of fp16's, middle and step are rounded towards 0: rounded
    // up they can take a code's value past 65504, which is the greatest of the group then)
    const float mid = __builtin_fmaf(8.f, st, mn);
    const bool far = fabsf(mid) + 8.f * st > 65408.f;
    buf[at] = far ? f2h_toward_0(mid) : f2h_bits(mid);
    buf[at + D] = far ? f2h_toward_0(st) : f2h_bits(st);
  }
  float mn0, st0;  // the first tile's, until they are in LDS
  MKV_DEV void start(int tile, Carry &) {
    first_tile = tile;
    fetch_meta(tile, mn0, st0);
  }
  MKV_DEV void put_tables() const { put_meta(first_tile, mn0, st0); }
  MKV_DEV void fetch(int tile, Raw &r, Carry &) const {
    const int tid = threadIdx.x, w = tid % (D / 8);
    if ((tile + 1) * kTile <= n) {
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int t = tid / (D / 8) + i * (2048 / D);
        r.k[i] = gld(reinterpret_cast<const uint32_t *>(kc + (int64_t)(tile * kTile + t) * (D / 2)) + w);
      }
    }
    const int t0 = min(tile * kTile + 4 * (tid >> 4), (n - 1) & ~3);  // (slots come in fours)
    const uint32_t *vp = reinterpret_cast<const uint32_t *>(vc + (int64_t)t0 * (D / 2) + (tid & 15) * (D / 8));
#pragma unroll
    for (int i = 0; i < NW; ++i) r.v[i] = gld(vp + i);
    fetch_meta(tile + 1, r.mn, r.st);
  }
  MKV_DEV void put(int tile, const Raw &r, Tile<D> &t) const {
    const int tid = threadIdx.x, w = tid % (D / 8);
    const uint16_t *buf = meta + (tile & 1) * 4 * D;
    if ((tile + 1) * kTile <= n) {
      const uint4 mid = *reinterpret_cast<const uint4 *>(buf + 8 * w), st = *reinterpret_cast<const uint4 *>(buf + D + 8 * w);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const uint32_t x0 = pk_fma(nib_pair(r.k[i], 0), st.x, mid.x), x1 = pk_fma(nib_pair(r.k[i], 1), st.y, mid.y);
        const uint32_t x2 = pk_fma(nib_pair(r.k[i], 2), st.z, mid.z), x3 = pk_fma(nib_pair(r.k[i], 3), st.w, mid.w);
        const uint32_t o[4] = {pk_lo(x0, x1), pk_lo(x2, x3), pk_hi(x0, x1), pk_hi(x2, x3)};
        put_k8(t, tid / (D / 8) + i * (2048 / D), 8 * w, o);
      }
    } else {  // (the last tile of a sequence at most)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int token = tid / (D / 8) + i * (2048 / D);
        const uint4 u = gld16(kres + token * D + 8 * w);
        const uint32_t o[4] = {u.x, u.y, u.z, u.w};
        put_k8(t, token, 8 * w, o);
      }
    }
    const int b = tid >> 4, rr = tid & 15;
#pragma unroll
    for (int g = 0; g < NGRP; ++g) {
      const uint2 mid = *reinterpret_cast<const uint2 *>(buf + 2 * D + g * kTile + 4 * b);
      const uint2 st = *reinterpret_cast<const uint2 *>(buf + 3 * D + g * kTile + 4 * b);
#pragma unroll
      for (int c = 0; c < 4; ++c) {  // channel 64 g + 4 rr + c: operand 4 g + c of the segment
        const uint32_t word = r.v[(4 * g + c) >> 1];
        put_v(t, 64 * g + 4 * rr + c, b, pk_fma(nib_pair(word, 2 * (c & 1)), st.x, mid.x),
              pk_fma(nib_pair(word, 2 * (c & 1) + 1), st.y, mid.y));
      }
    }
    put_meta(tile + 1, r.mn, r.st);
  }
};

// KVQuant: codes through tables of fp16 pairs (or, at 2 bits, quads), times the channel's threshold
// (keys) or the token's scale (values), which are fp16 values themselves; then the outliers.  A codebook may
// go past 1, and its values past fp16's end: keys and values are then held times a power of two (cb_scale),
// which goes into the tables and comes off the logits and outputs in float32.
template <int D, int BITS>
struct KvqLoader {
  static constexpr bool kFix = true;
  // (two tiles ahead it is no faster: 8 x 8192 tokens of 4 bits, 8 nodes, 52.2 us against 49.6.  Its
  // table lookups keep the LDS busy half the time)
  static constexpr int kDepth = 1;
  static constexpr int UK = kTile * D / 32, UV = kTile / 4 * D / 8;  // units of 32 keys, of 8 channels x 4 tokens
  const uint8_t *kc, *vc;
  const uint32_t *krow, *kout, *vout;
  const float *vsc;
  uint32_t *lutk, *lutv;  // LDS
  uint32_t *tau;          // LDS: thresholds of channel pairs
  float kscale, vscale;   // powers of two, at most 1
  uint32_t scales;        // both as fp16, in a scalar register
  uint4 lut4;             // this thread's part of the tables and thresholds until they are in LDS
  uint32_t tau2;
  int n, cap, nov, rowbytes;
  bool outliers;
  // the tile's range of key outliers, and where its second 32 tokens begin; read one tile ahead of the
  // entries themselves
  struct Range {
    uint32_t e0, emid, e1;
  };
  typedef Range Carry;
  struct Raw {
    uint32_t k[BITS], v[BITS];
    float s[4];
    Range r;
    uint32_t ko, vo;  // this thread's first key and value outlier
  };
  MKV_DEV Range range(int tile) const {
    return {gld(krow + min(tile * kTile, n)), gld(krow + min(tile * kTile + 32, n)), gld(krow + min(tile * kTile + 64, n))};
  }
  MKV_DEV void start(int tile, Carry &next) const { next = range(tile); }
  // The tables are read with the first tile and put into LDS behind its loads (all threads).
  MKV_DEV void load_tables(const float *cbtab, const float *kmeta) {
    static_assert(kTreeThreads * 4 >= 1024, "both tables of a codebook: one piece per thread");
    const int tid = threadIdx.x;
    lut4 = make_uint4(0u, 0u, 0u, 0u);
    kscale = cbtab[cb_scale(BITS)];
    vscale = cbtab[cb_scale(BITS) + 1];
    scales = __builtin_amdgcn_readfirstlane(pk_f16(kscale, vscale));
    if (tid < lut_half_words(BITS) / 2)
      lut4 = gld16(reinterpret_cast<const uint32_t *>(cbtab + kLutBase) + lut_offset(BITS) + 4 * tid);
    tau2 = tid < D / 2 ? pk_f16(gld(kmeta + 4 * tid), gld(kmeta + 4 * tid + 2)) : 0u;
  }
  MKV_DEV void put_tables() const {
    const int tid = threadIdx.x;
    if (tid < lut_half_words(BITS) / 2) {
      const float f = 4 * tid < lut_half_words(BITS) ? kscale : vscale;
      const uint32_t ff = pk_f16(f, f);
      reinterpret_cast<uint4 *>(lutk)[tid] =
          make_uint4(pk_mul(lut4.x, ff), pk_mul(lut4.y, ff), pk_mul(lut4.z, ff), pk_mul(lut4.w, ff));
    }
    if (tid < D / 2) tau[tid] = tau2;
  }
  MKV_DEV void fetch(int tile, Raw &r, Carry &next) const {
    const int tid = threadIdx.x;
    if (UK == kTreeThreads || tid < UK) {
      const int t = min(tile * kTile + tid / (D / 32), n - 1);
      const uint32_t *p = reinterpret_cast<const uint32_t *>(kc + (int64_t)t * rowbytes) + BITS * (tid % (D / 32));
#pragma unroll
      for (int i = 0; i < BITS; ++i) r.k[i] = gld(p + i);
    }
    if (UV == kTreeThreads || tid < UV) {
      const int t0 = min(tile * kTile + 4 * (tid / (D / 8)), (n - 1) & ~3);
      const uint32_t *p = reinterpret_cast<const uint32_t *>(vc + (int64_t)t0 * rowbytes) + BITS * (tid % (D / 8));
#pragma unroll
      for (int i = 0; i < BITS; ++i) r.v[i] = gld(p + i);
      const U4 s = gld16u(vsc + t0);
      r.s[0] = __builtin_bit_cast(float, s.x);
      r.s[1] = __builtin_bit_cast(float, s.y);
      r.s[2] = __builtin_bit_cast(float, s.z);
      r.s[3] = __builtin_bit_cast(float, s.w);
    }
    if (!outliers) return;
    r.r = next;
    if (r.r.e0 + tid < r.r.e1) r.ko = gld(kout + r.r.e0 + tid);
    if (tid < kTile) r.vo = gld(vout + min(tile * kTile + tid, n - 1));
    next = range(tile + 1);
  }
  // bits [at, at + 2 BITS) of a unit, as the packed pair they stand for
  MKV_DEV uint32_t pair(const uint32_t *lut, const uint32_t (&w)[BITS], int f) const {
    const int bit = 2 * BITS * f, i = bit >> 5, s = bit & 31;
    const uint32_t x = s + 2 * BITS <= 32 ? w[i] >> s : __builtin_amdgcn_alignbit(w[min(i + 1, BITS - 1)], w[i], s);
    return lut[x & ((1 << (2 * BITS)) - 1)];
  }
  // the quad of codes f as two packed pairs
  MKV_DEV uint2 quad(const uint32_t *lut, const uint32_t (&w)[BITS], int f) const {
    if constexpr (BITS == 2) return *reinterpret_cast<const uint2 *>(lut + 2 * ((w[f >> 2] >> (8 * (f & 3))) & 0xFFu));
    else return make_uint2(pair(lut, w, 2 * f), pair(lut, w, 2 * f + 1));
  }
  MKV_DEV void put(int tile, const Raw &r, Tile<D> &t) const {
    const int tid = threadIdx.x;
    if (UK == kTreeThreads || tid < UK) {
      const int token = tid / (D / 32), ch = 32 * (tid % (D / 32));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 a = quad(lutk, r.k, 2 * i), b = quad(lutk, r.k, 2 * i + 1);
        const uint4 u = *reinterpret_cast<const uint4 *>(tau + ch / 2 + 4 * i);
        const uint32_t o[4] = {pk_mul(a.x, u.x), pk_mul(a.y, u.y), pk_mul(b.x, u.z), pk_mul(b.y, u.w)};
        put_k8(t, token, ch + 8 * i, o);
      }
    }
    if (UV == kTreeThreads || tid < UV) {
      const int b = tid / (D / 8), ch = 8 * (tid % (D / 8)), left = n - (tile * kTile + 4 * b);
      float s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = j < left ? r.s[j] : 0.f;
      const uint32_t s01 = pk_f16(s[0], s[1]), s23 = pk_f16(s[2], s[3]);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint2 a = quad(lutv, r.v, c);
        put_v(t, ch + c, b, pk_mul(a.x, s01), pk_mul(a.y, s23));
      }
    }
  }
  MKV_DEV void fix(int tile, const Raw &r, Tile<D> &t) const {
    const int tid = threadIdx.x;
    const _Float16 ks = __builtin_bit_cast(h2v, scales)[0], vs = __builtin_bit_cast(h2v, scales)[1];
    auto scaled = [](uint32_t x, _Float16 s) {
      return __builtin_bit_cast(uint16_t, (_Float16)(__builtin_bit_cast(_Float16, (uint16_t)(x >> 16)) * s));
    };
    auto key = [&](uint32_t e, uint32_t x) {
      const int token = (outlier_tag(x) & 31) + (e >= r.r.emid ? 32 : 0);
      t.k[token * Tile<D>::KS + min(outlier_ch(x), D - 1)] = scaled(x, ks);
    };
    auto value = [&](int token, uint32_t x) {
      if (x != kNoOutlier) v_at(t, min(outlier_ch(x), D - 1), token >> 2)[token & 3] = scaled(x, vs);
    };
    if (r.r.e0 + tid < r.r.e1) key(r.r.e0 + tid, r.ko);
    for (uint32_t e = r.r.e0 + kTreeThreads + tid; e < r.r.e1; e += kTreeThreads) key(e, gld(kout + e));
    const int left = min(kTile, n - tile * kTile);
    if (tid < left) value(tid, r.vo);
    for (int i = kTile + tid; i < kTile * nov; i += kTreeThreads)  // (further slots)
      if ((i & 63) < left) value(i & 63, gld(vout + (int64_t)(i >> 6) * cap + tile * kTile + (i & 63)));
  }
};

// ---- the attention ------------------------------------------------------------------------------------
// Waves: WR of them take 16 RB rows each, and WT = 4 / WR share a tile's tokens.
template <int D, int RB, int WR>
struct TG {
  static constexpr int WT = 4 / WR, TW = kTile / WT, R = 16 * RB * WR;
  static constexpr int NB = TW == 16 ? 1 : 2;  // 16-token blocks of one step
  static constexpr int NM = D / 16, NQ = D / 32;
};

// A wave's rows: row 16 rb + lane % 16 of each lane, and what it has summed.
template <int D, int RB, int WR>
struct Rows {
  using G_ = TG<D, RB, WR>;
  h8v q[G_::NQ][RB];
  f4v o[G_::NM][RB];
  float m[RB], l[RB];
  unsigned long long mask[RB];  // the nodes that the row attends to
  bool any;                     // some row exists (the same in all lanes)
};

// The wave's tokens of a tile in LDS: all their logits, one move of the references, then the output 32 tokens
// at a time, so that one step's exponentials can run under the products of the one before (2-6 % less than
// logits 32 tokens at a time; two tiles in LDS with one barrier a tile gained nothing, and key rows without
// bank conflicts instead of padded ones cost more address registers than they gained).  References and
// logits are kept unscaled; the scale (and log2 e) enters with the reference in one fused operation before
// the exponential.
// Tokens at or past `left` do not exist; MASKED: nor does, for a row, a token that its mask does not name.
template <int D, int RB, int WR, bool MASKED>
MKV_DEV void attend_tile(Tile<D> &t, Rows<D, RB, WR> &x, int left, float qscale) {
  using C = TG<D, RB, WR>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int tok0 = (wave % C::WT) * C::TW;
  const float lazy = kLazy / qscale;
  constexpr int NT = C::TW / 16;  // 16-token blocks
  // a wave at its products goes before one that brings in the next tile (3-6 % over many rows)
  __builtin_amdgcn_s_setprio(1);
  f4v S[NT][RB];
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) S[b][rb] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int m = 0; m < C::NQ; ++m) {
      const h8v a = *reinterpret_cast<const h8v *>(t.k + (tok0 + 16 * b + lr) * Tile<D>::KS + 32 * m + 8 * lq);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) S[b][rb] = mfma32(a, x.q[m][rb], S[b][rb]);
    }
  if (MASKED || tok0 + C::TW > left) {
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int token = tok0 + 16 * b + 4 * lq + i;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          S[b][rb][i] = token < left && (!MASKED || ((x.mask[rb] >> token) & 1)) ? S[b][rb][i] : -INFINITY;
      }
  }
  float mx[RB];
  bool move = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    mx[rb] = -INFINITY;
#pragma unroll
    for (int b = 0; b < NT; ++b) {
      mx[rb] = fmaxf(fmaxf(mx[rb], S[b][rb][0]), S[b][rb][1]);
      mx[rb] = fmaxf(fmaxf(mx[rb], S[b][rb][2]), S[b][rb][3]);
    }
    move |= mx[rb] > x.m[rb] + lazy;
  }
  if (__any(move)) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float y = fmaxf(mx[rb], __shfl_xor(mx[rb], 16));
      y = fmaxf(y, __shfl_xor(y, 32));
      const bool up = y > x.m[rb];
      const float corr = up ? fexp2((x.m[rb] - y) * qscale) : 1.f;
      if (up) x.m[rb] = y;
      x.l[rb] *= corr;
#pragma unroll
      for (int m = 0; m < C::NM; ++m) x.o[m][rb] *= corr;
    }
  }
  const char *vt = reinterpret_cast<const char *>(t.v);
#pragma unroll
  for (int u = 0; u < NT / C::NB; ++u) {
    const int first = tok0 + 16 * C::NB * u;
    uint32_t P[RB][2 * C::NB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      // (a row that has seen nothing yet has no reference, and only logits of -infinity)
      const float ref = x.m[rb] == -INFINITY ? 0.f : __builtin_fmaf(-x.m[rb], qscale, kLift);
#pragma unroll
      for (int b = 0; b < C::NB; ++b) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fexp2(__builtin_fmaf(S[u * C::NB + b][rb][i], qscale, ref));
        x.l[rb] += (p[0] + p[1]) + (p[2] + p[3]);
        P[rb][2 * b] = pk_f16(p[0], p[1]);
        P[rb][2 * b + 1] = pk_f16(p[2], p[3]);
      }
    }
    const uint32_t v0 = 2 * kTile * lr + 8 * ((first / 4 + lq) ^ vswz(lr));
#pragma unroll
    for (int m = 0; m < C::NM; ++m) {
      const uint2 a0 = *reinterpret_cast<const uint2 *>(vt + v_offset(v0, m));
      if constexpr (C::NB == 2) {  // (first is a multiple of 32 tokens: 4 blocks on is bit 2 of the block)
        const uint2 a1 = *reinterpret_cast<const uint2 *>(vt + v_offset(v0 ^ 32, m));
        const h8v a = __builtin_bit_cast(h8v, make_uint4(a0.x, a0.y, a1.x, a1.y));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          x.o[m][rb] = mfma32(a, __builtin_bit_cast(h8v, make_uint4(P[rb][0], P[rb][1], P[rb][2], P[rb][3])), x.o[m][rb]);
      } else {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          x.o[m][rb] = mfma16(__builtin_bit_cast(h4v, a0), __builtin_bit_cast(h4v, make_uint2(P[rb][0], P[rb][1])), x.o[m][rb]);
      }
    }
  }
  __builtin_amdgcn_s_setprio(0);
}

// Tiles [begin, end) of the cache, each tile's loads issued before the kDepth tiles ahead of it are computed;
// `first()` runs after the first loads are on their way.
template <int D, int RB, int WR, class L, class F>
MKV_DEV void attend_range(L &ld, Tile<D> &t, Rows<D, RB, WR> &x, int begin, int end, float qscale, F first) {
  typename L::Raw raw[L::kDepth];
  typename L::Carry carry;
  if (begin < end) {
    ld.start(begin, carry);
#pragma unroll
    for (int i = 0; i < L::kDepth; ++i)
      if (begin + i < end) ld.fetch(begin + i, raw[i], carry);
    ld.put_tables();
  }
  first();
  __syncthreads();  // (the tables)
  for (int tile = begin; tile < end;) {
#pragma unroll
    for (int i = 0; i < L::kDepth; ++i) {
      if (tile >= end) break;  // (the same in all threads)
      ld.put(tile, raw[i], t);
      __syncthreads();
      if constexpr (L::kFix) {
        if (ld.outliers) {
          ld.fix(tile, raw[i], t);
          __syncthreads();
        }
      }
      if (tile + L::kDepth < end) ld.fetch(tile + L::kDepth, raw[i], carry);
      if (x.any) attend_tile<D, RB, WR, false>(t, x, ld.n - tile * kTile, qscale);
      __syncthreads();
      ++tile;
    }
  }
}

MKV_DEV float uniform(float x) {  // (in a scalar register)
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}
MKV_DEV float pow2_inverse(float x) { return __builtin_bit_cast(float, 0x7F000000u - __builtin_bit_cast(uint32_t, x)); }

// A weighted mean as fp16.  The weights' roundings can take it past the values it is a mean of by 2^-11: not
// past the last finite one, which would round to infinity.
MKV_DEV uint16_t mean_bits(float x) {
  constexpr float kLast = 65504.f, kPast = kLast * (1.f + 2.f / 2048.f);
  return f2h_bits(fabsf(x) < kPast ? fminf(fmaxf(x, -kLast), kLast) : x);
}

// What the kernel and the merge need to agree on.
struct TreeGeo {
  int Hkv, G, N, max_splits, chunk, max_new, items, row_blocks, S, even;  // even: all sequences have max_splits
};
// Splits of sequence s (a tile range each, by its capacity), and its first slot among all sequences'.
MKV_DEV int splits_of(const SeqDesc &sd, const TreeGeo &g) { return (sd.cap + g.chunk - 1) / g.chunk; }
MKV_DEV int64_t first_split(const SeqDesc &sd, int s, const TreeGeo &g) {
  // capacities are at most n0 + max_new + 3, so this many splits lie before it
  return (sd.row0 + (int64_t)s * (g.max_new + 3)) / g.chunk + s;
}
// A sequence's tiles, its drafted tokens being the last one, are dealt to its splits as evenly as they go.
struct TileRange {
  int begin, end;
};
MKV_DEV int tiles_of(int n) { return (n + kTile - 1) / kTile + 1; }
MKV_DEV TileRange tile_range(int tiles, int splits, int split) {
  const int q = tiles / splits, r = tiles % splits, begin = split * q + min(split, r);
  return {begin, begin + q + (split < r ? 1 : 0)};
}
// Which (sequence, kv head, split) an item is: the splits of a head next to each other, the heads of a
// sequence next.  Only splits that exist are launched: a workgroup that ends at once takes its place on the
// card before one that has work, which then waits (8 sequences of 3293 to 5398 tokens, 24 nodes: 67 us with
// one item per sequence, head and split of the longest).
struct Item {
  int s, h, split;
};
MKV_DEV Item item_of(int item, const SeqDesc *seqs, const TreeGeo &g) {
  if (g.even) return {item / g.max_splits / g.Hkv, item / g.max_splits % g.Hkv, item % g.max_splits};
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < g.S; s0 += 64) {
    const int mine = s0 + lane < g.S ? g.Hkv * ((gld(&seqs[s0 + lane].cap) + g.chunk - 1) / g.chunk) : 0;
    const int upto = wave_incl_scan(mine), all = __builtin_amdgcn_readlane(upto, 63);
    if (item < all) {
      const int l = __builtin_ctzll(__ballot(item < upto)), heads = __builtin_amdgcn_readlane(mine, l);
      const int splits = heads / g.Hkv, at = item - (__builtin_amdgcn_readlane(upto, l) - heads);
      return {s0 + l, at / splits, at % splits};
    }
    item -= all;
  }
  return {0, 0, 0};  // (no item is past the last sequence)
}

template <int D, int RB, int WR>
__global__ __launch_bounds__(kTreeThreads, RB == 2 ? 2 : 3) void k_tree_attn(const SeqDesc *__restrict__ seqs,
                                                            const int32_t *__restrict__ state,
                                                            const float *__restrict__ cbtab, TreeArgs a, TreeGeo geo,
                                                            float qscale) {
  using C = TG<D, RB, WR>;
  constexpr int R = C::R, WT = C::WT, NM = C::NM;
  __shared__ __attribute__((aligned(16))) Tile<D> tile;
  __shared__ __attribute__((aligned(16))) uint32_t s_lut[1024];
  __shared__ __attribute__((aligned(16))) uint32_t s_tau[D / 2];
  __shared__ float s_m[WT][R], s_l[WT][R];
  static_assert(WT == 1 || sizeof(float) * R * D <= sizeof(tile), "the waves' outputs are merged in the tile");
  const int item = blockIdx.x, yb = blockIdx.y;
  if (item >= geo.items) return;
  const Item it = item_of(item, seqs, geo);
  const int s = __builtin_amdgcn_readfirstlane(it.s), h = __builtin_amdgcn_readfirstlane(it.h);  // (in scalar registers)
  const int split = __builtin_amdgcn_readfirstlane(it.split);
  const SeqDesc &sd = seqs[s];
  const int n = state[((int64_t)s * geo.Hkv + h) * ST_WORDS + ST_COUNT];
  const int N = geo.N, G = geo.G, Hq = geo.Hkv * G;
  const int valid = a.n_valid ? min(max(a.n_valid[s], 0), N) : N;
  if (yb * R >= valid * G) return;
  const int tiles = tiles_of(n);
  const TileRange mine = tile_range(tiles, splits_of(sd, geo), split);
  if (mine.begin == mine.end) return;
  const bool tree = mine.end == tiles;
  const int begin = mine.begin, end = tree ? tiles - 1 : mine.end;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lq = lane >> 4;
  const int wr = wave / WT, wt = wave % WT;
  Rows<D, RB, WR> x;
  x.any = yb * R + wr * RB * 16 < valid * G;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = yb * R + (wr * RB + rb) * 16 + lr, node = row / G;
    const bool on = node < valid;
    const uint16_t *qp = a.q + (((int64_t)s * N + (on ? node : 0)) * Hq + h * G + row % G) * D;
#pragma unroll
    for (int m = 0; m < C::NQ; ++m) {
      const uint4 u = gld16h(qp + 32 * m + 8 * lq);
      x.q[m][rb] = __builtin_bit_cast(h8v, on ? u : make_uint4(0u, 0u, 0u, 0u));
    }
    // (bits of nodes that do not exist are dropped)
    x.mask[rb] = on && tree ? gld(a.mask + (int64_t)s * N + node) & (~0ull >> (64 - valid)) : 0ull;
    x.m[rb] = -INFINITY;
    x.l[rb] = 0.f;
#pragma unroll
    for (int m = 0; m < NM; ++m) x.o[m][rb] = f4v{0.f, 0.f, 0.f, 0.f};
  }
  // the drafted tokens, whose loads are issued first
  RowsLoader<D> nodes;
  nodes.K = a.k + ((int64_t)s * N * geo.Hkv + h) * D;
  nodes.V = a.v + ((int64_t)s * N * geo.Hkv + h) * D;
  nodes.stride = (int64_t)geo.Hkv * D;
  nodes.n = valid;
  typename RowsLoader<D>::Raw nraw;
  typename RowsLoader<D>::Carry none;
  if (tree) nodes.fetch(0, nraw, none);
  auto attend_nodes = [&](uint32_t vscale_pair) __attribute__((always_inline)) {
    if (!tree) return;
    // A value that is infinite or NaN must reach only the rows that attend to its node: it is left out
    // of the product, where a probability of 0 would make it NaN, and added to those rows.
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint32_t w = nraw.v[j][i];
        const uint32_t bad = ((w & 0x7C00u) == 0x7C00u ? 0xFFFFu : 0u) | ((w & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u);
        odd |= bad != 0u;
        nraw.v[j][i] = pk_mul(w & ~bad, vscale_pair);
      }
    nodes.put(0, nraw, tile);
    const bool any_odd = __syncthreads_or(odd);
    if (x.any) attend_tile<D, RB, WR, true>(tile, x, valid, qscale);
    if (any_odd) {  // (by the waves that have the node's logit, and with it a maximum)
      for (int j = wt * C::TW; j < min(valid, (wt + 1) * C::TW); ++j)
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = gld(nodes.V + j * nodes.stride + 16 * m + 4 * lq + i);
            if ((w & 0x7C00u) != 0x7C00u) continue;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              if ((x.mask[rb] >> j) & 1) x.o[m][rb][i] += h2f(w);
          }
    }
    __syncthreads();
  };
  float vscale = 1.f;  // what the outputs are times
  if (sd.method == FP16) {
    RowsLoader<D> ld;
    ld.K = reinterpret_cast<const uint16_t *>(sd.k) + h * stride_rows(sd, D);
    ld.V = reinterpret_cast<const uint16_t *>(sd.v) + h * stride_rows(sd, D);
    ld.stride = D;
    ld.n = n;
    attend_range<D, RB, WR>(ld, tile, x, begin, end, qscale, [&]() __attribute__((always_inline)) { attend_nodes(kOnePair); });
  } else if (sd.method == UQ) {
    UqLoader<D> ld;
    ld.kc = reinterpret_cast<const uint8_t *>(sd.kc) + h * stride_codes(sd);
    ld.vc = reinterpret_cast<const uint8_t *>(sd.vc) + h * stride_codes(sd);
    ld.kmeta = reinterpret_cast<const float *>(sd.kmeta) + h * stride_uq_kmeta(sd, D) * 2;
    ld.vmeta = reinterpret_cast<const float *>(sd.vmeta) + h * stride_uq_vmeta(sd, D) * 2;
    ld.kres = reinterpret_cast<const uint16_t *>(sd.kres) + (int64_t)h * kTile * D;
    ld.meta = reinterpret_cast<uint16_t *>(s_lut);
    ld.n = n;
    attend_range<D, RB, WR>(ld, tile, x, begin, end, qscale, [&]() __attribute__((always_inline)) { attend_nodes(kOnePair); });
  } else {
    auto run = [&](auto bits_tag) {
      constexpr int BITS = decltype(bits_tag)::value;
      KvqLoader<D, BITS> ld;
      ld.kc = reinterpret_cast<const uint8_t *>(sd.kc) + h * stride_codes(sd);
      ld.vc = reinterpret_cast<const uint8_t *>(sd.vc) + h * stride_codes(sd);
      ld.krow = reinterpret_cast<const uint32_t *>(sd.krow) + h * stride_krow(sd);
      ld.kout = reinterpret_cast<const uint32_t *>(sd.kout) + h * stride_kout(sd);
      ld.vout = reinterpret_cast<const uint32_t *>(sd.vout) + h * stride_vout(sd);
      ld.vsc = reinterpret_cast<const float *>(sd.vmeta) + h * stride_slots(sd);
      ld.lutk = s_lut;
      ld.lutv = s_lut + lut_half_words(BITS);
      ld.tau = s_tau;
      ld.n = n;
      ld.cap = sd.cap;
      ld.nov = sd.nov_slots;
      ld.rowbytes = sd.rowbytes;
      ld.outliers = sd.bp > 0;
      ld.load_tables(cbtab, reinterpret_cast<const float *>(sd.kmeta) + (int64_t)h * D * 2);
      // (the drafted values are scaled as the cache's are, the keys are not: the references of their logits are
      // before the cache's, and all of them back behind it)
      const float kback = pow2_inverse(ld.kscale);
      attend_range<D, RB, WR>(ld, tile, x, begin, end, uniform(qscale * kback), [&]() __attribute__((always_inline)) {
        attend_nodes(pk_hi(ld.scales, ld.scales));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x.m[rb] *= ld.kscale;
      });
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) x.m[rb] *= kback;
      vscale = ld.vscale;
    };
    if (sd.bits == 4) run(std::integral_constant<int, 4>{});
    else if (sd.bits == 3) run(std::integral_constant<int, 3>{});
    else run(std::integral_constant<int, 2>{});
  }
  // a row's four quads hold disjoint tokens
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    x.l[rb] += __shfl_xor(x.l[rb], 16);
    x.l[rb] += __shfl_xor(x.l[rb], 32);
    x.l[rb] *= vscale;  // (l is what o is divided by)
    x.m[rb] = __builtin_fmaf(x.m[rb], qscale, -kLift);  // from here on in log2, of what l and o are sums over
  }
  if constexpr (WT > 1) {
    // the waves that share rows: scaled to their common reference, then summed into the first
    if (lq == 0) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s_m[wt][(wr * RB + rb) * 16 + lr] = x.m[rb];
        s_l[wt][(wr * RB + rb) * 16 + lr] = x.l[rb];
      }
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = (wr * RB + rb) * 16 + lr;
      float M = s_m[0][row];
#pragma unroll
      for (int w = 1; w < WT; ++w) M = fmaxf(M, s_m[w][row]);
      float Ls = 0.f;
      // (without a maximum nothing was summed, or only NaN, which no maximum sees: it stays either way)
#pragma unroll
      for (int w = 0; w < WT; ++w) Ls += s_m[w][row] == -INFINITY ? s_l[w][row] : s_l[w][row] * fexp2(s_m[w][row] - M);
      const float f = x.m[rb] == -INFINITY ? 1.f : fexp2(x.m[rb] - M);
#pragma unroll
      for (int m = 0; m < NM; ++m) x.o[m][rb] *= f;
      x.m[rb] = M;
      x.l[rb] = Ls;
    }
    float *red = reinterpret_cast<float *>(&tile);
#pragma unroll 1
    for (int w = 1; w < WT; ++w) {
      if (wt == w) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int m = 0; m < NM; ++m)
            *reinterpret_cast<f4v *>(red + ((((wr * RB + rb) * NM + m) * 64) + lane) * 4) = x.o[m][rb];
      }
      __syncthreads();
      if (wt == 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int m = 0; m < NM; ++m)
            x.o[m][rb] += *reinterpret_cast<const f4v *>(red + ((((wr * RB + rb) * NM + m) * 64) + lane) * 4);
      }
      __syncthreads();
    }
    if (wt != 0) return;
  }
  if (geo.max_splits == 1) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = yb * R + (wr * RB + rb) * 16 + lr, node = row / G;
      if (node >= valid) continue;
      const float inv = 1.f / x.l[rb];
      uint16_t *op = a.out + (((int64_t)s * N + node) * Hq + h * G + row % G) * D;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) gst(op + 16 * m + 4 * lq + i, mean_bits(x.o[m][rb][i] * inv));
    }
    return;
  }
  float *part = a.workspace + (((first_split(sd, s, geo) + split) * geo.Hkv + h) * geo.row_blocks + yb) * (int64_t)(R * (D + 2));
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = (wr * RB + rb) * 16 + lr;
#pragma unroll
    for (int m = 0; m < NM; ++m) gst(reinterpret_cast<f4v *>(part + row * D + 16 * m + 4 * lq), x.o[m][rb]);
    if (lq == 0) gst(reinterpret_cast<f2v *>(part + R * D + row * 2), f2v{x.m[rb], x.l[rb]});
  }
}

// Merge of the splits: a thread takes 4 channels of a row, the loads of 8 splits at a time.
constexpr int kMergeLoads = 8;
template <int D>
__global__ __launch_bounds__(256) void k_tree_merge(const SeqDesc *__restrict__ seqs, const int32_t *__restrict__ state,
                                                    TreeArgs a, TreeGeo geo, int R) {
  constexpr int TPR = D / 4;  // threads per row
  const int N = geo.N, G = geo.G, Hq = geo.Hkv * G;
  const int blocks = (N * G + 256 / TPR - 1) / (256 / TPR);  // per (sequence, kv head)
  const int sh = blockIdx.x / blocks, h = sh % geo.Hkv, s = sh / geo.Hkv;
  const int row = (blockIdx.x % blocks) * (256 / TPR) + threadIdx.x / TPR, node = row / G, c = threadIdx.x % TPR * 4;
  const int valid = a.n_valid ? min(max(a.n_valid[s], 0), N) : N;
  if (node >= valid) return;
  const SeqDesc &sd = seqs[s];
  const int n = state[((int64_t)s * geo.Hkv + h) * ST_WORDS + ST_COUNT];
  const int used = min(splits_of(sd, geo), tiles_of(n));
  const int64_t step = (int64_t)geo.Hkv * geo.row_blocks * R * (D + 2);
  const float *part = a.workspace + ((first_split(sd, s, geo) * geo.Hkv + h) * geo.row_blocks + row / R) * (int64_t)(R * (D + 2));
  const float *ml = part + R * D + (row % R) * 2, *o = part + (row % R) * D + c;
  float M = -INFINITY, Ls = 0.f;
  f4v acc = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < used; p0 += kMergeLoads) {
    f2v x[kMergeLoads];  // (maximum, sum)
    f4v v[kMergeLoads];
#pragma unroll
    for (int i = 0; i < kMergeLoads; ++i) {
      const int64_t at = min(p0 + i, used - 1) * step;
      x[i] = gld(reinterpret_cast<const f2v *>(ml + at));
      v[i] = gld(reinterpret_cast<const f4v *>(o + at));
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kMergeLoads; ++i) top = fmaxf(top, x[i][0]);
    const float old = M == -INFINITY ? 0.f : fexp2(M - top);
    Ls *= old;
    acc *= old;
    M = top;
#pragma unroll
    for (int i = 0; i < kMergeLoads; ++i) {
      const float m = x[i][0];
      if (p0 + i >= used) continue;
      const float w = m == -INFINITY ? 1.f : fexp2(m - M);  // (no maximum: zeros, or NaN that is to be seen)
      Ls += x[i][1] * w;
      acc += v[i] * w;
    }
  }
  uint16_t *op = a.out + (((int64_t)s * N + node) * Hq + h * G + row % G) * D + c;
  const float inv = 1.f / Ls;
#pragma unroll
  for (int i = 0; i < 4; ++i) gst(op + i, mean_bits(acc[i] * inv));
}

template <int D, int RB, int WR>
hipError_t tree_impl(const Dev &dv, const Shape &sh, const TreePlan &plan, const TreeArgs &a, hipStream_t st) {
  const int items = plan.splits * sh.Hkv;
  const TreeGeo geo{sh.Hkv,   sh.G,  a.n_nodes,       plan.max_splits, plan.chunk,
                    sh.max_new, items, plan.row_blocks, sh.S,            plan.splits == sh.S * plan.max_splits};
  // the row blocks of a range are a multiple of 8 workgroups apart: on one XCD, whose L2 then holds the
  // range for all of them
  const dim3 grid((items + 7) & ~7, plan.row_blocks);
  hipLaunchKernelGGL((k_tree_attn<D, RB, WR>), grid, dim3(kTreeThreads), 0, st, dv.seqs, dv.state, dv.cbtab, a, geo,
                     kLog2e / sqrtf((float)D));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.max_splits == 1) return e;
  constexpr int RPB = 256 / (D / 4);
  const int blocks = (a.n_nodes * sh.G + RPB - 1) / RPB;
  hipLaunchKernelGGL(k_tree_merge<D>, dim3(sh.S * sh.Hkv * blocks), dim3(256), 0, st, dv.seqs, dv.state, a, geo, plan.rows);
  return hipGetLastError();
}

template <int D>
hipError_t tree_rows(const Dev &dv, const Shape &sh, const TreePlan &plan, const TreeArgs &a, hipStream_t st) {
  switch (plan.rows) {
    case 16: return tree_impl<D, 1, 1>(dv, sh, plan, a, st);
    case 32: return tree_impl<D, 1, 2>(dv, sh, plan, a, st);
    case 64: return tree_impl<D, 2, 2>(dv, sh, plan, a, st);
    default: return tree_impl<D, 2, 4>(dv, sh, plan, a, st);
  }
}

// ---- acceptance -----------------------------------------------------------------------------------------
// One workgroup per (sequence, kv head), a wave per token and 8 tokens at a time: each wave quantizes its
// token by itself (D / 64 channels a lane, reductions and ranks over the wave, no barriers), with the same
// rounded float32 steps as the decode append (append_dev.h), whose codes it gives bit for bit.  What a token
// needs of the ones before it: its place among the key outliers, from the waves' counts; the 4-token value
// blocks, put together in LDS; the rows of a uniform 4-bit key block, which ends a group of tokens.
// Bound by latency: two round trips and two barriers a group.  (One token after another by the append's
// own workgroup: up to six of KVQuant at 3 bits for 256 heads 25 us, so 6.4; 64 tokens of 4 bits 243 and 27.)
constexpr int kAcceptWaves = 8;

template <int D>
struct AcceptLds {
  float mid[2][16];                  // KVQ: midpoints of the key and of the value codebook, then infinity
  float cbv[16];                     // KVQ: value codebook
  float abs[kAcceptWaves][D];        // KVQ, several value outliers a token
  uint32_t row[kAcceptWaves][D / 8]; // a token's packed key codes
  uint32_t blk[3][D / 2];            // value codes of the group's 4-token blocks
  int outliers[kAcceptWaves];
  int take;
};

template <int D>
__global__ __launch_bounds__(64 * kAcceptWaves) void k_tree_accept(const SeqDesc *__restrict__ seqs, int32_t *state,
                                                                   const uint16_t *__restrict__ k,
                                                                   const uint16_t *__restrict__ v,
                                                                   const float *__restrict__ cbtab, int Hkv, int n_nodes,
                                                                   const int32_t *__restrict__ path,
                                                                   const int32_t *__restrict__ n_path, int max_path,
                                                                   int max_new, int32_t *counts) {
  constexpr int CH = D / 64, NT = 64 * kAcceptWaves;
  __shared__ AcceptLds<D> L;
  const int seq = blockIdx.x / Hkv, h = blockIdx.x % Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const SeqDesc &sd = seqs[seq];
  int32_t *st = state + ((int64_t)seq * Hkv + h) * ST_WORDS;
  const int32_t *nodes = path + (int64_t)seq * max_path;
  const int method = sd.method, bits = sd.bits, cap = sd.cap;
  int count = st[ST_COUNT], pos = st[ST_NEXT_POS], fill = st[ST_KOUT_FILL];
  const int want = min(max(n_path[seq], 0), max_path);
  if (tid == 0) L.take = want;
  __syncthreads();
  for (int i = tid; i < want; i += NT)
    if (nodes[i] < 0 || nodes[i] >= n_nodes) atomicMin(&L.take, i);
  const int words = method == UQ ? D / 2 : method == KVQ ? D * bits / 8 : 0;  // of a value block
  uint32_t *blocks = reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(sd.vc) + h * stride_codes(sd));
  for (int i = tid; i < 3 * (D / 2); i += NT) L.blk[i / (D / 2)][i % (D / 2)] = 0u;
  if (method == KVQ && tid < 48) {
    const int nc = 1 << bits, i = tid & 15;
    const float *cb = cbtab + cb_offset(bits);
    if (tid < 32) L.mid[tid >> 4][i] = i < nc - 1 ? cb[2 * nc + (tid >> 4) * (nc - 1) + i] : INFINITY;
    else L.cbv[i] = i < nc ? cb[nc + i] : 0.f;
  }
  __syncthreads();
  // the open value block goes on (its words by the threads that store them below)
  if (tid < words && (count & 3) != 0) L.blk[0][tid] = gld(blocks + (int64_t)(count >> 2) * words + tid);
  // (a method may have room for up to three tokens more, where it rounds its capacity up: they are not taken,
  // so that equal paths leave equal counts.  Up to there the outlier pools have room for every channel of every
  // token: the heads of a sequence hold the same tokens)
  const int take = min(L.take, min(cap, sd.n0 + max_new) - count);
  float2 tau[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) tau[i] = method == KVQ ? kvq_key_tau(sd, h, lane + 64 * i, D) : make_float2(0.f, 0.f);
  auto code_of = [&](float x, const float *mid) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < 15; ++i) c += x > mid[i] ? 1 : 0;
    return c;
  };
  auto before = [&](uint64_t m) { return __popcll(m & ((1ull << lane) - 1)); };
  __syncthreads();
  for (int done = 0; done < take;) {
    // the tokens of this group: up to the end of a key block, and as many as the key-outlier pool has room
    // for whatever they hold (a token that may not fit is dropped, as by the decode append)
    int m = min(kAcceptWaves, take - done);
    if (method == UQ) m = min(m, 64 - (count & 63));
    if (method == KVQ && sd.bp > 0) {
      if (fill + D > sd.pool_cap) break;
      m = min(m, (sd.pool_cap - fill) / D);
    }
    const int t = count + wave;
    const bool on = wave < m;
    uint32_t kx[CH], vx[CH];
    int kcode[CH];
    uint64_t kout[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) kx[i] = vx[i] = 0, kcode[i] = 0, kout[i] = 0;
    if (on) {
      const int64_t at = (((int64_t)seq * n_nodes + nodes[done + wave]) * Hkv + h) * D + lane;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        kx[i] = gld(k + at + 64 * i);
        vx[i] = gld(v + at + 64 * i);
      }
      uint32_t *blk = L.blk[(t >> 2) - (count >> 2)];
      if (method == FP16) {
        uint16_t *kr = reinterpret_cast<uint16_t *>(sd.k) + h * stride_rows(sd, D) + (int64_t)t * D + lane;
        uint16_t *vr = reinterpret_cast<uint16_t *>(sd.v) + h * stride_rows(sd, D) + (int64_t)t * D + lane;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          gst(kr + 64 * i, (uint16_t)kx[i]);
          gst(vr + 64 * i, (uint16_t)vx[i]);
        }
      } else if (method == UQ) {
        uint16_t *res = reinterpret_cast<uint16_t *>(sd.kres) + ((int64_t)h * 64 + (t & 63)) * D + lane;
#pragma unroll
        for (int i = 0; i < CH; ++i) {  // a lane's channels are one of each value group
          gst(res + 64 * i, (uint16_t)kx[i]);
          const float x = h2f(vx[i]), mn = wave_min(x), mx = wave_max(x), r = __fsub_rn(mx, mn);
          const float inv = r > 0.f ? __fdiv_rn(15.0f, r) : 0.f;
          const int code = (int)fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x, mn), inv)), 0.f), 15.f);
          or_uq_code(blk, lane + 64 * i, t & 3, code, D);
          if (lane == 0)
            (reinterpret_cast<float2 *>(sd.vmeta) + h * stride_uq_vmeta(sd, D))[(int64_t)t * CH + i] = make_float2(mn, __fdiv_rn(r, 15.0f));
        }
      } else {
        // key: codes under the frozen thresholds, packed; outliers wait for their place
        uint32_t *row = L.row[wave];
        if (lane < D / 8) row[lane] = 0u;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const float x = h2f(kx[i]);
          kcode[i] = code_of(__fmul_rn(x, tau[i].y), L.mid[0]);
          kout[i] = __ballot(sd.bp > 0 && fabsf(x) > tau[i].x);
          const int bit = bits * (lane + 64 * i);
          atomicOr(&row[bit >> 5], (uint32_t)kcode[i] << (bit & 31));
          if ((bit & 31) + bits > 32) atomicOr(&row[(bit >> 5) + 1], (uint32_t)kcode[i] >> (32 - (bit & 31)));
        }
        // value: the scale is the n_ov-th largest magnitude (0-based)
        const int nov = sd.bp > 0 ? sd.n_ov : 0;
        float ax[CH], s;
#pragma unroll
        for (int i = 0; i < CH; ++i) ax[i] = fabsf(h2f(vx[i]));
        if (nov <= 1) {
          s = wave_max(CH == 2 ? fmaxf(ax[0], ax[CH - 1]) : ax[0]);
          int ties = 0;
          float lower = -1.f;
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            ties += __popcll(__ballot(ax[i] == s));
            lower = fmaxf(lower, ax[i] < s ? ax[i] : -1.f);
          }
          if (nov == 1 && ties < 2) s = wave_max(lower);
        } else {
          float *all = L.abs[wave];
#pragma unroll
          for (int i = 0; i < CH; ++i) all[lane + 64 * i] = ax[i];
          __builtin_amdgcn_wave_barrier();
          s = 0.f;
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            int gt = 0, ge = 0;
            for (int j = 0; j < D; ++j) {
              gt += all[j] > ax[i] ? 1 : 0;
              ge += all[j] >= ax[i] ? 1 : 0;
            }
            const uint64_t hit = __ballot(gt <= nov && nov < ge);  // (every hit holds the same value)
            if (hit) s = __shfl(ax[i], __builtin_ctzll(hit));
          }
        }
        const float inv = s > 0.f ? __fdiv_rn(1.0f, s) : 0.f;
        uint32_t *vo = reinterpret_cast<uint32_t *>(sd.vout) + h * stride_vout(sd) + t;
        uint32_t *vd = reinterpret_cast<uint32_t *>(sd.vdel) + h * stride_vout(sd) + t;
        int total = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const float x = h2f(vx[i]);
          const int code = code_of(__fmul_rn(x, inv), L.mid[1]), c = lane + 64 * i;
          or_quad_code(blk, c, t & 3, code, bits);
          const uint64_t out = __ballot(sd.bp > 0 && ax[i] > s);
          const int r = total + before(out);
          if ((out >> lane & 1) && r < sd.nov_slots) {
            gst(vo + (int64_t)r * cap, outlier_entry(vx[i], t, code, c));
            gst(vd + (int64_t)r * cap, vdel_pack(__fsub_rn(x, __fmul_rn(s, L.cbv[code])), c));
          }
          total += __popcll(out);
        }
        for (int r = total + lane; r < sd.nov_slots; r += 64) {
          gst(vo + (int64_t)r * cap, kNoOutlier);
          gst(vd + (int64_t)r * cap, 0u);
        }
        if (lane == 0) gst(reinterpret_cast<float *>(sd.vmeta) + h * stride_slots(sd) + t, s);
        __builtin_amdgcn_wave_barrier();
        if (lane < D * bits / 32)
          gst(reinterpret_cast<uint32_t *>(reinterpret_cast<uint8_t *>(sd.kc) + h * stride_codes(sd) + (int64_t)t * sd.rowbytes) + lane,
              row[lane]);
        int n = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) n += __popcll(kout[i]);
        if (lane == 0) L.outliers[wave] = n;
      }
    }
    if (method == UQ) __builtin_amdgcn_s_waitcnt(0);  // the key rows, before other waves read them
    __syncthreads();
    if (method == KVQ) {
      int at = fill;
      for (int w = 0; w < m; ++w) {
        fill += L.outliers[w];
        at += w < wave ? L.outliers[w] : 0;
      }
      if (on) {
        uint32_t *pool = reinterpret_cast<uint32_t *>(sd.kout) + h * stride_kout(sd);
        int r = at;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          if (kout[i] >> lane & 1) gst(pool + r + before(kout[i]), outlier_entry(kx[i], t, kcode[i], lane + 64 * i));
          r += __popcll(kout[i]);
        }
        if (lane == 0) gst(reinterpret_cast<uint32_t *>(sd.krow) + h * stride_krow(sd) + t + 1, (uint32_t)r);
      }
    }
    const int first = count >> 2, last = (count + m - 1) >> 2;
    if (tid < words) {
      uint32_t open = 0u;  // what the next group's first block goes on from
      for (int b = first; b <= last; ++b) {
        open = L.blk[b - first][tid];
        gst(blocks + (int64_t)b * words + tid, open);
        L.blk[b - first][tid] = 0u;
      }
      if (((count + m) & 3) != 0) L.blk[0][tid] = open;
    }
    count += m;
    pos += m;
    done += m;
    if (method == UQ && (count & 63) == 0 && tid < D) {
      // a complete key block: thread c quantizes channel c
      const uint16_t *res = reinterpret_cast<const uint16_t *>(sd.kres) + (int64_t)h * 64 * D + tid;
      uq_key_block<D>(sd, h, (count >> 6) - 1, [&](int j) { return (uint32_t)gld(res + j * D); });
    }
    __syncthreads();
  }
  if (tid == 0) {
    st[ST_KOUT_FILL] = fill;
    set_counts(st, count, pos);
    if (counts != nullptr && h == 0) counts[seq] = count;
  }
}

}  // namespace

hipError_t launch_tree_attention(const Dev &dv, const Shape &sh, const TreePlan &plan, const TreeArgs &a, hipStream_t st) {
  return sh.D == 64 ? tree_rows<64>(dv, sh, plan, a, st) : tree_rows<128>(dv, sh, plan, a, st);
}

hipError_t launch_tree_accept(const Dev &dv, const Shape &sh, const uint16_t *k, const uint16_t *v, int n_nodes,
                              const int32_t *path, const int32_t *n_path, int max_path, int32_t *counts, hipStream_t st) {
  auto kernel = sh.D == 64 ? k_tree_accept<64> : k_tree_accept<128>;
  hipLaunchKernelGGL(kernel, dim3(sh.S * sh.Hkv), dim3(64 * kAcceptWaves), 0, st, dv.seqs, dv.state, k, v, dv.cbtab, sh.Hkv, n_nodes,
                     path, n_path, max_path, sh.max_new, counts);
  return hipGetLastError();
}

}  // namespace mkv
