// cure_packed_attn: attention of candidate trees, single tokens or chunks of prompts over a
// context whose tokens are packed in blocks of 64 with 8 bits a value (cure_kv_pack), the open
// rows behind it and the new rows themselves.
//
// Query row R of a kv-head is query head R % group of token R / group, so the heads that
// share keys share a tile. With C the bytes and s_k, s_v the scales of a token's block,
//   S = s_k (C_k Q^T),  P = s_v 2^(S - m),  l += P / s_v,  O^T += C_v^T P^T,  o = O / l
// in one pass over the keys with the reference m, near a running maximum of S + log2 s_v, and l in fp32.
// The value's scale is part of the exponent, so a block whose values are large and one
// whose values are small both have P in the range of 16 bits where they count at all. A wave takes scales as
// multiples of a power of two, by which it multiplies o at the end. Where one lies more than 2^32 from
// that, P and P / s_v no longer both fit fp32: l has a reference of its own from there on, the scores' maximum, and
// each score a second exponential.
//
// bf16: the bytes are widened to fp16, which holds them exactly, and the query rows are too, times
// a power of two for each row: what that loses is at most 2^-39 of the row's largest, where that is
// 2^-106 or more. P is rounded to fp16 for its product, 2^-11 where bf16 would take 2^-8 and add half
// as much again to the error that the output's own rounding makes; what lies 2^-21 below the largest P
// has fewer bits, down to 2^-32 of it. Open rows keep bf16's range: their products take P as two bf16
// values.
// fp32: fp32 throughout.
//
// 32x32 matrix instructions (x16 for 16 bits, x2 eight times for fp32), 32 query rows per wave. Lane
// l = 32 half + col owns query row col, and of a step's 32 tokens half of the scores:
//   S^T: A = token col's columns 32 s + 16 half + 8 u .. +7, B = query row col's;
//        D register r = score of token 8 (r / 4) + 4 half + r % 4
//   O^T: A = column 32 i + col of the tokens whose probabilities the lane holds in
//        registers 8 t .. 8 t + 7, B = those; D register r of block i = column 32 i + 8 (r / 4)
//        + 4 half + r % 4 of query row col.
// A packed block lies in memory as A wants it, 16 bytes to a lane: packed steps need no
// exchange between lanes. Many rows share what is widened through LDS, by 16x16x32 instructions and 16
// rows per wave, which leaves room for four waves to a SIMD:
//   lane l = 16 quad + col owns query row col and the scores of tokens 16 i + 4 quad + r;
//   S^T: A = token col's columns 32 s + 8 quad .. +7;  O^T: A = column 16 i + col of the lane's
//        eight tokens, D register r of block i = column 16 i + 4 quad + r.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "common.hpp"
#include "host_util.hpp"
#include "mfma_tile.hpp"
#include "packed.hpp"

namespace cure {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kStep = 32;            // tokens per step of the key loop
constexpr int kWaves = 4;            // waves per workgroup of a tile of few rows
constexpr int kRows = 32;            // query rows of such a wave, and of the tile
constexpr int kManyRows = 16;        // query rows of a wave where there are many
// Waves of such a tile on a SIMD. At d = 64 registers and LDS leave room for three workgroups (chunks of
// 256 to 512 tokens: 251 us, 271 with two).
template <int D>
constexpr int kPerSimd = D == 64 ? 6 : 4;
constexpr int kRing = 3;             // steps whose bytes are on their way or wait, of a tile of many rows
constexpr int kMaxSlots = 64;        // splits of a row's keys at most
constexpr float kNone = -3e38f;      // reference of a row that has seen nothing
constexpr int kAncWords = CURE_MAX_TREE_NODES / 32;
constexpr int64_t kMostTokens = INT32_MAX - 4096;    // of a sequence: steps' ends stay within 32 bits

struct Args {
  const void* q;
  const int8_t* pk;
  const int8_t* pv;
  const float* k_scale;
  const float* v_scale;
  int64_t blocks;
  const void* k;
  const void* v;
  int64_t cache_rows;
  void* o;
  float* lse;
  int32_t out_bf16;
  int32_t batch, n_max, hq, hkv, group;
  int64_t rows;
  float scale_log2;
  const int64_t* row_off;
  const int32_t* n_rows;
  const int64_t* blk_off;
  const int32_t* packed_len;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const int32_t* parent;
  int32_t* row_status;
  int32_t tile;                      // query rows of a tile
  int32_t tiles, tps, quantum, slots;    // tiles of a sequence; steps per split, which begin at multiples
                                     // of quantum, splits at most
  float* part_o;                     // [row][hq][slots][d]
  float* part_lse;                   // [row][hq][slots], of base 2
};

// A value at an address that the whole wave shares, through the scalar cache.
CURE_DEV float scalar_load(const float* p) {
  return *(const __attribute__((address_space(4))) float*)(uintptr_t)p;
}

CURE_DEV float first_lane(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// A sequence's sizes as the device has them. ok: they can be.
struct Seq {
  int64_t row0, block0, kv0;
  int n, packed, ctx;
  bool ok;
};
CURE_DEV Seq seq_of(const Args& a, int b) {
  Seq s;
  s.n = a.n_rows[b];
  s.packed = a.packed_len[b];
  s.ctx = a.ctx_len[b];
  s.block0 = a.blk_off[b];
  s.kv0 = a.kv_off[b];
  s.row0 = a.row_off ? a.row_off[b] : (int64_t)b * a.n_max;
  s.ok = s.n >= 0 && s.n <= a.n_max && s.packed >= 0 && s.ctx >= 0 && s.row0 >= 0 && s.row0 <= a.rows - s.n &&
         s.block0 >= 0 && s.block0 <= a.blocks - blocks_of(s.packed) && s.kv0 >= 0 &&
         s.kv0 <= a.cache_rows - s.ctx - s.n && (int64_t)s.packed + s.ctx + s.n <= kMostTokens;
  return s;
}

// Steps of 32 tokens that the rows up to packed row `last` see: packed ones, and all.
struct Steps {
  int packed, all;
};
CURE_DEV Steps steps_of(const Args& a, const Seq& s, int last) {
  const int64_t open = (int64_t)s.ctx + (a.parent ? s.n : last / a.group + 1);
  const int p = s.packed / kStep + (s.packed % kStep != 0);
  return Steps{p, p + (int)((open + kStep - 1) / kStep)};
}
// Splits of a tile's steps: n of `per`, the last one shorter.
struct Cut {
  int n, per;
};
__host__ CURE_DEV Cut cut_of(int steps, int tps, int slots, int quantum) {
  int n = (steps - 1) / tps + 1;
  if (n > slots) n = slots;
  const int per = ((steps - 1) / n / quantum + 1) * quantum;
  return Cut{(steps - 1) / per + 1, per};
}

// Eight values of an operand's lane: bytes, for which the query rows and P are fp16 where the
// rows are bf16, or rows' values.
struct Half8 {
  f16x8 x;
  // Bytes b as 1024 + (b + 128), whose low bits are fp16's, less 1152.
  CURE_DEV void bytes(uint32_t lo, uint32_t hi) {
    const f16x2 bias{(_Float16)1152.f, (_Float16)1152.f};
    const auto pair = [&](uint32_t w, uint32_t sel) {
      return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u, sel)) - bias;
    };
    const f16x2 p[4] = {pair(lo, 0x04010400u), pair(lo, 0x04030402u), pair(hi, 0x04010400u), pair(hi, 0x04030402u)};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i / 2][i % 2];
  }
  CURE_DEV void floats(const float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (_Float16)f[i];
  }
};
struct Bf8 {
  bf16x8 x;
  CURE_DEV void words(const u32x4* w) { x = __builtin_bit_cast(bf16x8, w[0]); }
  CURE_DEV void row(const RowVec<uint16_t, 16>& r, int u) {
    Pack8 p;
    p.u = make_uint4(r.w[4 * u], r.w[4 * u + 1], r.w[4 * u + 2], r.w[4 * u + 3]);
    x = p.v;
  }
  CURE_DEV void floats(const float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)f[i];
  }
  // What `floats` rounded off.
  CURE_DEV void rest(const float* f, const Bf8& high) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)(f[i] - (float)high.x[i]);
  }
};
struct Float8 {
  float x[8];
  CURE_DEV void words(const u32x4* w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i / 4][i % 4]);
  }
  CURE_DEV void bytes(uint32_t lo, uint32_t hi) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = (float)(int8_t)(lo >> (8 * i));
      x[4 + i] = (float)(int8_t)(hi >> (8 * i));
    }
  }
  CURE_DEV void row(const RowVec<float, 16>& r, int u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[8 * u + i]);
  }
  CURE_DEV void floats(const float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = f[i];
  }
};
CURE_DEV f32x16 mma(const Half8& a, const Half8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.x, b.x, c, 0, 0, 0);
}
CURE_DEV f32x16 mma(const Bf8& a, const Bf8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}
CURE_DEV f32x4 mma16(const Half8& a, const Half8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.x, b.x, c, 0, 0, 0);
}
CURE_DEV f32x4 mma16(const Bf8& a, const Bf8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x, b.x, c, 0, 0, 0);
}
CURE_DEV f32x16 mma(const Float8& a, const Float8& b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i], b.x[i], c, 0, 0, 0);
  return c;
}
// Operands beside bytes, and beside rows.
template <typename E>
struct Types;
template <>
struct Types<uint16_t> {
  using Byte = Half8;
  using Row = Bf8;
};
template <>
struct Types<float> {
  using Byte = Float8;
  using Row = Float8;
};

CURE_DEV f32x16 zeros() {
  f32x16 x;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 0.f;
  return x;
}

// x in another register: what a seldom taken branch replaces then keeps its own, and the other way needs no move.
CURE_DEV float moved(float x) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xe4, 0xf, 0xf, false)); }

// A lane's query row and what it has summed: kScores scores of a step, of which kLanes lanes
// share a row, and kBlocks blocks of output.
template <int kScores, int kLanes, int kBlocks, class Block>
struct Sums {
  static constexpr int kEach = sizeof(Block) / sizeof(float);
  float m = kNone, l = 0.f;                        // m is a whole number
  Block o[kBlocks];

  CURE_DEV Sums() {
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int r = 0; r < kEach; ++r) o[i][r] = 0.f;
  }
  // Scores x * factor of base 2 (-inf: not seen; factor > 0 there) of tokens whose values have scale 2^lv and
  // its reciprocal rv, in the wave's unit: their P. The reference moves to where the largest P is 2^7 to 2^8, which
  // leaves small ones of a million tokens precise in fp16, and does so where a lane's P sum up to more than 2^15, which
  // fp16 holds: at first, and seldom later. A maximum for each step would cost a tenth of it. A step
  // always comes that way with lv infinite, where rv is the scale's logarithm and l has a reference of its own, *own(),
  // and with lv NaN, where the scale is 0: the tokens count, their values do not.
  template <class Own>
  CURE_DEV void soften(const float (&x)[kScores], float factor, float lv, float rv, const Own& own, float (&p)[kScores]) {
    float added = exps(x, factor, lv - m, p);
    if (__builtin_expect(__any(!(added <= 0x1p15f)), 0)) {
      const bool apart = lv == INFINITY, none = lv != lv;
      lv = apart ? rv : lv;
      float high = x[0];
#pragma unroll
      for (int r = 1; r < kScores; ++r) high = fmaxf(high, x[r]);
      if (kLanes == 4) high = fmaxf(high, __shfl_xor(high, 16));
      high = max_halves(high) * factor;
      const float was = m;
      m = fmaxf(m, floorf(high + (none ? 0.f : lv)) - 7.f);
      const float f = fast_exp2(was - m);
#pragma unroll
      for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int r = 0; r < kEach; ++r) o[i][r] *= f;
      if (apart || none) {
        const float from = apart ? *own() : was, to = apart ? fmaxf(from, floorf(high)) : m;
        if (apart) *own() = to;
        l *= fast_exp2(from - to);
#pragma unroll
        for (int r = 0; r < kScores; ++r) l += fast_exp2(fmaf(x[r], factor, -to));
        rv = 0.f;
      } else {
        l *= f;
      }
      added = exps(x, factor, (none ? -INFINITY : lv) - m, p);
      m = moved(m);
      l = moved(l);
    }
    l = fmaf(added, rv, l);
  }
  CURE_DEV float exps(const float (&x)[kScores], float factor, float c, float (&p)[kScores]) const {
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < kScores; ++r) {
      p[r] = fast_exp2(fmaf(x[r], factor, c));
      sum[r % 2] += p[r];
    }
    return sum[0] + sum[1];
  }
  // The row's whole sum.
  CURE_DEV float all() const {
    float x = l;
    if (kLanes == 4) x += __shfl_xor(x, 16);
    return sum_halves(x);
  }
};
template <int D>
using FewSums = Sums<16, 2, D / 32, f32x16>;
template <int D>
using ManySums = Sums<8, 4, D / 16, f32x4>;

// The unit 2^z of a wave's value scales: 1, or near the first that lies more than 2^32 from that, where the wave
// meets it first; and whether others lie too far from it (apart). Within 2^32 of it, P / s_v of 2^31 tokens is below
// 2^100, and the P of a token whose score lies 24 below the largest above 2^-90. Open rows have scale 1.
struct ScaleUnit {
  uint32_t low = (127 - 32) << 23, span = (65 << 23) - 1;      // bits of the scales near enough: low .. low + span
  float down = 1.f;                                // 2^-z
  bool chosen = false, apart = false;
  CURE_DEV bool near(float s) const { return __float_as_uint(s) - low <= span; }
  // One that is not near, the same for the whole wave. m: the row's reference, l's own from here on where apart.
  template <class Own>
  CURE_DEV void meet(float s, float m, const Own& own) {
    const uint32_t bits = __float_as_uint(s), e = min(max(bits >> 23, 1u), 250u);
    if (bits == 0 || apart) return;
    if (chosen || __any(m > kNone)) {
      apart = true;
      *own() = m;
      return;
    }
    chosen = true;
    low = e > 32 ? (e - 32) << 23 : 1;
    span = (min(e + 33, 255u) << 23) - 1 - low;
    down = __uint_as_float((254 - e) << 23);
  }
  CURE_DEV float z() const { return (float)(127 - (int)(__float_as_uint(down) >> 23)); }
};
// A scale as soften takes it: in the unit, and its reciprocal.
struct ValueScale {
  float lv, rv;
  CURE_DEV ValueScale(float s, const ScaleUnit& u) {
    const float x = s > 0.f ? s * u.down : 1.f;
    lv = s > 0.f ? __builtin_amdgcn_logf(x) : NAN;
    rv = __builtin_amdgcn_rcpf(x);
    if (__builtin_expect(u.apart, 0)) {
      rv = s > 0.f ? __builtin_amdgcn_logf(s < 1.f ? s * 0x1p64f : s) - (s < 1.f ? 64.f : 0.f) - u.z() : -INFINITY;
      lv = INFINITY;
    }
  }
};

// The power of two by which a query row is brought to fp16, for its largest value to be in [2^14, 2^15),
// and its reciprocal.
struct HalfScale {
  float down, up;
  CURE_DEV explicit HalfScale(float high) {
    int e = (int)(__float_as_uint(high) >> 23) - 127 - 14;
    e = max(-120, min(e, 120));
    down = __uint_as_float((uint32_t)(127 - e) << 23);
    up = __uint_as_float((uint32_t)(127 + e) << 23);
  }
};
// Query rows as a few rows' products take them; returns what the scores are to be multiplied by.
template <int D>
CURE_DEV float byte_rows(const RowVec<uint16_t, 16> (&x)[D / 32], Half8 (&q)[D / 32][2]) {
  float high = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) high = fmaxf(high, fabsf(x[i].get(j)));
  const HalfScale s(max_halves(high));
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = x[i].get(8 * u + j) * s.down;
      q[i][u].floats(f);
    }
  return s.up;
}
template <int D>
CURE_DEV float byte_rows(const RowVec<float, 16> (&x)[D / 32], Float8 (&q)[D / 32][2]) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int u = 0; u < 2; ++u) q[i][u].row(x[i], u);
  return 1.f;
}
template <typename E, int D>
CURE_DEV void load_rows(const E* src, RowVec<E, 16> (&x)[D / 32]) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x[i].load(src + 32 * i);
}

// Values of a row that no query row need see: an infinity or NaN would reach the others through
// its zero probabilities.
CURE_DEV uint32_t finite_word(uint32_t w, uint16_t) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
CURE_DEV uint32_t finite_word(uint32_t w, float) { return (w & 0x7f800000u) == 0x7f800000u ? 0u : w; }

// Token of D register r in a lane's half, and of D register r % 4 of token block r / 4 in a lane's quad.
CURE_DEV int token_of(int half, int r) { return 8 * (r / 4) + 4 * half + r % 4; }
CURE_DEV int token_in(int quad, int r) { return 16 * (r / 4) + 4 * quad + r % 4; }

// An open step's values as the products take them, 16 bytes (two times 16, fp32) after the other: of
// few rows lane l's eight of block i and k-step t at [i][t][l], of many lane l's of block i at [i][l].
template <typename E, int D>
struct ValueTile {
  static constexpr int kWords = 8 * (int)sizeof(E) / 16;
  u32x4 x[D * 4][kWords];
  CURE_DEV const u32x4* few(int i, int t, int lane) const { return x[(2 * i + t) * kWave + lane]; }
  CURE_DEV const u32x4* many(int i, int lane) const { return x[i * kWave + lane]; }
};
// One unit of its making, four columns of eight tokens that a lane has: 4 * (D / 4) in all.
template <typename E, int D, bool kMany>
struct ValueUnit {
  RowVec<E, 4> x[8];
  static CURE_DEV int col_of(int unit) { return unit % (D / 4) * 4; }
  CURE_DEV void load(const E* rows, int64_t pitch, int t0, int most, int unit) {
    const int g = unit / (D / 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = kMany ? token_in(g, j) : token_of(g % 2, 8 * (g / 2) + j);
      x[j].load(rows + min(t0 + t, most) * pitch + col_of(unit));
    }
  }
  CURE_DEV void store(ValueTile<E, D>& tile, int unit) {
    const int g = unit / (D / 4), c0 = col_of(unit);
    const int at = kMany ? c0 / 16 * kWave + g * 16 + c0 % 16 : (2 * (c0 / 32) + g / 2) * kWave + g % 2 * 32 + c0 % 32;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int k = 0; k < RowVec<E, 4>::kWords; ++k) x[j].w[k] = finite_word(x[j].w[k], E());
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if constexpr (sizeof(E) == 2) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = __builtin_amdgcn_perm(x[2 * j + 1].w[c / 2], x[2 * j].w[c / 2], c % 2 ? 0x07060302u : 0x05040100u);
        tile.x[at + c][0] = w;
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) tile.x[at + c][k] = u32x4{x[4 * k].w[c], x[4 * k + 1].w[c], x[4 * k + 2].w[c], x[4 * k + 3].w[c]};
      }
    }
  }
};

// What a workgroup works on.
struct Work {
  Seq s;
  Steps steps;
  Cut cut;
  int b, hk, slot, r0, rows, node0;  // first packed row of the tile, of `rows`, and its node
  int begin, end;                    // steps
};

template <int kTileRows>
struct Trees {
  uint32_t anc[kTileRows][kAncWords];   // root paths of the tile's nodes, as bits
  int parent[CURE_MAX_TREE_NODES];
};

// Finds the workgroup's work, reports the sequence's status and forms the root paths. False: nothing
// to do. The grid: kv-heads, tiles, splits; sequences. A sequence's workgroups on one kv-head
// are hkv apart, so where that is a multiple of 8 they share an XCD's L2.
template <int kTileRows>
CURE_DEV bool locate(const Args& a, Work& w, Trees<kTileRows>& sh) {
  const int tid = threadIdx.x;
  w.b = blockIdx.y;
  w.hk = blockIdx.x % a.hkv;
  const int tile = blockIdx.x / a.hkv % a.tiles;
  w.slot = blockIdx.x / a.hkv / a.tiles;
  w.s = seq_of(a, w.b);
  const bool first = blockIdx.x == 0;
  if (!w.s.ok || w.s.n == 0) {
    if (first && tid == 0 && a.row_status) a.row_status[w.b] = w.s.ok ? CURE_OK : CURE_ERR_BAD_TREE;
    return false;
  }
  w.r0 = tile * a.tile;
  w.rows = w.s.n * a.group;
  if (w.r0 >= w.rows) return false;
  const int r_last = min(w.r0 + a.tile, w.rows) - 1;
  w.steps = steps_of(a, w.s, r_last);
  w.cut = cut_of(w.steps.all, a.tps, a.slots, a.quantum);
  w.begin = w.slot * w.cut.per;
  w.end = min(w.begin + w.cut.per, w.steps.all);
  if (w.begin >= w.end) return false;
  w.node0 = w.r0 / a.group;
  if (a.parent && (first || w.end > w.steps.packed)) {
    int p = -1;
    if (tid < w.s.n) p = a.parent[(int64_t)w.b * a.n_max + tid];
    const bool bad = tid < w.s.n && (p < -1 || p >= tid);
    const int any = __syncthreads_or(bad);
    if (first && tid == 0 && a.row_status) a.row_status[w.b] = any ? CURE_ERR_BAD_TREE : CURE_OK;
    if (tid < w.s.n) sh.parent[tid] = bad ? -1 : p;
    __syncthreads();
    if (tid <= r_last / a.group - w.node0) {
      uint32_t bits[kAncWords] = {};
      for (int j = w.node0 + tid; j >= 0; j = sh.parent[j]) {
#pragma unroll
        for (int i = 0; i < kAncWords; ++i) bits[i] |= j >> 5 == i ? 1u << (j & 31) : 0u;
      }
#pragma unroll
      for (int i = 0; i < kAncWords; ++i) sh.anc[tid][i] = bits[i];
    }
    __syncthreads();
  } else if (first && tid == 0 && a.row_status) {
    a.row_status[w.b] = CURE_OK;
  }
  return true;
}

// Which of an open step's tokens a node sees, as bits: t0 is the first one's index in the open rows.
template <int kTileRows>
CURE_DEV uint32_t seen_of(const Args& a, const Work& w, const Trees<kTileRows>& sh, int node, int t0) {
  const int own = t0 - w.s.ctx;                    // its index among the new rows
  if (!a.parent) {
    const int n = node - own + 1;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
  }
  const uint32_t* anc = sh.anc[node - w.node0];
  const int i = own >> 5, sft = own & 31;          // floor
  const uint32_t lo = i >= 0 && i < kAncWords ? anc[i] : 0u, hi = i + 1 >= 0 && i + 1 < kAncWords ? anc[i + 1] : 0u;
  uint32_t seen = sft ? lo >> sft | hi << (32 - sft) : lo;
  if (own < 0) seen |= own <= -32 ? ~0u : (1u << -own) - 1;
  return seen;
}

// Four columns from column j on of the tile's output row `at`, and the log-sum-exp of base 2 of a row.
template <int D>
CURE_DEV void write(const Args& a, const Work& w, int64_t at, int j, const f32x4& x) {
  if (w.cut.n > 1) *reinterpret_cast<f32x4*>(a.part_o + (at * a.slots + w.slot) * D + j) = x;
  else if (a.out_bf16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + j) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + j) = x;
}
CURE_DEV void write_lse(const Args& a, const Work& w, int64_t at, float m, float l) {
  const float lse2 = l > 0.f ? m + log2f(l) : -INFINITY;
  if (w.cut.n > 1) a.part_lse[at * a.slots + w.slot] = lse2;
  else if (a.lse) a.lse[at] = lse2 * kLn2;
}

// x 2^z for a whole number z.
CURE_DEV f32x4 in_units(f32x4 x, float z) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = ldexpf(x[i], (int)z);
  return x;
}

// Where a tile of few rows is joined: the same rows of each wave.
template <int D>
struct Out {
  float o[kWaves][kRows][D + 4];
  float m[kWaves][kRows], l[kWaves][kRows];        // l's unit is 2^m
  float unit[kWaves][kRows];                       // o's 2^unit; l's own references before
};
// Writes the tile's rows, the sums of what the waves have put into sh.
template <int D>
CURE_DEV void finish(const Args& a, const Work& w, const Out<D>& sh) {
  constexpr int kLanes = 16;                       // of a row, four columns each
  __syncthreads();
  for (int row = threadIdx.x / kLanes; row < kRows; row += kWaves * kWave / kLanes) {
    if (w.r0 + row >= w.rows) break;
    float m = kNone, unit = kNone, l = 0.f, f[kWaves];
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      m = fmaxf(m, sh.m[k][row]);
      unit = fmaxf(unit, sh.unit[k][row]);
    }
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      l += fast_exp2(sh.m[k][row] - m) * sh.l[k][row];
      f[k] = fast_exp2(sh.unit[k][row] - unit);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int R = w.r0 + row;
    const int64_t at = (w.s.row0 + R / a.group) * a.hq + w.hk * a.group + R % a.group;
#pragma unroll
    for (int j = threadIdx.x % kLanes * 4; j < D; j += kLanes * 4) {
      f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWaves; ++k) x += f[k] * *reinterpret_cast<const f32x4*>(&sh.o[k][row][j]);
      if (j == 0) write_lse(a, w, at, m, l);
      write<D>(a, w, at, j, in_units(x * inv, unit - m));
    }
  }
}

// What the lanes of a wave wrote to LDS is there for its others, and read before it changes.
CURE_DEV void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Scores of packed tokens, of which `left` are there, times `factor`; returns the factor that is
// left. A lane's tokens are kFar * (r / 4) + r % 4 behind its `own` first one.
template <int kFar, int kScores>
CURE_DEV float mask_packed(float (&x)[kScores], int left, float factor, int own) {
  if (left >= kStep) return factor;
  left -= own;
#pragma unroll
  for (int r = 0; r < kScores; ++r) x[r] = kFar * (r / 4) + r % 4 < left ? x[r] * factor : -INFINITY;
  return 1.f;
}
template <int kFar, int kScores>
CURE_DEV void mask_open(float (&x)[kScores], uint32_t seen, float factor, int own) {
  seen >>= own;
#pragma unroll
  for (int r = 0; r < kScores; ++r) x[r] = seen & (1u << (kFar * (r / 4) + r % 4)) ? x[r] * factor : -INFINITY;
}

// ---------------------------------------------------------------------------
// Up to 32 query rows to a tile: the waves take the steps in turn, each with all rows and sums of its
// own, which are joined at the end. Packed bytes go from memory to registers and into the
// matrix unit, a step ahead of their use; past the caches where one tile is all (kOnce), for nothing reads
// them twice (eight single tokens over 4096 to 32768: 57 us and 5.6 TB/s, 63 us without; 16 trees of 20 to 48
// nodes 61 us, 64 with). Memory bounds it for one tile, issue for several.
template <typename E, int D, bool kOnce>
__global__ __launch_bounds__(kWaves * kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void packed_few(Args a) {
  constexpr int kK = D / 32;                       // pieces of 32 columns
  using Byte = typename Types<E>::Byte;
  using RowF = typename Types<E>::Row;
  __shared__ __attribute__((aligned(16))) Out<D> out;
  __shared__ Trees<kRows> trees;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane % 32, half = lane / 32;
  Work w;
  if (!locate(a, w, trees)) return;

  // This lane's query row.
  const int R = min(w.r0 + col, w.rows - 1), node = R / a.group;
  const E* qsrc = static_cast<const E*>(a.q) + ((w.s.row0 + node) * a.hq + w.hk * a.group + R % a.group) * D + 16 * half;
  FewSums<D> sum;
  ScaleUnit scales;
  // Seldom used: from the thread's index, for no register to hold it.
  const auto own = [&] {
    int t = tid;
    asm("" : "+v"(t));
    return &out.unit[wave][t % 32];
  };
  const auto scale_of = [&](float s) {
    if (__builtin_expect(!scales.near(s), 0)) scales.meet(s, sum.m, own);
    return ValueScale(s, scales);
  };
  int step = w.begin + wave;
  const int packed_end = min(w.end, w.steps.packed);
  if (step < packed_end) {
    Byte q[kK][2];
    float qs;
    {
      RowVec<E, 16> x[kK];
      load_rows<E, D>(qsrc, x);
      qs = byte_rows<D>(x, q) * a.scale_log2;
    }
    struct Raw {
      u32x4 k[kK], v[kK];
      float ks, vs;
    };
    const auto fetch = [&](Raw& raw, int st) {
      const int64_t block = (w.s.block0 + st / 2) * a.hkv + w.hk;
      const int64_t at = block * (kBlockTokens * D) + st % 2 * (kStep * D) + lane * 16;
#pragma unroll
      for (int i = 0; i < kK; ++i) raw.k[i] = load_of<kOnce>(reinterpret_cast<const u32x4*>(a.pk + at + i * 1024));
#pragma unroll
      for (int i = 0; i < kK; ++i) raw.v[i] = load_of<kOnce>(reinterpret_cast<const u32x4*>(a.pv + at + i * 1024));
      raw.ks = scalar_load(a.k_scale + block);
      raw.vs = scalar_load(a.v_scale + block);
    };
    const auto work = [&](const Raw& raw, int st) {
      f32x16 y = zeros();
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Byte f;
          f.bytes(raw.k[i][2 * u], raw.k[i][2 * u + 1]);
          y = mma(f, q[i][u], y);
        }
      float x[16], p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = y[r];
      const float factor = mask_packed<8>(x, w.s.packed - st * kStep, raw.ks * qs, 4 * half);
      const ValueScale v = scale_of(raw.vs);
      sum.soften(x, factor, v.lv, v.rv, own, p);
      Byte pf[2];
      pf[0].floats(p);
      pf[1].floats(p + 8);
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          Byte f;
          f.bytes(raw.v[i][2 * t], raw.v[i][2 * t + 1]);
          sum.o[i] = mma(f, pf[t], sum.o[i]);
        }
    };
    // Two buffers in turn: a copy from one to the other would wait for its loads.
    Raw even, odd;
    fetch(even, step);
    fetch(odd, min(step + kWaves, packed_end - 1));
    while (true) {
      work(even, step);
      step += kWaves;
      if (step >= packed_end) break;
      fetch(even, min(step + kWaves, packed_end - 1));
      work(odd, step);
      step += kWaves;
      if (step >= packed_end) break;
      fetch(odd, min(step + kWaves, packed_end - 1));
    }
  }
  if (step < w.end) {
    const int64_t pitch = (int64_t)a.hkv * D;
    const int open = w.s.ctx + w.s.n;              // open and new rows
    const E* kp = static_cast<const E*>(a.k) + w.s.kv0 * pitch + w.hk * D;
    const E* vp = static_cast<const E*>(a.v) + w.s.kv0 * pitch + w.hk * D;
    RowF q[kK][2];
    {
      RowVec<E, 16> x[kK];
      load_rows<E, D>(qsrc, x);
#pragma unroll
      for (int i = 0; i < kK; ++i) {
        q[i][0].row(x[i], 0);
        q[i][1].row(x[i], 1);
      }
    }
    // The wave's own part of the LDS turns the values.
    static_assert(sizeof(ValueTile<E, D>) <= sizeof(out.o[0]), "");
    ValueTile<E, D>& tile = *reinterpret_cast<ValueTile<E, D>*>(out.o[wave]);
    ValueScale one = scale_of(1.f);
    one.lv = first_lane(one.lv);
    one.rv = first_lane(one.rv);
    for (; step < w.end; step += kWaves) {
      const int t0 = (step - w.steps.packed) * kStep;
      RowVec<E, 16> kx[kK];
      load_rows<E, D>(kp + min(t0 + col, open - 1) * pitch + 16 * half, kx);
      constexpr int kUnits = D / kWave;            // of values, per lane
      static_assert(kUnits <= 2, "");
      ValueUnit<E, D, false> unit[kUnits];
      const auto load_values = [&](int i) { unit[i].load(vp, pitch, t0, open - 1, i * kWave + lane); };
      load_values(0);
      f32x16 y = zeros();
#pragma unroll
      for (int i = 0; i < kK; ++i) {
        // In fp32 the second half waits for registers of keys that are done.
        if (kUnits > 1 && i == (sizeof(E) == 4 ? kK / 2 : 0)) {
          if (sizeof(E) == 4) __builtin_amdgcn_sched_barrier(0);
          load_values(kUnits - 1);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          RowF f;
          f.row(kx[i], u);
          y = mma(f, q[i][u], y);
        }
      }
#pragma unroll
      for (int i = 0; i < kUnits; ++i) unit[i].store(tile, i * kWave + lane);
      wave_sync();
      float x[16], p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = y[r];
      mask_open<8>(x, seen_of(a, w, trees, node, t0), a.scale_log2, 4 * half);
      sum.soften(x, 1.f, one.lv, one.rv, own, p);
      RowF pf[2], rest[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        pf[t].floats(p + 8 * t);
        if constexpr (sizeof(E) == 2) rest[t].rest(p + 8 * t, pf[t]);
      }
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          RowF f;
          f.words(tile.few(i, t, lane));
          sum.o[i] = mma(f, pf[t], sum.o[i]);
          if constexpr (sizeof(E) == 2) sum.o[i] = mma(f, rest[t], sum.o[i]);
        }
      wave_sync();
    }
  }
  const float l = sum.all();
  const float ref = scales.apart ? *own() : sum.m;
  wave_sync();
  int t = tid;                                     // as above
  asm("" : "+v"(t));
  const int c = t % 32, h = t % kWave / 32;
  if (h == 0) {
    out.m[wave][c] = ref;
    out.l[wave][c] = l;
    out.unit[wave][c] = sum.m + scales.z();
  }
#pragma unroll
  for (int i = 0; i < kK; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<f32x4*>(&out.o[wave][c][32 * i + 8 * (r / 4) + 4 * h]) =
          f32x4{sum.o[i][r], sum.o[i][r + 1], sum.o[i][r + 2], sum.o[i][r + 3]};
  finish<D>(a, w, out);
}

// ---------------------------------------------------------------------------
// More rows (bf16): 16 for each of kGroups waves, which share each step's keys and values. The first
// waves bring a step's bytes to LDS by DMA, 1 KB each, widen them and hand them on through LDS; an
// operand's 64 lanes of 16 bytes are 1 KB of LDS. Step i forms the probabilities and products of step
// i, the scores of step i + 1 and the widened tile of step i + 2, while the bytes of the kRing steps behind
// are on their way. Bound by issue: at
// 128 rows on four times 32768 tokens, 8 kv-heads, the kernel takes 95 us of the call's 103 (0.67 PFLOP/s), of
// which counters give the vector unit 46 % and the matrix unit 31 %, one seldom beside the other, and LDS 41 %. Tried
// and no faster: 32 rows and half as many waves (113 us), bytes brought through registers (108), the scores'
// products ahead of the softmax (108).
template <int D>
struct Tile {
  u32x4 k[2][D / 32][kWave];                       // of a block of 16 tokens and 32 columns
  ValueTile<uint16_t, D> v;
};
template <int D>
struct Stage {
  Tile<D> tile[3];
  u32x4 raw[kRing][2 * D / 32][kWave];
};
template <int i>
struct Turn {
  static constexpr int value = i;
};

template <int D, int kGroups>
__global__ __launch_bounds__(kGroups * kWave) __attribute__((amdgpu_waves_per_eu(kPerSimd<D>, kPerSimd<D>))) void packed_many(Args a) {
  using E = uint16_t;
  constexpr int kK = D / 32, kO = D / 16;
  constexpr int kBring = 2 * kK;                   // waves that bring 1 KB of a step: keys', then values'
  static_assert(kBring <= kGroups && kRing == 3, "");
  constexpr uint32_t kTileBytes = sizeof(Tile<D>), kRawBytes = 2 * kStep * D, kValues = sizeof(Tile<D>::k);
  __shared__ __attribute__((aligned(1024))) Stage<D> in;
  __shared__ Trees<kGroups * kManyRows> trees;
  __shared__ float refs[kGroups * kManyRows];      // l's own
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane % 16, quad = lane / 16, group = wave;
  Work w;
  if (!locate(a, w, trees)) return;

  const int R0 = w.r0 + group * kManyRows, R = min(R0 + col, w.rows - 1), node = R / a.group;
  const int last_node = min(R0 + kManyRows - 1, w.rows - 1) / a.group;
  const bool idle = R0 >= w.rows;                  // this wave's rows are not there
  const E* qsrc = static_cast<const E*>(a.q) + ((w.s.row0 + node) * a.hq + w.hk * a.group + R % a.group) * D + 8 * quad;
  ManySums<D> sum;
  ScaleUnit scales;
  const auto own = [&] { return &refs[group * kManyRows + col]; };
  // Value scales, one to a lane.
  const auto meet = [&](float s) __attribute__((always_inline)) {
    unsigned long long far;
    while (!scales.apart && (far = __ballot(s != 0.f && !scales.near(s))))
      scales.meet(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s), __ffsll(far) - 1)), sum.m, own);
  };

  const int packed_end = min(w.end, w.steps.packed), rounds = packed_end - w.begin;
  if (rounds > 0) {
    // This wave's bytes: from one half of a block to the other, and on to the next. Past the last step
    // there are none, which read as zeros.
    const int64_t block = (w.s.block0 + w.begin / 2) * a.hkv + w.hk, pitch = (int64_t)a.hkv * (kBlockTokens * D);
    const int8_t* src = (group < kK ? a.pk : a.pv) + block * (kBlockTokens * D) + w.begin % 2 * (kStep * D) + group % kK * 1024;
    int asked = 0;
    const uint32_t raw_lds = lds_addr(in.raw) + group * 1024;
    const auto dma = [&](uint32_t slot) {
      dma16_shared(raw_lds + slot, lane * 16, raw_rsrc(src, asked < rounds ? 1024 : 0));
      src += (w.begin + asked) % 2 ? pitch - kStep * D : kStep * D;
      ++asked;
    };
    if (group < kBring) {
#pragma unroll
      for (int i = 0; i < kRing; ++i) dma(i * kRawBytes);
    }

    Half8 q[kK];
    float qs;
    {
      RowVec<E, 8> x[kK];
      float high = 0.f;
#pragma unroll
      for (int i = 0; i < kK; ++i) {
        x[i].load(qsrc + 32 * i);
#pragma unroll
        for (int j = 0; j < 8; ++j) high = fmaxf(high, fabsf(x[i].get(j)));
      }
      const HalfScale s(max_halves(fmaxf(high, __shfl_xor(high, 16))));
#pragma unroll
      for (int i = 0; i < kK; ++i) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = x[i].get(j) * s.down;
        q[i].floats(f);
      }
      qs = s.up * a.scale_log2;
    }
    // Where this lane's 16 bytes belong: of keys columns 16 h .. of token t, whose quads 2 h and 2 h + 1
    // have eight each; of values column m of tokens 8 a + 4 h + c, whose quads h and 2 + h have dwords
    // a of the same parity.
    const int h = lane / 32, t = lane % 32;
    const bool keys = group < kK;
    char* const to0 = reinterpret_cast<char*>(in.tile) +
                      (keys ? (t / 16 * kK + group) * 1024 + (2 * h * 16 + t % 16) * 16
                            : kValues + ((group - kK) * 2 + t / 16) * 1024 + (h * 16 + t % 16) * 16);
    const int to1 = keys ? 256 : 512;
    const char* const from = reinterpret_cast<const char*>(in.raw) + group * 1024 + lane * 16;
    // Widens this wave's part of a step from a slot into a tile, and asks for the step that takes its place.
    u32x4 raw;
    const auto fetch = [&](uint32_t slot) {
      if (group >= kBring) return;
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(kRing - 1));
      asm volatile("" ::: "memory");
      raw = *reinterpret_cast<const u32x4*>(from + slot);
    };
    const auto widen = [&](uint32_t slot, uint32_t tile) {
      if (group >= kBring) return;
      Half8 f[2];
      f[0].bytes(raw[0], keys ? raw[1] : raw[2]);
      f[1].bytes(keys ? raw[2] : raw[1], raw[3]);
      *reinterpret_cast<u32x4*>(to0 + tile) = __builtin_bit_cast(u32x4, f[0].x);
      *reinterpret_cast<u32x4*>(to0 + tile + to1) = __builtin_bit_cast(u32x4, f[1].x);
      dma(slot);                                   // behind writes of what was read there
    };
    const char* const tiles = reinterpret_cast<const char*>(in.tile) + lane * 16;
    const auto operand = [&](uint32_t at) { return Half8{__builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(tiles + at))}; };
    float x[8];
    const auto scores = [&](uint32_t tile) {
      f32x4 y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kK; ++k) y[i] = mma16(operand(tile + (i * kK + k) * 1024), q[k], y[i]);
      }
#pragma unroll
      for (int r = 0; r < 8; ++r) x[r] = y[r / 4][r % 4];
    };
    // Scales of 64 blocks, a lane each: the keys' as factors of the scores, the values' as soften takes them.
    float key_of_block = 0.f, lv_of_block = 0.f, rv_of_block = 0.f;
    int block_of_lane0 = 0;                        // from the sequence's first one on
    const auto load_scales = [&](int step) __attribute__((always_inline)) {
      block_of_lane0 = step / 2;
      const int64_t at = (w.s.block0 + min(block_of_lane0 + lane, (packed_end - 1) / 2)) * a.hkv + w.hk;
      key_of_block = a.k_scale[at];
      const float s = a.v_scale[at];
      meet(s);
      const ValueScale v(s, scales);
      lv_of_block = v.lv;
      rv_of_block = v.rv;
      // Waited for here, and not at each step's use.
      asm volatile("" : "+v"(key_of_block), "+v"(lv_of_block), "+v"(rv_of_block));
    };
    const auto of_block = [&](float x, int at) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at)); };
    fetch(0);
    widen(0, 0);
    fetch(kRawBytes);
    widen(kRawBytes, kTileBytes);
    load_scales(w.begin);
    __syncthreads();
    scores(0);
    const auto step = [&](int i, auto turn) {
      constexpr uint32_t kNow = decltype(turn)::value, kNext = (kNow + 1) % 3, kAfter = (kNow + 2) % 3;
      fetch(kAfter * kRawBytes);
      if (!idle) {
        const int st = w.begin + i;
        if (__builtin_expect(st / 2 - block_of_lane0 == kWave, 0)) load_scales(st);
        const int at = st / 2 - block_of_lane0;
        const float factor = mask_packed<16>(x, w.s.packed - st * kStep, of_block(key_of_block, at) * qs, 4 * quad);
        float p[8];
        sum.soften(x, factor, of_block(lv_of_block, at), of_block(rv_of_block, at), own, p);
        Half8 pf;
        pf.floats(p);
        scores(kNext * kTileBytes);
#pragma unroll
        for (int k = 0; k < kO; ++k) sum.o[k] = mma16(operand(kNow * kTileBytes + kValues + k * 1024), pf, sum.o[k]);
      }
      widen(kAfter * kRawBytes, kAfter * kTileBytes);
      __syncthreads();
    };
    for (int i = 0;; i += 3) {
      step(i, Turn<0>());
      if (i + 1 >= rounds) break;
      step(i + 1, Turn<1>());
      if (i + 2 >= rounds) break;
      step(i + 2, Turn<2>());
      if (i + 3 >= rounds) break;
    }
    __builtin_amdgcn_s_waitcnt(0);                 // no DMA may land in what LDS holds next
    __syncthreads();
  }

  // Open steps: rows as they are, staged a step ahead.
  const int first = max(w.begin, w.steps.packed), more = max(0, w.end - first);
  if (more > 0) {
    const int64_t pitch = (int64_t)a.hkv * D;
    const int open = w.s.ctx + w.s.n;
    const E* kp = static_cast<const E*>(a.k) + w.s.kv0 * pitch + w.hk * D;
    const E* vp = static_cast<const E*>(a.v) + w.s.kv0 * pitch + w.hk * D;
    Bf8 q[kK];
#pragma unroll
    for (int i = 0; i < kK; ++i) {
      RowVec<E, 8> x;
      x.load(qsrc + 32 * i);
      q[i].x = __builtin_bit_cast(bf16x8, u32x4{x.w[0], x.w[1], x.w[2], x.w[3]});
    }
    const auto stage = [&](int i) {
      const int t0 = (first + i - w.steps.packed) * kStep;
      Tile<D>& t = in.tile[i % 2];
      // Keys: eight columns of a token to a unit.
      if (tid < kStep * (D / 8)) {
        const int tk = tid / (D / 8), c = tid % (D / 8);
        RowVec<E, 8> x;
        x.load(kp + min(t0 + tk, open - 1) * pitch + 8 * c);
        t.k[tk / 16][c / 4][c % 4 * 16 + tk % 16] = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
      }
      if (tid < D) {
        ValueUnit<E, D, true> unit;
        unit.load(vp, pitch, t0, open - 1, tid);
        unit.store(t.v, tid);
      }
    };
    meet(1.f);
    const ValueScale one(1.f, scales);
    stage(0);
    __syncthreads();
    for (int i = 0; i < more; ++i) {
      if (i + 1 < more) stage(i + 1);
      const int t0 = (first + i - w.steps.packed) * kStep;
      // Later tokens than all of the wave's rows are seen by none of them.
      if (!idle && (a.parent || t0 - w.s.ctx <= last_node)) {
        const Tile<D>& t = in.tile[i % 2];
        float x[8], p[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          f32x4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < kK; ++k) y = mma16(Bf8{__builtin_bit_cast(bf16x8, t.k[b][k][lane])}, q[k], y);
#pragma unroll
          for (int r = 0; r < 4; ++r) x[4 * b + r] = y[r];
        }
        mask_open<16>(x, seen_of(a, w, trees, node, t0), a.scale_log2, 4 * quad);
        sum.soften(x, 1.f, one.lv, one.rv, own, p);
        Bf8 pf, rest;
        pf.floats(p);
        rest.rest(p, pf);
#pragma unroll
        for (int k = 0; k < kO; ++k) {
          const Bf8 f{__builtin_bit_cast(bf16x8, *t.v.many(k, lane))};
          sum.o[k] = mma16(f, pf, sum.o[k]);
          sum.o[k] = mma16(f, rest, sum.o[k]);
        }
      }
      __syncthreads();
    }
  }
  // A row's quads have neighbouring columns: 64 bytes of it to a store.
  const float l = sum.all();
  if (R0 + col >= w.rows) return;
  const int64_t at = (w.s.row0 + node) * a.hq + w.hk * a.group + (R - node * a.group);
  const float inv = l > 0.f ? 1.f / l : 0.f, ref = scales.apart ? *own() : sum.m, z = sum.m - ref + scales.z();
  if (quad == 0) write_lse(a, w, at, ref, l);
#pragma unroll
  for (int i = 0; i < kO; ++i) write<D>(a, w, at, 16 * i + 4 * quad, in_units(sum.o[i] * inv, z));
}

// Joins the splits of a row by their log-sum-exps: D / 4 lanes per (row, head), in two round trips of loads and
// one more for each eight splits (128 rows of 32 heads in 16 splits, 33 MB: 9 us; 10.5 with the
// log-sum-exps read twice by every lane and four splits at a time).
template <int D>
__global__ __launch_bounds__(256) void packed_merge(Args a) {
  constexpr int kLanes = D / 4;
  const int b = blockIdx.y;
  const Seq s = seq_of(a, b);
  const int64_t i = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const int col = threadIdx.x % kLanes * 4;
  if (!s.ok || i >= (int64_t)s.n * a.hq) return;
  const int n = (int)(i / a.hq), head = (int)(i % a.hq);
  const int rows = s.n * a.group, r0 = (n * a.group + head % a.group) / a.tile * a.tile;
  const Cut cut = cut_of(steps_of(a, s, min(r0 + a.tile, rows) - 1).all, a.tps, a.slots, a.quantum);
  if (cut.n == 1) return;                          // written whole
  const int64_t at = (s.row0 + n) * a.hq + head;
  // A lane has every kLanes-th split's log-sum-exp and weight.
  constexpr int kMine = kMaxSlots / kLanes;
  const int lane = threadIdx.x % kLanes;
  float weight[kMine], m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int j = k * kLanes + lane;
    weight[k] = j < cut.n ? a.part_lse[at * a.slots + j] : -INFINITY;
    m = fmaxf(m, weight[k]);
  }
  for (int d = kLanes / 2; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d, kLanes));
  if (m == -INFINITY) m = 0.f;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    weight[k] = fast_exp2(weight[k] - m);
    sum += weight[k];
  }
  for (int d = kLanes / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d, kLanes);
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  const float* const from = a.part_o + at * a.slots * D + col;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int n = min(kLanes, cut.n - k * kLanes);
    // Eight loads at a time, past the last split its own again with a weight of 0.
    for (int j0 = 0; j0 < n; j0 += 8) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        acc += __shfl(weight[k], j0 + u, kLanes) * *reinterpret_cast<const f32x4*>(from + (k * kLanes + min(j0 + u, n - 1)) * D);
    }
  }
  acc *= sum > 0.f ? 1.f / sum : 0.f;
  if (a.out_bf16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + col) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + col) = acc;
  if (col == 0 && a.lse) a.lse[at] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// Host: tiles, splits and workspace.
int64_t steps_of(int32_t packed, int32_t ctx, int32_t n) {
  return ((int64_t)packed + kStep - 1) / kStep + ((int64_t)ctx + n + kStep - 1) / kStep;
}

// How a call is shared out: waves of a tile of many rows (0: few rows) and its rows, and splits.
struct Plan {
  int32_t groups, tile, tiles, tps, quantum, slots;
};

// A form of tile, and what its workgroup takes in us: a step alone on a CU, and at least, as a share of
// the CU; and besides its steps. Fitted to trees of 20 to 48 nodes (d = 128; few rows: 0.27 and 0.21 for
// 32 rows, many: 0.77 and 0.7 for 128, 1.05 for 256). Few rows do better where a workgroup has few steps (16 trees
// on 1024 to 4096 tokens 61 us, 90 with many), as more and smaller ones spread better, many rows where it has
// many (four trees of 32 nodes on 32768 tokens 101 us, 112 with few; a prompt of 2048 on 4000 262 and 288).
struct Form {
  int32_t groups, tile, quantum, per_cu;             // per_cu workgroups fit on a CU
  double alone, least, start;
};
constexpr double kJoin = 5;                          // of the launch that joins splits
constexpr double kJoined = 1200000;                  // values of splits written and joined in a microsecond
constexpr double kStream = 5900000;                  // bytes read in one
constexpr int kFewest = 4;                           // steps of a split

// Parts of a call: rows * hq * slots of d + 1 floats.
constexpr int64_t kMostBytes = int64_t(1) << 30;

// Planned from the host's sizes, with tiles for the n_max rows that the device's may reach.
Plan plan_of(int32_t dtype, int32_t batch, int64_t rows, int32_t n_max, int32_t hq, int32_t hkv, int32_t d, const int32_t* n,
             const int32_t* packed, const int32_t* ctx, int32_t kv_split) {
  const int64_t group = hq / hkv, cus = device_cu_count();
  int64_t most_rows = 0, longest = 1;
  for (int32_t b = 0; b < batch; ++b) {
    most_rows = std::max<int64_t>(most_rows, n[b] * group);
    if (n[b] > 0) longest = std::max(longest, steps_of(packed[b], ctx[b], n[b]));
  }
  const double room = kMostBytes / ((double)std::max<int64_t>(1, rows) * hq * (d + 1) * 4);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(longest, (int64_t)std::min((double)kMaxSlots, room)));
  double stream = 0;                                 // what the bytes of all sequences take
  for (int32_t b = 0; b < batch; ++b)
    if (n[b] > 0) stream += (double)steps_of(packed[b], ctx[b], n[b]) * hkv * (2 * kStep * d) / kStream;
  Plan best{};
  double best_time = -1;
  // As many splits as asked for, or those that should take least: as many turns of the longest, or all work
  // spread evenly and a quarter of one more. Tried are one, and half of, about and twice those with which
  // every place has one.
  const auto consider = [&](const Form& f, int64_t slots) {
    Plan p{f.groups, f.tile, (int32_t)std::max<int64_t>(1, (std::min<int64_t>(n_max, rows) * group + f.tile - 1) / f.tile), 0, f.quantum,
           (int32_t)std::max<int64_t>(1, std::min(slots, most))};
    p.tps = (int32_t)(((longest + p.slots - 1) / p.slots + f.quantum - 1) / f.quantum * f.quantum);
    int64_t groups = 0, high = 0;
    double work = 0;
    for (int32_t b = 0; b < batch; ++b) {
      if (n[b] <= 0) continue;
      const Cut c = cut_of((int)steps_of(packed[b], ctx[b], n[b]), p.tps, p.slots, f.quantum);
      const int64_t g = (n[b] * group + f.tile - 1) / f.tile * hkv * c.n;
      groups += g;
      work += (double)g * c.per;
      high = std::max<int64_t>(high, c.per);
    }
    // The launch's workgroups that find nothing to do keep some places from the others at first: eight
    // single tokens with 4096 to 32768 tokens take 64 us in 472 workgroups and 75 in 512.
    const int64_t at_once = f.per_cu * cus;
    const int64_t places = groups < (int64_t)hkv * p.tiles * p.slots * batch ? at_once - at_once / 16 : at_once;
    const int64_t beside = std::min<int64_t>(f.per_cu, (groups + cus - 1) / cus);
    const double step = std::max(f.alone, f.least * beside), start = f.start * (0.75 + 0.25 * beside), one = high * step + start;
    double time = std::min((double)((groups + places - 1) / places) * one,
                           std::max(one, (work * f.least + groups * start / f.per_cu) / cus + one / 4));
    time = std::max(time, stream);
    if (p.slots > 1) time += kJoin + (double)rows * hq * p.slots * d / kJoined;
    if (best_time >= 0 && time >= best_time) return;
    best_time = time;
    best = p;
  };
  const auto consider_all = [&](const Form& f) {
    if (kv_split > 0) return consider(f, kv_split);
    double total = 1;                                // steps of all workgroups
    for (int32_t b = 0; b < batch; ++b)
      if (n[b] > 0) total += (double)((n[b] * group + f.tile - 1) / f.tile * hkv) * steps_of(packed[b], ctx[b], n[b]);
    const int64_t useful = (longest + kFewest - 1) / kFewest;
    const int64_t even = (int64_t)std::min(std::ceil((double)longest * f.per_cu * cus / total), (double)kMaxSlots);
    int64_t last = 1;
    consider(f, 1);
    for (int64_t slots : {even / 2, even - 2, even - 1, even, 2 * even}) {
      slots = std::min(slots, useful);
      if (slots <= last) continue;
      consider(f, slots);
      last = slots;
    }
  };
  if (dtype == CURE_F32) {
    consider_all(d == 128 ? Form{0, kRows, kWaves, 2, 1.2, 1.15, 12} : Form{0, kRows, kWaves, 2, 0.63, 0.55, 12});
    return best;
  }
  consider_all(d == 128 ? Form{0, kRows, kWaves, 2, 0.27, 0.21, 8} : Form{0, kRows, kWaves, 2, 0.2, 0.18, 8});
  if (most_rows > 2 * kRows) {
    consider_all(d == 128 ? Form{8, 8 * kManyRows, 1, 2, 0.77, 0.7, 12} : Form{8, 8 * kManyRows, 1, 3, 0.55, 0.545, 12});
    // 256 rows where they are a sequence's all: its keys are then read and widened once.
    if (d == 128 && most_rows > 8 * kManyRows && most_rows <= 16 * kManyRows) consider_all(Form{16, 16 * kManyRows, 1, 1, 1.05, 1.05, 12});
  }
  return best;
}

size_t space_of(const Plan& p, int64_t rows, int32_t hq, int32_t d) {
  return p.slots == 1 ? 0 : (size_t)rows * hq * p.slots * (d + 1) * sizeof(float);
}

bool sizes_ok(int32_t batch, int32_t n_max, const int32_t* n, const int32_t* packed, const int32_t* ctx) {
  for (int32_t b = 0; b < batch; ++b)
    if (n[b] < 0 || n[b] > n_max || packed[b] < 0 || ctx[b] < 0) return false;
  return true;
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" size_t cure_packed_attn_workspace_size(int32_t batch, int64_t rows, int32_t n_max, int32_t hq,
                                                  int32_t hkv, int32_t d, const int32_t* host_n_rows,
                                                  const int32_t* host_packed_len,
                                                  const int32_t* host_ctx_len, int32_t kv_split) {
  if (batch <= 0 || rows <= 0 || n_max <= 0 || hq <= 0 || hkv <= 0 || hq % hkv || d <= 0 || kv_split < 0 ||
      !host_n_rows || !host_packed_len || !host_ctx_len ||
      !sizes_ok(batch, n_max, host_n_rows, host_packed_len, host_ctx_len))
    return 0;
  size_t most = 0;
  for (int32_t dtype : {CURE_F32, CURE_BF16})
    most = std::max(most, space_of(plan_of(dtype, batch, rows, n_max, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split), rows, hq, d));
  return most;
}

extern "C" cure_status cure_packed_attn(const void* q, const int8_t* pk, const int8_t* pv,
                                        const float* k_scale, const float* v_scale, int64_t blocks,
                                        const void* k, const void* v, int64_t cache_rows, void* o, float* lse,
                                        int32_t dtype, int32_t out_dtype, int32_t batch, int64_t rows,
                                        int32_t n_max, int32_t hq, int32_t hkv, int32_t d, float scale,
                                        const int64_t* row_off, const int32_t* n_rows,
                                        const int64_t* blk_off, const int32_t* packed_len,
                                        const int64_t* kv_off, const int32_t* ctx_len,
                                        const int32_t* parent, const int32_t* host_n_rows,
                                        const int32_t* host_packed_len, const int32_t* host_ctx_len,
                                        int32_t kv_split, int32_t* row_status, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  if ((dtype != CURE_F32 && dtype != CURE_BF16) || (out_dtype != CURE_F32 && out_dtype != CURE_BF16))
    return CURE_ERR_INVALID_ARG;
  if (batch < 0 || rows < 0 || n_max < 0 || blocks < 0 || cache_rows < 0 || hq <= 0 || hkv <= 0 || hq % hkv || d <= 0 ||
      kv_split < 0)
    return CURE_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale * kLog2e)) return CURE_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return CURE_ERR_UNSUPPORTED;
  if (batch > 65535 || (int64_t)n_max * hq > (int64_t(1) << 28) || (parent && n_max > CURE_MAX_TREE_NODES))
    return CURE_ERR_UNSUPPORTED;
  if (batch == 0) return CURE_OK;
  if (!n_rows || !blk_off || !packed_len || !kv_off || !ctx_len || !host_n_rows || !host_packed_len || !host_ctx_len)
    return CURE_ERR_INVALID_ARG;
  if (n_max > 0 && (!q || !k || !v || !o)) return CURE_ERR_INVALID_ARG;
  if (n_max > 0 && blocks > 0 && (!pk || !pv || !k_scale || !v_scale)) return CURE_ERR_INVALID_ARG;
  if (!row_off && n_max > 0 && rows / n_max < batch) return CURE_ERR_INVALID_ARG;      // padded rows
  if (!sizes_ok(batch, n_max, host_n_rows, host_packed_len, host_ctx_len)) return CURE_ERR_INVALID_ARG;
  for (int32_t b = 0; b < batch; ++b)
    if ((int64_t)host_packed_len[b] + host_ctx_len[b] + host_n_rows[b] > kMostTokens) return CURE_ERR_UNSUPPORTED;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if ((at(q) | at(pk) | at(pv) | at(k) | at(v) | at(o)) % 16) return CURE_ERR_INVALID_ARG;
  const Plan p = plan_of(dtype, batch, rows, n_max, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split);
  const size_t need = space_of(p, rows, hq, d);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CURE_ERR_WORKSPACE;
  if (need > 0 && at(workspace) % 16) return CURE_ERR_INVALID_ARG;
  const int64_t wgs = (int64_t)hkv * p.tiles * p.slots;
  const int threads = (p.groups ? p.groups : kWaves) * kWave;
  if (wgs * threads >= (int64_t(1) << 32)) return CURE_ERR_UNSUPPORTED;         // a launch counts threads in 32 bits
  float* part_o = static_cast<float*>(workspace);
  Args a{q, pk, pv, k_scale, v_scale, blocks, k, v, cache_rows, o, lse, out_dtype == CURE_BF16, batch, n_max, hq, hkv, hq / hkv,
         rows, scale * kLog2e, row_off, n_rows, blk_off, packed_len, kv_off, ctx_len, parent, row_status, p.tile, p.tiles, p.tps, p.quantum, p.slots,
         part_o, p.slots > 1 ? part_o + rows * hq * p.slots * d : nullptr};
  hipStream_t st = as_stream(stream);
  const dim3 grid((unsigned)wgs, (unsigned)batch), block(threads);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  const bool once = p.tiles == 1;
  if (dtype == CURE_F32 && once) d == 128 ? run(packed_few<float, 128, true>) : run(packed_few<float, 64, true>);
  else if (dtype == CURE_F32) d == 128 ? run(packed_few<float, 128, false>) : run(packed_few<float, 64, false>);
  else if (!p.groups && once) d == 128 ? run(packed_few<uint16_t, 128, true>) : run(packed_few<uint16_t, 64, true>);
  else if (!p.groups) d == 128 ? run(packed_few<uint16_t, 128, false>) : run(packed_few<uint16_t, 64, false>);
  else if (p.groups == 16) run(packed_many<128, 16>);
  else d == 128 ? run(packed_many<128, 8>) : run(packed_many<64, 8>);
  const cure_status launched = launch_status();
  if (launched != CURE_OK || p.slots == 1 || n_max == 0) return launched;
  const int per = 256 / (d / 4);
  // No sequence has more than `rows`, which parts of 1 GB bound to 2^21 rows and heads.
  const dim3 mgrid((unsigned)((std::min<int64_t>(n_max, rows) * hq + per - 1) / per), (unsigned)batch);
  if (d == 128) hipLaunchKernelGGL((packed_merge<128>), mgrid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((packed_merge<64>), mgrid, dim3(256), 0, st, a);
  return launch_status();
}
