// cure_packed_attn: attention of candidate trees, single tokens or chunks of prompts over a
// context whose tokens are packed in blocks of 64 with 8 bits a value (cure_kv_pack), the open
// rows behind it and the new rows themselves.
//
// Query row R of a kv-head is query head R % group of token R / group, so the heads that
// share keys share a tile. With C the bytes and s_k, s_v the scales of a token's block,
//   S = s_k (C_k Q^T),  P = s_v 2^(S - m),  l += P / s_v,  O^T += C_v^T P^T,  o = O / l
// in one pass over the keys with the reference m, a running maximum of S + log2 s_v, and l in fp32.
// The value's scale is part of the exponent, so a block whose values are large and one
// whose values are small both have P in the range of 16 bits where they count at all.
//
// bf16: the bytes are widened to fp16, which holds them exactly, and the query rows are too, times
// a power of two for each row: what that loses is below 2^-40 of the row's largest. P is rounded
// to fp16 for its product, 2^-12 where bf16 would take 2^-9 and add half as much again to the error that the
// output's own rounding makes. Open rows keep bf16's range: their products take P as two bf16 values.
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
// exchange between lanes.
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
constexpr int kWaves = 4;            // waves per workgroup
constexpr int kRows = 32;            // query rows of a wave
constexpr int kMaxGroups = 4;        // row groups of a workgroup at most
constexpr int kMaxSlots = 64;        // splits of a row's keys at most
constexpr float kNone = -3e38f;      // reference of a row that has seen nothing
constexpr int kAncWords = CURE_MAX_TREE_NODES / 32;

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
         s.kv0 <= a.cache_rows - s.ctx - s.n;
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
CURE_DEV Cut cut_of(const Args& a, int steps) {
  const int n = max(1, min((steps - 1) / a.tps + 1, a.slots));
  const int per = ((steps - 1) / n / a.quantum + 1) * a.quantum;
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

// Token of D register r in a lane's half.
CURE_DEV int token_of(int half, int r) { return 8 * (r / 4) + 4 * half + r % 4; }

// A lane's query row and what it has summed.
template <int D>
struct Sums {
  float m = kNone, l = 0.f;
  f32x16 o[D / 32];

  CURE_DEV Sums() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = zeros();
  }
  // Scores x * factor of base 2 (-inf: not seen; factor > 0 there) of tokens whose values have scale 2^lv and
  // its reciprocal rv: their P.
  CURE_DEV void soften(const f32x16& x, float factor, float lv, float rv, float (&p)[16]) {
    const float high = fmaf(max_halves(max_scores(x)), factor, lv);
    if (__any(high > m + kRescaleLog2)) {
      const float mn = fmaxf(m, high), f = fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= f;
    }
    const float c = lv - m;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = fast_exp2(fmaf(x[r], factor, c));
      sum[r % 2] += p[r];
    }
    l = fmaf(sum[0] + sum[1], rv, l);
  }
};

// The scale of a block's values as soften takes it. Blocks of zeros, and of values below
// 2^-93, have no products, and a scale that keeps their probabilities in range.
struct ValueScale {
  float lv, rv;
  bool any;
  CURE_DEV explicit ValueScale(float s) {
    any = s >= 0x1p-100f;
    lv = any ? __builtin_amdgcn_logf(s) : -60.f;
    rv = any ? 1.f / s : 0x1p60f;
  }
};

// Query rows as fp16: times 2^-e, for the largest of the row to be in [2^14, 2^15). Returns 2^e.
template <int D>
CURE_DEV float half_rows(const RowVec<uint16_t, 16> (&x)[D / 32], Half8 (&q)[D / 32][2]) {
  float high = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) high = fmaxf(high, fabsf(x[i].get(j)));
  high = max_halves(high);
  int e = (int)(__float_as_uint(high) >> 23) - 127 - 14;
  e = max(-120, min(e, 120));
  const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = x[i].get(8 * u + j) * down;
      q[i][u].floats(f);
    }
  return __uint_as_float((uint32_t)(127 + e) << 23);
}
template <int D>
CURE_DEV float half_rows(const RowVec<float, 16> (&x)[D / 32], Float8 (&q)[D / 32][2]) {
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

// Four, or two, values of a row that no query row need see: an infinity or NaN would reach the
// others through its zero probabilities.
CURE_DEV uint32_t finite2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
CURE_DEV float finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : x; }

// What a workgroup works on.
struct Work {
  Seq s;
  Steps steps;
  Cut cut;
  int b, hk, slot, r0, rows, node0;  // first packed row of the tile, of `rows`, and its node
  int begin, end;                    // steps
};

struct Trees {
  uint32_t anc[kRows * kMaxGroups][kAncWords];   // root paths of the tile's nodes, as bits
  int parent[CURE_MAX_TREE_NODES];
};

// Finds the workgroup's work, reports the sequence's status and forms the root paths. False: nothing
// to do. The grid: kv-heads, tiles, splits; sequences. A sequence's workgroups on one kv-head
// are hkv apart, so where that is a multiple of 8 they share an XCD's L2.
CURE_DEV bool locate(const Args& a, Work& w, Trees& sh) {
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
  w.cut = cut_of(a, w.steps.all);
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
CURE_DEV uint32_t seen_of(const Args& a, const Work& w, const Trees& sh, int node, int t0) {
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

// Where a workgroup's rows are joined and turned: a wave's 32 rows.
template <int D>
struct Out {
  float o[kWaves][kRows][D + 4];
  float m[kWaves][kRows], l[kWaves][kRows];
};

// Writes a tile's rows: kGroups groups of 32 rows, each the sum of kWaves / kGroups waves (wave w
// has rows of group w % kGroups). Nothing else may use sh any more.
template <int D, int kGroups>
CURE_DEV void finish(const Args& a, const Work& w, Out<D>& sh, Sums<D>& sum) {
  constexpr int kParts = kWaves / kGroups, kChunks = D / 4;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, col = lane % 32, half = lane / 32;
  const float l = sum_halves(sum.l);
  if (half == 0) {
    sh.m[wave][col] = sum.m;
    sh.l[wave][col] = l;
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<f32x4*>(&sh.o[wave][col][32 * i + 8 * (r / 4) + 4 * half]) =
          f32x4{sum.o[i][r], sum.o[i][r + 1], sum.o[i][r + 2], sum.o[i][r + 3]};
  __syncthreads();
  const bool whole = w.cut.n == 1;
  for (int c = tid; c < kGroups * kRows * kChunks; c += kWaves * kWave) {
    const int row = c / kChunks, j = c % kChunks * 4, group = row / kRows, rr = row % kRows;
    if (w.r0 + row >= w.rows) break;
    float m = kNone, ll = 0.f, f[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) m = fmaxf(m, sh.m[group + k * kGroups][rr]);
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      f[k] = fast_exp2(sh.m[group + k * kGroups][rr] - m);
      ll += f[k] * sh.l[group + k * kGroups][rr];
    }
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
    f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kParts; ++k) x += f[k] * *reinterpret_cast<const f32x4*>(&sh.o[group + k * kGroups][rr][j]);
    x *= inv;
    const int R = w.r0 + row;
    const int64_t at = (w.s.row0 + R / a.group) * a.hq + w.hk * a.group + R % a.group;
    if (j == 0) {
      const float lse2 = ll > 0.f ? m + log2f(ll) : -INFINITY;
      if (!whole) a.part_lse[at * a.slots + w.slot] = lse2;
      else if (a.lse) a.lse[at] = lse2 * kLn2;
    }
    if (!whole) *reinterpret_cast<f32x4*>(a.part_o + (at * a.slots + w.slot) * D + j) = x;
    else if (a.out_bf16)
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + j) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + j) = x;
  }
}

// Scores of packed tokens, of which `left` are there, times `factor`; returns the factor that is left.
CURE_DEV float mask_packed(f32x16& x, int half, int left, float factor) {
  if (left >= kStep) return factor;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = token_of(half, r) < left ? x[r] * factor : -INFINITY;
  return 1.f;
}

// ---------------------------------------------------------------------------
// Up to 32 query rows to a tile: the waves take the steps in turn, each with all rows and sums of its
// own, which are joined at the end. Packed bytes go from memory to registers and into the
// matrix unit, a step ahead of their use.
template <typename E, int D>
__global__ __launch_bounds__(kWaves * kWave, 2) void packed_few(Args a) {
  constexpr int kK = D / 32;                       // pieces of 32 columns
  using Byte = typename Types<E>::Byte;
  using RowF = typename Types<E>::Row;
  __shared__ __attribute__((aligned(16))) Out<D> out;
  __shared__ Trees trees;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int col = lane % 32, half = lane / 32;
  Work w;
  if (!locate(a, w, trees)) return;

  // This lane's query row.
  const int R = min(w.r0 + col, w.rows - 1), node = R / a.group;
  const E* qsrc = static_cast<const E*>(a.q) + ((w.s.row0 + node) * a.hq + w.hk * a.group + R % a.group) * D + 16 * half;
  Sums<D> sum;
  int step = w.begin + wave;
  const int packed_end = min(w.end, w.steps.packed);
  if (step < packed_end) {
    Byte q[kK][2];
    float qs;
    {
      RowVec<E, 16> x[kK];
      load_rows<E, D>(qsrc, x);
      qs = half_rows<D>(x, q) * a.scale_log2;
    }
    struct Raw {
      u32x4 k[kK], v[kK];
      float ks, vs;
    };
    const auto fetch = [&](Raw& raw, int st) {
      const int64_t block = (w.s.block0 + st / 2) * a.hkv + w.hk;
      const int64_t at = block * (kBlockTokens * D) + st % 2 * (kStep * D) + lane * 16;
#pragma unroll
      for (int i = 0; i < kK; ++i) raw.k[i] = *reinterpret_cast<const u32x4*>(a.pk + at + i * 1024);
#pragma unroll
      for (int i = 0; i < kK; ++i) raw.v[i] = *reinterpret_cast<const u32x4*>(a.pv + at + i * 1024);
      raw.ks = a.k_scale[block];
      raw.vs = a.v_scale[block];
    };
    Raw next;
    fetch(next, step);
    for (; step < packed_end; step += kWaves) {
      const Raw raw = next;
      fetch(next, min(step + kWaves, packed_end - 1));
      f32x16 x = zeros();
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Byte f;
          f.bytes(raw.k[i][2 * u], raw.k[i][2 * u + 1]);
          x = mma(f, q[i][u], x);
        }
      const ValueScale vs(raw.vs);
      float p[16];
      const float factor = mask_packed(x, half, w.s.packed - step * kStep, raw.ks * qs);
      sum.soften(x, factor, vs.lv, vs.rv, p);
      if (vs.any) {
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
      }
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
    for (; step < w.end; step += kWaves) {
      const int t0 = (step - w.steps.packed) * kStep;
      RowVec<E, 16> kx[kK];
      load_rows<E, D>(kp + min(t0 + col, open - 1) * pitch + 16 * half, kx);
      f32x16 x = zeros();
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          RowF f;
          f.row(kx[i], u);
          x = mma(f, q[i][u], x);
        }
      const uint32_t seen = seen_of(a, w, trees, node, t0);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = seen >> token_of(half, r) & 1 ? x[r] * a.scale_log2 : -INFINITY;
      float p[16];
      sum.soften(x, 1.f, 0.f, 1.f, p);
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
          const E* src = vp + 32 * i + col;
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const E e = src[min(t0 + token_of(half, 8 * t + j), open - 1) * pitch];
            y[j] = finite(sizeof(E) == 2 ? __uint_as_float((uint32_t)e << 16) : (float)e);
          }
          f.floats(y);
          sum.o[i] = mma(f, pf[t], sum.o[i]);
          if constexpr (sizeof(E) == 2) sum.o[i] = mma(f, rest[t], sum.o[i]);
        }
    }
  }
  finish<D, 1>(a, w, out, sum);
}

// ---------------------------------------------------------------------------
// More rows (bf16): kGroups groups of 32 query rows, a wave each, share a step's keys and
// values, which they widen together and hand on through LDS, two steps' room for each of the kWaves /
// kGroups sets of waves that take the steps in turn. An operand's 64 lanes of 16 bytes are 1 KB of
// LDS, written and read without conflicts.
template <int D>
struct Tile {
  u32x4 k[D / 32][2][kWave], v[D / 32][2][kWave];
};
template <int D, int kGroups>
union Many {
  Tile<D> tile[2][kWaves / kGroups];
  Out<D> out;
};

template <int D, int kGroups>
__global__ __launch_bounds__(kWaves * kWave, 2) void packed_many(Args a) {
  using E = uint16_t;
  constexpr int kK = D / 32;
  constexpr int kSets = kWaves / kGroups;
  constexpr int kThreads = kGroups * kWave;        // of a set
  constexpr int kUnits = kK * kWave / kThreads;    // 16-byte units of packed keys, and of values, per thread
  static_assert(kK * kWave % kThreads == 0 || kK * kWave < kThreads, "");
  constexpr int kMine = kUnits > 0 ? kUnits : 1;
  __shared__ __attribute__((aligned(16))) Many<D, kGroups> sh;
  __shared__ Trees trees;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int col = lane % 32, half = lane / 32;
  const int set = wave / kGroups, me = tid % kThreads;
  Work w;
  if (!locate(a, w, trees)) return;

  const int R0 = w.r0 + wave % kGroups * kRows, R = min(R0 + col, w.rows - 1), node = R / a.group;
  const int last_node = min(R0 + kRows - 1, w.rows - 1) / a.group;
  const E* qsrc = static_cast<const E*>(a.q) + ((w.s.row0 + node) * a.hq + w.hk * a.group + R % a.group) * D + 16 * half;
  const bool idle = R0 >= w.rows;                  // this wave's rows are not there
  Sums<D> sum;
  Half8 q[kK][2];
  float qs;
  {
    RowVec<E, 16> x[kK];
    load_rows<E, D>(qsrc, x);
    qs = half_rows<D>(x, q) * a.scale_log2;
  }
  const int packed_end = min(w.end, w.steps.packed);
  const int64_t pitch = (int64_t)a.hkv * D;
  const int open = w.s.ctx + w.s.n;
  const E* kp = static_cast<const E*>(a.k) + w.s.kv0 * pitch + w.hk * D;
  const E* vp = static_cast<const E*>(a.v) + w.s.kv0 * pitch + w.hk * D;

  struct Raw {
    u32x4 k[kMine], v[kMine];
  };
  const auto block_of = [&](int st) { return (w.s.block0 + st / 2) * a.hkv + w.hk; };
  const auto fetch = [&](Raw& raw, int st) {
    if (st >= packed_end || me >= kK * kWave) return;
    const int64_t at = block_of(st) * (kBlockTokens * D) + st % 2 * (kStep * D) + me * 16;
#pragma unroll
    for (int i = 0; i < kMine; ++i) raw.k[i] = *reinterpret_cast<const u32x4*>(a.pk + at + i * kThreads * 16);
#pragma unroll
    for (int i = 0; i < kMine; ++i) raw.v[i] = *reinterpret_cast<const u32x4*>(a.pv + at + i * kThreads * 16);
  };
  // A packed step's bytes, fetched before, or an open step's rows.
  const auto stage = [&](const Raw& raw, int st, Tile<D>& t) {
    if (st >= w.end) return;
    if (st < packed_end) {
      if (me >= kK * kWave) return;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int unit = me + i * kThreads, piece = unit / kWave, ln = unit % kWave;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Half8 f;
          f.bytes(raw.k[i][2 * u], raw.k[i][2 * u + 1]);
          t.k[piece][u][ln] = __builtin_bit_cast(u32x4, f.x);
          f.bytes(raw.v[i][2 * u], raw.v[i][2 * u + 1]);
          t.v[piece][u][ln] = __builtin_bit_cast(u32x4, f.x);
        }
      }
      return;
    }
    const int t0 = (st - w.steps.packed) * kStep;
    // Keys: 16 columns of a token to a unit.
    for (int unit = me; unit < kStep * (D / 16); unit += kThreads) {
      const int tok = unit / (D / 16), c = unit % (D / 16);
      RowVec<E, 16> x;
      x.load(kp + min(t0 + tok, open - 1) * pitch + 16 * c);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        t.k[c / 2][u][c % 2 * 32 + tok] = u32x4{x.w[4 * u], x.w[4 * u + 1], x.w[4 * u + 2], x.w[4 * u + 3]};
    }
    // Values: two columns of the eight tokens that a lane has in a k-step.
    for (int unit = me; unit < 4 * (D / 2); unit += kThreads) {
      const int c = unit % (D / 2) * 2, g = unit / (D / 2), h = g % 2, ks = g / 2;
      uint32_t x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = finite2(*reinterpret_cast<const uint32_t*>(vp + min(t0 + token_of(h, 8 * ks + j), open - 1) * pitch + c));
      u32x4 lo, hi;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
        hi[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
      }
      t.v[c / 32][ks][h * 32 + c % 32] = lo;
      t.v[c / 32][ks][h * 32 + c % 32 + 1] = hi;
    }
  };

  // Step `it` of the set is step w.begin + it * kSets + set. One step is staged ahead of the one at
  // work, and the bytes of the one after that are on their way.
  const int count = (w.end - w.begin + kSets - 1) / kSets;
  const auto step_of = [&](int it) { return w.begin + it * kSets + set; };
  Raw raw;
  fetch(raw, step_of(0));
  stage(raw, step_of(0), sh.tile[0][set]);
  fetch(raw, step_of(1));
  float ks = 0.f, vsc = 0.f;
  const auto scales = [&](int st) {
    if (st < packed_end) {
      ks = a.k_scale[block_of(st)];
      vsc = a.v_scale[block_of(st)];
    }
  };
  scales(step_of(0));
  __syncthreads();
  bool rows = false;                               // q holds the rows as they are
  Bf8 qr[kK][2];
  for (int it = 0; it < count; ++it) {
    const int st = step_of(it);
    const float ks_now = ks, vs_now = vsc;
    stage(raw, step_of(it + 1), sh.tile[(it + 1) % 2][set]);
    fetch(raw, step_of(it + 2));
    scales(step_of(it + 1));
    const Tile<D>& t = sh.tile[it % 2][set];
    if (st < packed_end && !idle) {
      f32x16 x = zeros();
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) x = mma(Half8{__builtin_bit_cast(f16x8, t.k[i][u][lane])}, q[i][u], x);
      const ValueScale vs(vs_now);
      float p[16];
      const float factor = mask_packed(x, half, w.s.packed - st * kStep, ks_now * qs);
      sum.soften(x, factor, vs.lv, vs.rv, p);
      if (vs.any) {
        Half8 pf[2];
        pf[0].floats(p);
        pf[1].floats(p + 8);
#pragma unroll
        for (int i = 0; i < kK; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) sum.o[i] = mma(Half8{__builtin_bit_cast(f16x8, t.v[i][u][lane])}, pf[u], sum.o[i]);
      }
    } else if (st < w.end && !idle) {
      const int t0 = (st - w.steps.packed) * kStep;
      if (!rows) {
        RowVec<E, 16> xr[kK];
        load_rows<E, D>(qsrc, xr);
#pragma unroll
        for (int i = 0; i < kK; ++i) {
          qr[i][0].row(xr[i], 0);
          qr[i][1].row(xr[i], 1);
        }
        rows = true;
      }
      // Later tokens than all of the wave's rows see nothing of it.
      if (a.parent || t0 - w.s.ctx <= last_node) {
        f32x16 x = zeros();
#pragma unroll
        for (int i = 0; i < kK; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) x = mma(Bf8{__builtin_bit_cast(bf16x8, t.k[i][u][lane])}, qr[i][u], x);
        const uint32_t seen = seen_of(a, w, trees, node, t0);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = seen >> token_of(half, r) & 1 ? x[r] * a.scale_log2 : -INFINITY;
        float p[16];
        sum.soften(x, 1.f, 0.f, 1.f, p);
        Bf8 pf[2], rest[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          pf[u].floats(p + 8 * u);
          rest[u].rest(p + 8 * u, pf[u]);
        }
#pragma unroll
        for (int i = 0; i < kK; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Bf8 f{__builtin_bit_cast(bf16x8, t.v[i][u][lane])};
            sum.o[i] = mma(f, pf[u], sum.o[i]);
            sum.o[i] = mma(f, rest[u], sum.o[i]);
          }
      }
    }
    __syncthreads();
  }
  finish<D, kGroups>(a, w, sh.out, sum);
}

// Joins the splits of a row by their log-sum-exps: D / 4 lanes per (row, head).
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
  const Cut cut = cut_of(a, steps_of(a, s, min(r0 + a.tile, rows) - 1).all);
  if (cut.n == 1) return;                          // written whole
  const int64_t at = (s.row0 + n) * a.hq + head;
  float m = -INFINITY, sum = 0.f;
  for (int j = 0; j < cut.n; ++j) m = fmaxf(m, a.part_lse[at * a.slots + j]);
  if (m == -INFINITY) m = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < cut.n; ++j) {
    const float w = fast_exp2(a.part_lse[at * a.slots + j] - m);
    sum += w;
    acc += w * *reinterpret_cast<const f32x4*>(a.part_o + (at * a.slots + j) * D + col);
  }
  acc *= sum > 0.f ? 1.f / sum : 0.f;
  if (a.out_bf16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + col) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + col) = acc;
  if (col == 0 && a.lse) a.lse[at] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// Host: tiles, splits and workspace.
struct Plan {
  int32_t groups, tiles, tps, quantum, slots;
};

// Parts of a call: rows * hq * slots of d + 1 floats.
constexpr int64_t kMostBytes = int64_t(1) << 30;

Plan plan_of(int32_t dtype, int32_t batch, int64_t rows, int32_t hq, int32_t hkv, int32_t d, const int32_t* n,
             const int32_t* packed, const int32_t* ctx, int32_t kv_split) {
  const int64_t group = hq / hkv;
  int64_t most_rows = 0;
  for (int32_t b = 0; b < batch; ++b) most_rows = std::max<int64_t>(most_rows, n[b] * group);
  Plan p;
  p.groups = dtype == CURE_F32 || most_rows <= kRows ? 1 : most_rows <= 2 * kRows ? 2 : 4;
  p.quantum = kWaves / p.groups;
  const int64_t tile = p.groups * kRows;
  int64_t total = 0, longest = 1;
  for (int32_t b = 0; b < batch; ++b) {
    if (n[b] <= 0) continue;
    const int64_t steps = ((int64_t)packed[b] + kStep - 1) / kStep + ((int64_t)ctx[b] + n[b] + kStep - 1) / kStep;
    total += (n[b] * group + tile - 1) / tile * hkv * steps;
    longest = std::max(longest, steps);
  }
  p.tiles = (int32_t)std::max<int64_t>(1, (most_rows + tile - 1) / tile);
  // Two workgroups per CU, of at least eight steps.
  const int64_t target = 2 * (int64_t)device_cu_count();
  int64_t tps = kv_split > 0 ? (longest + kv_split - 1) / kv_split : std::max<int64_t>(8, (total + target - 1) / target);
  tps = (tps + p.quantum - 1) / p.quantum * p.quantum;
  const int64_t room = kMostBytes / std::max<int64_t>(1, rows * hq * (d + 1) * 4);
  p.slots = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(longest + tps - 1) / tps, (int64_t)kMaxSlots, room}));
  p.tps = (int32_t)tps;
  return p;
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
    most = std::max(most, space_of(plan_of(dtype, batch, rows, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split), rows, hq, d));
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
  if (n_max > 0 && (!q || !pk || !pv || !k_scale || !v_scale || !k || !v || !o)) return CURE_ERR_INVALID_ARG;
  if (!row_off && n_max > 0 && rows / n_max < batch) return CURE_ERR_INVALID_ARG;      // padded rows
  if (!sizes_ok(batch, n_max, host_n_rows, host_packed_len, host_ctx_len)) return CURE_ERR_INVALID_ARG;
  for (int32_t b = 0; b < batch; ++b)
    if ((int64_t)host_packed_len[b] + host_ctx_len[b] + host_n_rows[b] > INT32_MAX - 4096) return CURE_ERR_UNSUPPORTED;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if ((at(q) | at(pk) | at(pv) | at(k) | at(v) | at(o)) % 16) return CURE_ERR_INVALID_ARG;
  const Plan p = plan_of(dtype, batch, rows, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split);
  const size_t need = space_of(p, rows, hq, d);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CURE_ERR_WORKSPACE;
  if (need > 0 && at(workspace) % 16) return CURE_ERR_INVALID_ARG;
  const int64_t wgs = (int64_t)hkv * p.tiles * p.slots;
  if (wgs * kWaves * kWave >= (int64_t(1) << 32)) return CURE_ERR_UNSUPPORTED;         // a launch counts threads in 32 bits
  float* part_o = static_cast<float*>(workspace);
  Args a{q, pk, pv, k_scale, v_scale, blocks, k, v, cache_rows, o, lse, out_dtype == CURE_BF16, batch, n_max, hq, hkv, hq / hkv,
         rows, scale * kLog2e, row_off, n_rows, blk_off, packed_len, kv_off, ctx_len, parent, row_status, p.groups * kRows, p.tiles, p.tps, p.quantum, p.slots,
         part_o, p.slots > 1 ? part_o + rows * hq * p.slots * d : nullptr};
  hipStream_t st = as_stream(stream);
  const dim3 grid((unsigned)wgs, (unsigned)batch), block(kWaves * kWave);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  if (dtype == CURE_F32) d == 128 ? run(packed_few<float, 128>) : run(packed_few<float, 64>);
  else if (p.groups == 1) d == 128 ? run(packed_few<uint16_t, 128>) : run(packed_few<uint16_t, 64>);
  else if (p.groups == 2) d == 128 ? run(packed_many<128, 2>) : run(packed_many<64, 2>);
  else d == 128 ? run(packed_many<128, 4>) : run(packed_many<64, 4>);
  const cure_status launched = launch_status();
  if (launched != CURE_OK || p.slots == 1 || n_max == 0) return launched;
  const int per = 256 / (d / 4);
  const dim3 mgrid((unsigned)(((int64_t)n_max * hq + per - 1) / per), (unsigned)batch);
  if (d == 128) hipLaunchKernelGGL((packed_merge<128>), mgrid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((packed_merge<64>), mgrid, dim3(256), 0, st, a);
  return launch_status();
}
