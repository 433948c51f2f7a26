// cure_packed_attn: attention of candidate trees, single tokens or chunks of prompts over a
// context whose tokens are packed in blocks of 64 with 8 bits a value (cure_kv_pack), the open
// rows behind it and the new rows themselves.
//
// Query row R of a kv-head is query head R % group of token R / group, so the heads that
// share keys share a tile. With c the bytes and s the scale of a token's block,
//   S^T = s_k (C_k Q^T),  P = 2^(S - m),  l += sum P,  O^T += C_v^T (s_v P)^T,  o = O / l
// in one pass over the keys with the running reference m and sum l in fp32. The bytes are
// widened to the queries' type, which holds them exactly, and the scales enter with the scores
// and the probabilities. For bf16 s_v P is rounded to bf16, as the matrix instruction takes no wider
// operand beside bf16 values; l sums P itself.
//
// 32x32 matrix instructions (x16 for bf16, x2 eight times for fp32), 32 query rows per wave. Lane
// l = 32 half + col owns query row col, and of a step's 32 tokens half of the scores:
//   S^T: A = token col's columns 32 s + 16 half + 8 u .. +7, B = query row col's;
//        D register r = score of token 8 (r / 4) + 4 half + r % 4
//   O^T: A = column 32 i + col of the tokens whose probabilities the lane holds in
//        registers 8 t .. 8 t + 7, B = those; D register r of block i = column 32 i + 8 (r / 4)
//        + 4 half + r % 4 of query row col.
// A packed block lies in memory as A wants it, 16 bytes to a lane, so packed steps go from
// memory to registers and into the matrix unit, without LDS and without exchange.
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

constexpr int kStep = 32;            // tokens per step of the key loop
constexpr int kWaves = 4;            // waves per workgroup, which take its steps in turn
constexpr int kRows = 32;            // query rows per tile
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
  int32_t tiles, tps, slots;         // tiles of a sequence, steps per split, splits at most
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
  const int per = ((steps - 1) / n / kWaves + 1) * kWaves;
  return Cut{(steps - 1) / per + 1, per};
}

// Eight values of an operand's lane, and the product of two.
template <typename E>
struct Frag;
template <>
struct Frag<uint16_t> {
  bf16x8 x;
  // Eight bytes: integers of seven bits and a sign are bf16 values, so the upper halves of
  // their fp32 forms are exact.
  CURE_DEV void bytes(uint32_t lo, uint32_t hi) {
    Pack8 p;
    const auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
    const auto byte = [](uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); };
    p.u = make_uint4(pair(byte(lo, 0), byte(lo, 1)), pair(byte(lo, 2), byte(lo, 3)), pair(byte(hi, 0), byte(hi, 1)),
                     pair(byte(hi, 2), byte(hi, 3)));
    x = p.v;
  }
  CURE_DEV void row(const RowVec<uint16_t, 16>& r, int u) {
    Pack8 p;
    p.u = make_uint4(r.w[4 * u], r.w[4 * u + 1], r.w[4 * u + 2], r.w[4 * u + 3]);
    x = p.v;
  }
  CURE_DEV void floats(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__bf16)f[i];
  }
  CURE_DEV void raw(int i, uint16_t v) { x[i] = __builtin_bit_cast(__bf16, v); }
};
template <>
struct Frag<float> {
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
  CURE_DEV void floats(const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = f[i];
  }
  CURE_DEV void raw(int i, float v) { x[i] = v; }
};
CURE_DEV f32x16 mma(const Frag<uint16_t>& a, const Frag<uint16_t>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}
CURE_DEV f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i], b.x[i], c, 0, 0, 0);
  return c;
}

// A value of a row that no query row need see: an infinity or NaN would reach the others
// through its zero probabilities.
CURE_DEV uint16_t finite(uint16_t x) { return (x & 0x7f80) == 0x7f80 ? 0 : x; }
CURE_DEV float finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.f : x; }

// Token of D register r in a lane's half.
CURE_DEV int token_of(int half, int r) { return 8 * (r / 4) + 4 * half + r % 4; }

template <int D>
struct Shared {
  float o[kWaves][kRows][D + 4];
  float m[kWaves][kRows], l[kWaves][kRows];
  uint32_t anc[kRows][kAncWords];    // root paths of the tile's nodes, as bits
  int parent[CURE_MAX_TREE_NODES];
};

template <typename E, int D>
__global__ __launch_bounds__(kWaves * kWave, 2) void packed_attn(Args a) {
  constexpr int kK = D / 32;                       // pieces of 32 columns
  __shared__ __attribute__((aligned(16))) Shared<D> sh;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int col = lane % 32, half = lane / 32;
  const int b = blockIdx.y;
  const int hk = blockIdx.x % a.hkv, tile = blockIdx.x / a.hkv % a.tiles, slot = blockIdx.x / a.hkv / a.tiles;
  const Seq s = seq_of(a, b);
  const bool first = blockIdx.x == 0;
  if (!s.ok || s.n == 0) {
    if (first && tid == 0 && a.row_status) a.row_status[b] = s.ok ? CURE_OK : CURE_ERR_BAD_TREE;
    return;
  }
  const int r0 = tile * kRows, rows = s.n * a.group;
  if (r0 >= rows) return;
  const int r_last = min(r0 + kRows, rows) - 1;
  const Steps steps = steps_of(a, s, r_last);
  const Cut cut = cut_of(a, steps.all);
  const int begin = slot * cut.per, end = min(begin + cut.per, steps.all);
  if (begin >= end) return;

  // The tree: its status, and the root paths of the tile's nodes where its rows are reached.
  const int node0 = r0 / a.group;
  if (a.parent && (first || end > steps.packed)) {
    int p = -1;
    if (tid < s.n) p = a.parent[(int64_t)b * a.n_max + tid];
    const bool bad = tid < s.n && (p < -1 || p >= tid);
    if (__syncthreads_or(bad)) p = bad ? -1 : p;
    if (first && a.row_status) {
      const int any = __syncthreads_or(bad);
      if (tid == 0) a.row_status[b] = any ? CURE_ERR_BAD_TREE : CURE_OK;
    }
    if (tid < s.n) sh.parent[tid] = p;
    __syncthreads();
    if (tid <= r_last / a.group - node0) {
      uint32_t bits[kAncWords] = {};
      for (int j = node0 + tid; j >= 0; j = sh.parent[j]) {
#pragma unroll
        for (int i = 0; i < kAncWords; ++i) bits[i] |= j >> 5 == i ? 1u << (j & 31) : 0u;
      }
#pragma unroll
      for (int i = 0; i < kAncWords; ++i) sh.anc[tid][i] = bits[i];
    }
    __syncthreads();
  } else if (first && tid == 0 && a.row_status) {
    a.row_status[b] = CURE_OK;
  }

  // This lane's query row.
  const int R = min(r0 + col, rows - 1), node = R / a.group;
  const int64_t qrow = (s.row0 + node) * a.hq + hk * a.group + R % a.group;
  Frag<E> q[kK][2];
  {
    const E* src = static_cast<const E*>(a.q) + qrow * D + 16 * half;
#pragma unroll
    for (int i = 0; i < kK; ++i) {
      RowVec<E, 16> x;
      x.load(src + 32 * i);
      q[i][0].row(x, 0);
      q[i][1].row(x, 1);
    }
  }
  float m = kNone, l = 0.f;
  f32x16 o[kK];
#pragma unroll
  for (int i = 0; i < kK; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;

  // Scores of base 2 (masked ones -inf) to probabilities times vs.
  const auto soften = [&](const f32x16& x, float vs, Frag<E> (&p)[2]) {
    float high = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) high = fmaxf(high, x[r]);
    high = max_halves(high);
    if (__any(high > m + kRescaleLog2)) {
      const float mn = fmaxf(m, high), f = fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int i = 0; i < kK; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= f;
    }
    float w[2][8];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e = fast_exp2(x[r] - m);
      l += e;
      w[r / 8][r % 8] = e * vs;
    }
    p[0].floats(w[0]);
    p[1].floats(w[1]);
  };

  int step = begin + wave;
  for (; step < min(end, steps.packed); step += kWaves) {
    const int64_t block = (s.block0 + step / 2) * a.hkv + hk;
    const int64_t at = block * (kBlockTokens * D) + step % 2 * (kStep * D) + lane * 16;
    u32x4 kw[kK], vw[kK];
#pragma unroll
    for (int i = 0; i < kK; ++i) kw[i] = *reinterpret_cast<const u32x4*>(a.pk + at + i * 1024);
#pragma unroll
    for (int i = 0; i < kK; ++i) vw[i] = *reinterpret_cast<const u32x4*>(a.pv + at + i * 1024);
    const float ks = a.k_scale[block] * a.scale_log2, vs = a.v_scale[block];
    f32x16 x;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
    for (int i = 0; i < kK; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        Frag<E> f;
        f.bytes(kw[i][2 * u], kw[i][2 * u + 1]);
        x = mma(f, q[i][u], x);
      }
    const int left = s.packed - step * kStep;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = token_of(half, r) < left ? x[r] * ks : -INFINITY;
    Frag<E> p[2];
    soften(x, vs, p);
#pragma unroll
    for (int i = 0; i < kK; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag<E> f;
        f.bytes(vw[i][2 * t], vw[i][2 * t + 1]);
        o[i] = mma(f, p[t], o[i]);
      }
  }
  const int64_t pitch = (int64_t)a.hkv * D;
  const int open = s.ctx + s.n;                    // open and new rows
  for (; step < end; step += kWaves) {
    const int t0 = (step - steps.packed) * kStep;
    const E* kp = static_cast<const E*>(a.k) + s.kv0 * pitch + hk * D;
    const E* vp = static_cast<const E*>(a.v) + s.kv0 * pitch + hk * D;
    f32x16 x;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
    const E* krow = kp + min(t0 + col, open - 1) * pitch + 16 * half;
#pragma unroll
    for (int i = 0; i < kK; ++i) {
      RowVec<E, 16> w;
      w.load(krow + 32 * i);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        Frag<E> f;
        f.row(w, u);
        x = mma(f, q[i][u], x);
      }
    }
    // Which of the step's tokens the row sees, as bits.
    const int own = t0 - s.ctx;                    // the first one's index among the new rows
    uint32_t seen;
    if (!a.parent) {
      const int n = node - own + 1;
      seen = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
    } else {
      const uint32_t* anc = sh.anc[node - node0];
      const int i = own >> 5, sft = own & 31;      // floor
      const uint32_t lo = i >= 0 && i < kAncWords ? anc[i] : 0u, hi = i + 1 >= 0 && i + 1 < kAncWords ? anc[i + 1] : 0u;
      seen = sft ? lo >> sft | hi << (32 - sft) : lo;
      if (own < 0) seen |= own <= -32 ? ~0u : (1u << -own) - 1;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = seen >> token_of(half, r) & 1 ? x[r] * a.scale_log2 : -INFINITY;
    Frag<E> p[2];
    soften(x, 1.f, p);
#pragma unroll
    for (int i = 0; i < kK; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag<E> f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          f.raw(j, finite(vp[min(t0 + token_of(half, 8 * t + j), open - 1) * pitch + 32 * i + col]));
        o[i] = mma(f, p[t], o[i]);
      }
  }

  // The waves' parts joined.
  l = sum_halves(l);
  if (half == 0) {
    sh.m[wave][col] = m;
    sh.l[wave][col] = l;
  }
#pragma unroll
  for (int i = 0; i < kK; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<f32x4*>(&sh.o[wave][col][32 * i + 8 * (r / 4) + 4 * half]) =
          f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
  __syncthreads();
  constexpr int kThreads = kWaves * kWave / kRows, kCols = D / kThreads;     // threads of a row, columns of each
  const int row = tid / kThreads, c0 = tid % kThreads * 4;
  if (r0 + row >= rows) return;
  float mm = kNone, ll = 0.f, f[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, sh.m[w][row]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    f[w] = fast_exp2(sh.m[w][row] - mm);
    ll += f[w] * sh.l[w][row];
  }
  const float inv = ll > 0.f ? 1.f / ll : 0.f;
  const int out_row = (r0 + row) / a.group;
  const int64_t at = (s.row0 + out_row) * a.hq + hk * a.group + (r0 + row) % a.group;
  const bool whole = cut.n == 1;
  const float lse2 = ll > 0.f ? mm + log2f(ll) : -INFINITY;
  if (tid % kThreads == 0) {
    if (!whole) a.part_lse[at * a.slots + slot] = lse2;
    else if (a.lse) a.lse[at] = lse2 * kLn2;
  }
#pragma unroll
  for (int c = 0; c < kCols; c += 4) {
    const int j = c0 + c * kThreads;
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += f[w] * *reinterpret_cast<const f32x4*>(&sh.o[w][row][j]);
    sum *= inv;
    if (!whole) *reinterpret_cast<f32x4*>(a.part_o + (at * a.slots + slot) * D + j) = sum;
    else if (a.out_bf16)
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + j) = u32x2{pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    else *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + j) = sum;
  }
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
  const int rows = s.n * a.group, r0 = (n * a.group + head % a.group) / kRows * kRows;
  const Cut cut = cut_of(a, steps_of(a, s, min(r0 + kRows, rows) - 1).all);
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
  int32_t tiles, tps, slots;
};

// Parts of a call: rows * hq * slots of d + 1 floats.
constexpr int64_t kMostBytes = int64_t(1) << 30;

Plan plan_of(int32_t batch, int64_t rows, int32_t hq, int32_t hkv, int32_t d, const int32_t* n, const int32_t* packed,
             const int32_t* ctx, int32_t kv_split) {
  const int64_t group = hq / hkv;
  int64_t total = 0, longest = 1, most_rows = 0;
  for (int32_t b = 0; b < batch; ++b) {
    if (n[b] <= 0) continue;
    const int64_t steps = ((int64_t)packed[b] + kStep - 1) / kStep + ((int64_t)ctx[b] + n[b] + kStep - 1) / kStep;
    total += (n[b] * group + kRows - 1) / kRows * hkv * steps;
    longest = std::max(longest, steps);
    most_rows = std::max<int64_t>(most_rows, n[b]);
  }
  Plan p;
  p.tiles = (int32_t)std::max<int64_t>(1, (most_rows * group + kRows - 1) / kRows);
  // Two workgroups per CU, of at least two steps for each wave.
  const int64_t target = 2 * (int64_t)device_cu_count();
  int64_t tps = kv_split > 0 ? (longest + kv_split - 1) / kv_split : std::max<int64_t>(2 * kWaves, (total + target - 1) / target);
  tps = (tps + kWaves - 1) / kWaves * kWaves;
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
  return space_of(plan_of(batch, rows, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split), rows, hq, d);
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
  const Plan p = plan_of(batch, rows, hq, hkv, d, host_n_rows, host_packed_len, host_ctx_len, kv_split);
  const size_t need = space_of(p, rows, hq, d);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CURE_ERR_WORKSPACE;
  if (need > 0 && at(workspace) % 16) return CURE_ERR_INVALID_ARG;
  const int64_t wgs = (int64_t)hkv * p.tiles * p.slots;
  if (wgs * kWaves * kWave >= (int64_t(1) << 32)) return CURE_ERR_UNSUPPORTED;         // a launch counts threads in 32 bits
  float* part_o = static_cast<float*>(workspace);
  Args a{q, pk, pv, k_scale, v_scale, blocks, k, v, cache_rows, o, lse, out_dtype == CURE_BF16, batch, n_max, hq, hkv, hq / hkv,
         rows, scale * kLog2e, row_off, n_rows, blk_off, packed_len, kv_off, ctx_len, parent, row_status, p.tiles, p.tps, p.slots,
         part_o, p.slots > 1 ? part_o + rows * hq * p.slots * d : nullptr};
  hipStream_t st = as_stream(stream);
  const dim3 grid((unsigned)wgs, (unsigned)batch), block(kWaves * kWave);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  if (dtype == CURE_BF16) d == 128 ? run(packed_attn<uint16_t, 128>) : run(packed_attn<uint16_t, 64>);
  else d == 128 ? run(packed_attn<float, 128>) : run(packed_attn<float, 64>);
  const cure_status launched = launch_status();
  if (launched != CURE_OK || p.slots == 1 || n_max == 0) return launched;
  const int per = 256 / (d / 4);
  const dim3 mgrid((unsigned)(((int64_t)n_max * hq + per - 1) / per), (unsigned)batch);
  if (d == 128) hipLaunchKernelGGL((packed_merge<128>), mgrid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((packed_merge<64>), mgrid, dim3(256), 0, st, a);
  return launch_status();
}
