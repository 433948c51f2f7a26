// cure_prompt_attn: causal attention of new tokens over their context and themselves
// (whole prompts, chunks of them, single tokens), sequences packed without padding.
// cure_prefix_attn: tree verification of sequences that share a prefix, whose keys and
// values are read once for all of them; each sequence's own context and tree are more work
// of the same launch, and a merge joins the parts by their log-sum-exps. 16 trees of 40 to 48 nodes
// on 8192 shared tokens, 32 heads of 128 over 8: 118 + 9 us.
//
// Both are one kernel over (tile of query rows, kv-head, split of the keys): query row R of
// a kv-head is query head R % group of token R / group, so the heads that share keys share
// a tile. A row sees the keys up to its own position (a prompt), all of them (a prefix, where
// the tokens are the nodes of all sequences, without those that a sequence does not have), or
// its context and the nodes on its root path (a tree).
//
//   S^T = K Q^T,  P = 2^(c S - m),  l += sum P,  O^T += V^T P^T,  o = O / l
// in one pass over the keys with the running reference m and sum l in fp32. P is rounded to
// bf16 for its product, as the matrix instruction takes no wider operand beside bf16
// values, and l sums the rounded values, so that o is a weighted mean of v exactly.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "common.hpp"
#include "host_util.hpp"
#include "mfma_tile.hpp"

namespace cure {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 32;            // tokens per step of the key loop
constexpr int kWaves = 4;            // waves per workgroup
constexpr int kRows = 32 * kWaves;   // query rows per tile of the bf16 kernel: 32 for each wave
constexpr int kNarrow = 32;          // query rows per tile of the fp32 kernel, whose waves share them
constexpr int kMaxPrefixBatch = 1024;
constexpr float kNone = -3e38f;      // reference of a row that has seen nothing
constexpr int kAncWords = CURE_MAX_TREE_NODES / 64;

// Division by a launch's constant: x / d = the high half of x * (2^32 / d + 1) while x * d < 2^32.
struct Div {
  int32_t d;
  uint32_t m;                        // 0: divide
  static Div by(int32_t d, int64_t x_max) {
    return Div{d, d > 1 && x_max * d < (int64_t(1) << 32) ? (uint32_t)((uint64_t(1) << 32) / (uint32_t)d + 1) : 0u};
  }
  CURE_DEV int operator()(int x) const { return m ? (int)__umulhi((uint32_t)x, m) : d == 1 ? x : x / d; }
};

// How keys are split: at most `most` splits of about tps tokens, at least one, which begin at
// multiples of `quantum`.
struct Splits {
  int32_t tps, most, quantum;
};

// Splits that rows of `keys` (at least one) keys have at most.
__host__ __device__ inline int32_t slots_of(const Splits& s, int64_t keys) {
  const int64_t n = (keys - 1) / s.tps + 1;
  return (int32_t)(n < s.most ? n : s.most);
}

// Where each sequence's parts lie, in calls whose workspace would be large with one number of
// slots for all rows. A prompt: row r, head h, split j at first + (r * hq + h) * splits + j. Own rows
// behind a prefix: the first split beside the prefix's, split j from 1 on at first + (r * hq + h) *
// (splits - 1) + j - 1.
struct Place {
  int64_t first;
  int32_t splits;                    // of the sequence's longest rows; 1: a prompt is written whole
};

struct Args {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  int32_t out_bf16;
  int32_t hq, hkv, group;
  Div by_group, by_hkv;
  int32_t batch, n_max;
  float scale_log2;
  int64_t rows;                      // rows of q and o
  const int64_t* row_off;            // prompt: first row of q and o per sequence
  const int32_t* n_rows;             // tokens, or nodes, per sequence
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const int32_t* parent;             // prefix: the trees
  int32_t* tree_status;
  int64_t prefix_off;
  int32_t prefix_len;
  int32_t tile, tile_log2;           // query rows of a tile
  int32_t tiles, own_tiles;          // prefix: tiles of all nodes, and of a sequence's
  Splits cut, own;                   // of a prompt's keys or the prefix, and of own rows
  int32_t slots;                     // of a row: the splits of a prompt, or the prefix's and then the own rows'
  float* part_o;                     // [row][hq][slots][d], or by place
  float* part_lse;                   // [row][hq][slots]
  Place* place;                      // [batch], or null
  int32_t merge0;                    // first token of a merge launch
};

// The place of sequence b's parts.
template <bool kPrefix>
CURE_DEV Place place_of(const Args& a, int b) {
  return a.place ? a.place[b] : Place{0, kPrefix ? a.own.most : a.cut.most};
}
// The part of a row and head for `slot`: rows of a prefix have a.slots together, and the others by place.
struct Parts {
  int64_t near, far;
  int32_t together;
  CURE_DEV int64_t operator()(int slot) const { return (slot < together ? near : far) + slot; }
};
template <bool kPrefix>
CURE_DEV Parts parts_of(const Args& a, const Place& p, int64_t row, int head) {
  const int64_t i = row * a.hq + head;
  if (!kPrefix) return Parts{p.first + i * p.splits, 0, INT32_MAX};
  return Parts{i * a.slots, p.first + i * (p.splits - 1) - a.slots, a.slots};
}

// The splits of `keys` (at least one) keys: n of `per` tokens, the last one shorter (a single
// one: all).
struct Cut {
  int n, per;
};
CURE_DEV Cut cut_of(const Splits& s, int keys) {
  if (s.most == 1) return Cut{1, keys};
  const int n = max(1, min((keys - 1) / s.tps + 1, s.most));
  const int per = ((keys - 1) / n / s.quantum + 1) * s.quantum;
  return Cut{(keys - 1) / per + 1, per};
}

// A sequence's rows, as the device's sizes have them: none where its context cannot be (the
// host's checks keep context and rows below 2^31 - 4096) or its rows lie outside those of q and o.
CURE_DEV int rows_of(const Args& a, int n_raw, int ctx, int64_t row0) {
  const int n = min(n_raw, a.n_max);
  const bool ok = ctx >= 0 && ctx <= INT32_MAX - 4096 - max(n, 0) && row0 >= 0 && row0 <= a.rows - n;
  return ok ? n : 0;
}

// What a workgroup works on: packed query rows r0 .. of `rows` in all, against cache rows
// key0 + [begin, end).
struct Work {
  int hk, r0, rows, slot, splits;
  int begin, end;
  int64_t key0;
  int64_t row0;                      // first row of the sequence (not for a prefix)
  int ctx;
  int b;
  Place place;                       // of a prompt
  bool tree;                         // a sequence's own rows, in cure_prefix_attn
};

// What cure_prefix_attn keeps in LDS beside the tiles: for the start of a workgroup alone the
// nodes before each sequence, or a tree's parents; then the root paths of its tile's nodes, as bits.
template <int kTileRows>
struct TreeSpace {
  unsigned long long anc[kTileRows][kAncWords];
};
struct StartSpace {
  int first[kMaxPrefixBatch + 1];
  int parent[CURE_MAX_TREE_NODES];
};
struct Shared {
  int* first;
  int* parent;
  unsigned long long (*anc)[kAncWords];
};
struct Nothing {};
template <class T>
CURE_DEV Shared shared_of(StartSpace& s, T& t) { return Shared{s.first, s.parent, t.anc}; }
CURE_DEV Shared shared_of(Nothing&, Nothing&) { return Shared{}; }

// Prompt: grid (kv-heads x tiles, splits, sequences); a sequence's last tiles, which see the
// most keys, come first. A sequence's tiles stay together, as they share its keys in the L2: dealt
// out in turn over the sequences, 16 prompts of 1 to 2048 tokens took 399 us instead of 253.
CURE_DEV bool locate_prompt(const Args& a, Work& w) {
  const int b = blockIdx.z, x = a.by_hkv(blockIdx.x);
  w.hk = blockIdx.x - x * a.hkv;
  const int n_raw = a.n_rows[b];
  w.ctx = a.ctx_len[b];
  w.row0 = a.row_off[b];
  w.key0 = a.kv_off[b];
  asm volatile("" : : "s"(n_raw), "s"(w.ctx), "s"(w.row0), "s"(w.key0));
  // A launch of the longest sequence's tiles is mostly workgroups without work: they end here.
  if (x * a.tile >= min(n_raw, a.n_max) * a.group) return false;
  w.place = place_of<false>(a, b);
  const int n = rows_of(a, n_raw, w.ctx, w.row0);
  w.rows = n * a.group;
  const int tiles = (w.rows + a.tile - 1) >> a.tile_log2;
  if (n <= 0 || x >= tiles) return false;
  w.r0 = (tiles - 1 - x) * a.tile;
  const int keys = w.ctx + a.by_group(min(w.r0 + a.tile, w.rows) - 1) + 1;
  const Cut c = cut_of(Splits{a.cut.tps, w.place.splits, a.cut.quantum}, keys);
  w.tree = false;
  w.slot = blockIdx.y;
  w.splits = c.n;
  w.begin = w.slot * c.per;
  w.end = min(w.begin + c.per, keys);
  return w.slot < c.n;
}

// Prefix: kv-heads x (tiles x splits of the prefix, then tiles x splits of each sequence's own
// rows). The prefix's tiles hold the existing nodes of all sequences in order, whose counts are
// summed here.
CURE_DEV bool locate_prefix(const Args& a, Work& w, const Shared& sh) {
  int x = a.by_hkv(blockIdx.x);
  w.hk = blockIdx.x - x * a.hkv;
  w.b = 0;
  const int shared_units = a.tiles * a.cut.most;
  w.tree = x >= shared_units;
  if (w.tree) {
    x -= shared_units;
    const int tile = x % a.own_tiles;
    x /= a.own_tiles;
    const int b = w.b = x % a.batch, s = x / a.batch;
    const int own_most = place_of<true>(a, b).splits;
    const int n_raw = a.n_rows[b];
    w.ctx = a.ctx_len[b];
    w.key0 = a.kv_off[b];
    asm volatile("" : : "s"(n_raw), "s"(w.ctx), "s"(w.key0));
    w.row0 = (int64_t)b * a.n_max;
    const int n = rows_of(a, n_raw, w.ctx, w.row0);
    w.rows = n * a.group;
    w.r0 = tile * a.tile;
    if (n <= 0) {                                  // the empty tree is valid, a context that cannot be is not
      if (tile == 0 && s == 0 && w.hk == 0 && threadIdx.x == 0 && a.tree_status)
        a.tree_status[b] = n_raw > 0 ? CURE_ERR_BAD_TREE : CURE_OK;
      return false;
    }
    const int keys = w.ctx + n;
    const Cut c = cut_of(Splits{a.own.tps, own_most, a.own.quantum}, keys);
    w.slot = a.cut.most + s;
    w.splits = c.n;
    w.begin = s * c.per;
    w.end = min(w.begin + c.per, keys);
    return s < c.n && w.r0 < w.rows;
  }
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    int sum = 0;
    if (lane == 0) sh.first[0] = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kWave) {
      const int b = b0 + lane;
      int v = b < a.batch ? min(max(a.n_rows[b], 0), a.n_max) : 0;
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int u = __shfl_up(v, d);
        if (lane >= d) v += u;
      }
      if (b < a.batch) sh.first[b + 1] = sum + v;
      sum += __shfl(v, kWave - 1);
    }
  }
  __syncthreads();
  const Cut c = cut_of(a.cut, a.prefix_len);
  w.rows = sh.first[a.batch] * a.group;
  w.r0 = x % a.tiles * a.tile;
  w.slot = x / a.tiles;
  w.splits = c.n;
  w.begin = w.slot * c.per;
  w.end = min(w.begin + c.per, a.prefix_len);
  w.key0 = a.prefix_off;
  w.ctx = a.prefix_len;
  w.row0 = 0;
  return w.slot < c.n && w.r0 < w.rows;
}

template <bool kPrefix>
CURE_DEV bool locate(const Args& a, Work& w, const Shared& sh) {
  return kPrefix ? locate_prefix(a, w, sh) : locate_prompt(a, w);
}

// The ancestor bits of the tile's nodes, for a workgroup of at least 256 threads whose work
// reaches the tree's rows; reports the tree's status. False: malformed.
CURE_DEV bool build_tree(const Args& a, const Work& w, const Shared& sh) {
  const int n = threadIdx.x, nodes = a.by_group(w.rows);
  int p = -1;
  if (n < nodes) p = a.parent[w.row0 + n];
  const bool ok = !__syncthreads_or(n < nodes && (p < -1 || p >= n));
  if (n == 0 && w.r0 == 0 && w.hk == 0 && a.tree_status) a.tree_status[w.b] = ok ? CURE_OK : CURE_ERR_BAD_TREE;
  if (!ok) return false;
  if (n < nodes) sh.parent[n] = p;
  __syncthreads();
  const int t0 = a.by_group(w.r0), t1 = a.by_group(min(w.r0 + a.tile, w.rows) - 1);
  if (n <= t1 - t0) {
    unsigned long long bits[kAncWords] = {};
    for (int j = t0 + n; j >= 0; j = sh.parent[j]) {
#pragma unroll
      for (int i = 0; i < kAncWords; ++i) bits[i] |= j >> 6 == i ? 1ull << (j & 63) : 0ull;
    }
#pragma unroll
    for (int i = 0; i < kAncWords; ++i) sh.anc[n][i] = bits[i];
  }
  __syncthreads();
  return true;
}

// Packed row R: its row of q and o, its query head, its node within the tile, and the last key
// that it sees with all before it.
struct Row {
  int64_t row;
  int head, node, last;
};
template <bool kPrefix>
CURE_DEV Row row_of(const Args& a, const Work& w, const Shared& sh, int R) {
  const int t = a.by_group(R);
  Row r;
  r.head = w.hk * a.group + (R - t * a.group);
  r.node = kPrefix ? t - a.by_group(w.r0) : 0;
  if (!kPrefix || w.tree) {
    r.row = w.row0 + t;
    r.last = kPrefix ? w.ctx - 1 : w.ctx + t;
    return r;
  }
  int lo = 0, hi = a.batch - 1;                    // the last sequence with first[b] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (sh.first[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  r.row = (int64_t)lo * a.n_max + (t - sh.first[lo]);
  r.last = w.ctx - 1;
  return r;
}

// The part of a row that this workgroup computes. Own rows read their place again where they need it.
template <bool kPrefix>
CURE_DEV int64_t part_at(const Args& a, const Work& w, const Row& me) {
  if (!kPrefix) return parts_of<false>(a, w.place, me.row, me.head)(w.slot);
  if (w.slot < a.slots) return (me.row * a.hq + me.head) * a.slots + w.slot;
  return parts_of<true>(a, a.place[w.b], me.row, me.head)(w.slot);
}

// Whether a row sees token t of its split: one up to `last`, or in a tree a node on its path.
template <bool kPrefix>
CURE_DEV bool sees(const Args& a, const Work& w, const Shared& sh, int t, int last, int node) {
  if (!kPrefix || !w.tree) return t <= last;
  const int j = t + w.begin - w.ctx, i = min(max(j, 0), CURE_MAX_TREE_NODES - 1);
  const bool on_path = (sh.anc[node][i >> 6] >> (i & 63)) & 1;
  return t <= last || (t + w.begin < w.end && on_path);
}

CURE_DEV void store8_f32(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
CURE_DEV void store8(const Args& a, int64_t idx, const float (&x)[8]) {
  if (a.out_bf16)
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.o) + idx) =
        make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  else
    store8_f32(reinterpret_cast<float*>(a.o) + idx, x);
}
CURE_DEV void store4(const Args& a, int64_t idx, float x0, float x1, float x2, float x3) {
  if (a.out_bf16) {
    uint2 pk;
    pk.x = pack_bf16x2(x0, x1);
    pk.y = pack_bf16x2(x2, x3);
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.o) + idx) = pk;
  } else {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.o) + idx) = make_float4(x0, x1, x2, x3);
  }
}

// ---------------------------------------------------------------------------
// bf16 kernel: 32 query rows per wave, 32x32x16 matrix instructions.
//
// Lane l = 32 half + col owns query row col of its wave, half of its scores:
//   S^T: A = K row col of the step's 32, columns 16 kk + 8 half .. +7; B = Q row col, same
//        columns; D register r = score of token 8 (r / 4) + 4 half + r % 4
//   O^T: k index 8 half + j of k-step ks stands for token 16 ks + 8 (j / 4) + 4 half + j % 4,
//        the probability that the lane holds; A = V^T by transposed LDS reads;
//        D register r of block i = column 32 i + 8 (r / 4) + 4 half + r % 4 of row col.
// Rings of kRing steps of K and of V in LDS are filled by DMA. Step h forms the scores of
// step h + 1, the probabilities of step h and the products of step h - 1: three parts that
// do not wait for each other, so the matrix instructions and the softmax's vector
// instructions of one wave interleave.
//
// 128 rows share a tile of keys, so that 2 workgroups of 4 waves fit a CU's registers (200 of
// 256 at head dim 128; 235 with a prefix, where the masks of the steps seen in part also keep 82
// scalar registers in lanes of a vector one, outside the main loop) and each key read from LDS serves 32 rows. Large prompts are bound by the
// matrix unit and the power it draws: a prompt of 8192 tokens, 32 heads of 128, took 488, 515 and
// 523 us on three cards (1.05 - 1.13 PFLOP/s of the 1.20 that a large product reaches), the unit busy
// 57 % of the cycles at 1.6 - 1.75 GHz; its instructions alone take 386 us. 16 prompts of 1 to 2048
// tokens take 236 us, 0.33 GB of
// queries and outputs among them that move at the workgroups' starts and ends. Single tokens are
// bound by the cache's way: 8 on 4k - 32k tokens 107 us, 5.9 TB/s of the 6.97 that a read reaches.
// Measured and slower: 64 rows per wave with one wave to a SIMD (2.4 times), 8 waves per workgroup
// (short prompts), rings of 8 steps at head dim 64.
template <int D>
struct Geo {
  static constexpr int kRing = 4;
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kBytes = kStep * kRowBytes;           // one step of K or V
  static constexpr int kDma = kBytes / 1024 / kWaves;        // 1 KB blocks per wave and tensor
  static_assert(kDma >= 1, "every wave moves part of each step");
  // Byte offset of a 16-byte chunk of a row, its index XORed by row so that a read's lanes
  // spread over the 64 banks. A K read takes 16 bytes from each of 32 rows; the hardware serves
  // it 16 lanes at a time, rows 0 - 3, 12 - 15, 20 - 27 and the others, which row bits 0, 1, 2 and
  // 4 tell apart. A transposed V read takes 32 or 64 bytes from each of 4 rows.
  static CURE_DEV int k_offset(int row, int chunk) {
    const int low = row & 3, b2 = (row >> 2) & 1, b4 = (row >> 4) & 1;
    const int f = D == 128 ? low << 2 | b4 << 1 | b2 : (low >> 1) << 2 | b4 << 1 | b2;
    return row * kRowBytes + ((chunk ^ f) << 4);
  }
  static CURE_DEV int v_offset(int row, int chunk) {
    const int low = row & 3, b2 = (row >> 2) & 1;
    const int f = D == 128 ? low << 2 | b2 << 1 : (low >> 1) << 2 | b2 << 1;
    return row * kRowBytes + ((chunk ^ f) << 4);
  }
};

// A row's probabilities of one step, as the products take them.
struct Probs {
  u32x4 u[2];
  CURE_DEV void set(int pair, bf16x2 v) { u[pair >> 2][pair & 3] = __builtin_bit_cast(uint32_t, v); }
  CURE_DEV bf16x8 operand(int ks) const { return __builtin_bit_cast(bf16x8, u[ks]); }
};

// kOnce: every key is read by one workgroup (no sequence has a second tile), and passes by the L2.
// us a call with that and without: 8 single tokens on 4k - 32k 107 and 123; 16 prompts of 1 to
// 2048 tokens 236 and 229, 4 of 2048 without groups 190 and 149.
template <int D, bool kPrefix, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, 2) void seq_attn(Args a) {
  using G = Geo<D>;
  constexpr int kRing = G::kRing;
  constexpr int kKK = D / 16;                      // k-steps of the scores
  constexpr int kBlk = D / 32;                     // 32-column blocks of the output
  constexpr int kAhead = 2;
  // Beyond what a step needs, the DMA of the kRing - 2 steps before it may be in flight.
  constexpr int kVmWait = waitcnt_vm((kRing - 2) * 2 * G::kDma);
  __shared__ __attribute__((aligned(1024))) unsigned char s_k[kRing * G::kBytes];
  __shared__ __attribute__((aligned(1024))) unsigned char s_v[kRing * G::kBytes];
  __shared__ typename std::conditional<kPrefix, StartSpace, Nothing>::type s_start;
  __shared__ typename std::conditional<kPrefix, TreeSpace<kRows>, Nothing>::type s_tree;
  const Shared sh = shared_of(s_start, s_tree);

  Work w;
  if (!locate<kPrefix>(a, w, sh)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;

  // The tile stream: per wave and step, kDma blocks of K and of V. The buffer resource
  // covers the step's own rows of the keys, so that the rest of a step reads as zeros and a
  // step past the split's end reads nothing; its base moves on in 64 bits.
  const uint32_t tok_bytes = (uint32_t)(a.hkv * G::kRowBytes);
  uint32_t k_src[G::kDma], v_src[G::kDma];
#pragma unroll
  for (int j = 0; j < G::kDma; ++j) {
    // The source of the chunk at this lane's place: XORed again, it is its own.
    const int byte = (wave * G::kDma + j) * 1024 + lane * 16;
    const int row = byte / G::kRowBytes, chunk = (byte % G::kRowBytes) >> 4;
    const uint32_t at = (uint32_t)row * tok_bytes + (uint32_t)(w.hk * G::kRowBytes);
    k_src[j] = at + G::k_offset(row, chunk) % G::kRowBytes;
    v_src[j] = at + G::v_offset(row, chunk) % G::kRowBytes;
  }
  const char* const kp = reinterpret_cast<const char*>(a.k) + (w.key0 + w.begin) * (int64_t)tok_bytes;
  const char* const vp = reinterpret_cast<const char*>(a.v) + (w.key0 + w.begin) * (int64_t)tok_bytes;
  const uint32_t k_lds = lds_addr(s_k), v_lds = lds_addr(s_v);
  const uint32_t dma0 = __builtin_amdgcn_readfirstlane(wave * G::kDma * 1024);
  const int steps = (w.end - w.begin + kStep - 1) / kStep;
  auto dma = [&](const char* p, const uint32_t (&src)[G::kDma], uint32_t lds, int h) {
    const int left = min(w.end - w.begin - h * kStep, kStep);
    const i32x4 rsrc = raw_rsrc(p + (int64_t)h * kStep * tok_bytes, left > 0 ? (uint32_t)left * tok_bytes : 0u);
#pragma unroll
    for (int j = 0; j < G::kDma; ++j) {
      if (kOnce) dma16(lds + dma0 + j * 1024, src[j], rsrc);
      else dma16_shared(lds + dma0 + j * 1024, src[j], rsrc);
    }
  };
#pragma unroll
  for (int h = 0; h < kRing; ++h) {
    dma(kp, k_src, k_lds + h * G::kBytes, h);
    if (h < kRing - 2) dma(vp, v_src, v_lds + h * G::kBytes, h);
  }

  // This lane's query row.
  const int R = w.r0 + wave * 32 + col;
  const bool row_ok = R < w.rows;
  const Row me = row_of<kPrefix>(a, w, sh, min(R, w.rows - 1));
  const int node = me.node;
  bf16x8 q[kKK];
  {
    const uint16_t* qrow = reinterpret_cast<const uint16_t*>(a.q) + (me.row * a.hq + me.head) * D;
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      Pack8 p;
      p.u = *reinterpret_cast<const uint4*>(qrow + kk * 16 + half * 8);
      q[kk] = p.v;
    }
  }
  // Keys that the wave's first and last row see, relative to the split; the steps it takes.
  const bool wave_ok = w.r0 + wave * 32 < w.rows;
  const int last = me.last - w.begin;
  const int first_last = __builtin_amdgcn_readfirstlane(last);
  const int last_last = __builtin_amdgcn_readlane(last, 31);
  const int my_steps = !wave_ok ? 0 : kPrefix ? steps : min(steps, max(0, (last_last + kStep) / kStep));
  const int full = min(my_steps, max(0, (first_last + 1) / kStep));   // steps that every row sees whole
  if (kPrefix && w.tree && w.end > w.ctx && !build_tree(a, w, sh)) {
    __builtin_amdgcn_s_waitcnt(0);                 // no DMA may land after the workgroup ends
    return;
  }

  // LDS addresses of this lane's operands in slot 0.
  uint32_t k_at[kKK];
#pragma unroll
  for (int kk = 0; kk < kKK; ++kk) k_at[kk] = k_lds + G::k_offset(col, 2 * kk + half);
  uint32_t v_at[kBlk];
  {
    const int j = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
    for (int i = 0; i < kBlk; ++i)
      v_at[i] = v_lds + G::v_offset(4 * half + (j >> 2), 4 * i + 2 * g + ((j & 3) >> 1)) + (j & 1) * 8;
  }

  f32x16 o[kBlk];
#pragma unroll
  for (int i = 0; i < kBlk; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  float m = 0.f, l = 0.f;
  const float c = a.scale_log2;
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  // Lambdas take ring slots as byte offsets: constants in the main loop.
  auto scores = [&](f32x16& x, uint32_t slot) {
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk)
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(k_at[kk] + slot), q[kk], x, 0, 0, 0);
  };
  auto values = [&](uint32_t slot, int ks, int i) {
    Pack8 f;
#pragma unroll
    for (int r = 0; r < 2; ++r) f.h[r] = lds_read_tr8(v_at[i] + slot + (16 * ks + 8 * r) * G::kRowBytes);
    return f;
  };
  // Probabilities against the reference m; returns `sum` with this lane's share of theirs.
  auto exps = [&](const f32x16& x, Probs& p, float sum) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bf16x2 v = {(__bf16)fast_exp2(fmaf(x[2 * j], c, -m)), (__bf16)fast_exp2(fmaf(x[2 * j + 1], c, -m))};
      p.set(j, v);
      sum = __builtin_amdgcn_fdot2_f32_bf16(v, ones, sum, false);
    }
    return sum;
  };
  // Not by max3_raw: the compiler would not wait for the scores (max_scores), and here a step's maximum is rare.
  auto row_max = [&](const f32x16& x) {
    float mx = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
    return max_halves(mx) * c;
  };
  // Takes over a step's sum. The reference moves where a row's maximum has risen by more than
  // 2^8, which no row's has while no lane's sum has grown by more.
  auto settle = [&](const f32x16& x, Probs& p, float sum) {
    if (__builtin_expect(__ballot(!(sum - l <= 256.f)) != 0, 0)) {
      const float mx = row_max(x);
      const bool grow = mx > m + kRescaleLog2;
      const float alpha = grow ? fast_exp2(m - mx) : 1.f;
      m = grow ? mx : m;
#pragma unroll
      for (int i = 0; i < kBlk; ++i) o[i] *= alpha;
      sum = exps(x, p, l * alpha);
    }
    l = sum;
  };
  // The products of a step that some rows see in part: a token that a row does not see must
  // not reach it, but 0 times an infinity or a NaN would. Where the step's values hold one, the
  // products take zeros in its place and the rows that do see it take it as it is.
  auto hidden_products = [&](const Probs& p, uint32_t slot, int h) {
    Pack8 f[2 * kBlk];
    float probe[2] = {0.f, 0.f};                   // a NaN from the first value that is not finite
#pragma unroll
    for (int n = 0; n < 2 * kBlk; ++n) f[n] = values(slot, n / kBlk, n % kBlk);
#pragma unroll
    for (int n = 0; n < 2 * kBlk; ++n)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        probe[n & 1] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{f[n].v[e], f[n].v[e + 1]},
                                                       bf16x2{(__bf16)0.f, (__bf16)0.f}, probe[n & 1], false);
    const bool finite = __ballot(probe[0] + probe[1] != 0.f) == 0;
    const auto clean = [](uint32_t u) {
      const uint32_t lo = (u & 0x7f80u) == 0x7f80u ? 0u : 0xffffu;
      const uint32_t hi = (u & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u;
      return u & (lo | hi);
    };
    if (__builtin_expect(!finite, 0)) {
#pragma unroll
      for (int n = 0; n < 2 * kBlk; ++n)
        f[n].u = make_uint4(clean(f[n].u.x), clean(f[n].u.y), clean(f[n].u.z), clean(f[n].u.w));
    }
#pragma unroll
    for (int n = 0; n < 2 * kBlk; ++n)
      o[n % kBlk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n].v, p.operand(n / kBlk), o[n % kBlk], 0, 0, 0);
    if (__builtin_expect(finite, 1)) return;
    for (int t = 0; t < kStep; ++t) {
      const bool seen = sees<kPrefix>(a, w, sh, h * kStep + t, last, node);
#pragma unroll
      for (int i = 0; i < kBlk; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {              // columns 32 i + 8 g + 4 half .. +3
          const uint32_t at = v_lds + slot + G::v_offset(t, 4 * i + g) + 8 * half;
          const u32x2 u = *(const __attribute__((address_space(3))) u32x2*)(uintptr_t)at;
          const float x[4] = {bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][4 * g + e] += seen && !(fabsf(x[e]) < INFINITY) ? x[e] : 0.f;
        }
    }
  };
  auto mask = [&](f32x16& x, int h) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      x[r] = sees<kPrefix>(a, w, sh, h * kStep + 8 * (r >> 2) + 4 * half + (r & 3), last, node) ? x[r] : -INFINITY;
  };
  // A step in the middle of a row's keys: scores of the next step into y, probabilities of this
  // one, whose scores are x, into n, products of the last one's, p; returns the running sum. Every
  // matrix instruction is followed by LDS reads for the one kAhead turns on and by an equal share
  // of the softmax, which the matrix unit's time hides.
  auto middle = [&](const f32x16& x, f32x16& y, const Probs& p, Probs& n, uint32_t k_slot, uint32_t v_slot) {
    constexpr int kPairs = 8 / kKK;                // pairs of probabilities per turn
    bf16x8 kf[kKK];
    Pack8 vf[kKK];
    float e0[8], e1[8], sum = l;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      kf[i] = lds_read16(k_at[i] + k_slot);
      vf[i] = values(v_slot, i / kBlk, i % kBlk);
    }
    const auto round = [&](int j) {                // pair j: scores 2 j and 2 j + 1
      const bf16x2 v = {(__bf16)e0[j], (__bf16)e1[j]};
      n.set(j, v);
      sum = __builtin_amdgcn_fdot2_f32_bf16(v, ones, sum, false);
    };
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll
    for (int i = 0; i < kKK; ++i) {
      y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], q[i], y, 0, 0, 0);
      if (i + kAhead < kKK) kf[i + kAhead] = lds_read16(k_at[i + kAhead] + k_slot);
#pragma unroll
      for (int j = kPairs * i; j < kPairs * (i + 1); ++j) {
        e0[j] = fast_exp2(fmaf(x[2 * j], c, -m));
        e1[j] = fmaf(x[2 * j + 1], c, -m);
      }
      __builtin_amdgcn_sched_barrier(0);
      o[i % kBlk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i].v, p.operand(i / kBlk), o[i % kBlk], 0, 0, 0);
      if (i + kAhead < kKK) vf[i + kAhead] = values(v_slot, (i + kAhead) / kBlk, (i + kAhead) % kBlk);
#pragma unroll
      for (int j = kPairs * i; j < kPairs * (i + 1); ++j) {
        e1[j] = fast_exp2(e1[j]);
        if (j >= kPairs) round(j - kPairs);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = 8 - kPairs; j < 8; ++j) round(j);
    return sum;
  };
  auto slot_of = [](int step) { return (uint32_t)(step % kRing) * G::kBytes; };
  // Step h begins: its slots (h + 1 of K, h - 1 of V) have landed for every wave, and those that
  // step h - 1 read (h of K, h - 2 of V) are refilled.
  auto begin = [&](int h, uint32_t k_slot, uint32_t v_slot) {
    __builtin_amdgcn_s_waitcnt(kVmWait);
    __syncthreads();
    dma(kp, k_src, k_lds + k_slot, h + kRing);
    dma(vp, v_src, v_lds + v_slot, h + kRing - 2);
  };

  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (!row_ok) {
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) q[kk] = bf16x8{};
  }
  // Scores and probabilities of the present step, of the next and of the one before.
  f32x16 x;
  Probs p;
  if (my_steps > 0) {
    scores(x, 0);
    if (full == 0) mask(x, 0);
    // The first reference: the row's maximum. A row that sees nothing here (a tree's node whose
    // path comes later) has no finite one: against kNone hidden scores have probabilities of
    // zero and the first score that is seen an infinite one, with which the reference moves.
    const float mx = row_max(x);
    m = mx == -INFINITY ? kNone : mx;
  }
  begin(0, 0, slot_of(kRing - 2));
  int h = 1;
  if (my_steps > 0) {
    l = exps(x, p, 0.f);
    scores(x, G::kBytes);
    // Steps that every row sees whole, a ring's turn at a time.
    for (; h + kRing <= full; h += kRing) {
#pragma unroll
      for (int j = 1; j <= kRing; ++j) {           // step h + j - 1, j modulo the ring
        f32x16 y;
        Probs n;
        begin(h + j - 1, slot_of(j), slot_of(j + kRing - 2));
        settle(x, n, middle(x, y, p, n, slot_of(j + 1), slot_of(j + kRing - 1)));
        x = y;
        p = n;
      }
    }
    // The rest of those, and the first step that is seen in part: its products come a step later.
    for (; h < my_steps && h <= full; ++h) {
      f32x16 y;
      Probs n;
      begin(h, slot_of(h), slot_of(h + kRing - 2));
      if (h == full) mask(x, h);
      settle(x, n, middle(x, y, p, n, slot_of(h + 1), slot_of(h + kRing - 1)));
      x = y;
      p = n;
    }
    // What is seen in part.
    for (; h <= my_steps; ++h) {
      begin(h, slot_of(h), slot_of(h + kRing - 2));
      hidden_products(p, slot_of(h + kRing - 1), h - 1);
      if (h < my_steps) {
        mask(x, h);
        settle(x, p, exps(x, p, l));
        scores(x, slot_of(h + 1));
      }
    }
  }
  for (; h <= steps; ++h) begin(h, slot_of(h), slot_of(h + kRing - 2));

  __builtin_amdgcn_s_waitcnt(0);                   // the rings' trailing DMA lands before exit
  if (!row_ok) return;
  const float lt = sum_halves(l);
  const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);   // a NaN stays one
  const float lse = lt == 0.f ? -INFINITY : (m + log2f(lt)) * kLn2;
  const bool whole = w.splits == 1 && !kPrefix;
  const int64_t pi = whole ? 0 : part_at<kPrefix>(a, w, me);
  const int64_t orow = me.row * a.hq + me.head;
  // Lanes l and l + 32 hold columns 0 - 3 and 4 - 7 of each eight of one row: they trade, so that each
  // has eight together, of every other eight.
#pragma unroll
  for (int i = 0; i < kBlk; ++i)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[i][4 * g + e] * inv),
                                                        __float_as_uint(o[i][4 * g + 4 + e] * inv), false, false);
        y[e] = __uint_as_float(r[0]);
        y[4 + e] = __uint_as_float(r[1]);
      }
      const int d0 = 32 * i + 8 * (g + half);
      if (whole) store8(a, orow * D + d0, y);
      else store8_f32(a.part_o + pi * D + d0, y);
    }
  if (half == 0) {
    if (!whole) a.part_lse[pi] = lse;
    else if (a.lse) a.lse[orow] = lse;
  }
}

// ---------------------------------------------------------------------------
// fp32 kernel: a tile is 32 query rows, which all four waves share, 32x32x2 fp32 matrix
// instructions, products and sums in fp32 throughout. Each wave takes every fourth step of the
// keys, with buffers and sums of its own, joined at the end.
//
// Lane l = 32 half + col owns query row col:
//   S^T: MFMA i of column group j takes k index half for column 8 j + 4 half + i, so one
//        16-byte read of K (row col, columns 8 j + 4 half .. +3) feeds four; D register r =
//        score of token 8 (r / 4) + 4 half + r % 4
//   O^T: MFMA r takes k index half for that token, the probability the lane holds; output
//        row c' of block i stands for column (D / 32) c' + i, so one read of V (the token's
//        row, columns (D / 32) col ..) feeds all D / 32 blocks.
// The scores of a wave's next step are formed together with the probabilities of the present
// one, whose vector instructions fill the matrix unit's time; then come the present one's
// products. K of the step after is asked for when the scores have read the buffer, V after the
// products, so that one buffer of each is enough and no wave waits for another.
//
// Bound by the matrix unit: 16 x 128 tokens on 8000, 32 heads of 128, take 2028 us, 133 TFLOP/s of
// the 154 that a large product reaches; at head dim 64 1026 us, 132. A prompt of 4096 tokens takes
// 1114 and 536 us. With tiles of 128 rows, 32 to a wave, those four launches took 2136, 1165, 1120
// and 624 us, and 4 x 32 tokens on 8000 164 instead of 146. Asking for K and V in pieces behind their
// reads was no faster, two accumulators of the scores slower.
template <int D>
struct GeoF32 {
  static constexpr int kRowBytes = 4 * D;
  static constexpr int kBytes = kStep * kRowBytes;
  static constexpr int kDma = kBytes / 1024;                 // 1 KB blocks per tensor
  static CURE_DEV int offset(int row, int chunk) { return row * kRowBytes + ((chunk ^ (row & 15)) << 4); }
};

template <int D, bool kPrefix>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 1 : 2) void seq_attn_f32(Args a) {
  using G = GeoF32<D>;
  constexpr int kJ = D / 8;                        // column groups of the scores
  constexpr int kBlk = D / 32;                     // output blocks
  constexpr int kGroups = D / 8;                   // of four columns that a lane ends up with
  constexpr int kAhead = 2;
  typedef float vfrag __attribute__((ext_vector_type(D / 32)));
  __shared__ __attribute__((aligned(1024))) unsigned char s_kv[kWaves][2][G::kBytes];   // [wave][K, V]
  __shared__ float s_m[kWaves][kNarrow], s_l[kWaves][kNarrow];
  __shared__ typename std::conditional<kPrefix, StartSpace, Nothing>::type s_start;
  __shared__ typename std::conditional<kPrefix, TreeSpace<kNarrow>, Nothing>::type s_tree;
  const Shared sh = shared_of(s_start, s_tree);

  Work w;
  if (!locate<kPrefix>(a, w, sh)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;

  const uint32_t tok_bytes = (uint32_t)(a.hkv * G::kRowBytes);
  uint32_t src[G::kDma];
#pragma unroll
  for (int j = 0; j < G::kDma; ++j) {
    const int byte = j * 1024 + lane * 16, row = byte / G::kRowBytes;
    src[j] = (uint32_t)row * tok_bytes +
             (uint32_t)(w.hk * G::kRowBytes + ((((byte % G::kRowBytes) >> 4) ^ (row & 15)) << 4));
  }
  const char* const kp = reinterpret_cast<const char*>(a.k) + (w.key0 + w.begin) * (int64_t)tok_bytes;
  const char* const vp = reinterpret_cast<const char*>(a.v) + (w.key0 + w.begin) * (int64_t)tok_bytes;
  const int steps = (w.end - w.begin + kStep - 1) / kStep;
  const unsigned char *const kt = s_kv[wave][0], *const vt = s_kv[wave][1];
  auto dma = [&](const char* p, const unsigned char* to, int h) {
    const int left = min(w.end - w.begin - h * kStep, kStep);
    const i32x4 rsrc = raw_rsrc(p + (int64_t)h * kStep * tok_bytes, left > 0 ? (uint32_t)left * tok_bytes : 0u);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // the reads of the buffer have their data
#pragma unroll
    for (int j = 0; j < G::kDma; ++j) dma16_shared(lds_addr(to) + j * 1024, src[j], rsrc);
  };
  // Everything but the last tensor asked for has landed.
  const auto landed = [] { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(G::kDma) : "memory"); };
  const auto all_landed = [] { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); };
  dma(kp, kt, wave);
  dma(vp, vt, wave);

  const int R = w.r0 + col;
  const Row me = row_of<kPrefix>(a, w, sh, min(R, w.rows - 1));
  const int node = me.node;
  f32x4 q[kJ];
  {
    const float* qrow = reinterpret_cast<const float*>(a.q) + (me.row * a.hq + me.head) * D;
#pragma unroll
    for (int j = 0; j < kJ; ++j) q[j] = *reinterpret_cast<const f32x4*>(qrow + 8 * j + 4 * half);
  }
  const int last = me.last - w.begin;
  const int first_last = __builtin_amdgcn_readfirstlane(last);
  const int last_last = __builtin_amdgcn_readlane(last, 31);
  const int my_steps = kPrefix ? steps : min(steps, max(0, (last_last + kStep) / kStep));
  if (kPrefix && w.tree && w.end > w.ctx && !build_tree(a, w, sh)) {
    all_landed();                                  // no DMA may land after the workgroup ends
    return;
  }

  const int k_off = G::offset(col, half);          // column group j: 32 j XORed onto it
  // V: row 8 (r / 4) + 4 half + r % 4. The swizzle takes a row's low four bits, so registers r
  // and r + 8 are 16 rows apart.
  int v_off[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int byte = col * (D / 32) * 4;
    v_off[r] = G::offset(8 * (r >> 2) + 4 * half + (r & 3), byte >> 4) + (byte & 15);
  }
  const auto key = [&](int j) { return *reinterpret_cast<const f32x4*>(kt + (k_off ^ (32 * j))); };
  const auto values = [&](int r) {
    return *reinterpret_cast<const vfrag*>(vt + (r >> 3) * 16 * G::kRowBytes + v_off[r & 7]);
  };

  f32x16 o[kBlk];
#pragma unroll
  for (int i = 0; i < kBlk; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  float m = kNone, l = 0.f;
  const float c = a.scale_log2;
  const auto tail = [&](int h) { return h * kStep + kStep - 1 > first_last; };   // some row sees step h in part
  const auto mask = [&](f32x16& x, int h) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      x[r] = sees<kPrefix>(a, w, sh, h * kStep + 8 * (r >> 2) + 4 * half + (r & 3), last, node) ? x[r] : -INFINITY;
  };
  const auto row_max = [&](const f32x16& x) {
    float mx = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
    return max_halves(mx) * c;
  };
  const auto exps = [&](const f32x16& x, f32x16& p, float sum) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = fast_exp2(fmaf(x[r], c, -m));
      sum += p[r];
    }
    return sum;
  };
  // Scores of the next step into y, probabilities of this one, whose scores are x, into p; returns
  // the running sum.
  const auto scores_and_exps = [&](f32x16& y, const f32x16& x, f32x16& p) {
    constexpr int kEach = 16 / kJ;                 // probabilities per column group
    f32x4 f[kJ];
    float sum = l;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) f[j] = key(j);
#pragma unroll
    for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      if (j + kAhead < kJ) f[j + kAhead] = key(j + kAhead);
#pragma unroll
      for (int i = 0; i < 4; ++i) y = __builtin_amdgcn_mfma_f32_32x32x2f32(f[j][i], q[j][i], y, 0, 0, 0);
#pragma unroll
      for (int r = kEach * j; r < kEach * (j + 1); ++r) {
        p[r] = fast_exp2(fmaf(x[r], c, -m));
        sum += p[r];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return sum;
  };
  // Takes over a step's sum; the reference moves as in the bf16 kernel.
  const auto settle = [&](const f32x16& x, f32x16& p, float sum) {
    if (__builtin_expect(__ballot(!(sum - l <= 256.f)) != 0, 0)) {
      const float mx = row_max(x);
      const bool grow = mx > m + kRescaleLog2;
      const float alpha = grow ? fast_exp2(m - mx) : 1.f;
      m = grow ? mx : m;
#pragma unroll
      for (int i = 0; i < kBlk; ++i) o[i] *= alpha;
      sum = exps(x, p, l * alpha);
    }
    l = sum;
  };
  const auto products = [&](const f32x16& p) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const vfrag f = values(r);
#pragma unroll
      for (int i = 0; i < kBlk; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[i], p[r], o[i], 0, 0, 0);
    }
  };
  const auto hidden_products = [&](const f32x16& p, int h) {
    float probe = 0.f;                             // a NaN from the first value that is not finite
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const vfrag f = values(r);
#pragma unroll
      for (int i = 0; i < kBlk; ++i) probe = fmaf(f[i], 0.f, probe);
    }
    if (__builtin_expect(__ballot(probe != 0.f) == 0, 1)) {
      products(p);
      return;
    }
    // As in the bf16 kernel: zeros for the values that are not finite, which the rows that see
    // them take as they are.
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const vfrag f = values(r);
#pragma unroll
      for (int i = 0; i < kBlk; ++i)
        o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(fabsf(f[i]) < INFINITY ? f[i] : 0.f, p[r], o[i], 0, 0, 0);
    }
    for (int t = 0; t < kStep; ++t) {
      const bool seen = sees<kPrefix>(a, w, sh, h * kStep + t, last, node);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int byte = (8 * (r >> 2) + 4 * half + (r & 3)) * (D / 32) * 4;
        const vfrag f = *reinterpret_cast<const vfrag*>(vt + G::offset(t, byte >> 4) + (byte & 15));
#pragma unroll
        for (int i = 0; i < kBlk; ++i)
          if (seen && !(fabsf(f[i]) < INFINITY)) o[i][r] += f[i];
      }
    }
  };

  const auto scores = [&](f32x16& x) {
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const f32x4 f = key(j);
#pragma unroll
      for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_32x32x2f32(f[i], q[j][i], x, 0, 0, 0);
    }
  };

  int h = wave;
  f32x16 x, p;
  if (h < my_steps) {
    landed();
    scores(x);
    dma(kp, kt, h + kWaves);
    if (tail(h)) mask(x, h);
    const float mx = row_max(x);
    m = mx == -INFINITY ? kNone : mx;
    all_landed();                                  // asked for in this order: V, the next K
  }
  // Steps that every row sees whole, but the last.
  for (; h + kWaves < my_steps && !tail(h); h += kWaves) {
    f32x16 y;
    landed();
    const float sum = scores_and_exps(y, x, p);
    dma(kp, kt, h + 2 * kWaves);
    settle(x, p, sum);
    landed();
    products(p);
    dma(vp, vt, h + kWaves);
    x = y;
  }
  // What is seen in part, and the last.
  for (; h < my_steps; h += kWaves) {
    if (tail(h)) mask(x, h);
    settle(x, p, exps(x, p, l));
    all_landed();
    hidden_products(p, h);
    if (h + kWaves >= my_steps) break;
    dma(vp, vt, h + kWaves);
    scores(x);
    dma(kp, kt, h + 2 * kWaves);
  }

  // The waves' sums are joined through the buffers, a quarter of the columns by each wave. Group g
  // of a lane's: columns kBlk c' + i for one or more rows c' of the blocks i, four consecutive ones.
  all_landed();
  const auto sums = [&](int i, int g) { return reinterpret_cast<f32x4*>(s_kv[i][0]) + g * kWave + lane; };
  static_assert(kGroups * kWave * sizeof(f32x4) <= G::kBytes, "a wave's sums fit its K buffer");
  l = sum_halves(l);
  if (half == 0) {
    s_m[wave][col] = m;
    s_l[wave][col] = l;
  }
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = o[e % kBlk][4 / kBlk * g + e / kBlk];
    *sums(wave, g) = y;
  }
  __syncthreads();
  if (R >= w.rows) return;
  m = kNone;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) m = fmaxf(m, s_m[i][col]);
  float lt = 0.f, weight[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    weight[i] = fast_exp2(s_m[i][col] - m);
    lt = fmaf(s_l[i][col], weight[i], lt);
  }
  const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);
  const float lse = lt == 0.f ? -INFINITY : (m + log2f(lt)) * kLn2;
  const bool whole = w.splits == 1 && !kPrefix;
  const int64_t pi = whole ? 0 : part_at<kPrefix>(a, w, me);
  const int64_t orow = me.row * a.hq + me.head;
#pragma unroll
  for (int u = 0; u < kGroups / kWaves; ++u) {
    const int g = wave * (kGroups / kWaves) + u, r = 4 / kBlk * g;
    f32x4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) y += *sums(i, g) * weight[i];
    y *= inv;
    const int d0 = kBlk * (8 * (r >> 2) + 4 * half + (r & 3));
    if (whole) store4(a, orow * D + d0, y[0], y[1], y[2], y[3]);
    else *reinterpret_cast<f32x4*>(a.part_o + pi * D + d0) = y;
  }
  if (wave == 0 && half == 0) {
    if (!whole) a.part_lse[pi] = lse;
    else if (a.lse) a.lse[orow] = lse;
  }
}

// ---------------------------------------------------------------------------
// Joins the parts of a row (a prompt's splits; a prefix's, then those of the own rows) by their
// log-sum-exps: D / 4 lanes per (row, head), four columns each. A launch and a round trip to memory
// for few rows (8 tokens of 32 heads 4.7 us), the parts' way for many (16 trees of 40 - 48 nodes, 32
// heads of 128, 9.3 us).
constexpr int kMerge = 8;

template <int D, bool kPrefix, bool kPlaced>
__global__ __launch_bounds__(256) void seq_merge(Args a) {
  constexpr int kLanes = D / 4;
  const int head = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const int col = (threadIdx.x % kLanes) * 4;
  const int i = a.merge0 + blockIdx.y, b = blockIdx.z;
  if (head >= a.hq) return;
  const int n_raw = a.n_rows[b], ctx = a.ctx_len[b];
  const Place place = kPlaced ? a.place[b] : Place{0, kPrefix ? a.own.most : a.cut.most};
  const int64_t row0 = kPrefix ? (int64_t)b * a.n_max : a.row_off[b], row = row0 + i;
  const int n = rows_of(a, n_raw, ctx, row0);
  if (i >= n) return;
  int shared, parts;                               // parts from slot 0 on, and in all
  if (kPrefix) {
    shared = cut_of(a.cut, a.prefix_len).n;
    parts = shared + cut_of(Splits{a.own.tps, place.splits, a.own.quantum}, ctx + n).n;
  } else {
    // The tile of this row's head decides how many keys its splits covered.
    const int rows = n * a.group, R = i * a.group + (head - a.by_group(head) * a.group);
    const int end = min(((R >> a.tile_log2) + 1) * a.tile, rows);
    shared = parts = cut_of(Splits{a.cut.tps, place.splits, a.cut.quantum}, ctx + a.by_group(end - 1) + 1).n;
    if (parts == 1) return;                        // written whole
  }
  const Parts part = parts_of<kPrefix>(a, place, row, head);
  const int64_t orow = row * a.hq + head;
  const int gap = kPrefix ? a.cut.most - shared : 0;   // slots that no split of the prefix has
  // kMerge parts at a time, all of whose loads are under way together. Parts that saw
  // nothing (a log-sum-exp of -inf) weigh nothing.
  float m = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 v[kMerge];
  float lse[kMerge];
  for (int s0 = 0; s0 < parts; s0 += kMerge) {
    float mn = m;
    bool none = true;
#pragma unroll
    for (int u = 0; u < kMerge; ++u) {
      const bool ok = s0 + u < parts;
      const int slot = s0 + u + (s0 + u < shared ? 0 : gap);
      const int64_t at = kPlaced ? part(slot) : part.near + slot;
      v[u] = ok ? *reinterpret_cast<const float4*>(a.part_o + at * D + col) : make_float4(0.f, 0.f, 0.f, 0.f);
      lse[u] = ok ? a.part_lse[at] : -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < kMerge; ++u) {
      mn = fmaxf(mn, lse[u]);
      none = none && lse[u] == -INFINITY;
    }
    if (none) continue;
    mn = mn == -INFINITY ? 0.f : mn;               // only NaNs, which come through
    const float w0 = fast_exp2((m - mn) * kLog2e);
    m = mn;
    sum *= w0;
    acc.x *= w0;
    acc.y *= w0;
    acc.z *= w0;
    acc.w *= w0;
#pragma unroll
    for (int u = 0; u < kMerge; ++u) {
      const float w = fast_exp2((lse[u] - mn) * kLog2e);
      sum += w;
      acc.x = fmaf(w, v[u].x, acc.x);
      acc.y = fmaf(w, v[u].y, acc.y);
      acc.z = fmaf(w, v[u].z, acc.z);
      acc.w = fmaf(w, v[u].w, acc.w);
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  store4(a, orow * D + col, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (col == 0 && a.lse) a.lse[orow] = sum == 0.f ? -INFINITY : m + logf(sum);
}

// ---------------------------------------------------------------------------
// Places the sequences' parts one after the other from `begin` on, by the device's sizes, in `capacity`
// slots. Where those exceed the host's, a sequence whose parts do not fit has one split.
constexpr int kPlaceThreads = 1024;  // at most

template <bool kPrefix>
__global__ __launch_bounds__(kPlaceThreads) void seq_place(Args a, int64_t begin, int64_t capacity) {
  __shared__ int64_t s_sum[kPlaceThreads / kWave];
  const int threads = blockDim.x, waves = threads / kWave;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t total = 0;                               // slots of the sequences before this turn's
  for (int b0 = 0; b0 < a.batch; b0 += threads) {
    const int b = b0 + threadIdx.x;
    int64_t row0 = 0, need = 0;
    int splits = 1, stride = 0;
    if (b < a.batch) {
      row0 = kPrefix ? (int64_t)b * a.n_max : a.row_off[b];
      const int ctx = a.ctx_len[b], n = rows_of(a, a.n_rows[b], ctx, row0);
      if (n > 0) splits = slots_of(kPrefix ? a.own : a.cut, ctx + n);
      stride = kPrefix ? splits - 1 : splits;
      if (splits > 1) need = (int64_t)n * a.hq * stride;
    }
    int64_t sum = need;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int64_t u = __shfl_up((long long)sum, d);
      if (lane >= d) sum += u;
    }
    if (lane == kWave - 1) s_sum[wave] = sum;
    __syncthreads();
    int64_t before = total + sum - need;
    for (int i = 0; i < waves; ++i) {
      if (i < wave) before += s_sum[i];
      total += s_sum[i];
    }
    __syncthreads();                               // the sums are read before the next turn's
    if (b < a.batch) a.place[b] = Place{begin + before - row0 * a.hq * stride, before + need <= capacity ? splits : 1};
  }
}

// ---------------------------------------------------------------------------
// Host: tiles, splits and workspace.
struct Plan {
  int tile;                          // query rows per tile
  int tiles;                         // most tiles of a sequence (a prefix: of all nodes)
  int own_tiles;                     // prefix: most tiles of a sequence's own rows
  Splits cut, own;
  int slots() const { return cut.most + own.most; }
};

// Keys that a workgroup works on at a time: the waves of a narrow tile take a step each.
int quantum_of(int tile) { return tile == kNarrow ? kStep * kWaves : kStep; }

// At least one whole quantum.
int64_t rounded(int64_t keys, int tile) {
  const int64_t quantum = quantum_of(tile);
  return std::max<int64_t>(1, (keys + quantum - 1) / quantum) * quantum;
}

// `most` splits of `keys`, or as many as there are quanta.
Splits splits_of(int64_t keys, int64_t most, int tile) {
  const int64_t quantum = quantum_of(tile);
  most = std::max<int64_t>(1, std::min<int64_t>({most, (keys + quantum - 1) / quantum, 65535}));
  return Splits{(int32_t)rounded((keys + most - 1) / most, tile), (int32_t)most, (int32_t)quantum};
}

// Splits that a plan considers of the longest keys.
constexpr int kCandidates[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
// Of the own rows behind a prefix: one sequence with one kv-head has a workgroup per CU with the last.
constexpr int kOwnCandidates[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};

// Estimated us, from measurements: a step of 32 keys on a CU (two workgroups there take turns:
// together they are little faster), and what a workgroup takes beside its steps, of which the way of
// its part of `rows` rows to memory and back at a CU's share of the bandwidth. At head dim 64 two
// workgroups of the fp32 kernel hide half of each other's start.
struct Cost {
  double key, start, part;
  Cost(int32_t dtype, int tile, int32_t d, double rows) {
    const bool bf16 = dtype == CURE_BF16;
    key = (bf16 ? (d == 128 ? 0.45 : 0.28) : (d == 128 ? 0.95 : 0.53)) / kStep;
    start = bf16 ? 5 : d == 128 ? 6 : 2.5;
    part = std::min<double>(tile, rows) * d * 8 / 27e3;
  }
};

int tile_of(int32_t dtype) { return dtype == CURE_F32 ? kNarrow : kRows; }

Plan prompt_plan(int32_t dtype, int32_t batch, int32_t hq, int32_t hkv, int32_t d, const int32_t* host_n_rows,
                 const int32_t* host_ctx_len, int32_t kv_split) {
  const int64_t cus = device_cu_count(), group = hq / hkv;
  const auto tiles_of = [&](int64_t n, int64_t tile) { return (n * group + tile - 1) / tile; };
  Plan p{};
  p.tile = tile_of(dtype);
  int64_t tiles = 0, keys = 0, longest = 0, total = 0;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = host_n_rows[b];
    tiles += tiles_of(n, p.tile);
    total += n;
    longest = std::max(longest, n);
    if (n > 0) keys = std::max<int64_t>(keys, n + host_ctx_len[b]);
  }
  p.tiles = (int)tiles_of(longest, p.tile);
  // A prompt of more than 65535 tokens has two tiles and more for every CU.
  int64_t most = kv_split > 0 ? kv_split : longest > 65535;
  if (most == 0) {
    // The splits of the longest keys that are estimated to take least time: that of the CUs
    // with the most workgroups, or of the longest workgroup. Measured us a call with 1, 2, 4 and 12
    // splits: one prompt of 2k 52, 72 (two); 4 chunks of 256 - 512 tokens on 2k - 16k, head dim
    // 64, 211, 185, 207, 222; 8 single tokens on 4k - 32k 385, 202, 120, 105.
    // Splits of fewer than 256 tokens cost more in starts and parts than they save: 4 x 32 tokens
    // on 2000 in fp32 69, 46, 53 and (6, 8 and 16 splits) 62, 66 and 94.
    const Cost cost(dtype, p.tile, d, (double)total * group / std::max<int64_t>(1, tiles));
    double best = 0;
    for (const int s : kCandidates) {
      const int64_t tps = rounded((keys + s - 1) / s, p.tile);
      if (s > 1 && tps < 256) break;
      int64_t units = 0;
      double work = 0;
      for (int b = 0; b < batch; ++b) {
        const int64_t n = host_n_rows[b], t = tiles_of(n, p.tile);
        const int64_t mean = host_ctx_len[b] + (n + 1) / 2 + std::min<int64_t>(n, p.tile / group) / 2;
        units += t * std::max<int64_t>(1, (mean + tps - 1) / tps);
        work += (double)t * mean;
      }
      units = std::max<int64_t>(1, units * hkv);
      if (longest * group <= 32) {
        // Single tokens and the like stream the cache once: as many workgroups as two per CU
        // (fp32 one: 8 single tokens on 8k, 4 kv-heads, head dim 128, 52 us with one and 60 with two),
        // whose tiles under way cover the memory's latency.
        if (s == 1 || units <= (dtype == CURE_BF16 ? 2 : 1) * cus) most = s;
        continue;
      }
      const double each = cost.start + (s > 1 ? cost.part : 0);
      const double all = (double)((units + cus - 1) / cus) * (work * hkv / units * cost.key + each);
      const double time = std::max(all, tps * cost.key + each) + (s > 1 ? 5 : 0);
      if (most == 0 || time < best) {
        most = s;
        best = time;
      }
    }
  }
  p.cut = splits_of(keys, most, p.tile);
  return p;
}

// Workgroups of a launch over a prefix's tiles and every sequence's own, existing or not, and whether
// their threads fit the 32 bits that a launch counts them in.
int64_t prefix_units(const Plan& p, int32_t batch, int32_t hkv, int64_t prefix_splits, int64_t own_splits) {
  return (p.tiles * prefix_splits + (int64_t)p.own_tiles * batch * own_splits) * hkv;
}
bool launchable(int64_t units) { return units < (int64_t(1) << 32) / (64 * kWaves); }

Plan prefix_plan(int32_t dtype, int32_t batch, int32_t hq, int32_t hkv, int32_t d, int32_t n_max,
                 int32_t prefix_len, const int32_t* host_ctx_len, const int32_t* host_n_nodes, int32_t kv_split) {
  const int64_t cus = device_cu_count(), group = hq / hkv;
  const auto tiles_of = [&](int64_t nodes, int64_t tile) { return (nodes * group + tile - 1) / tile; };
  int64_t nodes = 0, keys = 0;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = host_n_nodes[b];
    nodes += n;
    if (n > 0) keys = std::max<int64_t>(keys, n + host_ctx_len[b]);
  }
  Plan p{};
  p.tile = tile_of(dtype);
  // The device may hold other counts than the host's copies: tiles for every node there may
  // be, of which those past the last one end at once.
  p.tiles = (int)std::min<int64_t>(tiles_of((int64_t)batch * n_max, p.tile), INT32_MAX);
  p.own_tiles = (int)tiles_of(n_max, p.tile);
  const int64_t tiles = tiles_of(nodes, p.tile);
  // Own rows are split for themselves, as their number and lengths have nothing to do with the
  // prefix: workgroups and longest split of every candidate, up to one for each 256 keys or part of them.
  // us a call behind 200 shared tokens, with the estimate's splits and with one for each 256 keys: 16
  // trees of 48 nodes on 4000 104 (one) and 208, on 30000 579 (four) and 1245, 64 trees 2043 (two) and
  // 4969, where the workspace of the latter is 6 GB. 12 trees of 28 on 684 28 (one) and 32.
  struct Own {
    int64_t units, longest;
  };
  constexpr int kOwn = (int)(sizeof(kOwnCandidates) / sizeof(kOwnCandidates[0]));
  Own owns[kOwn] = {};
  int own_count = 0;
  double work = (double)tiles * prefix_len;
  for (int b = 0; b < batch; ++b)
    work += (double)tiles_of(host_n_nodes[b], p.tile) * ((int64_t)host_n_nodes[b] + host_ctx_len[b]);
  for (const int u : kOwnCandidates) {
    if (u > 1 && u > (keys + 255) / 256) break;
    const int64_t tps = rounded((keys + u - 1) / u, p.tile);
    Own& o = owns[own_count++];
    o.longest = std::min(tps, keys);
    for (int b = 0; b < batch; ++b) {
      const int64_t k = (int64_t)host_n_nodes[b] + host_ctx_len[b];
      o.units += tiles_of(host_n_nodes[b], p.tile) * std::max<int64_t>(1, (k + tps - 1) / tps) * hkv;
    }
  }
  // As for prompts, but all workgroups are one launch, in which those of own rows fill the CUs
  // around the prefix's. Measured us a call with 1, 2, 4 and 12 splits: 16 trees of 40 - 48 nodes on 8k
  // 131, 122, 137, 171; 32 single tokens on 16k, head dim 64, 169, 92, 52, 27 (24 with 16 and with 24, 26 with 32).
  int64_t most = kv_split, own = 1;
  const Cost cost(dtype, p.tile, d, (double)(nodes * group) / std::max<int64_t>(1, tiles));
  const double each = cost.start + cost.part;
  double best = 0;
  for (const int c : kCandidates) {
    const int64_t s = kv_split > 0 ? std::min(kv_split, prefix_len) : c;
    const int64_t tps = rounded((prefix_len + s - 1) / s, p.tile);
    if (c > 1 && (kv_split > 0 || tps < 256)) break;
    for (int i = 0; i < own_count; ++i) {
      const int64_t units = tiles * s * hkv + owns[i].units;
      const double unit = std::max(tps, owns[i].longest) * cost.key + each;
      const double time = std::max(unit, (work * hkv * cost.key + units * each) / cus + unit / 3);
      if (best == 0 || (time < best && launchable(prefix_units(p, batch, hkv, s, kOwnCandidates[i])))) {
        most = s;
        own = kOwnCandidates[i];
        best = time;
      }
    }
  }
  p.cut = splits_of(prefix_len, most, p.tile);
  p.own = splits_of(keys, own, p.tile);
  return p;
}

// Whether a call's parts go through the workspace: a prompt's where there are several.
bool in_parts(const Plan& p) { return p.slots() > 1; }

// A call's workspace: places of the sequences, if it has them, and `slots` parts of d columns and a
// log-sum-exp, of which the first `even` are the same for every row.
struct Space {
  bool placed;
  int32_t batch, d;
  int64_t slots, even;
  size_t place_bytes() const { return placed ? align_up((size_t)batch * sizeof(Place), 256) : 0; }
  size_t o_bytes() const { return align_up((size_t)slots * d * sizeof(float), 256); }
  size_t bytes() const { return place_bytes() + o_bytes() + align_up((size_t)slots * sizeof(float), 256); }
};

// Workspace up to which every row has the slots of the longest. Beyond, a launch of its own places the
// parts of each sequence by its own splits. 16 prompts of 2048 tokens beside one token on 128k, 32
// heads of 128: 1 MB and 1010 us, even 17 GB and 1140; 8 beside four, 2.2 GB even, 1116 and 1137. One
// prompt beside one token on 32k, 0.8 GB even, would take 133 us placed, and takes 126.
constexpr size_t kEvenBytes = size_t(1) << 30;

// rows * heads * slots, or a number that no workspace holds and whose bytes do not pass 64 bits.
constexpr int64_t kMostSlots = int64_t(1) << 46;
int64_t slots_in_all(int64_t rows, int64_t hq, int64_t slots) {
  return (double)rows * (double)hq * (double)slots < (double)kMostSlots ? rows * hq * slots : kMostSlots;
}

Space prompt_space(const Plan& p, int32_t batch, int64_t rows, int32_t hq, int32_t d, const int32_t* host_n_rows,
                   const int32_t* host_ctx_len) {
  const int64_t every = in_parts(p) ? slots_in_all(rows, hq, p.slots()) : 0;
  const Space even{false, batch, d, every, every};
  if (even.bytes() <= kEvenBytes) return even;
  int64_t slots = 0;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = host_n_rows[b];
    const int32_t splits = n > 0 ? slots_of(p.cut, n + host_ctx_len[b]) : 1;
    if (splits > 1) slots = std::min(slots + slots_in_all(n, hq, splits), kMostSlots);
  }
  return Space{true, batch, d, slots, 0};
}

// As for prompts. 256 trees of 48 nodes behind 200 shared tokens, one of them on 131072 of its own and the
// others on 100: 0.4 GB and 697 us, even 6.7 GB and 780; 64 of them 0.1 GB and 350 us, 1.7 GB and 374.
Space prefix_space(const Plan& p, int32_t batch, int32_t hq, int32_t d, int32_t n_max, const int32_t* host_ctx_len,
                   const int32_t* host_n_nodes) {
  const int64_t rows = (int64_t)batch * n_max, every = slots_in_all(rows, hq, p.slots());
  const Space even{false, batch, d, every, every};
  if (even.bytes() <= kEvenBytes) return even;
  int64_t slots = 0;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = host_n_nodes[b];
    if (n > 0) slots = std::min(slots + slots_in_all(n, hq, slots_of(p.own, n + host_ctx_len[b]) - 1), kMostSlots);
  }
  const int64_t fixed = slots_in_all(rows, hq, p.cut.most + 1);
  return Space{true, batch, d, fixed + slots, fixed};
}

void set_plan(Args& a, const Plan& p, const Space& space, void* ws) {
  a.tile = p.tile;
  a.tile_log2 = p.tile == kNarrow ? 5 : 7;
  static_assert(kNarrow == 1 << 5 && kRows == 1 << 7, "tiles of a power of two");
  a.tiles = p.tiles;
  a.own_tiles = p.own_tiles;
  a.cut = p.cut;
  a.own = p.own;
  a.slots = space.placed ? p.cut.most + 1 : p.slots();
  if (space.bytes() == 0) return;
  char* at = static_cast<char*>(ws);
  if (space.placed) a.place = reinterpret_cast<Place*>(at);
  at += space.place_bytes();
  a.part_o = reinterpret_cast<float*>(at);
  a.part_lse = reinterpret_cast<float*>(at + space.o_bytes());
}

template <bool kPrefix>
hipError_t launch_place(const Args& a, const Space& space, hipStream_t st) {
  const int threads = std::min((a.batch + kWave - 1) / kWave * kWave, kPlaceThreads);
  hipLaunchKernelGGL(seq_place<kPrefix>, dim3(1), dim3((unsigned)threads), 0, st, a, space.even, space.slots - space.even);
  return hipGetLastError();
}

template <bool kPrefix>
void launch_attn(const Args& a, int32_t dtype, int32_t d, dim3 grid, hipStream_t st) {
  const dim3 block(64 * kWaves);
  if (dtype == CURE_BF16) {
    const bool once = !kPrefix && a.tiles == 1;
    if (once && d == 128) hipLaunchKernelGGL((seq_attn<128, kPrefix, !kPrefix>), grid, block, 0, st, a);
    else if (once) hipLaunchKernelGGL((seq_attn<64, kPrefix, !kPrefix>), grid, block, 0, st, a);
    else if (d == 128) hipLaunchKernelGGL((seq_attn<128, kPrefix, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((seq_attn<64, kPrefix, false>), grid, block, 0, st, a);
  } else {
    if (d == 128) hipLaunchKernelGGL((seq_attn_f32<128, kPrefix>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((seq_attn_f32<64, kPrefix>), grid, block, 0, st, a);
  }
}

template <bool kPrefix>
void launch_merge(Args a, int32_t d, hipStream_t st) {
  const int heads = 1024 / d;
  constexpr int kTokens = 65535;                   // of a launch, whose grid holds them in 16 bits
  for (int64_t t = 0; t < a.n_max; t += kTokens) {
    a.merge0 = (int32_t)t;
    const dim3 grid((unsigned)((a.hq + heads - 1) / heads), (unsigned)std::min<int64_t>(a.n_max - t, kTokens),
                    (unsigned)a.batch);
    if (a.place && d == 128) hipLaunchKernelGGL((seq_merge<128, kPrefix, true>), grid, dim3(256), 0, st, a);
    else if (a.place) hipLaunchKernelGGL((seq_merge<64, kPrefix, true>), grid, dim3(256), 0, st, a);
    else if (d == 128) hipLaunchKernelGGL((seq_merge<128, kPrefix, false>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((seq_merge<64, kPrefix, false>), grid, dim3(256), 0, st, a);
  }
}

// The checks that both calls make of their operands.
cure_status check(const void* q, const void* k, const void* v, const void* o, int32_t dtype, int32_t out_dtype,
                  int32_t hq, int32_t hkv, int32_t d, float scale) {
  if (dtype != CURE_F32 && dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (out_dtype != CURE_F32 && out_dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (hq <= 0 || hkv <= 0 || hq % hkv != 0) return CURE_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return CURE_ERR_UNSUPPORTED;
  if (!(scale > 0.f) || !std::isfinite(scale * kLog2e)) return CURE_ERR_INVALID_ARG;
  if ((int64_t)hkv * d * 4 * kStep > INT32_MAX) return CURE_ERR_UNSUPPORTED;
  const uintptr_t in = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) |
                       reinterpret_cast<uintptr_t>(v);
  if (in % 16 != 0 || reinterpret_cast<uintptr_t>(o) % 16 != 0)
    return CURE_ERR_INVALID_ARG;
  return CURE_OK;
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" size_t cure_prompt_attn_workspace_size(int32_t batch, int64_t rows, int32_t hq, int32_t hkv, int32_t d,
                                                  const int32_t* host_n_rows, const int32_t* host_ctx_len,
                                                  int32_t kv_split) {
  if (batch <= 0 || rows <= 0 || hq <= 0 || hkv <= 0 || hq % hkv || d <= 0 || !host_n_rows || !host_ctx_len) return 0;
  size_t need = 0;                                 // of whichever type needs more
  for (const int32_t dtype : {CURE_F32, CURE_BF16}) {
    const Plan p = prompt_plan(dtype, batch, hq, hkv, d, host_n_rows, host_ctx_len, kv_split);
    need = std::max(need, prompt_space(p, batch, rows, hq, d, host_n_rows, host_ctx_len).bytes());
  }
  return need;
}

extern "C" cure_status cure_prompt_attn(const void* q, const void* k, const void* v, void* o, float* lse,
                                        int32_t dtype, int32_t out_dtype, int32_t batch, int64_t rows, int32_t hq,
                                        int32_t hkv, int32_t d, float scale, const int64_t* row_off,
                                        const int32_t* n_rows, const int64_t* kv_off, const int32_t* ctx_len,
                                        const int32_t* host_n_rows, const int32_t* host_ctx_len, int32_t kv_split,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  if (batch < 0 || rows < 0 || kv_split < 0) return CURE_ERR_INVALID_ARG;
  const cure_status bad = check(q, k, v, o, dtype, out_dtype, hq, hkv, d, scale);
  if (bad != CURE_OK) return bad;
  if (batch == 0 || rows == 0) return CURE_OK;
  if (!q || !k || !v || !o || !row_off || !n_rows || !kv_off || !ctx_len || !host_n_rows || !host_ctx_len)
    return CURE_ERR_INVALID_ARG;
  if (batch > 65535) return CURE_ERR_UNSUPPORTED;
  int64_t longest = 0;
  for (int b = 0; b < batch; ++b) {
    const int64_t n = host_n_rows[b], c = host_ctx_len[b];
    if (n < 0 || c < 0 || n > rows) return CURE_ERR_INVALID_ARG;
    if (n + c > INT32_MAX - 4096 || n * (hq / hkv) > INT32_MAX - 4096) return CURE_ERR_UNSUPPORTED;
    longest = std::max(longest, n);
  }
  if (longest == 0) return CURE_OK;
  const Plan p = prompt_plan(dtype, batch, hq, hkv, d, host_n_rows, host_ctx_len, kv_split);
  const Space space = prompt_space(p, batch, rows, hq, d, host_n_rows, host_ctx_len);
  const size_t need = space.bytes();
  if (need > 0 && (!workspace || workspace_bytes < need)) return CURE_ERR_WORKSPACE;
  if (need > 0 && reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return CURE_ERR_INVALID_ARG;
  if ((int64_t)p.tiles * hkv * 64 * kWaves >= (int64_t(1) << 32)) return CURE_ERR_UNSUPPORTED;
  Args a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  a.out_bf16 = out_dtype == CURE_BF16;
  a.hq = hq;
  a.hkv = hkv;
  a.group = hq / hkv;
  a.by_group = Div::by(a.group, std::max<int64_t>(longest * a.group, hq));
  a.by_hkv = Div::by(hkv, (int64_t)p.tiles * hkv);
  a.batch = batch;
  a.n_max = (int32_t)longest;
  a.scale_log2 = scale * kLog2e;
  a.rows = rows;
  a.row_off = row_off;
  a.n_rows = n_rows;
  a.kv_off = kv_off;
  a.ctx_len = ctx_len;
  set_plan(a, p, space, workspace);
  hipStream_t st = as_stream(stream);
  if (space.placed && launch_place<false>(a, space, st) != hipSuccess) return CURE_ERR_HIP;
  launch_attn<false>(a, dtype, d, dim3((unsigned)(hkv * p.tiles), (unsigned)p.cut.most, (unsigned)batch), st);
  if (hipGetLastError() != hipSuccess) return CURE_ERR_HIP;
  if (in_parts(p)) launch_merge<false>(a, d, st);
  return launch_status();
}

extern "C" size_t cure_prefix_attn_workspace_size(int32_t batch, int32_t hq, int32_t hkv, int32_t d, int32_t n_max,
                                                  int32_t prefix_len, const int32_t* host_ctx_len,
                                                  const int32_t* host_n_nodes, int32_t kv_split) {
  if (batch <= 0 || hq <= 0 || hkv <= 0 || hq % hkv || d <= 0 || n_max <= 0 || prefix_len < 0 || !host_ctx_len ||
      !host_n_nodes)
    return 0;
  if (prefix_len == 0) return cure_tree_attn_workspace_size(batch, hq, hkv, d, n_max, host_ctx_len, host_n_nodes, 0);
  size_t need = 0;                                 // of whichever type needs more
  for (const int32_t dtype : {CURE_F32, CURE_BF16}) {
    const Plan p = prefix_plan(dtype, batch, hq, hkv, d, n_max, prefix_len, host_ctx_len, host_n_nodes, kv_split);
    need = std::max(need, prefix_space(p, batch, hq, d, n_max, host_ctx_len, host_n_nodes).bytes());
  }
  return need;
}

extern "C" cure_status cure_prefix_attn(const void* q, const void* k, const void* v, void* o, float* lse,
                                        int32_t dtype, int32_t out_dtype, int32_t batch, int32_t hq, int32_t hkv,
                                        int32_t d, float scale, int64_t prefix_off, int32_t prefix_len,
                                        const int64_t* kv_off, const int32_t* ctx_len, const int32_t* n_nodes,
                                        const int32_t* parent, int32_t n_max, const int32_t* host_ctx_len,
                                        const int32_t* host_n_nodes, int32_t kv_split, int32_t* tree_status,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  if (batch < 0 || n_max < 0 || kv_split < 0 || prefix_off < 0 || prefix_len < 0) return CURE_ERR_INVALID_ARG;
  const cure_status bad = check(q, k, v, o, dtype, out_dtype, hq, hkv, d, scale);
  if (bad != CURE_OK) return bad;
  // Nothing shared, or no nodes: the tree attention is all there is.
  if (batch == 0 || n_max == 0 || prefix_len == 0)
    return cure_tree_attn(q, k, v, o, lse, dtype, out_dtype, batch, hq, hkv, d, scale, kv_off, ctx_len, n_nodes,
                          parent, n_max, host_ctx_len, host_n_nodes, 0, 0, tree_status, workspace, workspace_bytes,
                          stream);
  if (n_max > CURE_MAX_TREE_NODES || batch > kMaxPrefixBatch || prefix_len > INT32_MAX - 4096)
    return CURE_ERR_UNSUPPORTED;
  if (!q || !k || !v || !o || !kv_off || !ctx_len || !n_nodes || !parent || !host_ctx_len || !host_n_nodes)
    return CURE_ERR_INVALID_ARG;
  for (int b = 0; b < batch; ++b)
    if (host_ctx_len[b] < 0 || host_n_nodes[b] < 0 || host_n_nodes[b] > n_max) return CURE_ERR_INVALID_ARG;
  for (int b = 0; b < batch; ++b)
    if (host_ctx_len[b] > INT32_MAX - 4096) return CURE_ERR_UNSUPPORTED;
  if ((int64_t)batch * n_max * (hq / hkv) > INT32_MAX - 4096) return CURE_ERR_UNSUPPORTED;
  const Plan p = prefix_plan(dtype, batch, hq, hkv, d, n_max, prefix_len, host_ctx_len, host_n_nodes, kv_split);
  const Space space = prefix_space(p, batch, hq, d, n_max, host_ctx_len, host_n_nodes);
  const int64_t units = prefix_units(p, batch, hkv, p.cut.most, p.own.most);
  if (!launchable(units)) return CURE_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < space.bytes()) return CURE_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return CURE_ERR_INVALID_ARG;
  Args a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  a.out_bf16 = out_dtype == CURE_BF16;
  a.hq = hq;
  a.hkv = hkv;
  a.group = hq / hkv;
  a.by_group = Div::by(a.group, std::max<int64_t>((int64_t)batch * n_max * a.group, hq));
  a.by_hkv = Div::by(hkv, units);
  a.batch = batch;
  a.n_max = n_max;
  a.scale_log2 = scale * kLog2e;
  a.rows = (int64_t)batch * n_max;
  a.n_rows = n_nodes;
  a.kv_off = kv_off;
  a.ctx_len = ctx_len;
  a.parent = parent;
  a.tree_status = tree_status;
  a.prefix_off = prefix_off;
  a.prefix_len = prefix_len;
  set_plan(a, p, space, workspace);
  hipStream_t st = as_stream(stream);
  if (space.placed && launch_place<true>(a, space, st) != hipSuccess) return CURE_ERR_HIP;
  launch_attn<true>(a, dtype, d, dim3((unsigned)units), st);
  if (hipGetLastError() != hipSuccess) return CURE_ERR_HIP;
  launch_merge<true>(a, d, st);
  return launch_status();
}
