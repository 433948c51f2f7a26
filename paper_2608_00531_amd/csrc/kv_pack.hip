// cure_kv_pack: cache rows made blocks of 64 tokens in 8 bits with one scale for each
// block and kv head; cure_kv_unpack: blocks made rows.
//
//   a = max |x|,  scale = a / 127,  c = rint(127 x / a)
//
// The integer is the exact quotient's nearest, ties to even; ties are common in bf16, where x = a / 2
// is one. With 127 x exact (15 bits), q0 = x * (127 / a) and the exact remainder r = 127 x - q0 a,
// q0 + r / a is the quotient to fp32's last bit and a tie itself where it is one; no other quotient of
// two 8-bit integers times 127 lies near enough to a tie to round to it. For fp32 values x * (127 / a)
// is within 2^-16 of the quotient, so its nearest is right unless it lies between 0.49998 and 0.5 away;
// there the remainder 127 x - c a, which fp64 holds exactly (31 bits), says which.
//
// Bound by memory. Two waves take one block and head of K, two of V, 32 tokens each, whole, in
// registers: all their loads (8 KB of bf16 at head dim 128 each) are in flight together. A row's vectors lie
// in neighbouring lanes; the 16 tokens that a lane of V's layout holds are its own 16 loads, so that its
// bytes come together without exchange, and LDS turns them for the stores to be whole lines. Eight prompts
// of 501 to 4001 rows, 8 heads of 128: packed in 25 us and 4.4 TB/s (32 where the rows pass through the
// caches in the ordinary way), unpacked in 21 us and 5.1 TB/s (where its ordinary stores do better: 25).
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "host_util.hpp"
#include "packed.hpp"

namespace cure {
namespace {

struct Args {
  void* k;
  void* v;
  int64_t layer_stride, rows;
  int32_t n_max, hkv;
  const int64_t* kv_off;
  const int32_t* n_rows;
  int8_t* pk;
  int8_t* pv;
  float* k_scale;
  float* v_scale;
  int64_t block_stride, blocks;
  const int64_t* blk_off;
  const int32_t* from;               // first token of the sequence
  int32_t* row_status;
};

// What a workgroup takes of a sequence: tokens t0 .. of block `block`, n of them wanted, the
// first of which is row `row`; a head of it.
struct Part {
  int64_t row, block;
  int n, skip, head;                 // skip: the block's tokens before the first one wanted
};

// False: nothing to do.
CURE_DEV bool part_of(const Args& a, bool whole_blocks, Part& p) {
  const int b = blockIdx.y, index = blockIdx.x / a.hkv;
  const int n = a.n_rows[b], from = a.from[b];
  const int64_t row0 = a.kv_off[b], block0 = a.blk_off[b];
  const bool ok = n >= 0 && n <= a.n_max && from >= 0 && row0 >= 0 && row0 <= a.rows - n && block0 >= 0 &&
                  block0 <= a.blocks - blocks_of((int64_t)from + n) && !(whole_blocks && from % kBlockTokens);
  if (blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.row_status[b] = ok ? CURE_OK : CURE_ERR_BAD_TREE;
  if (!ok || n == 0) return false;
  const int64_t t0 = ((int64_t)(from / kBlockTokens) + index) * kBlockTokens;      // the block's first token
  const int64_t begin = t0 > from ? t0 : from, end = min(t0 + kBlockTokens, (int64_t)from + n);
  if (begin >= end) return false;
  p.head = blockIdx.x % a.hkv;
  p.skip = (int)(begin - t0);
  p.n = (int)(end - begin);
  p.row = row0 + (begin - from);
  p.block = block0 + t0 / kBlockTokens;
  return true;
}

// rint(127 x / a), ties to even; inv is near 127 / a.
CURE_DEV float to_int(float x, float a, float inv) {
  float c = rintf(x * inv);
  const double r = 2.0 * fma(-(double)c, (double)a, 127.0 * (double)x), m = fabs(r);
  if (m > (double)a || (m == (double)a && ((int)c & 1))) c += copysignf(1.f, (float)r);
  return c;
}

// Words' low bytes.
CURE_DEV uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// How a block's values become integers. Where 127 / a or 127 x would overflow they are scaled by a power of
// two first: what that rounds off is far below a / 254.
template <typename E>
struct Quant {
  static constexpr float kMagic = 12582912.f;      // 1.5 * 2^23: a sum's low bits are the integer
  float up, top, inv, unit;
  CURE_DEV explicit Quant(float a) {
    up = a < 0x1p-100f ? 0x1p100f : a > 0x1p100f ? 0x1p-100f : 1.f;
    top = a * up;
    inv = top > 0.f ? 127.f / top : 0.f;
    unit = inv * (1.f / 127.f);
  }
  // 16 values as bytes.
  CURE_DEV u32x4 bytes(float (&x)[16]) const {
    if (up != 1.f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= up;
    }
    uint32_t y[16];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float f;
      if (sizeof(E) == 2) {
        const float q = x[i] * inv;
        f = fmaf(fmaf(-q, top, 127.f * x[i]), unit, q) + kMagic;
      } else {
        f = fmaf(x[i], inv, kMagic);
        off = fmaxf(off, fabsf(fmaf(x[i], inv, kMagic - f)));
      }
      y[i] = __float_as_uint(f);
    }
    if (sizeof(E) == 4 && __builtin_expect(__any(!(off <= 0.49998f)), 0)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = (uint32_t)(int)to_int(x[i], top, inv);
    }
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = bytes_of(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    return out;
  }
};

// What a wave's lanes take of a half of a block. K: unit i is 16 columns of a token, and 16 bytes of the
// block. V: D / 32 columns of the 16 tokens 8 a + 4 h + c, each column 16 bytes of the block.
template <int D>
struct Lanes {
  static constexpr int kUnits = D / 32;            // of K, per lane
  static constexpr int kCols = D / 32;             // of V, per lane
  // Token of unit i or of V's load i, the part that all lanes share and the lane's own, and the lane's column.
  static CURE_DEV int k_token(int i) { return i * (kWave * 16 / D); }
  static CURE_DEV int k_own(int lane) { return lane / (D / 16); }
  static CURE_DEV int k_col(int lane) { return lane % (D / 16) * 16; }
  static CURE_DEV int k_byte(int t, int j) { return j / 32 * 1024 + j % 32 / 16 * 512 + t * 16; }
  static CURE_DEV int v_token(int i) { return i / 4 * 8 + i % 4; }
  static CURE_DEV int v_own(int lane) { return lane / 32 * 4; }
  static CURE_DEV int v_col(int lane) { return lane % 32 * kCols; }
  static CURE_DEV int v_byte(int lane, int j) { return j / 32 * 1024 + lane / 32 * 512 + j % 32 * 16; }
};

// The wave's part of a workgroup's: keys or values, and the tokens of a half.
struct Role {
  int lane, half;
  bool values;
  CURE_DEV Role() {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    lane = threadIdx.x % kWave;
    half = wave % 2;
    values = wave >= 2;
  }
};

// Has the values widened anew: kept in fp32 from the maximum on, they would take twice the registers.
template <class Row, int kRows>
CURE_DEV void forget(Row (&x)[kRows]) {
#pragma unroll
  for (int i = 0; i < kRows; ++i)
#pragma unroll
    for (int j = 0; j < Row::kWords; ++j) asm volatile("" : "+v"(x[i].w[j]));
}

template <typename E, int D>
__global__ __launch_bounds__(4 * kWave, sizeof(E) == 2 ? 7 : 5) void kv_pack(Args a) {
  using L = Lanes<D>;
  __shared__ float highs[4];
  __shared__ __attribute__((aligned(16))) u32x4 turn[4][D * 2];
  Part p;
  if (!part_of(a, true, p)) return;
  const Role r;
  const int lane = r.lane, n = p.n - 32 * r.half;  // tokens of this half, or fewer than none
  const int64_t pitch = (int64_t)a.hkv * D, layer = blockIdx.z;
  const E* src = static_cast<const E*>(r.values ? a.v : a.k) + layer * a.layer_stride + (p.row + 32 * r.half) * pitch +
                 (int64_t)p.head * D;
  const int64_t block = (layer * a.block_stride + p.block) * a.hkv + p.head;
  int8_t* dst = (r.values ? a.pv : a.pk) + block * (kBlockTokens * D) + r.half * (kBlockTokens / 2 * D);
  // The block's largest, of both halves.
  const auto highest = [&](float high) {
    high = wave_max(high);
    if (lane == 0) highs[threadIdx.x / kWave] = high;
    __syncthreads();
    high = fmaxf(highs[2 * r.values], highs[2 * r.values + 1]);
    if (lane == 0 && r.half == 0) (r.values ? a.v_scale : a.k_scale)[block] = high / 127.f;
    return high;
  };
  float high = 0.f;
  if (!r.values) {
    RowVec<E, 16> x[L::kUnits];
    const int own = L::k_own(lane);
    const uint32_t at = own * (uint32_t)pitch + L::k_col(lane);
    if (n >= kBlockTokens / 2) {
#pragma unroll
      for (int i = 0; i < L::kUnits; ++i) x[i].template load<true>(src + L::k_token(i) * pitch + at);
    } else {
#pragma unroll
      for (int i = 0; i < L::kUnits; ++i) {
        x[i].clear();
        if (L::k_token(i) + own < n) x[i].template load<true>(src + L::k_token(i) * pitch + at);
      }
    }
#pragma unroll
    for (int i = 0; i < L::kUnits; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) high = fmaxf(high, fabsf(x[i].get(j)));
    const Quant<E> q(highest(high));
    forget(x);
#pragma unroll
    for (int i = 0; i < L::kUnits; ++i) {
      float f[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = x[i].get(j);
      *reinterpret_cast<u32x4*>(dst + L::k_byte(L::k_token(i) + own, L::k_col(lane))) = q.bytes(f);
    }
    return;
  }
  RowVec<E, L::kCols> x[16];
  const int own = L::v_own(lane);
  const uint32_t at = own * (uint32_t)pitch + L::v_col(lane);
  if (n >= kBlockTokens / 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i].template load<true>(src + L::v_token(i) * pitch + at);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i].clear();
      if (L::v_token(i) + own < n) x[i].template load<true>(src + L::v_token(i) * pitch + at);
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int j = 0; j < L::kCols; ++j) high = fmaxf(high, fabsf(x[i].get(j)));
  const Quant<E> q(highest(high));
  forget(x);
#pragma unroll
  for (int j = 0; j < L::kCols; ++j) {
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = x[i].get(j);
    turn[threadIdx.x / kWave][L::v_byte(lane, L::v_col(lane) + j) / 16] = q.bytes(f);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < L::kCols; ++j) reinterpret_cast<u32x4*>(dst)[j * kWave + lane] = turn[threadIdx.x / kWave][j * kWave + lane];
}

// The largest scale that 127 times is finite. The one above it, of a block that holds fp32's largest value, is
// taken as this.
constexpr float kMostScale = 0x1.020406p+121f;

// Waits for what is loaded once, and not at every store that takes some of it, which would wait for the stores
// before too.
template <int kVecs>
CURE_DEV void arrived(u32x4 (&w)[kVecs]) {
#pragma unroll
  for (int i = 0; i < kVecs; ++i) asm volatile("" : "+v"(w[i]));
}

// The same pieces the other way.
template <typename E, int D>
__global__ __launch_bounds__(4 * kWave) void kv_unpack(Args a) {
  using L = Lanes<D>;
  Part p;
  if (!part_of(a, false, p)) return;
  const Role r;
  const int lane = r.lane, skip = p.skip - 32 * r.half;
  const int64_t pitch = (int64_t)a.hkv * D, layer = blockIdx.z;
  E* dst = static_cast<E*>(r.values ? a.v : a.k) + layer * a.layer_stride + (p.row - skip) * pitch + (int64_t)p.head * D;
  const int64_t block = (layer * a.block_stride + p.block) * a.hkv + p.head;
  const bool all = skip <= 0 && skip + p.n >= kBlockTokens / 2;
  float scale = (r.values ? a.v_scale : a.k_scale)[block];
  scale = scale > kMostScale ? kMostScale : scale;
  const int8_t* src = (r.values ? a.pv : a.pk) + block * (kBlockTokens * D) + r.half * (kBlockTokens / 2 * D);
  const auto value = [&](const u32x4& w, int i) { return (float)(int8_t)(w[i / 4] >> (i % 4 * 8)) * scale; };
  const auto wanted = [&](int t) { return t >= skip && t < skip + p.n; };
  if (!r.values) {
    const int own = L::k_own(lane);
    const uint32_t at = own * (uint32_t)pitch + L::k_col(lane);
    u32x4 w[L::kUnits];
#pragma unroll
    for (int i = 0; i < L::kUnits; ++i)
      w[i] = *reinterpret_cast<const u32x4*>(src + L::k_byte(L::k_token(i) + own, L::k_col(lane)));
    arrived(w);
#pragma unroll
    for (int i = 0; i < L::kUnits; ++i) {
      RowVec<E, 16> x;
#pragma unroll
      for (int j = 0; j < 16; j += 2) x.put2(j, value(w[i], j), value(w[i], j + 1));
      if (all || wanted(L::k_token(i) + own)) x.store(dst + L::k_token(i) * pitch + at);
    }
    return;
  }
  const int own = L::v_own(lane);
  const uint32_t at = own * (uint32_t)pitch + L::v_col(lane);
  u32x4 w[L::kCols];
#pragma unroll
  for (int j = 0; j < L::kCols; ++j) w[j] = *reinterpret_cast<const u32x4*>(src + L::v_byte(lane, L::v_col(lane) + j));
  arrived(w);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    RowVec<E, L::kCols> x;
#pragma unroll
    for (int j = 0; j < L::kCols; j += 2) x.put2(j, value(w[j], i), value(w[j + 1], i));
    if (all || wanted(L::v_token(i) + own)) x.store(dst + L::v_token(i) * pitch + at);
  }
}

// The checks that both calls make, and the launch. touched: blocks of a sequence; *nothing: there is nothing to do.
cure_status check(const Args& a, int64_t touched, int32_t dtype, int32_t n_layers, int32_t d, int32_t batch, bool* nothing) {
  *nothing = false;
  if (dtype != CURE_F32 && dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (n_layers < 1 || a.rows < 0 || a.hkv <= 0 || d <= 0 || batch < 0 || a.n_max < 0 || a.blocks < 0)
    return CURE_ERR_INVALID_ARG;
  if (n_layers > 1 && (a.layer_stride < 0 || a.block_stride < 0)) return CURE_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return CURE_ERR_UNSUPPORTED;
  // A launch counts threads in 32 bits, and offsets within some rows are of 32.
  if (batch > 65535 || n_layers > 65535 || a.hkv > 1 << 20 || touched * a.hkv * (4 * kWave) >= (int64_t(1) << 32))
    return CURE_ERR_UNSUPPORTED;
  *nothing = batch == 0;
  if (batch == 0) return CURE_OK;
  if (!a.kv_off || !a.n_rows || !a.blk_off || !a.from || !a.row_status) return CURE_ERR_INVALID_ARG;
  if (a.n_max > 0) {
    if (a.rows > 0 && (!a.k || !a.v)) return CURE_ERR_INVALID_ARG;
    if (a.blocks > 0 && (!a.pk || !a.pv || !a.k_scale || !a.v_scale)) return CURE_ERR_INVALID_ARG;
    const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    if ((at(a.k) | at(a.v) | at(a.pk) | at(a.pv)) % 16 || (at(a.k_scale) | at(a.v_scale)) % 4) return CURE_ERR_INVALID_ARG;
    if (n_layers > 1 && a.layer_stride % (dtype == CURE_BF16 ? 8 : 4)) return CURE_ERR_INVALID_ARG;
  }
  return CURE_OK;
}

// Workgroups: blocks that a sequence's rows can touch (one more where they need not begin with
// one) x heads, sequences, layers.
template <bool kPack>
cure_status launch(Args a, int32_t dtype, int32_t n_layers, int32_t d, int32_t batch, void* stream) {
  bool nothing;
  const int64_t touched = a.n_max == 0 ? 1 : blocks_of(a.n_max) + (kPack ? 0 : 1);
  const cure_status st = check(a, touched, dtype, n_layers, d, batch, &nothing);
  if (st != CURE_OK || nothing) return st;
  if (n_layers <= 1) a.layer_stride = a.block_stride = 0;
  const dim3 grid((unsigned)(touched * a.hkv), (unsigned)batch, (unsigned)n_layers), block(4 * kWave);
  hipStream_t s = as_stream(stream);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
  if (kPack) {
    if (dtype == CURE_BF16) d == 128 ? run(kv_pack<uint16_t, 128>) : run(kv_pack<uint16_t, 64>);
    else d == 128 ? run(kv_pack<float, 128>) : run(kv_pack<float, 64>);
  } else {
    if (dtype == CURE_BF16) d == 128 ? run(kv_unpack<uint16_t, 128>) : run(kv_unpack<uint16_t, 64>);
    else d == 128 ? run(kv_unpack<float, 128>) : run(kv_unpack<float, 64>);
  }
  return launch_status();
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" cure_status cure_kv_pack(const void* k, const void* v, int32_t dtype, int32_t n_layers,
                                    int64_t layer_stride, int64_t rows, int32_t hkv, int32_t d,
                                    int32_t batch, int32_t n_max, const int64_t* kv_off,
                                    const int32_t* n_rows, int8_t* pk, int8_t* pv, float* k_scale,
                                    float* v_scale, int64_t block_stride, int64_t blocks,
                                    const int64_t* blk_off, const int32_t* packed_len,
                                    int32_t* row_status, void* stream) {
  return launch<true>(Args{const_cast<void*>(k), const_cast<void*>(v), layer_stride, rows, n_max, hkv, kv_off, n_rows, pk, pv,
                           k_scale, v_scale, block_stride, blocks, blk_off, packed_len, row_status},
                      dtype, n_layers, d, batch, stream);
}

extern "C" cure_status cure_kv_unpack(const int8_t* pk, const int8_t* pv, const float* k_scale,
                                      const float* v_scale, int64_t block_stride, int64_t blocks,
                                      const int64_t* blk_off, const int32_t* first, void* k, void* v,
                                      int32_t dtype, int32_t n_layers, int64_t layer_stride, int64_t rows,
                                      int32_t hkv, int32_t d, int32_t batch, int32_t n_max,
                                      const int64_t* kv_off, const int32_t* n_rows, int32_t* row_status,
                                      void* stream) {
  return launch<false>(Args{k, v, layer_stride, rows, n_max, hkv, kv_off, n_rows, const_cast<int8_t*>(pk),
                            const_cast<int8_t*>(pv), const_cast<float*>(k_scale), const_cast<float*>(v_scale), block_stride,
                            blocks, blk_off, first, row_status},
                       dtype, n_layers, d, batch, stream);
}
