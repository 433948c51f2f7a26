// cure_rope_append: new rows' queries and keys normalised per head and rotated by
// their positions, keys and values written to the cache rows after each
// sequence's context -- what cure_tree_attn and the prompt attention read.
// cure_rope_frequencies: the rotation's frequencies, on the host.
//
//   x^  = x * rsqrt(mean(x^2) + eps) * w         (queries and keys, where weights are given)
//   y_a = m (x^_a cos t - x^_b sin t),  y_b = m (x^_a sin t + x^_b cos t),  t = pos * f_i
// for the rot / 2 pairs (a, b) of a head: (i, i + rot / 2), or (2i, 2i + 1) when
// interleaved; the other columns pass through. A prompt's row n has position
// base + n, a tree's node base + depth(n), so that after cure_commit has moved a path's
// rows to consecutive slots each still carries its own position.
//
// Everything is computed in fp32 from the inputs' own type and rounded once, to the
// nearest, at the store. The angle is reduced in fp64 (pos * f / 2 pi minus its whole
// part): far positions have angles of 10^5 and more, of which fp32 keeps 2^-7.
//
// Bound by memory: each row is read and written once (8 prompts of 501 to 4001 tokens, 17931 rows of
// 32 + 8 heads of 128: 89 us, 4.93 TB/s, the rate of a large copy), few rows by one launch and its two round
// trips to memory (32 rows 5.6 us). One workgroup takes up to kMaxRows
// rows of one sequence; the depth of a tree's nodes and the rows' cosines and sines are
// formed once per workgroup, in LDS, and serve all of a row's heads. A head's columns lie
// in d / (16 bytes) neighbouring lanes, so the norm's sum and the exchange with the lanes
// that hold the other half of the pairs stay inside a wave.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "host_util.hpp"

namespace cure {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 4;          // rows per workgroup
constexpr int kMaxPairs = 128;       // rotated pairs of a head (d <= 256)
constexpr int kBatch = 4;            // vectors in flight per thread

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct Args {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_ld, k_ld, v_ld;
  int64_t rows, cache_rows;
  int32_t n_max, rows_per_wg;
  const int64_t* row_off;
  const int32_t* n_rows;
  const int32_t* parent;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const int32_t* pos_off;
  int32_t hq, hkv, d;
  const void* q_weight;
  const void* k_weight;
  float eps, inv_d, mscale;
  const float* inv_freq;
  int32_t rot;
  void* q_out;
  void* k_cache;
  void* v_cache;
  int32_t* row_status;
};

// 16 bytes of a row as fp32, and back (one rounding, to nearest even).
template <typename E>
struct Vec;
template <>
struct Vec<uint16_t> {
  static constexpr int kN = 8;
  static CURE_DEV void widen(u32x4 u, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(u[i]);
      x[2 * i + 1] = bf16_hi(u[i]);
    }
  }
  static CURE_DEV u32x4 narrow(const float* x) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    return u;
  }
};
template <>
struct Vec<float> {
  static constexpr int kN = 4;
  static CURE_DEV void widen(u32x4 u, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(u[i]);
  }
  static CURE_DEV u32x4 narrow(const float* x) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(x[i]);
    return u;
  }
};

// Sum over the kLanes lanes of a head (an aligned group).
template <int kLanes>
CURE_DEV float group_sum(float x) {
  x += partner<1>(x);
  x += partner<2>(x);
  x += partner<4>(x);
  if (kLanes > 8) x += partner<8>(x);
  if (kLanes > 16) x += partner<16>(x);
  if (kLanes > 32) x = sum_halves(x);
  return x;
}

// kLanes: lanes per head, the power of two (8 to 64) that holds its vectors.
template <typename E, int kLanes, bool kInterleaved>
__global__ __launch_bounds__(kThreads) void rope_append(Args a) {
  using V = Vec<E>;
  constexpr int kN = V::kN;
  constexpr int kGroups = kThreads / kLanes;       // heads in work at a time
  __shared__ int s_anc[CURE_MAX_TREE_NODES], s_depth[CURE_MAX_TREE_NODES];
  __shared__ __attribute__((aligned(16))) float s_cos[kMaxRows][kMaxPairs], s_sin[kMaxRows][kMaxPairs];

  const int b = blockIdx.y, tid = threadIdx.x;
  const int n0 = blockIdx.x * a.rows_per_wg;
  const int heads = a.hq + 2 * a.hkv;
  const int lane = tid % kLanes;                   // within the head
  const int col = lane * kN;
  const bool in = col < a.d;

  // Vectors in work: kBatch heads per thread, from head `head` of row n0 + r on, kGroups
  // apart. The loads of the first need no more than the row's place.
  u32x4 x[kBatch];
  int r = 0, h = tid / kLanes;
  const auto settle = [&](int& r, int& h) {
    while (h >= heads) {
      h -= heads;
      ++r;
    }
  };
  const auto fetch = [&](int64_t row0, int rows) {
    int rr = r, hh = h;
#pragma unroll
    for (int u = 0; u < kBatch; ++u, hh += kGroups) {
      settle(rr, hh);
      x[u] = u32x4{0, 0, 0, 0};
      if (!in || rr >= rows) continue;
      const int64_t row = row0 + n0 + rr;
      const int hk = hh - a.hq;
      const E* src = hk < 0 ? static_cast<const E*>(a.q) + row * a.q_ld + (int64_t)hh * a.d
                     : hk < a.hkv ? static_cast<const E*>(a.k) + row * a.k_ld + (int64_t)hk * a.d
                                  : static_cast<const E*>(a.v) + row * a.v_ld + (int64_t)(hk - a.hkv) * a.d;
      x[u] = *reinterpret_cast<const u32x4*>(src + col);
    }
  };

  // One round trip: the sequence's sizes, its tree, the frequencies, the weights and,
  // where rows are padded and so in place whatever the sizes are, the first vectors.
  const bool tree = a.parent != nullptr;
  int p = -1;
  if (tree && tid < a.n_max) p = a.parent[(int64_t)b * a.n_max + tid];
  if (!a.row_off) fetch((int64_t)b * a.n_max, min(a.rows_per_wg, a.n_max - n0));
  u32x4 wq16{0, 0, 0, 0}, wk16{0, 0, 0, 0};        // this lane's norm weights
  if (in && a.q_weight) wq16 = *reinterpret_cast<const u32x4*>(static_cast<const E*>(a.q_weight) + col);
  if (in && a.k_weight) wk16 = *reinterpret_cast<const u32x4*>(static_cast<const E*>(a.k_weight) + col);
  const int pairs = a.rot / 2;
  const float freq0 = pairs > 0 ? a.inv_freq[tid % pairs] : 0.f;
  const int64_t row0 = a.row_off ? a.row_off[b] : (int64_t)b * a.n_max;
  const int N = a.n_rows[b];
  const int L = a.ctx_len[b];
  const int64_t off = a.kv_off[b];
  const int64_t base = (int64_t)L + (a.pos_off ? a.pos_off[b] : 0);
  bool bad = N < 0 || N > a.n_max || L < 0 || row0 < 0 || row0 > a.rows - N ||
             (a.hkv > 0 && (off < 0 || off > a.cache_rows - L - N));
  // Depths by pointer doubling: p becomes the ancestor 2^round up (-1: past the root), depth
  // the steps up to it. Up to 64 nodes every wave does it by itself, with lane exchanges; more
  // (at most 8 rounds for 256) go through LDS.
  int depth = p >= 0;
  if (tree && a.n_max <= kWave) {
    const int l = tid % kWave;
    p = l < a.n_max ? a.parent[(int64_t)b * a.n_max + l] : -1;
    bad = bad || __ballot(l < N && (p < -1 || p >= l)) != 0;
    p = l < N && !bad ? p : -1;
    depth = p >= 0;
    while (__ballot(p >= 0)) {
      const int up = __shfl(p, max(p, 0)), more = __shfl(depth, max(p, 0));
      depth += p >= 0 ? more : 0;
      p = p >= 0 ? up : -1;
    }
  } else if (tree) {
    bad = __syncthreads_or(bad || (tid < N && (p < -1 || p >= tid)));
    if (!bad) {
      if (tid < N) {
        s_anc[tid] = p;
        s_depth[tid] = depth;
      }
      while (__syncthreads_or(tid < N && p >= 0)) {
        int up = -1, more = 0;
        if (tid < N && p >= 0) {
          up = s_anc[p];
          more = s_depth[p];
        }
        __syncthreads();
        if (tid < N && p >= 0) {
          p = up;
          s_anc[tid] = up;
          s_depth[tid] += more;
        }
      }
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.row_status[b] = bad ? CURE_ERR_BAD_TREE : CURE_OK;
  if (bad || n0 >= N) return;
  const int nrows = min(a.rows_per_wg, N - n0);
  if (a.row_off) fetch(row0, nrows);

  // The half layout's partner lane, and the index of this lane's first pair.
  const bool turned = col < a.rot;
  const bool low = col < pairs;
  const int hop = pairs / kN;                      // lanes between the halves
  const int other = threadIdx.x % kWave + (turned ? (low ? hop : -hop) : 0);
  const int pair0 = !turned ? 0 : kInterleaved ? col / 2 : (low ? col : col - pairs);

  for (int i = tid; i < (nrows * pairs + kWave - 1) / kWave * kWave; i += kThreads) {
    const int row = min(i / max(pairs, 1), nrows - 1), f = i - row * pairs;
    int up = n0 + row;
    if (tree) up = a.n_max <= kWave ? __shfl(depth, up) : s_depth[up];
    if (i >= nrows * pairs) continue;
    const float freq = i == tid ? freq0 : a.inv_freq[f];
    double turn = (double)(base + up) * (double)freq * 0.15915494309189535;   // / 2 pi
    turn -= rint(turn);
    float sn, cs;
    sincospif(2.f * (float)turn, &sn, &cs);
    s_cos[row][f] = cs * a.mscale;
    s_sin[row][f] = sn * a.mscale;
  }
  __syncthreads();

  float wq[kN], wk[kN];
  V::widen(wq16, wq);
  V::widen(wk16, wk);
  // Uniform over the workgroup, as the exchanges inside a wave need every lane.
  const int items = nrows * heads;
  for (int i0 = 0; i0 < items; i0 += kBatch * kGroups) {
    if (i0 > 0) fetch(row0, nrows);
#pragma unroll
    for (int u = 0; u < kBatch; ++u, h += kGroups) {
      settle(r, h);
      const bool live = in && r < nrows;
      const int row = min(r, kMaxRows - 1);
      const bool query = h < a.hq, value = h >= a.hq + a.hkv;
      float y[kN];
      V::widen(x[u], y);
      if (a.q_weight || a.k_weight) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < kN; ++j) ss = fmaf(y[j], y[j], ss);
        ss = group_sum<kLanes>(ss);
        const float rs = rsqrtf(fmaf(ss, a.inv_d, a.eps));
        const bool norm = query ? a.q_weight != nullptr : a.k_weight != nullptr;
#pragma unroll
        for (int j = 0; j < kN; ++j) y[j] = norm ? y[j] * rs * (query ? wq[j] : wk[j]) : y[j];
      }
      // The pairs from pair0 on, a multiple of as many as are read: 16 bytes of LDS at a time (8
      // for the two pairs of four interleaved columns).
      constexpr int kReads = kInterleaved ? kN / 2 : kN, kWide = kReads < 4 ? kReads : 4;
      typedef float wide __attribute__((ext_vector_type(kWide)));
      float z[kN], c[kReads], s[kReads];
#pragma unroll
      for (int j = 0; j < kReads; j += kWide) {
        const wide cv = *reinterpret_cast<const wide*>(&s_cos[row][pair0 + j]);
        const wide sv = *reinterpret_cast<const wide*>(&s_sin[row][pair0 + j]);
#pragma unroll
        for (int i = 0; i < kWide; ++i) {
          c[j + i] = cv[i];
          s[j + i] = sv[i];
        }
      }
      if (kInterleaved) {
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
          z[j] = fmaf(y[j], c[j / 2], -(y[j + 1] * s[j / 2]));
          z[j + 1] = fmaf(y[j], s[j / 2], y[j + 1] * c[j / 2]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const float o = __shfl(y[j], other);
          z[j] = fmaf(y[j], c[j % kReads], low ? -(o * s[j % kReads]) : o * s[j % kReads]);
        }
      }
      if (!live) continue;
      const int64_t n = n0 + r;
      const int hk = h - a.hq;
      E* dst = query ? static_cast<E*>(a.q_out) + ((row0 + n) * a.hq + h) * a.d
                     : static_cast<E*>(value ? a.v_cache : a.k_cache) + ((off + L + n) * a.hkv + hk - (value ? a.hkv : 0)) * a.d;
      *reinterpret_cast<u32x4*>(dst + col) = value ? x[u] : V::narrow(turned ? z : y);
    }
  }
}

template <typename E, bool kInterleaved>
void launch(const Args& a, dim3 grid, hipStream_t st) {
  constexpr int kMost = 2 * kMaxPairs / Vec<E>::kN;      // lanes of the widest head
  const int lanes = a.d / Vec<E>::kN;
  const dim3 block(kThreads);
  if (lanes <= 8) hipLaunchKernelGGL((rope_append<E, 8, kInterleaved>), grid, block, 0, st, a);
  else if (lanes <= 16) hipLaunchKernelGGL((rope_append<E, 16, kInterleaved>), grid, block, 0, st, a);
  else if (kMost == 32 || lanes <= 32) hipLaunchKernelGGL((rope_append<E, 32, kInterleaved>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_append<E, kMost, kInterleaved>), grid, block, 0, st, a);
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" cure_status cure_rope_append(const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                                        const void* v, int64_t v_ld, int32_t dtype, int64_t rows,
                                        int32_t batch, int32_t n_max, const int64_t* row_off,
                                        const int32_t* n_rows, const int32_t* parent,
                                        const int64_t* kv_off, const int32_t* ctx_len,
                                        const int32_t* pos_off, int32_t hq, int32_t hkv, int32_t d,
                                        const void* q_weight, const void* k_weight, float eps,
                                        const float* inv_freq, int32_t rot, uint32_t flags,
                                        float mscale, void* q_out, void* k_cache, void* v_cache,
                                        int64_t cache_rows, int32_t* row_status, void* stream) {
  if (dtype != CURE_F32 && dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (batch < 0 || n_max < 0 || rows < 0 || cache_rows < 0 || hq < 0 || hkv < 0 || d <= 0 ||
      rot < 0 || rot > d || (flags & ~CURE_ROPE_INTERLEAVED))
    return CURE_ERR_INVALID_ARG;
  if (hq == 0 && hkv == 0) return CURE_ERR_INVALID_ARG;
  if (batch == 0) return CURE_OK;
  if (!n_rows || !kv_off || !ctx_len || !row_status || (rot > 0 && !inv_freq)) return CURE_ERR_INVALID_ARG;
  if (n_max > 0) {
    if ((hq > 0 && (!q || !q_out)) || (hkv > 0 && (!k || !v || !k_cache || !v_cache)))
      return CURE_ERR_INVALID_ARG;
    if (!row_off && rows / n_max < batch) return CURE_ERR_INVALID_ARG;   // padded rows
  }
  if (!std::isfinite(mscale) || ((q_weight || k_weight) && !(eps >= 0.f && std::isfinite(eps))))
    return CURE_ERR_INVALID_ARG;
  const int64_t elem = dtype == CURE_BF16 ? 2 : 4;
  if (d % 16 != 0 || d > 2 * kMaxPairs || rot % 16 != 0) return CURE_ERR_UNSUPPORTED;
  if (parent && n_max > CURE_MAX_TREE_NODES) return CURE_ERR_UNSUPPORTED;
  if (batch > 65535 || hq > 65535 || hkv > 65535) return CURE_ERR_UNSUPPORTED;
  if ((hq > 0 && q_ld < (int64_t)hq * d) ||
      (hkv > 0 && (k_ld < (int64_t)hkv * d || v_ld < (int64_t)hkv * d)))
    return CURE_ERR_INVALID_ARG;
  if (hq > 0 && q == q_out && q_ld != (int64_t)hq * d) return CURE_ERR_INVALID_ARG;   // rows would overlap
  // Rows move as 16-byte vectors.
  uintptr_t at = reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight);
  if (hq > 0) at |= reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(q_out);
  if (hkv > 0)
    at |= reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(k_cache) |
          reinterpret_cast<uintptr_t>(v_cache);
  if (at % 16 != 0) return CURE_ERR_INVALID_ARG;
  if ((hq > 0 && q_ld * elem % 16) || (hkv > 0 && (k_ld * elem % 16 || v_ld * elem % 16)))
    return CURE_ERR_INVALID_ARG;
  Args a{q, k, v, q_ld, k_ld, v_ld, rows, cache_rows, n_max, 1, row_off, n_rows, parent, kv_off,
         ctx_len, pos_off, hq, hkv, d, q_weight, k_weight, eps, 1.f / (float)d, mscale, inv_freq,
         rot, q_out, k_cache, v_cache, row_status};
  // Few rows are dealt out one to a workgroup; many share its start-up. us a call with one and
  // with four: 1024 rows of 32 + 8 heads of 128 8.5 and 12.2, 2048 14.6 and 15.1, 4096 22.3 and 21.6;
  // 2048 of 8 + 1 heads of 64 8.7 and 5.7. Large rows would turn later, small ones earlier: at 2048 the
  // former lose 3 % by it, the latter gain a third.
  if ((int64_t)batch * n_max >= 2048) a.rows_per_wg = kMaxRows;
  const int64_t most = row_off ? std::min<int64_t>(n_max, rows) : n_max;   // rows that a sequence can have
  const int64_t wgs = std::max<int64_t>(1, (most + a.rows_per_wg - 1) / a.rows_per_wg);
  if (wgs * kThreads >= (int64_t(1) << 32)) return CURE_ERR_UNSUPPORTED;   // a launch counts threads in 32 bits
  const dim3 grid((unsigned)wgs, (unsigned)batch);
  const bool interleaved = flags & CURE_ROPE_INTERLEAVED;
  hipStream_t st = as_stream(stream);
  if (dtype == CURE_BF16) interleaved ? launch<uint16_t, true>(a, grid, st) : launch<uint16_t, false>(a, grid, st);
  else interleaved ? launch<float, true>(a, grid, st) : launch<float, false>(a, grid, st);
  return launch_status();
}

extern "C" cure_status cure_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor,
                                             double orig_len, double p0, double p1,
                                             float* host_inv_freq, float* host_mscale) {
  if (rot < 0 || rot % 2 || !(base > 1.0) || !std::isfinite(base) || (rot > 0 && !host_inv_freq) || !host_mscale)
    return CURE_ERR_INVALID_ARG;
  if (scaling < CURE_ROPE_PLAIN || scaling > CURE_ROPE_RAMP) return CURE_ERR_INVALID_ARG;
  if (scaling != CURE_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return CURE_ERR_INVALID_ARG;
  if (scaling >= CURE_ROPE_BANDS &&
      (!(orig_len > 0.0) || !std::isfinite(orig_len) || !std::isfinite(p0) || !std::isfinite(p1)))
    return CURE_ERR_INVALID_ARG;
  if (scaling == CURE_ROPE_BANDS && !(p0 > 0.0 && p1 > p0)) return CURE_ERR_INVALID_ARG;
  if (scaling == CURE_ROPE_RAMP && !(p1 > 0.0 && p0 > p1)) return CURE_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586;
  *host_mscale = 1.f;
  if (scaling == CURE_ROPE_BASE && rot > 2) base *= std::pow(factor, (double)rot / (rot - 2));
  // Ramp: the pairs that make p0 (p1) turns over the original length bound it.
  double first = 0.0, last = 0.0;
  if (scaling == CURE_ROPE_RAMP) {
    const auto pair_of = [&](double turns) {
      return rot * std::log(orig_len / (turns * two_pi)) / (2.0 * std::log(base));
    };
    first = std::max(std::floor(pair_of(p0)), 0.0);
    last = std::min(std::ceil(pair_of(p1)), (double)(rot - 1));
    if (last <= first) last = first + 0.001;
    *host_mscale = (float)(0.1 * std::log(factor) + 1.0);
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    if (scaling == CURE_ROPE_LINEAR) {
      f /= factor;
    } else if (scaling == CURE_ROPE_BANDS) {
      // Wavelengths up to orig / p1 stay, those from orig / p0 on are stretched by the
      // factor, and those between blend.
      const double turns = orig_len * f / two_pi;
      const double keep = std::min(1.0, std::max(0.0, (turns - p0) / (p1 - p0)));
      f = f * keep + f / factor * (1.0 - keep);
    } else if (scaling == CURE_ROPE_RAMP) {
      const double stretch = std::min(1.0, std::max(0.0, (i - first) / (last - first)));
      f = f / factor * stretch + f * (1.0 - stretch);
    }
    host_inv_freq[i] = (float)f;
  }
  return CURE_OK;
}
