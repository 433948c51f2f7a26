// What packing and the attention over a packed cache share: the block's layout and the
// vectors that both move.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace cure {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlockTokens = CURE_PACK_TOKENS;

// Blocks that n tokens take.
__host__ __device__ inline int64_t blocks_of(int64_t n) { return (n + kBlockTokens - 1) / kBlockTokens; }

// Loads of what a kernel reads once, which need not stay in its caches; others.
template <bool kOnce, typename T>
CURE_DEV T load_of(const T* p) {
  return kOnce ? __builtin_nontemporal_load(p) : *p;
}

// N values of a row, consecutive, as the dwords that hold them; widened to fp32, and back
// with one rounding, to nearest even. N * sizeof(E) is 4, 8 or a multiple of 16.
template <typename E, int N>
struct RowVec {
  static constexpr int kWords = N * (int)sizeof(E) / 4;
  uint32_t w[kWords];

  CURE_DEV void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  template <bool kOnce = false>
  CURE_DEV void load(const E* p) {
    if (kWords == 1) {
      w[0] = load_of<kOnce>(reinterpret_cast<const uint32_t*>(p));
      return;
    }
    if (kWords == 2) {
      const u32x2 x = load_of<kOnce>(reinterpret_cast<const u32x2*>(p));
      w[0] = x[0];
      w[1 % kWords] = x[1];
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const u32x4 x = load_of<kOnce>(reinterpret_cast<const u32x4*>(p) + i / 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[(i + j) % kWords] = x[j];
    }
  }
  CURE_DEV void store(E* p) const {
    if (kWords == 1) {
      *reinterpret_cast<uint32_t*>(p) = w[0];
      return;
    }
    if (kWords == 2) {
      *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1 % kWords]};
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; i += 4)
      reinterpret_cast<u32x4*>(p)[i / 4] =
          u32x4{w[i % kWords], w[(i + 1) % kWords], w[(i + 2) % kWords], w[(i + 3) % kWords]};
  }
  CURE_DEV float get(int i) const {
    if (sizeof(E) == 4) return __uint_as_float(w[i]);
    return i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
  }
  // Values i and i + 1, i even.
  CURE_DEV void put2(int i, float a, float b) {
    if (sizeof(E) == 4) {
      w[i] = __float_as_uint(a);
      w[(i + 1) % kWords] = __float_as_uint(b);
    } else {
      w[i / 2] = pack_bf16x2(a, b);
    }
  }
};

}  // namespace cure
