// What the matrix-core attention kernels share: operand types, buffer resources, the
// DMA of K/V tiles into LDS, its swizzled layout and LDS operand reads (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace cure {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kRsrcWord3 = 0x00020000;     // raw (untyped) 32-bit access, gfx9 family

// A raw buffer resource over `bytes` bytes at `base`, as four wave-uniform
// dwords (SGPRs): base address (48 bits, stride 0), record count in bytes,
// and the gfx9-family word for untyped 32-bit access. Built from integer
// words rather than converted from the opaque resource type, which the
// compiler would spill through a per-thread memory copy.
CURE_DEV i32x4 raw_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu)),
               __builtin_amdgcn_readfirstlane((int)bytes),
               __builtin_amdgcn_readfirstlane(kRsrcWord3)};
}

CURE_DEV uint32_t lds_addr(const void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const lds_void*)p);
}

// LDS reads at a 32-bit LDS address: with a per-lane base and a compile-time
// constant the constant travels in the instruction's 16-bit offset field.
CURE_DEV bf16x8 lds_read16(uint32_t addr) {
  return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)addr;
}
CURE_DEV i16x4 lds_read_tr8(uint32_t addr) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)addr);
}

// 64 lanes x 16 bytes from a buffer resource straight into LDS: lane i's bytes
// land at lds_base + 16 * i (lds_base travels in M0). Out-of-range offsets
// read as zero. A DMA may follow the write of its M0 after one wait state, which the
// compiler does not add for an instruction that it cannot see into.
// dma16 marks the bytes as read once; dma16_shared leaves them to the L2, for
// workgroups that read the same ones.
CURE_DEV void dma16(uint32_t lds_base, uint32_t voff, i32x4 rsrc) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_base)
               : "memory");
}
CURE_DEV void dma16_shared(uint32_t lds_base, uint32_t voff, i32x4 rsrc) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_base)
               : "memory");
}

union Pack8 {
  uint4 u;
  bf16x8 v;
  i16x4 h[2];
};

// Three-input maximum as one v_max3_f32. Written as assembly because fmaxf
// first canonicalises every operand that may be a signalling NaN (an extra
// instruction per score); scores here are finite dot products or -inf. The compiler
// puts no wait states between a matrix instruction and assembly that reads its
// result, so no operand may be such a result that nothing else has read: max_scores.
CURE_DEV float max3_raw(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// Maximum of the scores of one matrix result (and of m). The canonicalised score is read by an
// instruction that the compiler sees and delays until the result is there, and every
// other score's read depends on it: one instruction more than the maxima alone.
template <class V>
CURE_DEV float max_scores(const V& x) {
  constexpr int n = sizeof(V) / sizeof(float);
  float m = __builtin_canonicalizef(x[0]);
#pragma unroll
  for (int r = 1; r < n; r += 2) m = max3_raw(m, x[r], x[r + 1 < n ? r + 1 : r]);
  return m;
}
template <class V>
CURE_DEV float max_scores(const V& x, float m) {
  constexpr int n = sizeof(V) / sizeof(float);
  m = max3_raw(m, __builtin_canonicalizef(x[0]), x[1]);
#pragma unroll
  for (int r = 2; r < n; r += 2) m = max3_raw(m, x[r], x[r + 1]);
  return m;
}
constexpr int kTile = 64;            // tokens per K/V tile
constexpr float kRescaleLog2 = 8.f;       // lazy rescale threshold (log2 units)

template <int D>
struct TileGeo {
  static constexpr int kChunks = D / 8;             // 16-byte chunks per row
  static constexpr int kRowBytes = D * 2;
  static constexpr int kTileBytes = kTile * kRowBytes;
  static constexpr int kBlocks = kTileBytes / 1024;  // 1 KB DMA blocks per tile
  // Swizzle: the chunk index is XORed with a row-dependent value. Any value
  // keeps the layout correct (the DMA and every reader apply the same XOR); it
  // only decides which LDS banks one instruction touches. At head dim 128 the
  // chunk bits are (r1^r2, r1, r2, r0) of the row bits r0..r2: with it neither
  // the K operand reads (16 bytes per lane, 16 rows) nor the transposed V reads
  // (8 bytes per lane, 4 rows per 16 lanes) have bank conflicts, as measured
  // with SQ_LDS_BANK_CONFLICT on gfx950 (the earlier permutation of the row
  // bits cost 4 stall cycles per K read and 2 per V read).
  static CURE_DEV int swz(int row) {
    if (kChunks == 16) {
      const int r0 = row & 1, r1 = (row >> 1) & 1, r2 = (row >> 2) & 1;
      return (r1 ^ r2) | (r1 << 1) | (r2 << 2) | (r0 << 3);
    }
    return ((row & 3) << 1) | ((row >> 2) & 1);
  }
  static CURE_DEV int offset(int row, int chunk) {   // byte offset inside a tile
    return row * kRowBytes + ((chunk ^ swz(row)) << 4);
  }
};

// s_waitcnt immediate: at most `vm` vector-memory operations outstanding, no
// wait on export, all LDS/scalar-memory operations complete (gfx9 encoding:
// vmcnt[3:0] in bits 3:0, vmcnt[5:4] in bits 15:14, expcnt in 6:4).
constexpr int waitcnt_vm(int vm) { return (vm & 15) | ((vm >> 4) << 14) | (7 << 4); }

}  // namespace cure
