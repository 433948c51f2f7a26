// Host code of the packed cache's operators and of sampling under sanitizers: argument checks and launch
// plans over ordinary, degenerate and the largest sizes. No call reaches a kernel launch.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "cure.h"

static int failures = 0;

static void expect(bool ok, const char* what) {
  if (!ok) {
    std::printf("FAIL %s\n", what);
    ++failures;
  }
}

int main() {
  void* const P = reinterpret_cast<void*>(uintptr_t(0x1000));
  const auto ints = [&] { return static_cast<const int32_t*>(P); };
  const auto longs = [&] { return static_cast<const int64_t*>(P); };
  const int32_t big = INT32_MAX;
  struct Heads {
    int32_t hq, hkv, d;
  };
  const std::vector<Heads> heads = {{1, 1, 64}, {32, 8, 128}, {8, 1, 64}, {4096, 1, 128}, {4096, 4096, 128}, {1 << 20, 1 << 20, 64}};
  for (const int32_t n : {0, 1, 32, 33, 256, 65535, 1 << 20, big})
    for (const int32_t packed : {0, 1, 63, 64, 65, 32768, 1 << 24, big - 70000, big})
      for (const int32_t ctx : {0, 1, 500, big})
        for (const Heads& h : heads)
          for (const int32_t split : {0, 1, 2, 7, 64, 65, big})
            for (const int64_t rows : {int64_t(3) * n, INT64_MAX}) {
              const std::vector<int32_t> hn = {n, 0, n}, hp = {packed, 3, 64}, hc = {ctx, 1, 0};
              const size_t need = cure_packed_attn_workspace_size(3, rows, n, h.hq, h.hkv, h.d, hn.data(), hp.data(), hc.data(), split);
              expect(need <= size_t(1) << 30, "workspace");
              for (const int32_t dtype : {CURE_F32, CURE_BF16}) {
                // Calls of several parts stop for their workspace, those that are too large before; the others would launch.
                const bool large = (int64_t)n * h.hq > (int64_t(1) << 28) || (int64_t)packed + ctx + n > big - 4096;
                if (!large && (need == 0 || split < 2 || rows == INT64_MAX)) continue;
                const int st = cure_packed_attn(P, (const int8_t*)P, (const int8_t*)P, (const float*)P, (const float*)P, INT64_MAX, P, P,
                                                INT64_MAX, P, nullptr, dtype, dtype, 3, rows, n, h.hq, h.hkv, h.d, 0.1f, nullptr, ints(),
                                                longs(), ints(), longs(), ints(), nullptr, hn.data(), hp.data(), hc.data(), split,
                                                nullptr, P, 1, nullptr);
                expect(st == CURE_ERR_WORKSPACE || st == CURE_ERR_UNSUPPORTED, "attention");
                if (st != CURE_ERR_WORKSPACE && st != CURE_ERR_UNSUPPORTED) return 1;
              }
            }

  const auto pack = [&](int32_t layers, int64_t stride, int32_t hkv, int32_t n_max, int64_t blocks, int32_t d) {
    return cure_kv_pack(P, P, CURE_BF16, layers, stride, INT64_MAX, hkv, d, 2, n_max, longs(), ints(), (int8_t*)P, (int8_t*)P, (float*)P,
                        (float*)P, stride, blocks, longs(), ints(), (int32_t*)P, nullptr);
  };
  expect(pack(2, INT64_MAX, 8, 64, INT64_MAX, 128) == CURE_ERR_INVALID_ARG, "pack stride");
  expect(pack(big, INT64_MAX - 7, 8, 64, INT64_MAX, 128) == CURE_ERR_UNSUPPORTED, "pack layers");
  expect(pack(1, 0, big, big, INT64_MAX, 64) == CURE_ERR_UNSUPPORTED, "pack heads");
  expect(pack(1, 0, 1, big, INT64_MAX, 64) == CURE_ERR_UNSUPPORTED, "pack rows");
  expect(pack(1, 0, 8, 64, INT64_MAX, big) == CURE_ERR_UNSUPPORTED, "pack head dim");
  const auto sample = [&](int32_t batch, int32_t rows, int32_t vocab, int64_t ld) {
    return cure_sample(P, CURE_F32, batch, rows, vocab, ld, nullptr, nullptr, nullptr, nullptr, (const float*)P, nullptr, (int32_t*)P,
                       nullptr, nullptr, nullptr);
  };
  expect(sample(big, big, 100, INT64_MAX) == CURE_ERR_UNSUPPORTED, "sample rows");
  expect(sample(1, 1, big, INT64_MAX) == CURE_ERR_UNSUPPORTED, "sample vocabulary");
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
