// Host code of the rotary, prompt and shared-prefix operators under sanitizers: argument checks,
// frequencies and launch plans over ordinary, degenerate and the largest sizes. No call reaches a
// kernel launch.
#include <climits>
#include <cmath>
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
  const int32_t big = INT32_MAX;
  const std::vector<int32_t> lengths = {0, 1, 2, 31, 32, 33, 127, 129, 4097, 65535, 65536, 1 << 20, big - 5000};
  struct Heads {
    int32_t hq, hkv, d;
  };
  const std::vector<Heads> heads = {{1, 1, 64}, {32, 8, 128}, {8, 1, 64}, {65535, 1, 128}, {4096, 4096, 128}};
  const std::vector<int32_t> splits = {0, 1, 7, 65535, big};

  for (const int32_t n : lengths)
    for (const int32_t ctx : lengths)
      for (const Heads& h : heads)
        for (const int32_t split : splits) {
          const std::vector<int32_t> hn = {n, 1, 0}, hc = {ctx, 0, 5};
          const int64_t rows = (int64_t)n + 1;
          cure_prompt_attn_workspace_size(3, rows, h.hq, h.hkv, h.d, hn.data(), hc.data(), split);
          for (const int32_t dtype : {CURE_F32, CURE_BF16}) {
            // Calls of several parts stop for their workspace; the others would launch.
            if (split < 2 || n == 0 || n > 65535 || (int64_t)n + ctx <= 128) continue;
            const int st = cure_prompt_attn(P, P, P, P, nullptr, dtype, dtype, 3, rows, h.hq, h.hkv, h.d, 0.1f, (const int64_t*)P,
                                            (const int32_t*)P, (const int64_t*)P, (const int32_t*)P, hn.data(), hc.data(),
                                            split, P, 1, nullptr);
            expect(st == CURE_ERR_WORKSPACE || st == CURE_ERR_UNSUPPORTED, "prompt");
            if (st != CURE_ERR_WORKSPACE && st != CURE_ERR_UNSUPPORTED) return 1;
          }
        }

  for (const int32_t batch : {1, 3, 1024})
    for (const int32_t n_max : {1, 48, 256})
      for (const int32_t prefix : {1, 33, 16384, 1 << 24, big - 4096})
        for (const int32_t ctx : {0, 1, 500, big - 5000})
          for (const Heads& h : heads)
            for (const int32_t split : splits) {
              std::vector<int32_t> hn(batch, n_max), hc(batch, ctx);
              hn[0] = 0;
              const size_t need = cure_prefix_attn_workspace_size(batch, h.hq, h.hkv, h.d, n_max, prefix, hc.data(),
                                                                  hn.data(), split);
              expect(need > 0, "prefix workspace");
              const int st = cure_prefix_attn(P, P, P, P, nullptr, CURE_BF16, CURE_BF16, batch, h.hq, h.hkv, h.d, 0.1f, 0,
                                              prefix, (const int64_t*)P, (const int32_t*)P, (const int32_t*)P,
                                              (const int32_t*)P, n_max, hc.data(), hn.data(), split, nullptr, P, 1, nullptr);
              expect(st == CURE_ERR_WORKSPACE || st == CURE_ERR_UNSUPPORTED, "prefix");
              if (st != CURE_ERR_WORKSPACE && st != CURE_ERR_UNSUPPORTED) return 1;
            }

  std::vector<float> f(128);
  float m = 0.f;
  for (int32_t rot = 0; rot <= 256; rot += 2)
    for (int32_t scaling = CURE_ROPE_PLAIN; scaling <= CURE_ROPE_RAMP; ++scaling)
      for (const double factor : {1.0, 3.5, 1e6})
        for (const double orig : {1.0, 4096.0, 1e9}) {
          const double p0 = scaling == CURE_ROPE_RAMP ? 32.0 : 1.0, p1 = scaling == CURE_ROPE_RAMP ? 1.0 : 4.0;
          const int st = cure_rope_frequencies(rot, 10000.0, scaling, factor, orig, p0, p1, f.data(), &m);
          expect(st == CURE_OK, "frequencies");
          for (int32_t i = 0; i < rot / 2; ++i) expect(std::isfinite(f[i]) && f[i] >= 0.f, "a frequency");
        }

  const auto append = [&](int64_t rows, int32_t batch, int32_t n_max, int32_t hq, int32_t hkv, int32_t d, int64_t ld) {
    return cure_rope_append(P, ld, P, ld, P, ld, CURE_BF16, rows, batch, n_max, nullptr, (const int32_t*)P, nullptr,
                            (const int64_t*)P, (const int32_t*)P, nullptr, hq, hkv, d, nullptr, nullptr, 0.f, (const float*)P,
                            d, 0, 1.f, P, P, P, INT64_MAX, (int32_t*)P, nullptr);
  };
  expect(append(INT64_MAX, 2, big, big, 1, 64, INT64_MAX) == CURE_ERR_UNSUPPORTED, "append heads");
  expect(append(10, 2, 6, 2, 1, 64, 128) == CURE_ERR_INVALID_ARG, "append rows");
  expect(append(12, 2, 6, 2, 1, 64, 127) == CURE_ERR_INVALID_ARG, "append distance");
  expect(append(12, 2, 6, 2, 1, 320, 1 << 20) == CURE_ERR_UNSUPPORTED, "append head dim");
  std::printf("%d failure(s)\n", failures);
  return failures != 0;
}
