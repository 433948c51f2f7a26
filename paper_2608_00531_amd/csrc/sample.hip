// cure_sample: one token drawn for each logits row, with temperature, top-k, top-p and
// min-p, from a given uniform number.
//
// In the order (value descending, index ascending), with w_j = exp((x_j - m) / T) or nothing
// past 64 T below the maximum m, what each filter keeps is a run from the front, and the
// token is the entry at which the kept weights' running sum passes u W. So a row needs
// three places in its order: by a count (top-k), by a sum of weights (top-p, and the token) and by
// a value (min-p). All are found alike, without sorting: a histogram over bins of the
// logits holds each bin's count and weight, a scan over the bins says in which one the place
// lies, and that bin is divided again until it holds a single value, whose entries differ
// by index alone.
//
// Whether an entry is kept or drawn must not depend on how the work is split, so weights
// are summed in bins as integers: relative to the upper edge of a bin of width T / 64 a weight
// is in (exp(-1/64), 1], and 2^44 times it, rounded, leaves room for 2^20 of them. Over the bins
// the sums are formed in fp64, in one order.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "host_util.hpp"

namespace cure {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;
constexpr int kBins = 4096;
constexpr int kPer = kBins / kThreads;             // bins of a thread
constexpr double kRange = 64.0;                    // weights reach 64 T below the maximum
constexpr double kUnit = 0x1p44;
constexpr int kMaxVocab = 1 << 20;

struct Args {
  const void* logits;
  int32_t rows, vocab;
  int64_t ld;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniform;
  const int32_t* n_rows;
  int32_t* token;
  float* logprob;
  int32_t* kept;
};

CURE_DEV float widen(uint16_t x) { return bf16_to_f32(x); }
CURE_DEV float widen(float x) { return x; }

// Order-preserving integer of a finite value; both zeros alike.
CURE_DEV uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
CURE_DEV float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// exp(-y) for 0 <= y <= 1/64: the series' next term is below 2^-54.
CURE_DEV double exp_small(double y) {
  double p = 1.0 / 720;
  p = fma(-y, p, 1.0 / 120);
  p = fma(-y, p, 1.0 / 24);
  p = fma(-y, p, 1.0 / 6);
  p = fma(-y, p, 0.5);
  p = fma(-y, p, 1.0);
  return fma(-y, p, 1.0);
}

// A place in the order: the entries before it, their weight.
struct Place {
  int count;
  double mass;
};
// The run up to a place: everything above `key`, and the first `ties` entries that equal it.
struct Run {
  uint32_t key;
  int ties, count;
  double mass;
};

enum Query { kCount, kMass, kDraw, kValue };       // entries, weight reached, weight passed, values from a key on

struct Shared {
  uint32_t cnt[kBins];
  unsigned long long mass[kBins];
  // Saved scan of the first histogram.
  uint32_t sum_cnt[kWaves];
  double sum_mass[kWaves];
  uint32_t found_bin;
  Place found;
  uint32_t lo, hi;
  uint32_t seg[kWaves];
  float max[kWaves];
};

// A row's map from values to weights and bins.
struct Scale {
  double m, inv_t, limit;            // 64 T
  CURE_DEV double below(float x) const { return m - (double)x; }
  CURE_DEV bool has(float x) const { return below(x) <= limit; }
  CURE_DEV int bin(float x) const { return min((int)(below(x) * inv_t * kRange), kBins - 1); }
  CURE_DEV double weight(float x) const { return exp(-below(x) * inv_t); }
  // Units of exp(-bin / 64) that an entry of the bin has.
  CURE_DEV unsigned long long units(float x, int bin) const {
    return (unsigned long long)rint(kUnit * exp_small(fmax(fma(below(x), inv_t, -bin * (1.0 / kRange)), 0.0)));
  }
};
CURE_DEV double edge(int bin) { return exp(-bin * (1.0 / kRange)) / kUnit; }

template <typename E>
struct Row {
  const E* x;
  int vocab;
  template <typename F>
  CURE_DEV void each(F&& f) const {
    for (int i = threadIdx.x; i < vocab; i += kThreads) f(widen(x[i]), i);
  }
};

// Finds in the histogram the first bin, in order, at which the place lies: its index (or -1),
// and what is before it. weight(bin) is one unit's worth; bins are in descending order of value.
template <typename W, typename Hit>
CURE_DEV int find_bin(Shared& sh, const Place& base, W&& weight, Hit&& hit) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  uint32_t c = 0;
  double w = 0.0;
  for (int i = 0; i < kPer; ++i) {
    const int bin = tid * kPer + i;
    c += sh.cnt[bin];
    if (sh.cnt[bin]) w += (double)sh.mass[bin] * weight(bin);
  }
  // Running sums over the threads, in one order.
  uint32_t ci = c;
  double wi = w;
  for (int d = 1; d < kWave; d *= 2) {
    const uint32_t cu = __shfl_up(ci, d);
    const double wu = __shfl_up(wi, d);
    if (lane >= d) {
      ci += cu;
      wi += wu;
    }
  }
  __syncthreads();
  if (lane == kWave - 1) {
    sh.sum_cnt[wave] = ci;
    sh.sum_mass[wave] = wi;
  }
  if (tid == 0) sh.found_bin = kBins;
  __syncthreads();
  Place p = base;
  for (int i = 0; i < wave; ++i) {
    p.count += sh.sum_cnt[i];
    p.mass += sh.sum_mass[i];
  }
  const uint32_t c_up = __shfl_up(ci, 1);
  const double w_up = __shfl_up(wi, 1);
  if (lane > 0) {
    p.count += c_up;
    p.mass += w_up;
  }
  // The first bin that is hit, else the last one that holds anything.
  int mine = kBins;
  Place at = p;
  for (int i = 0; i < kPer && mine == kBins; ++i) {
    const int bin = tid * kPer + i;
    const int n = sh.cnt[bin];
    const double mass = n ? (double)sh.mass[bin] * weight(bin) : 0.0;
    if (hit(bin, n, Place{p.count + n, p.mass + mass})) {
      mine = bin;
      at = p;
    }
    p.count += n;
    p.mass += mass;
  }
  if (mine < kBins) atomicMin(&sh.found_bin, (uint32_t)mine);
  __syncthreads();
  int found = (int)sh.found_bin;
  if (found == kBins) {
    // Rounding kept a sum from its target: the last bin that holds anything.
    __syncthreads();
    if (tid == 0) sh.found_bin = 0;
    __syncthreads();
    int last = -1;
    Place q = p;
    Place lq = p;
    for (int i = kPer - 1; i >= 0 && last < 0; --i) {
      const int bin = tid * kPer + i;
      const int n = sh.cnt[bin];
      q.count -= n;
      if (n) {
        q.mass -= (double)sh.mass[bin] * weight(bin);
        last = bin;
        lq = q;
      }
    }
    if (last >= 0) atomicMax(&sh.found_bin, (uint32_t)last);
    __syncthreads();
    found = (int)sh.found_bin;
    if (last == found) sh.found = lq;
  } else if (mine == found) {
    sh.found = at;
  }
  __syncthreads();
  return found;
}

// The run of `query`: count entries, or weight `target`, or values from key `from` on, at most
// `most` entries. sh holds the first histogram, which is made again where it was replaced.
template <typename E>
CURE_DEV Run find_run(Shared& sh, const Row<E>& row, const Scale& sc, Query query, int count, double target, uint32_t from) {
  const int tid = threadIdx.x;
  const auto hit = [&](const Place& upto) {
    return query == kCount ? upto.count >= count : query == kMass ? upto.mass >= target : upto.mass > target;
  };
  // First histogram, once every thread has read the last one.
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) {
    sh.cnt[i] = 0;
    sh.mass[i] = 0;
  }
  __syncthreads();
  row.each([&](float x, int) {
    if (!sc.has(x)) return;
    const int bin = sc.bin(x);
    atomicAdd(&sh.cnt[bin], 1u);
    atomicAdd(&sh.mass[bin], sc.units(x, bin));
  });
  __syncthreads();
  const int from_bin = query == kValue ? sc.bin(value_of(from)) : 0;
  const int bin = find_bin(sh, Place{0, 0.0}, edge,
                           [&](int b, int n, const Place& upto) { return query == kValue ? b == from_bin : n > 0 && hit(upto); });
  Place base = sh.found;
  // The keys of the bin's entries.
  __syncthreads();
  if (tid == 0) {
    sh.lo = ~0u;
    sh.hi = 0;
  }
  __syncthreads();
  row.each([&](float x, int) {
    if (!sc.has(x) || sc.bin(x) != bin) return;
    atomicMin(&sh.lo, key_of(x));
    atomicMax(&sh.hi, key_of(x));
  });
  __syncthreads();
  uint32_t lo = sh.lo, hi = sh.hi;
  if (lo > hi) return Run{from, 0, base.count, base.mass};         // by value, and none in that bin
  const double unit = edge(bin);
  while (true) {
    if (query == kValue && from > hi) return Run{from, 0, base.count, base.mass};
    // Bins of keys, the largest first.
    const uint32_t width = (hi - lo) / kBins + 1;
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) {
      sh.cnt[i] = 0;
      sh.mass[i] = 0;
    }
    __syncthreads();
    row.each([&](float x, int) {
      if (!sc.has(x) || sc.bin(x) != bin) return;
      const uint32_t k = key_of(x);
      if (k < lo || k > hi) return;
      const int i = (int)((hi - k) / width);
      atomicAdd(&sh.cnt[i], 1u);
      atomicAdd(&sh.mass[i], sc.units(x, bin));
    });
    __syncthreads();
    // By value: the bin that holds `from`, or the first one below the run.
    const int at = find_bin(sh, base, [&](int) { return unit; }, [&](int b, int n, const Place& upto) {
      return query == kValue ? (from <= lo ? b == kBins - 1 : b == (int)((hi - from) / width)) : n > 0 && hit(upto);
    });
    base = sh.found;
    const int n = sh.cnt[at];
    const double mass = n ? (double)sh.mass[at] * unit : 0.0;
    if (query == kValue && from <= lo) return Run{lo, n, base.count + n, base.mass + mass};     // all of them: none equals it below
    const uint32_t top = hi - (uint32_t)at * width, bottom = top - lo < width ? lo : top - width + 1;
    if (width == 1 || n == 0) {
      if (query == kValue) return Run{top, n, base.count + n, base.mass + mass};
      // One value: so many of its entries.
      const double each = mass / n;
      int ties = query == kCount ? count - base.count
                                 : (int)fmin((double)n, fmax(1.0, query == kMass ? ceil((target - base.mass) / each)
                                                                                 : floor((target - base.mass) / each) + 1.0));
      ties = max(1, min(ties, n));
      return Run{top, ties, base.count + ties, base.mass + ties * each};
    }
    lo = bottom;
    hi = top;
  }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void sample_rows(Args a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int b = blockIdx.x / a.rows, n = blockIdx.x % a.rows;
  const int64_t r = blockIdx.x;
  const float t = a.temperature ? a.temperature[b] : 1.f, top_p = a.top_p ? a.top_p[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f;
  const int top_k = a.top_k ? a.top_k[b] : 0;
  const float u = a.uniform[r];
  const auto answer = [&](int token, float logprob, int kept) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = logprob;
    if (a.kept) a.kept[r] = kept;
  };
  if ((a.n_rows && n >= a.n_rows[b]) || !(t >= 0.f) || t == INFINITY || top_p != top_p || min_p != min_p || u != u) {
    if (tid == 0) answer(CURE_NO_TOKEN, -INFINITY, 0);
    return;
  }
  const Row<E> row{static_cast<const E*>(a.logits) + r * a.ld, a.vocab};
  float high = -INFINITY;
  bool bad = false;
  row.each([&](float x, int) {
    bad = bad || !(x < INFINITY);
    high = fmaxf(high, x);
  });
  high = wave_max(high);
  if (lane == 0) sh.max[wave] = high;
  bad = __syncthreads_or(bad);
  for (int w = 0; w < kWaves; ++w) high = fmaxf(high, sh.max[w]);
  if (bad || high == -INFINITY) {
    if (tid == 0) answer(CURE_NO_TOKEN, -INFINITY, 0);
    return;
  }
  const double td = t == 0.f ? 1.0 : (double)t;
  const Scale sc{(double)high, 1.0 / td, t == 0.f ? 0.0 : kRange * td};
  Run run, drawn;
  if (t == 0.f) {
    run = drawn = Run{key_of(high), 1, 1, 1.0};
  } else {
    run = find_run(sh, row, sc, kCount, top_k > 0 ? min(top_k, a.vocab) : a.vocab, 0.0, 0);
    if (top_p < 1.f) {
      const Run p = find_run(sh, row, sc, kMass, 0, fmax(0.0, (double)top_p) * run.mass, 0);
      if (p.count < run.count) run = p;
    }
    if (min_p > 0.f) {
      // The smallest key whose weight reaches min_p (the maximum's does, or is kept all the same).
      uint32_t lo = key_of((float)(sc.m - sc.limit)), hi = key_of(high);
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (sc.weight(value_of(mid)) >= (double)min_p) hi = mid;
        else lo = mid + 1;
      }
      const bool one = !(1.f >= min_p);
      const Run v = one ? Run{key_of(high), 1, 1, 1.0} : find_run(sh, row, sc, kValue, 0, 0.0, lo);
      if (v.count < run.count) run = v;
    }
    drawn = find_run(sh, row, sc, kDraw, 0, fmax(0.0, (double)u) * run.mass, 0);
    // Rounding, or a number of one and more: the last entry kept.
    if (drawn.count > run.count) drawn = find_run(sh, row, sc, kCount, run.count, 0.0, 0);
  }
  // The drawn.ties-th entry of that value, by index: waves count in parts of the row.
  const int part = ((a.vocab + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int i0 = wave * part, i1 = min(i0 + part, a.vocab);
  int found = 0;
  for (int i = i0 + lane; i - lane < i1; i += kWave)
    found += __popcll(__ballot(i < i1 && widen(row.x[min(i, a.vocab - 1)]) > -INFINITY && key_of(widen(row.x[min(i, a.vocab - 1)])) == drawn.key));
  if (lane == 0) sh.seg[wave] = found;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += sh.seg[w];
  if (before < drawn.ties && before + found >= drawn.ties) {
    for (int i = i0 + lane; i - lane < i1; i += kWave) {
      const bool is = i < i1 && key_of(widen(row.x[min(i, a.vocab - 1)])) == drawn.key;
      const unsigned long long hits = __ballot(is);
      const int here = __popcll(hits & ((1ull << lane) - 1));
      if (is && before + here + 1 == drawn.ties)
        answer(i, (float)(-sc.below(value_of(drawn.key)) * sc.inv_t - log(run.mass)), run.count);
      before += __popcll(hits);
    }
  }
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" size_t cure_sample_workspace_size(int32_t batch, int32_t rows, int32_t vocab) {
  (void)batch;
  (void)rows;
  (void)vocab;
  return 0;
}

extern "C" cure_status cure_sample(const void* logits, int32_t dtype, int32_t batch, int32_t rows,
                                   int32_t vocab, int64_t ld, const float* temperature,
                                   const int32_t* top_k, const float* top_p, const float* min_p,
                                   const float* uniform, const int32_t* n_rows, int32_t* token,
                                   float* logprob, int32_t* kept, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  (void)workspace;
  (void)workspace_bytes;
  if (dtype != CURE_F32 && dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (batch < 0 || rows < 0 || vocab < 1 || ld < vocab) return CURE_ERR_INVALID_ARG;
  if (vocab > kMaxVocab) return CURE_ERR_UNSUPPORTED;
  const int64_t total = (int64_t)batch * rows;
  if (total >= (int64_t(1) << 31) / kThreads) return CURE_ERR_UNSUPPORTED;
  if (total == 0) return CURE_OK;
  if (!logits || !uniform || !token) return CURE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == CURE_BF16 ? 2 : 4)) return CURE_ERR_INVALID_ARG;
  const Args a{logits, rows, vocab, ld, temperature, top_k, top_p, min_p, uniform, n_rows, token, logprob, kept};
  const dim3 grid((unsigned)total), block(kThreads);
  if (dtype == CURE_BF16) hipLaunchKernelGGL((sample_rows<uint16_t>), grid, block, 0, as_stream(stream), a);
  else hipLaunchKernelGGL((sample_rows<float>), grid, block, 0, as_stream(stream), a);
  return launch_status();
}
