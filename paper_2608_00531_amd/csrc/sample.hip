// cure_sample: one token drawn for each logits row, with temperature, top-k, top-p and
// min-p, from a given uniform number.
//
// In the order (value descending, index ascending), with w_j = exp((x_j - m) / T) or nothing
// past 64 T below the maximum m, what each filter keeps is a run from the front, and the
// token is the entry at which the kept weights' running sum passes u W. So a row needs a few
// places in its order: by a count (top-k), by a sum of weights (top-p, and the token) and by
// a value (min-p). They are found alike, without sorting: a histogram over bins of the values
// holds what each bin has, sums over groups of 64 bins say in which group a place lies, and
// a scan of that group's bins in which bin.
//
// Whether an entry is kept or drawn must not depend on how the work is split. Counts are
// integers, weights are formed in fp64 once for each bin or summed as integers, and the bins' sums
// are added in one order.
//
// One workgroup takes a row, so that every bin is in one LDS. A row is read twice, for its histogram and for the
// drawn value's entries. 544 bf16 rows of 128256 take 60 us: the first reading and the bins' computation 30 (the LDS
// additions hide behind them and cost one), the search 17, the second reading 16, less what overlaps. 32 CUs have
// three of the rows and the others two: 512 rows take 52 us. One row takes 25, ten of them its first reading by one
// CU and the rest latency of the steps behind it.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "host_util.hpp"

namespace cure {
namespace {

constexpr double kRange = 64.0;                    // weights reach 64 T below the maximum
constexpr int kMostWaves = 16;                     // of a workgroup
constexpr int kMaxVocab = 1 << 20;
constexpr int kList = 1024;                        // entries of a bin that are put in order in a list, at most

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

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

// A row's settings. none: no token can be drawn by them.
struct Settings {
  float t, top_p, min_p, u;
  int top_k;
  bool none;
};
CURE_DEV Settings settings_of(const Args& a, int64_t r) {
  const int b = (int)(r / a.rows), n = (int)(r % a.rows);
  Settings s;
  s.t = a.temperature ? a.temperature[b] : 1.f;
  s.top_p = a.top_p ? a.top_p[b] : 1.f;
  s.min_p = a.min_p ? a.min_p[b] : 0.f;
  s.top_k = a.top_k ? a.top_k[b] : 0;
  s.u = a.uniform[r];
  s.none = (a.n_rows && n >= a.n_rows[b]) || !(s.t >= 0.f) || s.t == INFINITY || s.top_p != s.top_p || s.min_p != s.min_p ||
           s.u != s.u;
  return s;
}
CURE_DEV void answer(const Args& a, int64_t r, int token, float logprob, int kept) {
  a.token[r] = token;
  if (a.logprob) a.logprob[r] = logprob;
  if (a.kept) a.kept[r] = kept;
}
CURE_DEV void no_answer(const Args& a, int64_t r) { answer(a, r, CURE_NO_TOKEN, -INFINITY, 0); }

// exp(y) for -709 < y <= 0: 2^k e^f with |f| <= ln 2 / 2, whose series' next term is below 2^-57.
CURE_DEV double exp_of(double y) {
  const double k = rint(y * 1.4426950408889634074);
  const double f = fma(k, -2.3190468138462996e-17, fma(k, -0.6931471805599453094, y));      // ln 2 in two parts
  const double f2 = f * f, f4 = f2 * f2;
  const auto pair = [&](double a, double b) { return fma(f, b, a); };
  const double low = fma(f2, pair(0.5, 1.0 / 6), pair(1.0, 1.0));
  const double mid = fma(f2, pair(1.0 / 720, 1.0 / 5040), pair(1.0 / 24, 1.0 / 120));
  const double high = fma(f2, pair(1.0 / 3628800, 1.0 / 39916800), pair(1.0 / 40320, 1.0 / 362880));
  const double top = pair(1.0 / 479001600, 1.0 / 6227020800);
  return ldexp(fma(f4, fma(f4, fma(f4, top, high), mid), low), (int)k);
}

// A row's map from values to weights.
struct Scale {
  double m, inv_t, limit;            // limit: 64 T
  CURE_DEV double below(float x) const { return m - (double)x; }
  CURE_DEV bool has(float x) const { return below(x) <= limit; }
  CURE_DEV double weight(float x) const { return exp_of(-below(x) * inv_t); }
};
CURE_DEV Scale scale_of(float high, float t) {
  const double td = t == 0.f ? 1.0 : (double)t;    // T = 0: only what equals the maximum
  return Scale{(double)high, 1.0 / td, t == 0.f ? 0.0 : kRange * td};
}

// Sums over the wave.
template <int kStage>
CURE_DEV double with_partner(double v) {
  return v + __hiloint2double(cure::partner<kStage>(__double2hiint(v)), cure::partner<kStage>(__double2loint(v)));
}
CURE_DEV double wave_sum(double x) {
  x = with_partner<1>(x);
  x = with_partner<2>(x);
  x = with_partner<4>(x);
  x = with_partner<8>(x);
  x = with_partner<16>(x);
  return with_partner<32>(x);
}
CURE_DEV int wave_sum(int x) {
  x += cure::partner<1>(x);
  x += cure::partner<2>(x);
  x += cure::partner<4>(x);
  x += cure::partner<8>(x);
  x += cure::partner<16>(x);
  return x + cure::partner<32>(x);
}

// Entries and their weight.
struct Amount {
  int n;
  double w;
};
CURE_DEV Amount operator+(Amount a, Amount b) { return Amount{a.n + b.n, a.w + b.w}; }
// Of one lane, the same for all.
CURE_DEV Amount lane_of(Amount a, int lane) {
  const auto read = [&](int x) { return __builtin_amdgcn_readlane(x, lane); };
  return Amount{read(a.n), __hiloint2double(read(__double2hiint(a.w)), read(__double2loint(a.w)))};
}
// Of the lane below, nothing for the first.
CURE_DEV Amount lower(Amount a) {
  const auto move = [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x138, 0xf, 0xf, false); };
  return Amount{move(a.n), __hiloint2double(move(__double2hiint(a.w)), move(__double2loint(a.w)))};
}
// One step of a scan: what a DPP pattern brings from a lower lane is added in the rows of kRows, and
// nothing where it brings none.
template <int kPattern, int kRows>
CURE_DEV Amount with_lower(Amount a) {
  const auto move = [](int x) { return __builtin_amdgcn_update_dpp(0, x, kPattern, kRows, 0xf, false); };
  return a + Amount{move(a.n), __hiloint2double(move(__double2hiint(a.w)), move(__double2loint(a.w)))};
}
// Sum over the lanes up to this one: in rows of 16, then row 0's last lane to row 1 and 2's to 3, then
// lane 31 to the upper half.
CURE_DEV Amount wave_scan(Amount a) {
  a = with_lower<0x111, 0xf>(a);
  a = with_lower<0x112, 0xf>(a);
  a = with_lower<0x114, 0xf>(a);
  a = with_lower<0x118, 0xf>(a);
  a = with_lower<0x142, 0xa>(a);
  return with_lower<0x143, 0xc>(a);
}

// A bin in the order: what lies before it, and what it holds.
struct Found {
  int pos;
  Amount before, in;
};

// The bins of a row for one wave: kGroups groups of 64 positions in descending order of value, whose
// sums lie in LDS; bin(pos) gives what a position holds.
template <int kGroups, typename Bin>
struct Order {
  static constexpr int kEach = (kGroups + kWave - 1) / kWave;      // groups of a lane
  Bin bin;
  Amount group[kEach], before, upto;               // of the lane

  CURE_DEV Order(const int* n, const double* w, Bin b) : bin(b) {
    Amount mine{0, 0.0};
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      group[j] = Amount{n[lane_id() * kEach + j], w[lane_id() * kEach + j]};
      mine = mine + group[j];
    }
    upto = wave_scan(mine);
    before = lower(upto);
  }
  CURE_DEV Amount all() const { return lane_of(upto, kWave - 1); }

  // The first position that holds something and up to which hit(amount) is true; where rounding
  // keeps it from being so, the last one that holds something. There has to be one.
  template <typename Hit>
  CURE_DEV Found find(const Hit& hit) const {
    const bool any = upto.n > before.n;
    unsigned long long is = __ballot(any && hit(upto));
    const int lane = is ? __ffsll(is) - 1 : 63 - __clzll(__ballot(any));
    int at = -1;
    bool sure = false;
    Amount run = before, base = before;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const Amount next = run + group[j];
      if (group[j].n > 0 && !sure) {
        at = j;
        base = run;
        sure = hit(next);
      }
      run = next;
    }
    const int g = lane * kEach + __builtin_amdgcn_readlane(at, lane);
    base = lane_of(base, lane);
    const Amount in = bin(g * kWave + lane_id());
    const Amount sum = wave_scan(in);
    is = __ballot(in.n > 0 && hit(base + sum));
    const int l = is ? __ffsll(is) - 1 : 63 - __clzll(__ballot(in.n > 0));
    return Found{g * kWave + l, base + lane_of(lower(sum), l), lane_of(in, l)};
  }
};

// How many of n entries of weight `each` behind `before` reach (or pass) a target.
CURE_DEV int ties_to(double target, Amount before, Amount in, bool pass) {
  const double each = in.w / in.n, x = (target - before.w) / each;
  return (int)fmin((double)in.n, fmax(1.0, pass ? floor(x) + 1.0 : ceil(x)));
}

// ---------------------------------------------------------------------------
// Any values, and fp32 in general: bins of width T / 32 below the maximum. Relative to its upper edge an entry of a
// bin has a weight in (exp(-1/32), 1], and 2^43 times it, rounded, leaves room for 2^20 of them
// in an integer of 64 bits. The bin of a place is gathered and put in order; where it holds too many entries
// it is divided by their keys until it holds a single value.
constexpr int kBins = 2048;
constexpr double kPerT = 32.0;                     // bins of a width T
constexpr int kGroups = kBins / kWave;
constexpr double kUnit = 0x1p43;
static_assert(kUnit * kMaxVocab <= 0x1p63, "a bin may hold the whole row");

// Order-preserving integer of a finite value; both zeros alike.
CURE_DEV uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
CURE_DEV float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// 2^43 exp(-f / 32) for 0 <= f <= 1, rounded: the series' next term is below 2^-55, and 1.5 * 2^52 added leaves
// the integer in the low bits.
CURE_DEV unsigned long long units_of(double f) {
  constexpr double u = -1.0 / kPerT;
  constexpr double c2 = u * u / 2, c3 = c2 * u / 3, c4 = c3 * u / 4, c5 = c4 * u / 5, c6 = c5 * u / 6, c7 = c6 * u / 7;
  double p = fma(f, kUnit * c7, kUnit * c6);
  p = fma(f, p, kUnit * c5);
  p = fma(f, p, kUnit * c4);
  p = fma(f, p, kUnit * c3);
  p = fma(f, p, kUnit * c2);
  p = fma(f, p, kUnit * u);
  p = fma(f, p, kUnit) + 0x1.8p52;
  return (unsigned long long)__double_as_longlong(p) & ((1ull << 51) - 1);
}

struct Binned : Scale {
  double per;                        // bins of a unit
  CURE_DEV explicit Binned(const Scale& s) : Scale(s), per(s.inv_t * kPerT) {}
  CURE_DEV int bin(float x) const { return min((int)(below(x) * per), kBins - 1); }
  // Units of exp(-bin / 32) that an entry of the bin has.
  CURE_DEV unsigned long long units(float x, int bin) const { return units_of(below(x) * per - bin); }
};
CURE_DEV double edge(int bin) { return exp_of(-bin * (1.0 / kPerT)) / kUnit; }

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

enum Query { kCount, kMass, kDraw };               // entries, weight reached, weight passed

struct Shared {
  uint32_t cnt[kBins];
  unsigned long long mass[kBins];
  uint32_t sum_cnt[kMostWaves];
  double sum_mass[kMostWaves];
  uint32_t found_bin;
  Place found;
  uint32_t lo, hi;
  uint32_t seg[kMostWaves];
  float max[kMostWaves];
  // For places found in the first histogram.
  int group_n[kWave];                // of groups, and zeros
  double group_w[kWave];
  Found at;
  int query;
  double target;
  Amount run;
  int listed;
  uint32_t key[kList];
  int index[kList];
  int order[kList];
};

CURE_DEV float widen(uint16_t x) { return bf16_to_f32(x); }
CURE_DEV float widen(float x) { return x; }

template <typename E, int kThreads>
struct Row {
  const E* x;
  int vocab;
  template <typename F>
  CURE_DEV void each(F&& f) const {
    each_at([&](float v, int) { f(v); });
  }
  template <typename F>
  CURE_DEV void each_at(F&& f) const {
    constexpr int kAhead = 4;
    if (sizeof(E) == 2) {
      for (int i = threadIdx.x; i < vocab; i += kThreads) f(widen(x[i]), i);
      return;
    }
    int i = threadIdx.x * 4;
    for (; i + (kAhead - 1) * 4 * kThreads + 4 <= vocab; i += kAhead * 4 * kThreads) {
      u32x4 w[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) __builtin_memcpy(&w[u], x + i + u * 4 * kThreads, 16);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(__uint_as_float(w[u][j]), i + u * 4 * kThreads + j);
    }
    for (; i < vocab; i += 4 * kThreads)
      for (int j = 0; j < 4; ++j)
        if (i + j < vocab) f(widen(x[i + j]), i + j);
  }
};

// Finds in the histogram the first bin, in order, at which the place lies: its index (or -1),
// and what is before it. weight(bin) is one unit's worth; bins are in descending order of value.
template <int kThreads, typename W, typename Hit>
CURE_DEV int find_bin(Shared& sh, const Place& base, W&& weight, Hit&& hit) {
  constexpr int kPer = kBins / kThreads;           // bins of a thread
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
    if (hit(n, Place{p.count + n, p.mass + mass})) {
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

// The run of `query`: count entries, or weight `target`. sh holds the first histogram, which is made
// again where it was replaced.
template <typename E, int kThreads>
CURE_DEV Run find_run(Shared& sh, const Row<E, kThreads>& row, const Binned& sc, Query query, int count, double target) {
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
  row.each([&](float x) {
    if (!sc.has(x)) return;
    const int bin = sc.bin(x);
    atomicAdd(&sh.cnt[bin], 1u);
    atomicAdd(&sh.mass[bin], sc.units(x, bin));
  });
  __syncthreads();
  const int bin = find_bin<kThreads>(sh, Place{0, 0.0}, edge, [&](int n, const Place& upto) { return n > 0 && hit(upto); });
  Place base = sh.found;
  // The keys of the bin's entries.
  __syncthreads();
  if (tid == 0) {
    sh.lo = ~0u;
    sh.hi = 0;
  }
  __syncthreads();
  row.each([&](float x) {
    if (!sc.has(x) || sc.bin(x) != bin) return;
    atomicMin(&sh.lo, key_of(x));
    atomicMax(&sh.hi, key_of(x));
  });
  __syncthreads();
  uint32_t lo = sh.lo, hi = sh.hi;
  const double unit = edge(bin);
  while (true) {
    // Bins of keys, the largest first.
    const uint32_t width = (hi - lo) / kBins + 1;
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) {
      sh.cnt[i] = 0;
      sh.mass[i] = 0;
    }
    __syncthreads();
    row.each([&](float x) {
      if (!sc.has(x) || sc.bin(x) != bin) return;
      const uint32_t k = key_of(x);
      if (k < lo || k > hi) return;
      const int i = (int)((hi - k) / width);
      atomicAdd(&sh.cnt[i], 1u);
      atomicAdd(&sh.mass[i], sc.units(x, bin));
    });
    __syncthreads();
    const int at = find_bin<kThreads>(sh, base, [&](int) { return unit; }, [&](int n, const Place& upto) { return n > 0 && hit(upto); });
    base = sh.found;
    const int n = sh.cnt[at];
    const double mass = n ? (double)sh.mass[at] * unit : 0.0;
    const uint32_t top = hi - (uint32_t)at * width, bottom = top - lo < width ? lo : top - width + 1;
    if (width == 1 || n == 0) {
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

// The entry up to which the row's order has `count` entries, or weight `target`: found in the first
// histogram, whose groups are summed, by gathering its bin. False: the bin holds too many.
struct Entry {
  uint32_t key;
  int index;
  Amount upto;
};
template <typename E, int kThreads>
CURE_DEV bool find_entry(Shared& sh, const Row<E, kThreads>& row, const Binned& sc, Query query, int count, double target, Entry& out) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const auto hit = [&](Amount x) { return query == kCount ? x.n >= count : query == kMass ? x.w >= target : x.w > target; };
  __syncthreads();
  if (wave == 0) {
    const auto holds = [&](int pos) {
      const int n = (int)sh.cnt[pos];
      return Amount{n, n ? (double)sh.mass[pos] * edge(pos) : 0.0};
    };
    const Order<kGroups, decltype(holds)> order(sh.group_n, sh.group_w, holds);
    const Found f = order.find(hit);
    if (lane == 0) {
      sh.at = f;
      sh.listed = 0;
    }
  }
  __syncthreads();
  const Found f = sh.at;
  if (f.in.n > kList) return false;
  // Values somewhat beyond the bin's, by which to tell most entries without 64-bit arithmetic.
  const float low = (float)(sc.m - (f.pos + 1.001) / sc.per), high = (float)(sc.m - (f.pos - 0.001) / sc.per);
  row.each_at([&](float x, int i) {
    if (!(x >= low && x <= high) || !sc.has(x) || sc.bin(x) != f.pos) return;
    const int k = atomicAdd(&sh.listed, 1);
    sh.key[k] = key_of(x);
    sh.index[k] = i;
  });
  __syncthreads();
  const int n = f.in.n;
  for (int i = tid; i < n; i += kThreads) {
    const uint32_t k = sh.key[i];
    const int at = sh.index[i];
    int before = 0;
    for (int j = 0; j < n; ++j) before += sh.key[j] > k || (sh.key[j] == k && sh.index[j] < at);
    sh.order[before] = i;
  }
  __syncthreads();
  if (wave == 0) {
    const double unit = edge(f.pos);
    int found = n - 1;
    Amount upto = f.before;
    unsigned long long sum = 0;
    for (int i0 = 0; i0 < n; i0 += kWave) {
      const int i = min(i0 + lane, n - 1);
      unsigned long long u = i0 + lane < n ? sc.units(value_of(sh.key[sh.order[i]]), f.pos) : 0;
      for (int d = 1; d < kWave; d *= 2) {
        const unsigned long long up = __shfl_up(u, d);
        if (lane >= d) u += up;
      }
      const Amount here{f.before.n + i + 1, f.before.w + (double)(sum + u) * unit};
      const unsigned long long is = __ballot(i0 + lane < n && hit(here));
      const int l = is ? __ffsll(is) - 1 : min(kWave, n - i0) - 1;
      upto = lane_of(here, l);
      if (is) {
        found = i0 + l;
        break;
      }
      sum += __shfl(u, kWave - 1);
    }
    if (lane == 0) {
      sh.lo = sh.key[sh.order[found]];
      sh.query = sh.index[sh.order[found]];
      sh.run = upto;
    }
  }
  __syncthreads();
  out = Entry{sh.lo, sh.query, sh.run};
  return true;
}

// The smallest key whose weight reaches min_p, which is at most 1.
CURE_DEV uint32_t key_from(const Binned& sc, float min_p) {
  uint32_t lo = key_of((float)(sc.m - sc.limit)), hi = key_of((float)sc.m);
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (sc.weight(value_of(mid)) >= (double)min_p) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

template <typename E, int kThreads>
CURE_DEV void sample_any(Shared& sh, const Args& a, int64_t r, const Settings& s) {
  constexpr int kWaves = kThreads / kWave;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const Row<E, kThreads> row{static_cast<const E*>(a.logits) + r * a.ld, a.vocab};
  float high = -INFINITY;
  bool bad = false;
  for (int i = tid; i < kBins; i += kThreads) {
    sh.cnt[i] = 0;
    sh.mass[i] = 0;
  }
  row.each([&](float x) {
    bad = bad || !(x < INFINITY);
    high = fmaxf(high, x);
  });
  high = wave_max(high);
  if (lane == 0) sh.max[wave] = high;
  bad = __syncthreads_or(bad);
  for (int w = 0; w < kWaves; ++w) high = fmaxf(high, sh.max[w]);
  if (bad || high == -INFINITY) {
    if (tid == 0) no_answer(a, r);
    return;
  }
  const Binned sc(scale_of(high, s.t));
  const double u = fmax(0.0, (double)s.u), top_p = fmax(0.0, (double)s.top_p);
  // The first histogram, and its groups' sums.
  row.each([&](float x) {
    if (!sc.has(x)) return;
    const int bin = sc.bin(x);
    atomicAdd(&sh.cnt[bin], 1u);
    atomicAdd(&sh.mass[bin], sc.units(x, bin));
  });
  __syncthreads();
  for (int g = wave; g < kWave; g += kWaves) {
    const int pos = g * kWave + lane, n = g < kGroups ? (int)sh.cnt[pos] : 0;
    Amount sum{0, 0.0};
    if (__ballot(n > 0)) sum = Amount{wave_sum(n), wave_sum(n ? (double)sh.mass[pos] * edge(pos) : 0.0)};
    if (lane == 0) {
      sh.group_n[g] = sum.n;
      sh.group_w[g] = sum.w;
    }
  }
  __syncthreads();
  Amount run{0, 0.0};
  for (int g = 0; g < kGroups; ++g) run = run + Amount{sh.group_n[g], sh.group_w[g]};
  const Amount whole = run;
  const bool by_k = s.t > 0.f && s.top_k > 0 && s.top_k < run.n, by_p = s.t > 0.f && s.top_p < 1.f, by_min = s.t > 0.f && s.min_p > 0.f;
  int reach = 1;                                   // entries whose weight is at least min_p
  if (by_min && s.min_p <= 1.f) {
    const float from = value_of(key_from(sc, s.min_p));
    int n = 0;
    row.each([&](float x) { n += x >= from; });
    n = wave_sum(n);
    if (lane == 0) sh.seg[wave] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kWaves; ++w) n += sh.seg[w];
    reach = max(1, min(n, whole.n));
  }
  // Place q of the order that a row needs, if it does: top-k, top-p, min-p, the token; and the last
  // entry kept, where rounding or a number of one and more lead past it. One loop, for the search to be in
  // the code once.
  struct Wanted {
    bool is;
    Query query;
    int count;
    double target;
  };
  const auto wanted = [&](int q, const Amount& kept, int drawn) {
    if (q == 0) return Wanted{by_k, kCount, s.top_k, 0.0};
    if (q == 1) return Wanted{by_p, kMass, 0, top_p * kept.w};
    if (q == 2) return Wanted{by_min && reach < kept.n, kCount, reach, 0.0};
    if (q == 3) return s.t == 0.f ? Wanted{true, kCount, 1, 0.0} : Wanted{true, kDraw, 0, u * kept.w};
    return Wanted{drawn > kept.n, kCount, kept.n, 0.0};
  };
  const int q0 = s.t == 0.f ? 3 : 0;
  if (s.t == 0.f) run = Amount{1, 1.0};
  const Amount start = run;
  Entry e;
  bool quick = true;
#pragma unroll 1
  for (int q = q0; q < 5 && quick; ++q) {
    const Wanted w = wanted(q, run, q > 3 ? e.upto.n : 0);
    if (!w.is) continue;
    quick = find_entry(sh, row, sc, w.query, w.count, w.target, e);
    if (quick && q < 3 && e.upto.n < run.n) run = e.upto;
  }
  if (quick) {
    if (tid == 0) answer(a, r, e.index, (float)(-sc.below(value_of(e.key)) * sc.inv_t - log(run.w)), run.n);
    return;
  }
  // A bin that holds too many: by keys.
  Amount kept = start;
  Run drawn{key_of(high), 1, 1, 1.0};
#pragma unroll 1
  for (int q = q0; q < 5; ++q) {
    const Wanted w = wanted(q, kept, drawn.count);
    if (!w.is) continue;
    const Run found = find_run(sh, row, sc, w.query, w.count, w.target);
    if (q >= 3) drawn = found;
    else if (found.count < kept.n) kept = Amount{found.count, found.mass};
  }
  // The drawn.ties-th entry of that value, by index: waves count in parts of the row.
  const int part = ((a.vocab + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  const int i0 = wave * part, i1 = min(i0 + part, a.vocab);
  const auto is_it = [&](int i) {
    const float x = widen(row.x[min(i, a.vocab - 1)]);
    return i < i1 && x > -INFINITY && key_of(x) == drawn.key;
  };
  int found = 0;
  for (int i = i0; i < i1; i += kWave) found += __popcll(__ballot(is_it(i + lane)));
  __syncthreads();
  if (lane == 0) sh.seg[wave] = found;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += sh.seg[w];
  if (before >= drawn.ties || before + found < drawn.ties) return;
  for (int i = i0; i < i1; i += kWave) {
    const bool is = is_it(i + lane);
    const unsigned long long hits = __ballot(is);
    const int here = __popcll(hits & ((1ull << lane) - 1));
    if (is && before + here + 1 == drawn.ties)
      answer(a, r, i + lane, (float)(-sc.below(value_of(drawn.key)) * sc.inv_t - log(kept.w)), kept.n);
    before += __popcll(hits);
  }
}

constexpr int kThreads32 = 1024;

__global__ __launch_bounds__(kThreads32) void sample_f32(Args a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Settings s = settings_of(a, r);
  if (!s.none) sample_any<float, kThreads32>(sh, a, r, s);
  else if (threadIdx.x == 0) no_answer(a, r);
}

// ---------------------------------------------------------------------------
// bf16: a bin is a value, of which [2^-30, 2^10) has 40 octaves of 128 to either sign, and zero. Weights
// are formed once for each bin in use, so that an entry costs four packed integer instructions
// and one LDS addition. Eight waves take a row and three rows share a CU, which hide each other's latency: 768
// rows take 72 us, and 90 with 16 waves to a row and two to a CU; a single row 27 and 27. Rows with
// other magnitudes that count go the general way, entry by entry: one row of 128256 with an entry of 1100
// takes 166 us, 544 of them 411, and one of a single such value, whose additions all meet in one bin, 3.5 ms.
constexpr int kOctaves = 40 * 128;                 // bins of one sign
constexpr int kSign = 8192;                        // a negative value's, whose byte offset has its sign bit
constexpr int kPlaces = 2 * kOctaves;              // in a row's order
constexpr uint32_t kFirst16 = ((127 - 30) << 7) - 1;      // bits of the value below 2^-30
constexpr int kLowest = kSign + kOctaves - 1, kHighest = kOctaves - 1; // the bins of the largest magnitudes
constexpr int kZero = 0, kMinusZero = kSign;    // behind either, of the smallest
constexpr uint32_t kMinusInf2 = 0xff80ff80u;
constexpr int kGroups16 = kPlaces / kWave;
constexpr int kGroupSlots = (kGroups16 + kWave - 1) / kWave * kWave;   // of groups, and zeros
constexpr int kTies = 2048;                        // entries of one value that are put in order in a list, at most

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));


CURE_DEV u16x2 both(uint32_t x) { return __builtin_bit_cast(u16x2, x * 0x10001u); }
// Bins of two values, times 4.
CURE_DEV uint32_t bins_of(uint32_t w) {
  const u16x2 mag = __builtin_bit_cast(u16x2, w & 0x7fff7fffu);
  u16x2 t = __builtin_elementwise_min(__builtin_elementwise_sub_sat(mag, both(kFirst16)), both(kOctaves - 1));
  uint32_t one = 0x10001u;
  asm("" : "+s"(one));                             // a minimum with a known 1 would become comparisons
  t = __builtin_elementwise_max(t, __builtin_elementwise_min(mag, __builtin_bit_cast(u16x2, one))) << 2;
  return (w & 0x80008000u) | __builtin_bit_cast(uint32_t, t);
}
constexpr uint32_t kLowest4 = 4 * kLowest;
static_assert(kLowest4 < 0x10000 && 4 * kSign == 0x8000, "");
CURE_DEV float value_of_bin(int bin) {
  const int t = bin % kSign;
  return __uint_as_float(t ? (uint32_t)(t + kFirst16) << 16 | (bin >= kSign ? 0x80000000u : 0u) : 0u);
}
// The bin at a place of the order: positive values from the top down, zero, negative ones. The last
// place is that of minus zero, whose entries are counted with zero's.
CURE_DEV int bin_at(int pos) { return pos < kOctaves ? kOctaves - 1 - pos : kSign + (pos + 1) % kOctaves; }

struct Shared16 {
  union {
    int cnt[kSign + kOctaves];
    struct {                                       // between the two signs' bins
      int positive[kOctaves];
      double group_w[kGroupSlots];
      int group_n[kGroupSlots];
      int list[kTies];
    };
  };
  int listed, bad, lowest, first, reach, other, odd;
  int bin, ties, kept;
  float logprob;
  int seg[kMostWaves];
};
static_assert(sizeof(Shared16) <= 53760 && kOctaves + 3 * kGroupSlots + kTies <= kSign, "three to a CU");

// A row's entries, eight at least, as 16-byte vectors: vector i * kThreads + thread for i < n, entries
// past the end as -inf.
template <int kThreads>
struct Row16 {
  const uint16_t* x;
  int vocab, n;

  // Index of the vector's first entry: the last vectors overlap, and what they repeat is -inf.
  CURE_DEV int first(int i) const { return min((i * kThreads + (int)threadIdx.x) * 8, vocab - 8); }
  CURE_DEV u32x4 load(int i) const {
    u32x4 w;
    __builtin_memcpy(&w, x + first(i), 16);        // rows need not begin with 16 bytes
    return w;
  }
  CURE_DEV u32x4 masked(u32x4 w, int i) const {
    const int at = (i * kThreads + (int)threadIdx.x) * 8, f = first(i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool is = f + j >= at && f + j < vocab;
      if (!is) w[j / 2] = j % 2 ? (w[j / 2] & 0xffffu) | (kMinusInf2 & 0xffff0000u) : (w[j / 2] & 0xffff0000u) | (kMinusInf2 & 0xffffu);
    }
    return w;
  }
  // f(vector, i) for each, kAhead of whose loads are under way at a time beside the last ones'.
  static constexpr int kAhead = 4;
  template <typename F>
  CURE_DEV void each(const F& f) const {
    struct Ahead {
      u32x4 w[kAhead];
    };
    const auto fetch = [&](Ahead& a, int i) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) a.w[u] = load(min(i * kAhead + u, n - 1));
    };
    const auto take = [&](const Ahead& a, int i) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) f(a.w[u], i * kAhead + u);
    };
    const int whole = (n - 1) / kAhead;            // so many times kAhead that have no end among them
    Ahead even, odd;                               // in turn: a copy would wait for its loads
    fetch(even, 0);
    for (int i = 0; i < whole; i += 2) {
      fetch(odd, i + 1);
      take(even, i);
      if (i + 1 == whole) {
        even = odd;
        break;
      }
      fetch(even, i + 2);
      take(odd, i + 1);
    }
#pragma unroll 1
    for (int i = whole * kAhead; i < n; ++i) {
      f(masked(even.w[0], i), i);
#pragma unroll
      for (int u = 0; u + 1 < kAhead; ++u) even.w[u] = even.w[u + 1];
    }
  }
};

// False, once all threads have left sh: the row has to go the general way.
template <int kThreads>
CURE_DEV bool sample_exact(Shared16& sh, const Args& a, int64_t r, const Settings& s) {
  constexpr int kWaves = kThreads / kWave, kWaveGroups = kGroups16 / kWaves;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  if (a.vocab < 8) return false;
  const Row16<kThreads> row{static_cast<const uint16_t*>(a.logits) + r * a.ld, a.vocab, (a.vocab + 8 * kThreads - 1) / (8 * kThreads)};
  for (int i = tid; i < (kSign + kOctaves) / 4; i += kThreads) reinterpret_cast<u32x4*>(sh.cnt)[i] = u32x4{0, 0, 0, 0};
  if (tid == 0) {
    sh.listed = sh.bad = sh.lowest = sh.reach = sh.other = 0;
    sh.first = kPlaces;
  }
  __syncthreads();
  const auto count = [&](uint32_t bin4) { atomicAdd(reinterpret_cast<int*>(reinterpret_cast<char*>(sh.cnt) + bin4), 1); };
  // What lies in the lowest bin is not counted there: -inf, as masked entries are, would have the lanes
  // of a wave wait for each other.
  int low = 0;                                     // finite ones
  bool bad = false;
  row.each([&](const u32x4& w, int) {
    uint32_t b[4];
    u16x2 high = both(0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b[j] = bins_of(w[j]);
      high = __builtin_elementwise_max(high, __builtin_bit_cast(u16x2, b[j]));
    }
    if (__builtin_expect(__any(high[0] == kLowest4 || high[1] == kLowest4), 0)) {
      // One word after the other, in a loop that is short.
      u32x4 left = w;
#pragma unroll 1
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t v = e ? left[0] >> 16 : left[0] & 0xffffu, bin4 = bins_of(v) & 0xffffu;
          if (bin4 != kLowest4) count(bin4);
          else low += v < 0xff80u;
          bad = bad || v > 0xff80u;
        }
        left = u32x4{left[1], left[2], left[3], left[0]};
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      count(b[j] & 0xffffu);
      count(b[j] >> 16);
    }
  });
  if (__any(low > 0)) {
    low = wave_sum(low);
    if (lane == 0) atomicAdd(&sh.lowest, low);
  }
  if (bad) sh.bad = 1;
  __syncthreads();
  // Other bins that stand for more than one value: +inf and NaNs, and magnitudes that have no bins.
  if (tid == 0) {
    sh.odd = sh.cnt[kHighest] > 0 || sh.cnt[kZero + 1] > 0 || sh.cnt[kMinusZero + 1] > 0;
    sh.cnt[kZero] += sh.cnt[kMinusZero];
    sh.cnt[kMinusZero] = 0;
  }
  __syncthreads();
  if (sh.odd) {
    bool other = false;
    row.each([&](const u32x4& w, int) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t v = w[j / 2] >> (j % 2 * 16) & 0xffffu, mag = v & 0x7fffu;
        bad = bad || mag > 0x7f80u || v == 0x7f80u;
        other = other || (mag > 0 && mag <= kFirst16) || (v < 0x8000u && mag >= kFirst16 + kOctaves - 1);
      }
    });
    if (bad) sh.bad = 1;
    if (other) sh.other = 1;
    __syncthreads();
  }
  // A wave's groups of 64 places, every kWaves-th one: which are used, and the first place that is.
  const auto group_of = [&](int i) { return i * kWaves + wave; };
  uint32_t used = 0;
  int mine = kPlaces;
#pragma unroll
  for (int i = kWaveGroups - 1; i >= 0; --i) {
    const int pos = group_of(i) * kWave + lane, n = sh.cnt[bin_at(pos)];
    if (n > 0) mine = pos;
    used |= __any(n > 0) ? 1u << i : 0u;
  }
  if (lane < kGroupSlots / kWaves) {
    sh.group_n[group_of(lane)] = 0;
    sh.group_w[group_of(lane)] = 0.0;
  }
  mine = -wave_max(-mine);
  if (lane == 0 && mine < kPlaces) atomicMin(&sh.first, mine);
  __syncthreads();
  const bool empty = sh.first == kPlaces;          // but for the lowest bin
  if (sh.bad || (empty && sh.lowest == 0)) {
    if (tid == 0) no_answer(a, r);
    return true;
  }
  const Scale sc = scale_of(value_of_bin(empty ? kLowest : bin_at(sh.first)), s.t);
  if (sh.other || (sh.lowest > 0 && (empty || sc.has(value_of_bin(kLowest))))) {
    __syncthreads();
    return false;
  }
  // What a place of the order holds.
  const auto holds = [&](int pos) {
    const int bin = bin_at(pos), n = sh.cnt[bin];
    const float x = value_of_bin(bin);
    if (n == 0 || !sc.has(x)) return Amount{0, 0.0};
    return Amount{n, n * sc.weight(x)};
  };
  int reach = 0;                                   // entries whose weight is at least min_p
#pragma unroll 1
  for (; used; used &= used - 1) {
    const int g = group_of(__ffs(used) - 1);
    const Amount in = holds(g * kWave + lane);
    if (in.w >= in.n * (double)s.min_p) reach += in.n;
    const Amount sum{wave_sum(in.n), wave_sum(in.w)};
    if (lane == 0) {
      sh.group_n[g] = sum.n;
      sh.group_w[g] = sum.w;
    }
  }
  reach = wave_sum(reach);
  if (lane == 0 && reach) atomicAdd(&sh.reach, reach);
  __syncthreads();
  if (wave == 0) {
    const Order<kGroups16, decltype(holds)> order(sh.group_n, sh.group_w, holds);
    Amount run = s.t == 0.f ? Amount{1, 1.0} : order.all();    // what is kept so far
    Found f{0, {0, 0.0}, {0, 0.0}};
    int ties = 0;
    // top-k, top-p, min-p, the token; and the last entry kept, where rounding or a number of one
    // and more lead past it.
#pragma unroll 1
    for (int q = s.t == 0.f ? 3 : 0; q < 5; ++q) {
      int n = 0;                                   // so many entries, or (0) a weight
      double target = 0.0;
      if (q == 0) {
        if (s.top_k <= 0 || s.top_k >= run.n) continue;
        n = s.top_k;
      } else if (q == 1) {
        if (!(s.top_p < 1.f)) continue;
        target = fmax(0.0, (double)s.top_p) * run.w;
      } else if (q == 2) {
        n = max(1, sh.reach);
        if (!(s.min_p > 0.f) || n >= run.n) continue;
      } else if (q == 3) {
        target = fmax(0.0, (double)s.u) * run.w;
      } else {
        if (f.before.n + ties <= run.n) break;
        n = run.n;
      }
      f = order.find([&](Amount x) { return n ? x.n >= n : q == 1 ? x.w >= target : x.w > target; });
      ties = n ? min(n - f.before.n, f.in.n) : ties_to(target, f.before, f.in, q == 3);
      const Amount upto = f.before + Amount{ties, ties * (f.in.w / f.in.n)};
      if (q < 3 && upto.n < run.n) run = upto;
    }
    if (lane == 0) {
      const int bin = bin_at(f.pos);
      sh.bin = bin;
      sh.ties = ties;
      sh.kept = run.n;
      sh.logprob = (float)(-sc.below(value_of_bin(bin)) * sc.inv_t - log(run.w));
    }
  }
  __syncthreads();
  // The ties-th entry of that value, by index.
  const int bin = sh.bin, n = sh.cnt[bin];
  // Zero where a word's entries have the bin's value.
  const uint32_t mask = bin == kZero ? 0x7fff7fffu : ~0u, bits = (__float_as_uint(value_of_bin(bin)) >> 16) * 0x10001u;
  const auto off = [&](uint32_t w) { return __builtin_bit_cast(u16x2, (w & mask) ^ bits); };
  if (n <= kTies) {
    row.each([&](const u32x4& w, int i) {
      u16x2 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = off(w[j]);
      const u16x2 low = __builtin_elementwise_min(__builtin_elementwise_min(x[0], x[1]), __builtin_elementwise_min(x[2], x[3]));
      if (low[0] && low[1]) return;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (x[j / 2][j % 2] == 0) sh.list[atomicAdd(&sh.listed, 1)] = row.first(i) + j;
    });
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const int me = sh.list[i];
      int before = 0;
      for (int j = 0; j < n; ++j) before += sh.list[j] < me;
      if (before == sh.ties - 1) answer(a, r, me, sh.logprob, sh.kept);
    }
    return true;
  }
  // Many: counted by vectors, waves and lanes, in the entries' order.
  int left = sh.ties;
  for (int i = 0; i < row.n; ++i) {
    const u32x4 w = row.masked(row.load(i), i);
    int mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u16x2 x = off(w[j]);
      mine += (x[0] == 0) + (x[1] == 0);
    }
    const int upto = wave_scan(Amount{mine, 0.0}).n;
    if (lane == kWave - 1) sh.seg[wave] = upto;
    __syncthreads();
    int before = 0, all = 0;
    for (int k = 0; k < kWaves; ++k) {
      before += k < wave ? sh.seg[k] : 0;
      all += sh.seg[k];
    }
    before += upto - mine;
    if (before < left && before + mine >= left) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u16x2 x = off(w[j]);
        if (x[0] == 0 && ++before == left) answer(a, r, row.first(i) + 2 * j, sh.logprob, sh.kept);
        if (x[1] == 0 && ++before == left) answer(a, r, row.first(i) + 2 * j + 1, sh.logprob, sh.kept);
      }
    }
    left -= all;
    __syncthreads();
    if (left <= 0) break;
  }
  return true;
}

constexpr int kThreads16 = 512;

__global__ __launch_bounds__(kThreads16, 6) void sample_bf16(Args a) {
  __shared__ union {
    Shared16 own;
    Shared any;
  } space;
  const int64_t r = blockIdx.x;
  const Settings s = settings_of(a, r);
  if (s.none) {
    if (threadIdx.x == 0) no_answer(a, r);
  } else if (!sample_exact<kThreads16>(space.own, a, r, s)) {
    sample_any<uint16_t, kThreads16>(space.any, a, r, s);
  }
}

}  // namespace
}  // namespace cure

using namespace cure;

extern "C" cure_status cure_sample(const void* logits, int32_t dtype, int32_t batch, int32_t rows,
                                   int32_t vocab, int64_t ld, const float* temperature,
                                   const int32_t* top_k, const float* top_p, const float* min_p,
                                   const float* uniform, const int32_t* n_rows, int32_t* token,
                                   float* logprob, int32_t* kept, void* stream) {
  if (dtype != CURE_F32 && dtype != CURE_BF16) return CURE_ERR_INVALID_ARG;
  if (batch < 0 || rows < 0 || vocab < 1 || ld < vocab) return CURE_ERR_INVALID_ARG;
  if (vocab > kMaxVocab) return CURE_ERR_UNSUPPORTED;
  const int64_t total = (int64_t)batch * rows;
  if (total >= (int64_t(1) << 31) / 1024) return CURE_ERR_UNSUPPORTED;
  if (total == 0) return CURE_OK;
  if (!logits || !uniform || !token) return CURE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == CURE_BF16 ? 2 : 4)) return CURE_ERR_INVALID_ARG;
  const Args a{logits, rows, vocab, ld, temperature, top_k, top_p, min_p, uniform, n_rows, token, logprob, kept};
  const auto run = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(threads), 0, as_stream(stream), a);
  };
  if (dtype == CURE_F32) run(sample_f32, kThreads32);
  else run(sample_bf16, kThreads16);
  return launch_status();
}
