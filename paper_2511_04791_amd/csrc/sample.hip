// Sampling from a row of V logits x (temperature T, top-k, top-p, min-p, a given uniform number u).
//
// Tokens are ranked by falling logit, ties by the lower index, and weigh w = exp((max - x) / -T).  Each filter
// keeps a run of ranks from the first: top-k the first k; top-p, of those, rank r where the mass before it is
// less than p times theirs; min-p those with w >= min-p (the largest has w = 1).  The token is the first rank
// whose kept cumulative mass exceeds u times the kept mass S.
//
// So every step looks for a place in the ranking, and a row need not be sorted: a histogram over
// d = (max - x) / T gives the mass before each of its bins, and only the tokens of the few bins that can hold
// the places looked for are listed, sorted and summed.  Tokens with d >= kSpan (e^-48 each, 3.8e-16 of the largest's over a row of
// 2^18) are left out: less than two units in the last place of S in 64 bits, where S is 1, and less beside larger sums.
//
// Sums do not depend on the order of atomics: a token adds an integer to its bin, 2^45 + (1 - v) 2^33, with
// v = e^-(d - d_bin) in (1 - 2^-6.4, 1] its weight relative to the bin's first.  The count stands in bits 45 on,
// the sum of up to 2^18 terms under 2^(26.6 + 18) below.  Each term rounds by 2^-34 of the token's weight.
//
// A row is read twice (its maximum, the histogram), a third time where the places lie past the largest few hundred tokens,
// which the second pass lists as it goes; by one workgroup, or in slices by several where there are few rows.
//
// us of the steps for 256 float32 rows of 128256 logits, a CU each, 68 a call: maximum 17 (131 MB, 7.7 TB/s), histogram 19,
// its sums 5, third pass 15, sorting 2, the answer 3; the rest is the launch and the rows that take longest.  One row on one CU:
// 5, 18, 5, 9 to 13, 2, 3: the histogram is bound by its LDS additions (12 us without any arithmetic) and the arithmetic in 64 bits
// (16 without additions), the rest by latency.  256 bf16 rows 60 a call.  Rows that narrow takes are far slower: 256 rows of
// deviation 0.5 at T = 2 383, 256 bf16 rows of deviation 0.8 around 10 (thousands of tokens of one value) 358, 64 such 362 and 333.
//
// 1024 threads leave a thread 128 registers, which is not enough for sample_row and sample_count, where every step and a call of
// narrow meet: sample_count spills 24 (float32) and 21 (bf16) with 144 and 128 bytes of scratch a lane, sample_row 2 and none, 48 bytes.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "serving_ops.h"
#include "wave_ops.h"

namespace duet {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 4096, kSubBins = 2048, kBinsPerThread = kBins / kThreads;
constexpr double kSpan = 48.0, kBinsPerUnit = kBins / kSpan, kBinWidth = kSpan / kBins;
constexpr int kCountShift = 45;
constexpr double kFraction = 8589934592.0;  // 2^33
constexpr int kList = 2048;                 // tokens listed and sorted; more are narrowed down by their bits
constexpr int kListPerThread = kList / kThreads;

__device__ __forceinline__ float as_float(const __bf16& x) { return static_cast<float>(x); }
__device__ __forceinline__ float as_float(const float& x) { return x; }

// Larger logits have larger keys; both zeros the same one, NaN and -inf (masked tokens) key 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x > -INFINITY ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// A place in the ranking: n tokens and their mass before it.
struct Place {
  uint32_t n;
  double mass;
};

// A run of listed tokens of one bin, summed; `first`: it begins with the bin's first.
struct Run {
  uint32_t first, n;
  u64 fraction;
};

struct Shared {
  union {
    u64 hist[kBins];
    double mass[kBins + 1];  // mass before each bin, once the histogram is summed
  };
  uint32_t before[kBins + 1];  // tokens before each bin
  u64 list[kList];             // (~key, index): in rank order when sorted
  uint32_t guesses[kList + 1];
  union {
    Run runs[kWaves];
    struct {
      double wave_mass[kWaves];
      uint32_t wave_count[kWaves];
    };
  };
  Place place;
  int found[5];
  double value;
  float wave_max[kWaves], wave_low[kWaves];
  uint32_t key, listed, wanted;
  int at, pos, last_pos;
};

struct Row {
  double max, scale;  // of a gap to bins
  // (max - x) / T in bins; not below kBins for masked tokens, NaN among them.
  __device__ __forceinline__ double bins(float x) const { return (max - x) * scale; }
  __device__ __forceinline__ double bins_of_key(uint32_t k) const { return bins(of_key(k)); }
};
__device__ __forceinline__ double weight_of(double bins) { return exp(-bins * kBinWidth); }
// (1 - v) 2^33 to the nearest: the series of 1 - e^-y, y = x kBinWidth, x in [0, 1), up to y^3, and y^4 by the cubic nearest
// to it there; within 2^-37.
__device__ __forceinline__ uint32_t fraction_of(double bins) {
  constexpr double w = kBinWidth, f = kFraction, q = f * w * w * w * w / 24;
  const double x = __builtin_amdgcn_fract(bins);
  return (uint32_t)fma(x, fma(x, fma(x, f * w * w * w / 6 - 2 * q, -f * w * w / 2 + 1.25 * q), f * w - 0.25 * q), 0.5 + q / 128);
}
__device__ __forceinline__ u64 token_bits(double bins) { return (1ull << kCountShift) + fraction_of(bins); }
__device__ __forceinline__ uint32_t count_of(u64 h) { return (uint32_t)(h >> kCountShift); }
__device__ __forceinline__ double scale_of(int bin) { return weight_of(bin); }
__device__ __forceinline__ double mass_of(uint32_t n, u64 fraction, double scale) {
  return (n - (double)fraction / kFraction) * scale;
}
__device__ __forceinline__ double mass_of(u64 h, double scale) {
  return mass_of(count_of(h), h & ((1ull << kCountShift) - 1), scale);
}

// A row's logits.  If its largest is infinite, the infinities count as 0 and the rest as masked.
template <typename T>
struct Logits {
  const T* x;
  int n;
  bool infinite;

  __device__ __forceinline__ float plain(float v) const { return infinite ? (v == INFINITY ? 0.f : -INFINITY) : v; }
  __device__ __forceinline__ float at(int i) const { return plain(as_float(x[i])); }

  // f(four logits, index of the first): a wave takes 64 vectors of four past the first boundary at a time, U such in flight;
  // the up to 258 tokens before and after those come one a lane, with three masked ones.  Whole waves call f.
  template <int U, typename F>
  __device__ __forceinline__ void fours(F f) const {
    typedef T Four __attribute__((ext_vector_type(4)));
    const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
    const int off = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) & 3);
    const int head = min(n, (4 - off) & 3), units = (n - head) / 256, rest = n - 256 * units;
    const Four* p = reinterpret_cast<const Four*>(x + head);
    if (wave < units) {
      // Each vector's registers are loaded again as soon as it is used.
      Four v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = p[64 * min(wave + u * kWaves, units - 1) + lane];
      for (int i = wave; i < units; i += U * kWaves) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = i + u * kWaves;
          if (k < units) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = as_float(v[u][e]);
            if (infinite)
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = plain(y[e]);
            f(y, head + 4 * (64 * k + lane));
          }
          v[u] = p[64 * min(k + U * kWaves, units - 1) + lane];
        }
      }
    }
    if (64 * wave < rest) {
      const int k = tid < head ? tid : 256 * units + tid;
      const float y[4] = {tid < rest ? at(k) : -INFINITY, -INFINITY, -INFINITY, -INFINITY};
      f(y, k);
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    fours<2>([&](const float* v, int i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(v[e], i + e);
    });
  }
};

// A value of the lane one (two, four, eight) before in its row of 16, of the last lane of the row before, of the last of the
// first two rows, for an inclusive scan over the wave; zero where there is none.  Vector instructions: no LDS round trip.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t before_in_wave(uint32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 before_in_wave(u64 x) {
  return (u64)before_in_wave<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | before_in_wave<CTRL, ROWS>((uint32_t)x);
}
template <typename F>
__device__ __forceinline__ void scan_steps(F step) {
  step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
}
__device__ __forceinline__ void scan_place(uint32_t* n, double* m) {
  scan_steps([&](auto ctrl, auto rows) {
    constexpr int c = decltype(ctrl)::value, r = decltype(rows)::value;
    *n += before_in_wave<c, r>(*n);
    *m += __longlong_as_double(before_in_wave<c, r>((u64)__double_as_longlong(*m)));
  });
}

// ---- narrowing by bits: any number of tokens in a bin ------------------------------------------------

// The first of the n bins (rank order) with reached(place after it); its place before it.  The last bin holding
// a token where none reaches.  fixed_bin >= 0: all are parts of that bin of the first histogram.
template <typename F>
__device__ int find_bin(Shared& s, int n, int fixed_bin, Place at, F reached, Place* before) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, per = n / kThreads;
  uint32_t c = 0;
  double m = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    c += count_of(s.hist[b]);
    m += mass_of(s.hist[b], scale_of(fixed_bin >= 0 ? fixed_bin : b));
  }
  uint32_t ci = c;
  double mi = m;
  scan_place(&ci, &mi);
  if (lane == 63) s.wave_count[wave] = ci, s.wave_mass[wave] = mi;
  if (tid == 0) s.at = 1 << 30;
  __syncthreads();
  Place p = at;
  for (int w = 0; w < wave; ++w) p.n += s.wave_count[w], p.mass += s.wave_mass[w];
  p.n += ci - c;
  p.mass += mi - m;
  Place mine = p, last_place = p;
  int first = -1, last = -1;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    const u64 h = s.hist[b];
    if (!h) continue;
    last = b, last_place = p;
    p.n += count_of(h);
    p.mass += mass_of(h, scale_of(fixed_bin >= 0 ? fixed_bin : b));
    if (first < 0 && reached(p)) first = b, mine = last_place;
  }
  if (first >= 0) atomicMin(&s.at, first);
  __syncthreads();
  if (s.at == 1 << 30) {
    __syncthreads();
    if (tid == 0) s.at = -1;
    __syncthreads();
    if (last >= 0) atomicMax(&s.at, last);
    __syncthreads();
    first = last, mine = last_place;
  }
  const int found = s.at;
  if (first == found) s.place = mine;
  __syncthreads();
  *before = s.place;
  __syncthreads();
  return found;
}

// The key that holds the place, how many of the tokens with that key come before or at it, and the place after those.
struct Found {
  uint32_t key, ties;
  Place end;
};

// reached(place): whether the place is at or past the one looked for.
template <typename T, typename F>
__device__ Found find(Shared& s, const Logits<T>& x, const Row& row, F reached) {
  const int tid = threadIdx.x;
  auto inside = [&](auto f) {
    x.each([&](float v, int) {
      const double d = row.bins(v);
      if (d < kBins) f(key_of(v), d);
    });
  };
  auto clear = [&](int n) {
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) s.hist[i] = 0;
    __syncthreads();
  };
  clear(kBins);
  inside([&](uint32_t, double d) { atomicAdd(&s.hist[(int)d], token_bits(d)); });
  __syncthreads();
  Place before{0, 0.0};
  const int bin = find_bin(s, kBins, -1, before, reached, &before);
  // The bin's largest and smallest key.
  if (tid == 0) s.key = 0, s.wanted = 0xffffffffu;
  __syncthreads();
  inside([&](uint32_t k, double d) {
    if ((int)d == bin) atomicMax(&s.key, k), atomicMin(&s.wanted, k);
  });
  __syncthreads();
  uint32_t hi = s.key, lo = s.wanted;
  while (true) {
    int shift = 0;
    while (((hi - lo) >> shift) >= kSubBins) ++shift;
    clear(kSubBins);
    inside([&](uint32_t k, double d) {
      if (k <= hi && k >= lo) atomicAdd(&s.hist[(hi - k) >> shift], token_bits(d));
    });
    __syncthreads();
    const int sub = find_bin(s, kSubBins, bin, before, reached, &before);
    const uint32_t n = count_of(s.hist[sub]);
    hi -= (uint32_t)sub << shift;
    lo = hi - min(hi - lo, (1u << shift) - 1);
    if (shift == 0) {
      const double w = weight_of(row.bins_of_key(hi));
      // ties before or at the place: the fewest with which it is reached
      uint32_t a = 1, b = n;
      while (a < b) {
        const uint32_t c = (a + b) / 2;
        if (reached(Place{before.n + c, before.mass + c * w})) b = c;
        else a = c + 1;
      }
      return Found{hi, a, Place{before.n + a, before.mass + a * w}};
    }
  }
}

// Index of the n-th token (from 1) with this key.
template <typename T>
__device__ int index_of(Shared& s, const Logits<T>& x, uint32_t key, uint32_t n) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int per = ((x.n + kWaves - 1) / kWaves + 63) / 64 * 64;  // a wave's tokens
  const int lo = wave * per, hi = min(x.n, lo + per);
  auto is = [&](int i) { return i + lane < hi && key_of(x.at(min(i + lane, x.n - 1))) == key; };
  uint32_t c = 0;
  for (int i = lo; i < hi; i += 64) c += __popcll(__ballot(is(i)));
  __syncthreads();
  if (lane == 0) s.wave_count[wave] = c;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s.wave_count[w];
  if (before < n && n <= before + c) {
    for (int i = lo; i < hi; i += 64) {
      const bool one = is(i);
      const u64 all = __ballot(one);
      if (one && before + __popcll(all & ((1ull << lane) - 1)) + 1 == n) s.at = i + lane;
      before += __popcll(all);
    }
  }
  __syncthreads();
  return s.at;
}

struct Settings {
  uint32_t top_k;  // 0: off
  double top_p;    // 1: off
  double min_p;    // 0: off, at most 1
  double u;
};
struct Pick {
  int index;
  float prob;
};

template <typename T>
__device__ __attribute__((noinline)) Pick narrow(Shared& s, Logits<T> x, Row row, Settings c) {
  const uint32_t k = c.top_k ? c.top_k : 0xffffffffu;
  Place kept = find(s, x, row, [&](const Place& p) { return p.n >= k; }).end;
  if (c.top_p < 1) {
    const double need = c.top_p * kept.mass;
    const uint32_t n = kept.n;
    kept = find(s, x, row, [&](const Place& p) { return p.n >= n || p.mass >= need; }).end;
  }
  if (c.min_p > 0) {
    __syncthreads();
    if (threadIdx.x == 0) s.wanted = 0;
    __syncthreads();
    uint32_t own = 0;
    x.each([&](float v, int) { own += weight_of(row.bins(v)) >= c.min_p; });
    atomicAdd(&s.wanted, own);
    __syncthreads();
    const uint32_t n = s.wanted;
    __syncthreads();
    if (n < kept.n) kept = find(s, x, row, [&](const Place& p) { return p.n >= n; }).end;
  }
  const double target = c.u * kept.mass;
  const uint32_t n = kept.n;
  const Found f = find(s, x, row, [&](const Place& p) { return p.n >= n || p.mass > target; });
  const int i = index_of(s, x, f.key, f.ties);
  return Pick{i, (float)(weight_of(row.bins_of_key(f.key)) / kept.mass)};
}

// ---- the histogram and a short list -------------------------------------------------------------------

// s.list[0 .. n) into rising order; n <= kList, no two alike.  Each wave sorts runs of 64 in registers; runs are then joined
// two by two, a token's place being its place in its own and, by bisection, in the other.
__device__ void sort_list(Shared& s, int n) {
  const int tid = threadIdx.x, lane = tid & 63;
  for (int r = tid >> 6; 64 * r < n; r += kWaves) {
    u64 v = 64 * r + lane < n ? s.list[64 * r + lane] : ~0ull;
    for (int k = 2; k <= 64; k <<= 1)
      for (int step = k >> 1; step > 0; step >>= 1) {
        const u64 other = __shfl_xor(v, step);
        if ((v > other) == (((lane & k) == 0) == ((lane & step) == 0))) v = other;
      }
    if (64 * r + lane < n) s.list[64 * r + lane] = v;
  }
  __syncthreads();
  for (int len = 64; len < n; len *= 2) {
    u64 v[kListPerThread];
    int to[kListPerThread];
#pragma unroll
    for (int j = 0; j < kListPerThread; ++j) {
      const int i = tid + j * kThreads;
      if (i >= n) continue;
      v[j] = s.list[i];
      const int other = (i / len ^ 1) * len;
      int at = 0;
      for (int step = len; step > 0; step >>= 1)
        if (at + step <= len && other + at + step <= n && s.list[other + at + step - 1] < v[j]) at += step;
      to[j] = (i & ~(2 * len - 1)) + (i & (len - 1)) + at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kListPerThread; ++j)
      if (tid + j * kThreads < n) s.list[to[j]] = v[j];
    __syncthreads();
  }
}

__device__ __forceinline__ u64 entry(float v, int i) { return (u64)(~key_of(v)) << 32 | (uint32_t)i; }

// Lanes of the mask before this one.
__device__ __forceinline__ uint32_t lanes_before(u64 mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Of a wave's N tokens a lane, token(e), those that are in[e], to the list's end.
template <int N, typename F>
__device__ __forceinline__ void put(Shared& s, const bool* in, F token) {
  u64 all[N];
  uint32_t n = 0, at = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) all[e] = __ballot(in[e]), n += __popcll(all[e]);
  if (!n) return;
  if ((threadIdx.x & 63) == 0) at = atomicAdd(&s.listed, n);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (!all[e]) continue;
    const uint32_t to = at + lanes_before(all[e]);
    if (in[e] && to < kList) s.list[to] = token(e);
    at += __popcll(all[e]);
  }
}

// The bins that a row's places may lie in: those of top-k's end, top-p's, min-p's and the token's.
struct Wanted {
  int lo[4], hi[4];  // empty where hi < lo
  int last;
  Place all;  // the whole row
  __device__ __forceinline__ bool has(int b) const {
    bool in = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) in |= b >= lo[i] && b <= hi[i];
    return in;
  }
};

// Sums the histogram: its place before every bin stays in s.mass and s.before, that of the whole row past the last.
__device__ Wanted decide(Shared& s, const Settings& c) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  uint32_t n[kBinsPerThread], cn = 0;
  double m[kBinsPerThread], cm = 0;
  double scale = scale_of(tid * kBinsPerThread);
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) {
    const u64 h = s.hist[tid * kBinsPerThread + i];
    n[i] = count_of(h);
    m[i] = mass_of(h, scale);
    scale *= 0.9883496471138451;  // e^-kBinWidth
    cn += n[i];
    cm += m[i];
  }
  uint32_t in = cn;
  double im = cm;
  scan_place(&in, &im);
  if (lane == 63) s.wave_count[wave] = in, s.wave_mass[wave] = im;
  if (tid < 5) s.found[tid] = kBins;
  if (tid == 0) s.at = -1, s.wanted = 0;
  __syncthreads();
  Place low{0, 0.0}, all{0, 0.0};
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) low = all;
    all.n += s.wave_count[w];
    all.mass += s.wave_mass[w];
  }
  low.n += in - cn;
  low.mass += im - cm;
  Place high[kBinsPerThread];
  int last = -1;
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) {
    const int b = tid * kBinsPerThread + i;
    s.mass[b] = low.mass;
    s.before[b] = low.n;
    low = high[i] = Place{low.n + n[i], low.mass + m[i]};
    if (n[i]) last = b;
  }
  if (tid == 0) s.mass[kBins] = all.mass, s.before[kBins] = all.n;
  if (last >= 0 && !(__ballot(last >= 0) >> lane >> 1)) atomicMax(&s.at, last);
  // The first bin holding a token with reached(place after it) goes to slot q; the last bin if there is none.
  auto look = [&](int q, auto reached) {
    int b = kBins;
#pragma unroll
    for (int i = kBinsPerThread - 1; i >= 0; --i)
      if (n[i] && reached(high[i])) b = tid * kBinsPerThread + i;
    const u64 some = __ballot(b < kBins);  // bins rise with the lanes: the first lane has the wave's least
    if (b < kBins && !(some & ((1ull << lane) - 1))) atomicMin(&s.found[q], b);
  };
  const bool k = c.top_k && c.top_k < all.n;
  if (k) look(0, [&](const Place& q) { return q.n >= c.top_k; });
  __syncthreads();
  last = s.at;
  Wanted w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w.lo[i] = 0, w.hi[i] = -1;
  w.all = all;
  const int kb = k ? min(s.found[0], last) : last;
  int plo = last, phi = last, mb = last;
  if (c.top_p < 1) {
    const double least = c.top_p * (k ? s.mass[kb] : all.mass), most = c.top_p * (k ? s.mass[kb + 1] : all.mass);
    look(1, [&](const Place& q) { return q.mass >= least; });
    look(2, [&](const Place& q) { return q.mass >= most; });
    __syncthreads();
    plo = min(kb, s.found[1]), phi = min(kb, s.found[2]);
  }
  // The bin that weights of min-p lie in.  No float's logarithm is nearer to a bin's edge than 1.7e-10 bins, and the roundings of a
  // token's and of this are under 1e-11: tokens of earlier bins weigh more than min-p and those of later ones less.
  if (c.min_p > 0) mb = min((int)(-log(c.min_p) * kBinsPerUnit), kBins - 1);
  const int elo = min(min(kb, plo), mb), ehi = min(min(kb, phi), mb);
  const double tlo = c.u * s.mass[elo], thi = c.u * s.mass[ehi + 1];
  look(3, [&](const Place& q) { return q.mass > tlo; });
  look(4, [&](const Place& q) { return q.mass > thi; });
  __syncthreads();
  w.lo[3] = min(ehi, min(last, s.found[3]));
  w.hi[3] = min(ehi, min(last, s.found[4]));
  if (k && (c.top_p < 1 || kb <= ehi)) w.lo[0] = w.hi[0] = kb;
  if (c.top_p < 1 && plo <= ehi) w.lo[1] = plo, w.hi[1] = min(phi, ehi);
  if (c.min_p > 0 && mb <= ehi) w.lo[2] = w.hi[2] = mb;
  w.last = max(max(w.hi[0], w.hi[1]), max(w.hi[2], w.hi[3]));
  uint32_t wanted = 0;
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i)
    if (w.has(tid * kBinsPerThread + i)) wanted += n[i];
  if (wanted) atomicAdd(&s.wanted, wanted);
  __syncthreads();
  return w;
}

// The token from the sorted list of n tokens, which holds all of the wanted bins; before_bin(b): the place before a bin.
template <typename F>
__device__ Pick finish(Shared& s, int n, const Row& row, const Settings& c, const Wanted& w, F before_bin) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  constexpr int P = kListPerThread;
  double d[P], scale[P];  // d: in bins
  int bin[P];
  uint32_t fraction[P];
  Run run[P];
  const bool busy = wave * 64 * P < n;  // waves past the list only meet the barriers
  auto bins_at = [&](int i) { return row.bins_of_key(~(uint32_t)(s.list[i] >> 32)); };
  auto join = [](const Run& a, const Run& b) { return b.first ? b : Run{a.first, a.n + b.n, a.fraction + b.fraction}; };
  Run sum{0, 0, 0}, left{0, 0, 0};
  if (busy) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int i = tid * P + j;
      const int k = min(i, n - 1);
      d[j] = bins_at(k);
      bin[j] = (int)d[j];
      fraction[j] = fraction_of(d[j]);
      const Run one{i == 0 || i >= n || (int)bins_at(k - 1) != bin[j], 1, fraction[j]};
      sum = j ? join(sum, one) : one;
      run[j] = sum;
      scale[j] = scale_of(bin[j]);
    }
    scan_steps([&](auto ctrl, auto rows) {
      constexpr int c = decltype(ctrl)::value, r = decltype(rows)::value;
      sum = join(Run{before_in_wave<c, r>(sum.first), before_in_wave<c, r>(sum.n), before_in_wave<c, r>(sum.fraction)}, sum);
    });
    if (lane == 63) s.runs[wave] = sum;
    left = Run{before_in_wave<0x138, 0xf>(sum.first), before_in_wave<0x138, 0xf>(sum.n), before_in_wave<0x138, 0xf>(sum.fraction)};
  }
  if (tid == 0) s.pos = 1 << 30, s.last_pos = -1, s.at = -1, s.value = w.all.mass;
  __syncthreads();
  Place high[P];
  if (busy) {
    Run before{0, 0, 0};
    for (int v = 0; v < wave; ++v) before = join(before, s.runs[v]);
    left = lane ? join(before, left) : before;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const Run r = join(left, run[j]);
      const Place b = before_bin(bin[j]);
      high[j] = Place{b.n + r.n, b.mass + mass_of(r.n, r.fraction, scale[j])};
    }
  }
  auto listed = [&](int j) { return tid * P + j < n && bin[j] <= w.last; };
  const bool k = c.top_k && c.top_k < w.all.n;
  if (k)
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (listed(j) && high[j].n == c.top_k) s.value = high[j].mass;
  int last = -1;
#pragma unroll
  for (int j = 0; j < P; ++j)
    if (listed(j)) last = tid * P + j;
  if (last >= 0 && !(__ballot(last >= 0) >> lane >> 1)) atomicMax(&s.last_pos, last);
  __syncthreads();
  Place kept{k ? c.top_k : w.all.n, s.value};
  auto leave = [&](int at) {  // an index known when compiled keeps the array in registers
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (at == tid * P + j) s.place = high[j];
  };
  // The first listed rank at or past a place, the last one where none is.
  auto first = [&](auto reached) {
    int i = 1 << 30;
#pragma unroll
    for (int j = P - 1; j >= 0; --j)
      if (listed(j) && reached(high[j])) i = tid * P + j;
    const u64 some = __ballot(i < 1 << 30);
    if (i < 1 << 30 && !(some & ((1ull << lane) - 1))) atomicMin(&s.pos, i);
    __syncthreads();
    const int at = s.pos == 1 << 30 ? s.last_pos : s.pos;
    leave(at);
    __syncthreads();
    if (tid == 0) s.pos = 1 << 30;
    return at;
  };
  if (c.top_p < 1 && w.lo[1] <= w.hi[1]) {
    const double need = c.top_p * kept.mass;
    first([&](const Place& p) { return p.mass >= need; });
    if (s.place.n < kept.n) kept = s.place;
    __syncthreads();
  }
  if (c.min_p > 0 && w.lo[2] <= w.hi[2]) {
    int own = -1;
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (listed(j) && bin[j] == w.lo[2] && weight_of(d[j]) >= c.min_p) own = tid * P + j;
    if (own >= 0) atomicMax(&s.at, own);
    __syncthreads();
    leave(s.at);
    if (s.at < 0 && tid == 0) s.place = before_bin(w.lo[2]);
    __syncthreads();
    if (s.place.n < kept.n) kept = s.place;
    __syncthreads();
  }
  const double target = c.u * kept.mass;
  const int at = first([&](const Place& p) { return p.mass > target; });
#pragma unroll
  for (int j = 0; j < P; ++j)
    if (at == tid * P + j) s.value = weight_of(d[j]);
  __syncthreads();
  return Pick{(int)(uint32_t)s.list[at], (float)(s.value / kept.mass)};
}

// ---- one row: the pieces that one workgroup, or several, run --------------------------------------------

// What a row's request asks for; the first rank alone needs no more than the maximum.
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, int r, double* inv_t, bool* greedy) {
  const float t = a.temperature ? a.temperature[r] : 1.f;
  const int top_k = a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
  *inv_t = 1.0 / t;
  *greedy = !(t > 0.f) || top_k == 1 || top_p <= 0.f;
  return Settings{(uint32_t)max(top_k, 0), top_p < 1.f ? top_p : 1.0, min_p > 0.f ? fmin(1.0, (double)min_p) : 0.0,
                  u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.0};
}

// A slice's largest logit (and, for the first rank alone, its lowest index), and the smallest of the maxima of groups of 32
// threads, or of `waves` waves (a power of two): some 130 tokens of a row lie above the smallest of 32 such, 32 at least if
// the groups have a token each.
struct Part {
  float max, low;
  int index, pad;
};
template <typename T>
__device__ Part largest(Shared& s, const Logits<T>& x, int waves, bool greedy) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  float most = -INFINITY;
  int index = 0;
  if (greedy) {
    x.each([&](float v, int i) {
      if (v > most || (v == most && i < index)) most = v, index = i;
    });
  } else {
    x.template fours<8>([&](const float* v, int) { most = fmaxf(most, fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]))); });
  }
  float low = most, high = most;
  for (int off = 1; off < 64; off <<= 1) {
    high = fmaxf(high, __shfl_xor(high, off));
    const float other = __shfl_xor(low, off);
    low = off < 32 || waves ? fmaxf(low, other) : fminf(low, other);
  }
  if (lane == 0) s.wave_max[wave] = high, s.wave_low[wave] = low;
  if (tid == 0) s.at = 0x7fffffff;
  __syncthreads();
  // Each lane a wave's: their maximum, and the least of the groups' (the lanes past the sixteenth repeat them).
  high = s.wave_max[lane & (kWaves - 1)], low = s.wave_low[lane & (kWaves - 1)];
#pragma unroll
  for (int off = 1; off < kWaves; off <<= 1) {
    high = fmaxf(high, __shfl_xor(high, off));
    const float other = __shfl_xor(low, off);
    low = off < waves ? fmaxf(low, other) : fminf(low, other);
  }
  if (greedy) {
    if (most == high && high > -INFINITY) atomicMin(&s.at, index);
    __syncthreads();
    index = s.at;
  }
  return Part{high, low, index, 0};
}

__device__ __forceinline__ void answer(const SampleArgs& a, int r, int index, float prob) {
  if (threadIdx.x) return;
  a.ids[r] = index;
  if (a.probs) a.probs[r] = prob;
}

// The slice's tokens into s.hist; those not below `low` into the wave's part of s.list, as far as there is room.  Returns how
// many those are.
constexpr int kWaveList = kList / kWaves;
template <typename T>
__device__ int count(Shared& s, const Logits<T>& x, int first, const Row& row, float low) {
  u64* list = s.list + (threadIdx.x >> 6) * kWaveList;
  int n = 0;
  x.template fours<4>([&](const float* v, int i) {
    double d[4];
    u64 bits[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = row.bins(v[e]), bits[e] = token_bits(d[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d[e] < kBins) atomicAdd(&s.hist[(int)d[e]], bits[e]);
    if (__ballot(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) >= low))
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = v[e] >= low && d[e] < kBins;
        const u64 all = __ballot(in);
        if (!all) continue;
        const int at = n + lanes_before(all);
        if (in && at < kWaveList) list[at] = entry(v[e], first + i + e);
        n += __popcll(all);
      }
  });
  return n;
}

// The wanted bins as `n` runs apart from each other, in rank order.  The bins fall with the logits, so a run is one of logits,
// from .. to; its tokens take the places start .. start + tokens - 1 among all of the runs' and its bins begin at `bin`, with
// `slope` tokens each.
struct Edges {
  float from[4], to[4], slope[4];
  int bin[4];
  uint32_t start[5];
  int n, pad[2];
};
// Lane 2 q (and 2 q + 1) of each wave finds by bisection the smallest key of run q (past it), that is with bins below hi + 1 (lo).
__device__ Edges edges_of(const Shared& s, const Row& row, const Wanted& w) {
  const int lane = threadIdx.x & 63;
  int lo[4], hi[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) lo[q] = w.hi[q] < w.lo[q] ? kBins : w.lo[q], hi[q] = w.hi[q] < w.lo[q] ? kBins - 1 : w.hi[q];
  auto order = [&](int i, int j) {
    if (lo[j] < lo[i]) {
      const int l = lo[i], h = hi[i];
      lo[i] = lo[j], hi[i] = hi[j], lo[j] = l, hi[j] = h;
    }
  };
  order(0, 1), order(2, 3), order(0, 2), order(1, 3), order(1, 2);
  // Runs that meet become one, in the last of them; empty ones stand behind all others.
#pragma unroll
  for (int q = 1; q < 4; ++q)
    if (lo[q] < kBins && lo[q] <= hi[q - 1] + 1) {
      lo[q] = lo[q - 1], hi[q] = max(hi[q], hi[q - 1]);
      lo[q - 1] = kBins, hi[q - 1] = kBins - 1;
    }
  uint32_t below = 0, at = 0xff800000u;  // the keys of masked tokens, and past every finite logit's
  int edge = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (lane == 2 * q) edge = lo[q] == kBins ? -1 : hi[q] + 1;
    if (lane == 2 * q + 1) edge = lo[q] == kBins ? -1 : lo[q];
  }
  // The key of the edge's place on the scale, if rounding left it near enough; else all of them.
  const uint32_t near = key_of((float)(row.max - edge / row.scale));
  if (near > 0x00800010u && near < 0xff7ffff0u && row.bins_of_key(near + 2) < edge && !(row.bins_of_key(near - 2) < edge))
    below = near - 2, at = near + 2;
  while (at - below > 1) {
    const uint32_t mid = below + (at - below) / 2;
    if (row.bins_of_key(mid) < edge) at = mid;
    else below = mid;
  }
  Edges e;
  e.n = e.pad[0] = e.pad[1] = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) e.from[q] = e.to[q] = INFINITY, e.slope[q] = 0, e.bin[q] = 0;  // holds no finite logit
  uint32_t start = 0;
#pragma unroll
  for (int q = 0; q < 5; ++q) e.start[q] = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t from = __shfl(at, 2 * q), to = __shfl(at, 2 * q + 1) - 1;
    if (lo[q] == kBins || to < from) continue;  // min-p's bin may have room for no logit
    const uint32_t tokens = s.before[hi[q] + 1] - s.before[lo[q]];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i == e.n) {
        e.from[i] = of_key(from), e.to[i] = of_key(to), e.bin[i] = lo[q], e.start[i] = start;
        e.slope[i] = (float)tokens / (hi[q] + 1 - lo[q]);
      }
    start += tokens;
    ++e.n;
#pragma unroll
    for (int i = 1; i < 5; ++i)
      if (i >= e.n) e.start[i] = start;
  }
  return e;
}

// The list of the runs' n tokens into rising order: a token's place is guessed, as if its run's were spread evenly over its
// bins (and, where T is bf16, those of one logit, by their index, over the gap to the next), and the few tokens with one guess
// are put in order by comparing them all; by sort_list where more than kAlike have one.  us of 25 / 480 / 900 tokens:
// 1.8 / 2.1 / 2.4, by sort_list 1.2 / 4.1 / 6.5.
constexpr uint32_t kAlike = 64;
template <typename T>
__device__ void sort_runs(Shared& s, int n, const Row& row, const Edges& edges, int vocab) {
  constexpr int P = kListPerThread;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  u64 v[P];
  uint32_t guess[P], slot[P];
#pragma unroll
  for (int j = 0; j < P; ++j) s.guesses[tid + j * kThreads] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (tid + j * kThreads >= n) continue;
    v[j] = s.list[tid + j * kThreads];
    const uint32_t key = ~(uint32_t)(v[j] >> 32);
    const double d = row.bins_of_key(key);
    float slope = edges.slope[0];
    int bin = edges.bin[0];
    uint32_t start = edges.start[0], end = edges.start[1];
#pragma unroll
    for (int q = 1; q < 4; ++q)
      if (q < edges.n && d >= edges.bin[q])
        slope = edges.slope[q], bin = edges.bin[q], start = edges.start[q], end = edges.start[q + 1];
    float x = (float)(d - bin) * slope;
    if (std::is_same<T, __bf16>::value) {
      const float next = fminf((float)(row.bins_of_key(key - 0x10000u) - bin) * slope, (float)(end - start));
      x = fminf(fmaf(next - x, (float)(int)(uint32_t)v[j] / (float)vocab, x), next);
    }
    guess[j] = min(start + (uint32_t)x, min(end, (uint32_t)kList) - 1);
    slot[j] = atomicAdd(&s.guesses[guess[j]], 1u);
  }
  __syncthreads();
  // Tokens before each guess.
  uint32_t c[P], sum = 0, most = 0;
#pragma unroll
  for (int j = 0; j < P; ++j) c[j] = s.guesses[P * tid + j], sum += c[j], most = max(most, c[j]);
  uint32_t in = sum;
  scan_steps([&](auto ctrl, auto rows) { in += before_in_wave<decltype(ctrl)::value, decltype(rows)::value>(in); });
  if (lane == 63) s.wave_count[wave] = in;
  if (__syncthreads_or(most > kAlike)) return sort_list(s, n);
  uint32_t before = in - sum;
  for (int w = 0; w < wave; ++w) before += s.wave_count[w];
#pragma unroll
  for (int j = 0; j < P; ++j) s.guesses[P * tid + j] = before, before += c[j];
  if (tid == kThreads - 1) s.guesses[kList] = before;
  __syncthreads();
  uint32_t from[P], to[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (tid + j * kThreads >= n) continue;
    from[j] = s.guesses[guess[j]], to[j] = s.guesses[guess[j] + 1];
    s.list[from[j] + slot[j]] = v[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (tid + j * kThreads >= n) continue;
    uint32_t at = from[j];
    for (uint32_t i = from[j]; i < to[j]; ++i) at += s.list[i] < v[j];
    slot[j] = at;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < P; ++j)
    if (tid + j * kThreads < n) s.list[slot[j]] = v[j];
  __syncthreads();
}

// The slice's tokens within the N runs into s.list.
template <int N, typename T>
__device__ __forceinline__ void gather_runs(Shared& s, const Logits<T>& x, int first, const Edges& edges) {
  x.template fours<4>([&](const float* v, int i) {
    auto in = [&](int e) {  // the median of a logit and a run's ends is the logit
      bool any = false;
#pragma unroll
      for (int q = 0; q < N; ++q) any |= __builtin_amdgcn_fmed3f(v[e], edges.from[q], edges.to[q]) == v[e];
      return any;
    };
    const bool wanted[4] = {in(0), in(1), in(2), in(3)};
    put<4>(s, wanted, [&](int e) { return entry(v[e], first + i + e); });
  });
}
template <typename T>
__device__ void gather(Shared& s, const Logits<T>& x, int first, const Edges& edges) {
  if (edges.n == 1) gather_runs<1>(s, x, first, edges);
  else if (edges.n == 2) gather_runs<2>(s, x, first, edges);
  else gather_runs<4>(s, x, first, edges);
}

// Whether a list of the tokens not below `low` holds every wanted bin: it does the bins before the one that `low` lies in.
__device__ __forceinline__ bool list_serves(const Row& row, const Wanted& w, float low) {
  const double b = row.bins(low);
  return w.last < (b < kBins ? (int)b : kBins);
}

// Of the waves' parts of the list, `n` in this wave's, the tokens of the wanted bins, as one list.
__device__ void keep_wanted(Shared& s, int n, const Row& row, const Wanted& w) {
  const int lane = threadIdx.x & 63;
  u64 v[kWaveList / 64];
#pragma unroll
  for (int j = 0; j < kWaveList / 64; ++j)
    v[j] = lane + 64 * j < n ? s.list[(threadIdx.x >> 6) * kWaveList + lane + 64 * j] : ~0ull;
  if (threadIdx.x == 0) s.listed = 0;
  __syncthreads();
  bool in[kWaveList / 64];
#pragma unroll
  for (int j = 0; j < kWaveList / 64; ++j) in[j] = v[j] != ~0ull && w.has((int)row.bins_of_key(~(uint32_t)(v[j] >> 32)));
  put<kWaveList / 64>(s, in, [&](int j) { return v[j]; });
  __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_row(SampleArgs a) {
  __shared__ Shared s;
  const int r = blockIdx.x, tid = threadIdx.x;
  Logits<T> x{static_cast<const T*>(a.logits) + (size_t)r * a.row_stride, a.vocab, false};
  double inv_t;
  bool greedy;
  const Settings c = settings_of(a, r, &inv_t, &greedy);
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) s.hist[tid + i * kThreads] = 0;
  Part p = largest(s, x, 0, greedy);
  if (p.max == -INFINITY) return answer(a, r, -1, 0.f);
  if (greedy) return answer(a, r, p.index, 1.f);
  x.infinite = p.max == INFINITY;
  const float low = x.plain(p.low);
  const Row row{x.plain(p.max), inv_t * kBinsPerUnit};
  const int listed = count(s, x, 0, row, low);
  const bool whole = __syncthreads_and(listed <= kWaveList);
  const Wanted w = decide(s, c);
  if (whole && list_serves(row, w, low)) {
    keep_wanted(s, listed, row, w);
    sort_list(s, s.listed);
  } else if (s.wanted > kList) {
    const Pick pick = narrow(s, x, row, c);
    return answer(a, r, pick.index, pick.prob);
  } else {
    const Edges edges = edges_of(s, row, w);
    if (tid == 0) s.listed = 0;
    __syncthreads();
    gather(s, x, 0, edges);
    __syncthreads();
    sort_runs<T>(s, s.listed, row, edges, x.n);
  }
  const int n = s.listed;
  const Pick pick = finish(s, n, row, c, w, [&](int b) { return Place{s.before[b], s.mass[b]}; });
  answer(a, r, pick.index, pick.prob);
}

// ---- several workgroups a row, for few rows -------------------------------------------------------------
//
// Each takes a slice: sample_max leaves the slices' maxima, sample_count adds up their histograms and lists, sample_list
// lists the tokens of the wanted bins if that list does not serve.  The last of a row's workgroups to finish a step goes
// on with the row alone.  What they share goes past the XCDs' L2 caches by device-scope accesses.

constexpr int kMaxSlices = 8;
struct Split {
  u64 hist[kBins];
  u64 list[kList];
  double mass[kBins];      // the place before each bin, left for sample_list
  uint32_t before[kBins];
  Part part[kMaxSlices];
  Edges edges;
  Wanted wanted;
  uint32_t listed, counted, gathered, open;  // tokens listed, slices done with each step, whether sample_list is needed
};

template <typename V>
__device__ __forceinline__ V load_shared(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename V>
__device__ __forceinline__ void store_shared(V* p, V v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename T>
__device__ __forceinline__ Logits<T> slice_of(const SampleArgs& a, int r, int* first) {
  const int per = (a.vocab + gridDim.x - 1) / gridDim.x;
  *first = min((int)blockIdx.x * per, a.vocab);
  return Logits<T>{static_cast<const T*>(a.logits) + (size_t)r * a.row_stride + *first, min(per, a.vocab - *first), false};
}

// Adds a wave's list of n tokens to the row's; more than `room` do not fit, and are counted all the same.
__device__ void send_list(Split* row, const u64* list, int n, int room) {
  const int lane = threadIdx.x & 63;
  if (n == 0) return;
  uint32_t at = 0;
  const uint32_t more = n > room ? kList + 1 : n;
  if (lane == 0) at = __hip_atomic_fetch_add(&row->listed, more, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  at = __builtin_amdgcn_readfirstlane(at);
  for (int i = lane; i < min(n, room); i += 64)
    if (at + i < kList) store_shared(&row->list[at + i], list[i]);
}

// Whether the workgroup is the last of the row's to arrive; then the row's list is in s.list, unless it is too long.
// What the workgroups hand over are device-scope atomic accesses, past the L2 of an XCD, and such an addition or store is done once
// it is counted off.  So it is enough that each wave waits for its own before the barrier and the arrival; the orders are relaxed,
// as a release would also write back the L2 and an acquire empty it, where none of this lies.
__device__ bool last_of_row(Shared& s, Split* row, uint32_t* arrived) {
  const int tid = threadIdx.x;
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the wave's stores and additions have completed
  __syncthreads();
  if (tid == 0)
    s.at = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  __syncthreads();
  if (!s.at) return false;
  if (tid == 0) s.listed = load_shared(&row->listed);
  __syncthreads();
  for (uint32_t i = tid; i < min(s.listed, (uint32_t)kList); i += kThreads) s.list[i] = load_shared(&row->list[i]);
  __syncthreads();
  return true;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_max(SampleArgs a, Split* split) {
  __shared__ Shared s;
  const int r = blockIdx.y, tid = threadIdx.x;
  Split* row = split + r;
  for (int i = blockIdx.x * kThreads + tid; i < kBins; i += gridDim.x * kThreads) row->hist[i] = 0;
  if (blockIdx.x == 0 && tid == 0) row->listed = row->counted = row->gathered = row->open = 0;
  double inv_t;
  bool greedy;
  (void)settings_of(a, r, &inv_t, &greedy);
  int first;
  const Logits<T> x = slice_of<T>(a, r, &first);
  Part p = largest(s, x, gridDim.x / 2, greedy);
  if (p.max > -INFINITY) p.index += first;  // a slice without a token keeps the index past all others
  if (tid == 0) row->part[blockIdx.x] = p;
}

// The row's part from its slices'; the infinities of a row whose largest is infinite count as 0 from here on.
template <typename T>
__device__ Part join_parts(const Split* row, Logits<T>* x) {
  Part p{-INFINITY, INFINITY, 0x7fffffff, 0};
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const Part q = row->part[i];
    if (q.max > p.max || (q.max == p.max && q.index < p.index)) p.max = q.max, p.index = q.index;
    p.low = fminf(p.low, q.low);
  }
  x->infinite = p.max == INFINITY;
  return p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_count(SampleArgs a, Split* split) {
  __shared__ Shared s;
  const int r = blockIdx.y, tid = threadIdx.x;
  Split* row = split + r;
  double inv_t;
  bool greedy;
  const Settings c = settings_of(a, r, &inv_t, &greedy);
  int first;
  Logits<T> x = slice_of<T>(a, r, &first);
  const Part p = join_parts(row, &x);
  if (p.max == -INFINITY || greedy) {
    if (blockIdx.x == 0) answer(a, r, p.max == -INFINITY ? -1 : p.index, p.max == -INFINITY ? 0.f : 1.f);
    return;
  }
  const float low = x.plain(p.low);
  const Row scale{x.plain(p.max), inv_t * kBinsPerUnit};
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) s.hist[tid + i * kThreads] = 0;
  __syncthreads();
  const int listed = count(s, x, first, scale, low);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) {
    const u64 h = s.hist[tid + i * kThreads];
    if (h) (void)__hip_atomic_fetch_add(&row->hist[tid + i * kThreads], h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  send_list(row, s.list + (tid >> 6) * kWaveList, listed, kWaveList);
  if (!last_of_row(s, row, &row->counted)) return;
#pragma unroll
  for (int i = 0; i < kBinsPerThread; ++i) s.hist[tid + i * kThreads] = load_shared(&row->hist[tid + i * kThreads]);
  __syncthreads();
  const Wanted w = decide(s, c);
  x = Logits<T>{static_cast<const T*>(a.logits) + (size_t)r * a.row_stride, a.vocab, x.infinite};
  if (s.listed <= kList && list_serves(scale, w, low)) {
    const int n = s.listed;
    sort_list(s, n);
    const Pick pick = finish(s, n, scale, c, w, [&](int b) { return Place{s.before[b], s.mass[b]}; });
    return answer(a, r, pick.index, pick.prob);
  }
  if (s.wanted > kList) {
    const Pick pick = narrow(s, x, scale, c);
    return answer(a, r, pick.index, pick.prob);
  }
  const Edges edges = edges_of(s, scale, w);
  for (int i = tid; i < kBins; i += kThreads) row->mass[i] = s.mass[i], row->before[i] = s.before[i];
  if (tid == 0) row->edges = edges, row->wanted = w, row->listed = 0, row->open = 1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_list(SampleArgs a, Split* split) {
  __shared__ Shared s;
  const int r = blockIdx.y, tid = threadIdx.x;
  Split* row = split + r;
  if (!row->open) return;
  double inv_t;
  bool greedy;
  const Settings c = settings_of(a, r, &inv_t, &greedy);
  int first;
  Logits<T> x = slice_of<T>(a, r, &first);
  const Part p = join_parts(row, &x);
  const Row scale{x.plain(p.max), inv_t * kBinsPerUnit};
  if (tid == 0) s.listed = 0;
  __syncthreads();
  const Edges edges = row->edges;
  gather(s, x, first, edges);
  __syncthreads();
  const int each = (s.listed + kWaves - 1) / kWaves, from = (tid >> 6) * each;
  send_list(row, s.list + from, max(0, min(each, (int)s.listed - from)), kList);
  if (!last_of_row(s, row, &row->gathered)) return;
  const int n = s.listed;
  sort_runs<T>(s, n, scale, edges, a.vocab);
  const Wanted w = row->wanted;
  const Pick pick = finish(s, n, scale, c, w, [&](int b) { return Place{row->before[b], row->mass[b]}; });
  answer(a, r, pick.index, pick.prob);
}

}  // namespace

// Slices of a row.  One workgroup pays for no hand-over; several share the passes.  us of a call with 1 / 2 / 4 / 8 / 16, top-p
// of float32 rows: 128256 logits, 1 row 49 / 44 / 36 / 33 / 35, 32 rows 56 / 49 / 41 / 40 / 67, 64 rows 57 / 52 / 46 / 69 / 114,
// 128 rows 61 / 62 / 81 / 125; 50000 logits, 1 row 27 / 31 / 29 / 30 / 32, 64 rows 32 / 37 / 37 / 60; 16384, 1 row 20 / 27.
int sample_slices(int rows, int vocab) {
  if (vocab < (1 << 16) || rows > 64) return 1;
  return rows > 32 ? 4 : 8;
}

size_t sample_workspace(int rows, int vocab) { return sample_slices(rows, vocab) > 1 ? rows * sizeof(Split) : 0; }

namespace {
template <typename T>
hipError_t launch(const SampleArgs& a, void* workspace, hipStream_t s) {
  const int slices = sample_slices(a.rows, a.vocab);
  if (slices == 1) {
    hipLaunchKernelGGL(sample_row<T>, dim3(a.rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  }
  Split* split = static_cast<Split*>(workspace);
  const dim3 grid(slices, a.rows);
  hipLaunchKernelGGL(sample_max<T>, grid, dim3(kThreads), 0, s, a, split);
  hipLaunchKernelGGL(sample_count<T>, grid, dim3(kThreads), 0, s, a, split);
  hipLaunchKernelGGL(sample_list<T>, grid, dim3(kThreads), 0, s, a, split);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  return a.dtype == DUET_BF16 ? launch<__bf16>(a, workspace, s) : launch<float>(a, workspace, s);
}

}  // namespace duet
