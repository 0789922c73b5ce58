// Sampling from a row of V logits x (temperature T, top-k, top-p, min-p, a given uniform number u).
//
// Tokens are ranked by falling logit, ties by the lower index, and weigh w = exp((max - x) / -T).  Each filter
// keeps a run of ranks from the first: top-k the first k; top-p, of those, rank r where the mass before it is
// less than p times theirs; min-p those with w >= min-p (the largest has w = 1).  The token is the first rank
// whose kept cumulative mass exceeds u times the kept mass S.
//
// So every step looks for a place in the ranking, and a row need not be sorted: a histogram over
// d = (max - x) / T gives the mass before each of its bins, and the bin that holds the place is narrowed by
// the bits of its logits, down to one value, whose tokens weigh the same.  The mass of tokens with d >= kSpan
// (e^-48 each, at most 4e-16 of the largest's over a row) is less than a unit in the last place of S in 64 bits.
//
// Sums do not depend on the order of atomics: a token adds an integer to its bin, 2^45 + (1 - v) 2^33, with
// v = e^-(d - d_bin) in (1 - 2^-6.4, 1] its weight relative to the bin's first.  The count stands in bits 45 on,
// the sum of up to 2^18 terms under 2^(26.6 + 18) below.  Each term rounds by 2^-34 of the token's weight.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "wave_ops.h"

namespace duet {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 4096, kSubBins = 2048;
constexpr double kSpan = 48.0, kBinsPerUnit = kBins / kSpan, kBinWidth = kSpan / kBins;
constexpr int kCountShift = 45;
constexpr double kFraction = 8589934592.0;  // 2^33

__device__ __forceinline__ float logit(const __bf16* x) { return static_cast<float>(*x); }
__device__ __forceinline__ float logit(const float* x) { return *x; }

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

struct Shared {
  unsigned long long hist[kBins];
  double mass[kWaves];
  uint32_t count[kWaves];
  uint32_t key;
  int found;
  Place place;
};

struct Row {
  double max, inv_t;
  __device__ double gap(uint32_t key) const {
    const double x = of_key(key);
    return x == max ? 0.0 : (max - x) * inv_t;  // infinite past an infinite max
  }
  __device__ int bin(double d) const { return min((int)(d * kBinsPerUnit), kBins - 1); }
};

__device__ __forceinline__ unsigned long long token_bits(double d, int bin) {
  return (1ull << kCountShift) + (unsigned long long)((1.0 - exp(bin * kBinWidth - d)) * kFraction + 0.5);
}
__device__ __forceinline__ uint32_t count_of(unsigned long long h) { return (uint32_t)(h >> kCountShift); }
__device__ __forceinline__ double mass_of(unsigned long long h, int bin) {
  return (count_of(h) - (double)(h & ((1ull << kCountShift) - 1)) / kFraction) * exp(-bin * kBinWidth);
}

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
    m += mass_of(s.hist[b], fixed_bin >= 0 ? fixed_bin : b);
  }
  uint32_t ci = c;
  double mi = m;
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t cu = __shfl_up(ci, off);
    const double mu = __shfl_up(mi, off);
    if (lane >= off) ci += cu, mi += mu;
  }
  if (lane == 63) s.count[wave] = ci, s.mass[wave] = mi;
  if (tid == 0) s.found = 1 << 30;
  __syncthreads();
  Place p = at;
  for (int w = 0; w < wave; ++w) p.n += s.count[w], p.mass += s.mass[w];
  p.n += ci - c;
  p.mass += mi - m;
  Place mine = p, last_place = p;
  int first = -1, last = -1;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    const unsigned long long h = s.hist[b];
    if (!h) continue;
    last = b, last_place = p;
    p.n += count_of(h);
    p.mass += mass_of(h, fixed_bin >= 0 ? fixed_bin : b);
    if (first < 0 && reached(p)) first = b, mine = last_place;
  }
  if (first >= 0) atomicMin(&s.found, first);
  __syncthreads();
  if (s.found == 1 << 30) {
    __syncthreads();
    if (tid == 0) s.found = -1;
    __syncthreads();
    if (last >= 0) atomicMax(&s.found, last);
    __syncthreads();
    first = last, mine = last_place;
  }
  const int found = s.found;
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
__device__ Found find(Shared& s, const T* x, int vocab, const Row& row, F reached) {
  const int tid = threadIdx.x;
  auto each = [&](auto f) {
    for (int i = tid; i < vocab; i += kThreads) {
      const uint32_t k = key_of(logit(x + i));
      if (!k) continue;
      const double d = row.gap(k);
      if (d < kSpan) f(k, d);
    }
  };
  auto clear = [&](int n) {
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) s.hist[i] = 0;
    __syncthreads();
  };
  clear(kBins);
  each([&](uint32_t, double d) { atomicAdd(&s.hist[row.bin(d)], token_bits(d, row.bin(d))); });
  __syncthreads();
  Place before{0, 0.0};
  const int bin = find_bin(s, kBins, -1, before, reached, &before);
  // The bin's keys: from the largest down to one past the smallest.
  if (tid == 0) s.key = 0, s.found = -1;
  __syncthreads();
  each([&](uint32_t k, double d) {
    if (row.bin(d) == bin) atomicMax(&s.key, k);
  });
  __syncthreads();
  uint32_t hi = s.key;
  __syncthreads();
  if (tid == 0) s.key = 0xffffffffu;
  __syncthreads();
  each([&](uint32_t k, double d) {
    if (row.bin(d) == bin) atomicMin(&s.key, k);
  });
  __syncthreads();
  uint32_t lo = s.key;
  while (true) {
    int shift = 0;
    while (((hi - lo) >> shift) >= kSubBins) ++shift;
    clear(kSubBins);
    each([&](uint32_t k, double d) {
      if (k <= hi && k >= lo) atomicAdd(&s.hist[(hi - k) >> shift], token_bits(d, bin));
    });
    __syncthreads();
    const int sub = find_bin(s, kSubBins, bin, before, reached, &before);
    const uint32_t n = count_of(s.hist[sub]);
    hi -= (uint32_t)sub << shift;
    lo = hi - min(hi - lo, (1u << shift) - 1);
    if (shift == 0) {
      const double w = exp(-row.gap(hi));
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
__device__ int index_of(Shared& s, const T* x, int vocab, uint32_t key, uint32_t n) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int per = ((vocab + kWaves - 1) / kWaves + 63) / 64 * 64;  // a wave's tokens
  const int lo = wave * per, hi = min(vocab, lo + per);
  uint32_t c = 0;
  for (int i = lo; i < hi; i += 64) c += __popcll(__ballot(i + lane < hi && key_of(logit(x + min(i + lane, vocab - 1))) == key));
  __syncthreads();
  if (lane == 0) s.count[wave] = c;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += s.count[w];
  if (before < n && n <= before + c) {
    for (int i = lo; i < hi; i += 64) {
      const bool is = i + lane < hi && key_of(logit(x + min(i + lane, vocab - 1))) == key;
      const unsigned long long all = __ballot(is);
      if (is && before + __popcll(all & ((1ull << lane) - 1)) + 1 == n) s.found = i + lane;
      before += __popcll(all);
    }
  }
  __syncthreads();
  return s.found;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_row(SampleArgs a) {
  __shared__ Shared s;
  const int r = blockIdx.x, tid = threadIdx.x;
  const T* x = static_cast<const T*>(a.logits) + (size_t)r * a.row_stride;
  if (tid == 0) s.key = 0;
  __syncthreads();
  uint32_t most = 0;
  for (int i = tid; i < a.vocab; i += kThreads) most = max(most, key_of(logit(x + i)));
  atomicMax(&s.key, most);
  __syncthreads();
  most = s.key;
  __syncthreads();
  const float t = a.temperature ? a.temperature[r] : 1.f;
  if (!most || !(t > 0.f)) {  // nothing left, or the largest
    const int i = most ? index_of(s, x, a.vocab, most, 1) : -1;
    if (tid == 0) {
      a.ids[r] = i;
      if (a.probs) a.probs[r] = most ? 1.f : 0.f;
    }
    return;
  }
  const Row row{of_key(most), 1.0 / t};
  const int top_k = a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
  // The last kept rank.
  const uint32_t all = 0xffffffffu;
  uint32_t most_n = top_k > 0 ? top_k : all;
  auto kept = find(s, x, a.vocab, row, [&](const Place& p) { return p.n >= most_n; });
  if (top_p < 1.f) {
    const double need = fmax(0.0, (double)top_p) * kept.end.mass;
    const uint32_t n = kept.end.n;
    kept = find(s, x, a.vocab, row, [&](const Place& p) { return p.n >= n || p.mass >= need; });
  }
  if (min_p > 0.f) {
    // Count the tokens of at least that weight.
    __syncthreads();
    if (tid == 0) s.key = 0;
    __syncthreads();
    uint32_t c = 0;
    const double least = fmin(1.0, (double)min_p);
    for (int i = tid; i < a.vocab; i += kThreads) {
      const uint32_t k = key_of(logit(x + i));
      c += k && exp(-row.gap(k)) >= least;
    }
    atomicAdd(&s.key, c);
    __syncthreads();
    const uint32_t n = min(s.key, kept.end.n);
    __syncthreads();
    if (n < kept.end.n) kept = find(s, x, a.vocab, row, [&](const Place& p) { return p.n >= n; });
  }
  float u = a.u[r];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  const double target = u * kept.end.mass;
  const uint32_t n = kept.end.n;
  const auto pick = find(s, x, a.vocab, row, [&](const Place& p) { return p.n >= n || p.mass > target; });
  const int i = index_of(s, x, a.vocab, pick.key, pick.ties);
  if (tid == 0) {
    a.ids[r] = i;
    if (a.probs) a.probs[r] = (float)(exp(-row.gap(pick.key)) / kept.end.mass);
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  if (a.dtype == DUET_BF16) hipLaunchKernelGGL(sample_row<__bf16>, dim3(a.rows), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(sample_row<float>, dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace duet
