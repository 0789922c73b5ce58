// The QKV split with the position rotation on the way (rotary position embedding): the query and key
// rows of the projection are turned by their token's position, keys and values enter the paged cache.
//
// A pair (a, b) of a head's row turns by t = p f: a' = a cos t - b sin t, b' = a sin t + b cos t, with p the
// position of the token on the pair's axis and f the pair's frequency.  Dimensions past rot_dim and
// values are copied.  p f / 2 pi is formed in 64 bits (at position 100000 the product alone would lose
// 2^-8 of a radian in 32) and brought within an eighth of a turn of a quarter there; sine, cosine and the
// rotation are 32-bit, with one rounding to the stored type.
//
// Bound by memory: the projection is read once, the same bytes are written.  A workgroup takes the rows of one request
// whose positions lie on one page (up to 16; one decode row), forms their sines and cosines once in LDS (all heads turn
// alike), and moves some of the columns of all of them: a thread a unit of 32 bytes a row (of queries and keys two 16-byte
// chunks, eight rows in flight, neighbours at neighbouring chunks: with the two side by side a kernel that only copied took twice
// as long).  The first loads go out before the sines are formed.  Values go to a dim-major page, a whole page's 32 or 64
// contiguous bytes a dim, of a page that the chunk covers in part, value by value.
//
// Request r (rows q_start .. q_start + q_len - 1) has the page groups from q_start / 16 + 2 r on: more than it needs,
// whatever its first slot, and groups past its last page end at once.
//
// 8224 rows of 64 + 2 x 8 heads of 128 in bf16 take 77 us (4.4 TB/s; a large copy reaches 5.1), 2112 rows of 32 + 2 x 8 heads
// 15 (3.4 TB/s: a chain of latencies of 3 us before the first store), in float32 31 (3.3 TB/s).  256 decode rows in bf16 7.9, one
// 3.5: half of the former's 1056 workgroups are empty, two groups a request, and the kernel for up to kRopeTable requests, with
// check_pages in it, has 97 registers: four waves a SIMD instead of the five of 96.  One kernel for both orders of pairs took
// 1.2 us more for the 2112 rows.  Rows past the last are loaded as that again: with branches around the loads those waited for each
// other (8224 rows 159 us).  A single row alone is told apart (256 decode rows 8.9 us without).
//
// Up to kRopeTable requests travel with the launch's arguments; more are uploaded, a launch of its own (2 to 4 us on the GPU, as
// much on the host).  The upload clears the error word; without it one more workgroup reads the page ids of the whole batch
// and stores the word, if the caller has a workspace for it.  One decode row: 15.8 us a call with the upload, 10.3 with the
// workgroup, 8.5 without a workspace.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rope_device.h"
#include "serving_ops.h"
#include "wave_ops.h"

namespace duet {
namespace {

template <typename T, bool ADJACENT, typename Table>
__global__ __launch_bounds__(256) void rope_split(RopeSplitArgs s, Table requests) {
  constexpr int N = Chunk<T>::N;
  constexpr bool kPassed = std::is_same<Table, Passed>::value;
  __shared__ float2 turn[16][kMaxPairs];
  const int d = s.head_dim, pairs = s.rot_dim / 2, tid = threadIdx.x;
  int group = blockIdx.x;
  if (kPassed && s.err) {
    static_assert(sizeof(Passed::at) <= sizeof(turn), "the check keeps the requests where the sines go");
    if (group == 0) {
      if constexpr (kPassed)
        if (blockIdx.y == 0) check_pages(s, requests, reinterpret_cast<int2*>(turn));
      return;
    }
    --group;
  }
  const int r = uniform(find_request(s.num_reqs, [&](int x) { return first_group(requests.row(x), x) <= group; }));
  const Group at = group_of(requests[r], r, group);
  const int n = at.rows, pos = at.pos, row = at.row, slot = pos & 15;
  if (n <= 0) return;
  const int id = s.page_table[(size_t)r * s.max_pages + at.page];
  const bool ok = page_ok(id, s.num_phys_pages);
  if (!kPassed && !ok && blockIdx.y == 0 && tid == 0) atomicOr(s.err, 1);
  // The thread's unit.  Its first loads, 16 of 16 bytes, go out before the sines are formed and wait for neither the page id nor
  // those: eight rows of a unit of queries or keys, all sixteen of one of values.
  const int units = d / (2 * N), nqk = s.h_q + s.h_kv, width = (nqk + s.h_kv) * d;
  const int qk_units = nqk * units, all = qk_units + s.h_kv * d / N, u = blockIdx.y * 256 + tid;
  const T* src = static_cast<const T*>(s.qkv) + (size_t)row * width;
  const bool qk = u < qk_units, there = u < all;
  const int head = u / units, k = u - head * units;
  // A unit's two chunks: those that turn together, of halves, else two half a head apart or half of what is copied; so that
  // neighbours take neighbouring chunks.  A column of values.
  const bool together = !ADJACENT && k < pairs / N;
  const int from = ADJACENT || together ? 0 : s.rot_dim - pairs, half = ADJACENT ? d / 2 : together ? pairs : (d - s.rot_dim) / 2;
  const int c0 = from + k * N, c1 = c0 + half;
  const int col = (u - qk_units) * N;
  uint4 a[16];
  auto load = [&](int t0, uint4* v) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const T* y = src + (size_t)min(t0 + t, n - 1) * width + head * d;
      v[t] = *reinterpret_cast<const uint4*>(y + c0);
      v[8 + t] = *reinterpret_cast<const uint4*>(y + c1);
    }
  };
  constexpr int J = 16 * kMaxPairs / 256;
  int p[J];
  double f[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (256 * j >= n * pairs) break;
    const int i = min(tid + 256 * j, n * pairs - 1), t = i / pairs, pair = i - t * pairs;
    p[j] = s.positions ? s.positions[(size_t)s.pair_axis[pair] * s.tokens + row + t] : pos + t;
    f[j] = s.turns[pair];
  }
  if (n == 1) {
    const T* y = src + (qk ? head * d + c0 : nqk * d + col);
    if (there) a[0] = *reinterpret_cast<const uint4*>(y);
    if (qk) a[8] = *reinterpret_cast<const uint4*>(y + half);
  } else if (qk) {
    load(0, a);
  } else if (there) {
#pragma unroll
    for (int t = 0; t < 16; ++t)
      a[t] = *reinterpret_cast<const uint4*>(src + (size_t)min(t, n - 1) * width + nqk * d + col);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (256 * j >= n * pairs) break;
    const int i = min(tid + 256 * j, n * pairs - 1), t = i / pairs;
    turn[t][i - t * pairs] = cos_sin_of(p[j] * f[j]);
  }
  __syncthreads();
  if (!there) return;
  if (qk) {
    const bool is_q = head < s.h_q;
    if (!is_q && !ok) return;
    T* dst;
    size_t stride;
    if (is_q) {
      dst = static_cast<T*>(s.q) + ((size_t)row * s.h_q + head) * d;
      stride = (size_t)s.h_q * d;
    } else {
      dst = static_cast<T*>(s.k_cache) + (((size_t)id * s.h_kv + head - s.h_q) * 16 + slot) * d;
      stride = d;
    }
    auto store = [&](int t0, uint4* v) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if (t0 + t >= n) break;
        const float2* turns = turn[t0 + t];
        if constexpr (ADJACENT) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int c = h ? c1 : c0;
            if (c >= s.rot_dim) continue;
            Chunk<T> x = __builtin_bit_cast(Chunk<T>, v[8 * h + t]);
#pragma unroll
            for (int e = 0; e < N; e += 2) {
              const float2 z = turns[(c + e) / 2];
              const float v0 = static_cast<float>(x.v[e]), v1 = static_cast<float>(x.v[e + 1]);
              x.v[e] = static_cast<T>(v0 * z.x - v1 * z.y);
              x.v[e + 1] = static_cast<T>(v0 * z.y + v1 * z.x);
            }
            v[8 * h + t] = __builtin_bit_cast(uint4, x);
          }
        } else if (together) {
          Chunk<T> x = __builtin_bit_cast(Chunk<T>, v[t]), y = __builtin_bit_cast(Chunk<T>, v[8 + t]);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 z = turns[c0 + e];
            const float v0 = static_cast<float>(x.v[e]), v1 = static_cast<float>(y.v[e]);
            x.v[e] = static_cast<T>(v0 * z.x - v1 * z.y);
            y.v[e] = static_cast<T>(v0 * z.y + v1 * z.x);
          }
          v[t] = __builtin_bit_cast(uint4, x);
          v[8 + t] = __builtin_bit_cast(uint4, y);
        }
        T* y = dst + (t0 + t) * stride;
        *reinterpret_cast<uint4*>(y + c0) = v[t];
        *reinterpret_cast<uint4*>(y + c1) = v[8 + t];
      }
    };
    store(0, a);
    if (n > 8) load(8, a), store(8, a);
    return;
  }
  if (!ok) return;
  T* v = static_cast<T*>(s.v_cache) + (((size_t)id * s.h_kv + col / d) * d + col % d) * 16 + slot;
  Chunk<T> x[16];
#pragma unroll
  for (int t = 0; t < 16; ++t) x[t] = __builtin_bit_cast(Chunk<T>, a[t]);
  if (n < 16) {
#pragma unroll
    for (int t = 0; t < 16; ++t)
      if (t < n)
#pragma unroll
        for (int e = 0; e < N; ++e) v[e * 16 + t] = x[t].v[e];
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
#pragma unroll
    for (int t = 0; t < 16; t += N) {
      Chunk<T> y;
#pragma unroll
      for (int i = 0; i < N; ++i) y.v[i] = x[t + i].v[e];
      *reinterpret_cast<uint4*>(v + e * 16 + t) = __builtin_bit_cast(uint4, y);
    }
}

template <typename T, bool ADJACENT>
hipError_t launch(const RopeSplitArgs& a, const int4* requests, hipStream_t s) {
  const int n = 16 / sizeof(T), d = a.head_dim;
  const int units = (a.h_q + a.h_kv) * d / (2 * n) + a.h_kv * d / n;
  const int groups = a.tokens / 16 + 2 * a.num_reqs, columns = (units + 255) / 256;
  if (a.num_reqs <= kRopeTable) {
    Passed p;
    for (int r = 0; r < a.num_reqs; ++r) p.at[r] = make_int2(requests[r].y, requests[r].w);
    p.at[a.num_reqs] = make_int2(a.tokens, 0);
    hipLaunchKernelGGL((rope_split<T, ADJACENT, Passed>), dim3(groups + (a.err ? 1 : 0), columns), dim3(256), 0, s, a, p);
  } else {
    hipLaunchKernelGGL((rope_split<T, ADJACENT, Uploaded>), dim3(groups, columns), dim3(256), 0, s, a, Uploaded{a.meta});
  }
  return hipGetLastError();
}
template <typename T>
hipError_t launch(const RopeSplitArgs& a, const int4* requests, hipStream_t s) {
  return a.adjacent ? launch<T, true>(a, requests, s) : launch<T, false>(a, requests, s);
}

}  // namespace

hipError_t launch_rope_split(const RopeSplitArgs& a, const int4* requests, hipStream_t s) {
  if (a.tokens <= 0 && !a.err) return hipSuccess;  // with an error word one workgroup clears that
  return a.dtype == DUET_BF16 ? launch<__bf16>(a, requests, s) : launch<float>(a, requests, s);
}

}  // namespace duet
