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
// alike), and then some of the columns of all of them: a thread a unit of 32 bytes a row (of queries and keys the two
// 16-byte chunks that turn together), eight rows in flight.  Values go to a dim-major page, a whole page's 32 or 64
// contiguous bytes a dim, of a page that the chunk covers in part, value by value.
//
// Request r (rows q_start .. q_start + q_len - 1) has the page groups from q_start / 16 + 2 r on: more than it needs,
// whatever its first slot, and groups past its last page end at once.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "wave_ops.h"

namespace duet {
namespace {

// (cos, sin) of `rev` turns.  The Taylor series of both on |t| <= pi / 4: the first terms left out are
// t^11 / 11! < 2e-9 and t^12 / 12! < 2e-10, under half a unit in the last place of the results.
__device__ __forceinline__ float2 cos_sin_of(double rev) {
  const double quarter = rint(4.0 * rev);
  const float t = (float)((rev - 0.25 * quarter) * 6.283185307179586);
  const float z = t * t;
  const float s = fmaf(t * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), t);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int q = (int)(quarter - 4.0 * floor(0.25 * quarter));
  const float x = q & 1 ? s : c, y = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y);
}

__device__ __forceinline__ int first_group(const RopeSplitArgs& s, int r) { return (s.meta[r].y >> 4) + 2 * r; }

template <typename T>
struct Chunk {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};

constexpr int kMaxPairs = 64;

template <typename T>
__global__ __launch_bounds__(256) void rope_split(RopeSplitArgs s) {
  constexpr int N = Chunk<T>::N;
  __shared__ float2 turn[16][kMaxPairs];
  const int group = blockIdx.x, d = s.head_dim, pairs = s.rot_dim / 2, tid = threadIdx.x;
  const int r = uniform(find_request(s.num_reqs, [&](int x) { return first_group(s, x) <= group; }));
  const int4 m = s.meta[r];
  const int page = (m.w >> 4) + group - first_group(s, r);
  const int pos = max(m.w, 16 * page), n = min(m.w + m.z, 16 * page + 16) - pos;
  if (n <= 0) return;
  const int row = m.y + pos - m.w, slot = pos & 15;
  const int id = s.page_table[(size_t)r * s.max_pages + (pos >> 4)];
  const bool ok = page_ok(id, s.num_phys_pages);
  if (!ok && blockIdx.y == 0 && tid == 0) atomicOr(s.err, 1);
  for (int i = tid; i < n * pairs; i += 256) {
    const int t = i / pairs, pair = i - t * pairs;
    const int p = s.positions ? s.positions[(size_t)s.pair_axis[pair] * s.tokens + row + t] : pos + t;
    turn[t][pair] = cos_sin_of(p * s.turns[pair]);
  }
  __syncthreads();
  const int units = d / (2 * N), nqk = s.h_q + s.h_kv, width = (nqk + s.h_kv) * d;
  const int qk_units = nqk * units, all = qk_units + s.h_kv * d / N;
  const T* src = static_cast<const T*>(s.qkv) + (size_t)row * width;
  for (int u = blockIdx.y * 256 + tid; u < all; u += gridDim.y * 256) {
    if (u < qk_units) {
      const int head = u / units, k = u - head * units, turned = pairs / N;  // units that turn
      const bool is_q = head < s.h_q;
      if (!is_q && !ok) continue;
      // The unit's two chunks, and the pair of its first element(s).
      const bool halves = k < turned && !s.adjacent;
      const int c0 = halves ? k * N : 2 * k * N, c1 = halves ? c0 + pairs : c0 + N;
      const T* x = src + head * d;
      T* dst;
      size_t stride;
      if (is_q) {
        dst = static_cast<T*>(s.q) + ((size_t)row * s.h_q + head) * d;
        stride = (size_t)s.h_q * d;
      } else {
        dst = static_cast<T*>(s.k_cache) + (((size_t)id * s.h_kv + head - s.h_q) * 16 + slot) * d;
        stride = d;
      }
      const bool turns = k < turned;
#pragma unroll
      for (int t0 = 0; t0 < 16; t0 += 8) {
        if (t0 >= n) break;
        uint4 a[8], b[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const T* y = x + (size_t)min(t0 + t, n - 1) * width;
          a[t] = *reinterpret_cast<const uint4*>(y + c0);
          b[t] = *reinterpret_cast<const uint4*>(y + c1);
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          if (t0 + t >= n) break;
          if (turns) {
            Chunk<T> p = __builtin_bit_cast(Chunk<T>, a[t]), q = __builtin_bit_cast(Chunk<T>, b[t]);
            const float2* cs = turn[t0 + t] + k * N;
            if (s.adjacent) {
#pragma unroll
              for (int e = 0; e < N / 2; ++e)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  T* w = h ? q.v : p.v;
                  const float2 z = cs[h * N / 2 + e];
                  const float v0 = static_cast<float>(w[2 * e]), v1 = static_cast<float>(w[2 * e + 1]);
                  w[2 * e] = static_cast<T>(v0 * z.x - v1 * z.y);
                  w[2 * e + 1] = static_cast<T>(v0 * z.y + v1 * z.x);
                }
            } else {
#pragma unroll
              for (int e = 0; e < N; ++e) {
                const float2 z = cs[e];
                const float v0 = static_cast<float>(p.v[e]), v1 = static_cast<float>(q.v[e]);
                p.v[e] = static_cast<T>(v0 * z.x - v1 * z.y);
                q.v[e] = static_cast<T>(v0 * z.y + v1 * z.x);
              }
            }
            a[t] = __builtin_bit_cast(uint4, p);
            b[t] = __builtin_bit_cast(uint4, q);
          }
          T* y = dst + (t0 + t) * stride;
          *reinterpret_cast<uint4*>(y + c0) = a[t];
          *reinterpret_cast<uint4*>(y + c1) = b[t];
        }
      }
      continue;
    }
    if (!ok) continue;
    const int col = (u - qk_units) * N;
    T* v = static_cast<T*>(s.v_cache) + (((size_t)id * s.h_kv + col / d) * d + col % d) * 16 + slot;
    Chunk<T> x[16];
#pragma unroll
    for (int t = 0; t < 16; ++t)
      x[t] = __builtin_bit_cast(Chunk<T>, *reinterpret_cast<const uint4*>(src + (size_t)min(t, n - 1) * width + nqk * d + col));
    if (n < 16) {
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t < n)
#pragma unroll
          for (int e = 0; e < N; ++e) v[e * 16 + t] = x[t].v[e];
      continue;
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
}

}  // namespace

hipError_t launch_rope_split(const RopeSplitArgs& a, hipStream_t s) {
  if (a.tokens <= 0) return hipSuccess;
  const int n = a.dtype == DUET_BF16 ? 8 : 4, d = a.head_dim;
  const int units = (a.h_q + a.h_kv) * d / (2 * n) + a.h_kv * d / n;
  const int groups = a.tokens / 16 + 2 * a.num_reqs;
  const dim3 grid(groups, (units + 255) / 256);
  if (a.dtype == DUET_BF16) hipLaunchKernelGGL(rope_split<__bf16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rope_split<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace duet
