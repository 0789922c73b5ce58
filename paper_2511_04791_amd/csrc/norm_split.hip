// The QKV split with a norm of each head and the position rotation on the way, into pages of the projection's type or
// into 8-bit ones.
//
// A head's row x of a query or key becomes y = x w / sqrt(mean(x^2) + eps), in 32 bits, then its pairs turn as in
// rope_split.hip; values are copied.  8-bit pages hold e4m3 values times a power of two that the d values of a token's
// head share: the smallest that brings the largest of them to 448, e4m3's largest, so the exponent follows from the bits of
// the largest value and the division is exact; one rounding in all, after the rotation.
//
// Bound by memory, and laid out as rope_split.hip: a workgroup takes the rows of one request on one page, a thread two
// 16-byte chunks of a head's row (or eight columns of values) for all of them, so a head's row lies in neighbouring lanes, 4 to
// 16 of them, and its sum or maximum is taken by that many lanes' moves inside a row of 16.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cache_ops.h"
#include "rope_device.h"
#include "wave_ops.h"

namespace duet {
namespace {

template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// Over the 4, 8 or 16 neighbouring lanes that hold a head's row; every lane gets the same bits.
template <typename F>
__device__ __forceinline__ float over_lanes(float x, int lanes, F f) {
  x = f(x, moved<0xB1>(x));                    // lanes 1, 0, 3, 2
  x = f(x, moved<0x4E>(x));                    // lanes 2, 3, 0, 1
  if (lanes >= 8) x = f(x, moved<0x141>(x));   // mirrored in 8
  if (lanes >= 16) x = f(x, moved<0x140>(x));  // mirrored in 16
  return x;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float most(float a, float b) { return fmaxf(a, b); }

// The exponent's byte of a row whose largest finite magnitude is m: 448 is 1.75 2^8, so the power is 2^(exponent - 8), or
// the next where the fraction is above 0.75.  At least 2^-126.
__device__ __forceinline__ int scale_byte(float m) { return max((int)((__float_as_uint(m) + 0x1fffffu) >> 23) - 8, 1); }
__device__ __forceinline__ float inverse_scale(int e) { return __uint_as_float((unsigned)(254 - e) << 23); }
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
// Two values over the scale, as e4m3 in the low or high half; infinities become NaN (x times 0 is).
template <bool HIGH>
__device__ __forceinline__ int packed8(float a, float b, float inv, int old) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(fmaf(a, 0.f, a * inv), fmaf(b, 0.f, b * inv), old, HIGH);
}

template <typename T, bool ADJACENT, bool EIGHT, typename Table>
__global__ __launch_bounds__(256) void norm_split(NormSplitArgs x, Table requests) {
  constexpr int N = Chunk<T>::N;
  constexpr bool kPassed = std::is_same<Table, Passed>::value;
  __shared__ float2 turn[16][kMaxPairs];
  const RopeSplitArgs& s = x.rope;
  const int d = s.head_dim, pairs = s.rot_dim / 2, tid = threadIdx.x;
  int group = blockIdx.x;
  if (kPassed && s.err) {
    if (group == 0) {
      if constexpr (kPassed)
        if (blockIdx.y == 0) check_pages(s, requests, reinterpret_cast<int2*>(turn));
      return;
    }
    --group;
  }
  const int r = uniform(find_request(s.num_reqs, [&](int i) { return first_group(requests.row(i), i) <= group; }));
  const Group at = group_of(requests[r], r, group);
  const int n = at.rows, pos = at.pos, row = at.row, slot = pos & 15;
  if (n <= 0) return;
  const int id = s.page_table[(size_t)r * s.max_pages + at.page];
  const bool ok = page_ok(id, s.num_phys_pages);
  if (!kPassed && !ok && blockIdx.y == 0 && tid == 0) atomicOr(s.err, 1);
  // Units as in rope_split.hip; those of values start on a multiple of 16, so that a head's lie in one row of lanes.
  const int units = d / (2 * N), nqk = s.h_q + s.h_kv, width = (nqk + s.h_kv) * d;
  const int qk_units = nqk * units, v_units = (qk_units + 15) & ~15, u = blockIdx.y * 256 + tid;
  const T* src = static_cast<const T*>(s.qkv) + (size_t)row * width;
  const bool qk = u < qk_units;
  const int head = u / units, k = u - head * units;
  const bool together = !ADJACENT && k < pairs / N;
  const int from = ADJACENT || together ? 0 : s.rot_dim - pairs, half = ADJACENT ? d / 2 : together ? pairs : (d - s.rot_dim) / 2;
  const int c0 = from + k * N, c1 = c0 + half;
  const int col = (u - v_units) * N;
  const bool value = !qk && col >= 0 && col < s.h_kv * d;
  uint4 a[16];
  auto load = [&](int t0) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const T* y = src + (size_t)min(t0 + t, n - 1) * width + head * d;
      a[t] = *reinterpret_cast<const uint4*>(y + c0);
      a[8 + t] = *reinterpret_cast<const uint4*>(y + c1);
    }
  };
  if (qk) {
    load(0);
  } else if (value) {
#pragma unroll
    for (int t = 0; t < 16; ++t)
      a[t] = *reinterpret_cast<const uint4*>(src + (size_t)min(t, n - 1) * width + nqk * d + col);
  }
  for (int i = tid; i < n * pairs; i += 256) {
    const int t = i / pairs, pair = i - t * pairs;
    const int p = s.positions ? s.positions[(size_t)s.pair_axis[pair] * s.tokens + row + t] : pos + t;
    turn[t][pair] = cos_sin_of(p * s.turns[pair]);
  }
  __syncthreads();
  if (qk) {
    const bool is_q = head < s.h_q;
    if (!is_q && !ok) return;
    const T* w = static_cast<const T*>(is_q ? x.wq : x.wk);
    float w0[N], w1[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      w0[e] = w ? static_cast<float>(w[c0 + e]) : 1.f;
      w1[e] = w ? static_cast<float>(w[c1 + e]) : 1.f;
    }
    const size_t slab = (size_t)id * s.h_kv + head - s.h_q;
    auto one = [&](int t, int t0) {
      const Chunk<T> v0 = __builtin_bit_cast(Chunk<T>, a[t]), v1 = __builtin_bit_cast(Chunk<T>, a[8 + t]);
      float y0[N], y1[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y0[e] = static_cast<float>(v0.v[e]), y1[e] = static_cast<float>(v1.v[e]);
      if (x.norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) sum = fmaf(y0[e], y0[e], fmaf(y1[e], y1[e], sum));
        sum = over_lanes(sum, units, add);
        const float inv = 1.f / sqrtf(sum / d + x.eps);
#pragma unroll
        for (int e = 0; e < N; ++e) y0[e] *= inv * w0[e], y1[e] *= inv * w1[e];
      }
      const float2* turns = turn[t0 + t];
      if constexpr (ADJACENT) {
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          if (c0 < s.rot_dim) {
            const float2 z = turns[(c0 + e) / 2];
            const float p = y0[e], q = y0[e + 1];
            y0[e] = p * z.x - q * z.y, y0[e + 1] = p * z.y + q * z.x;
          }
          if (c1 < s.rot_dim) {
            const float2 z = turns[(c1 + e) / 2];
            const float p = y1[e], q = y1[e + 1];
            y1[e] = p * z.x - q * z.y, y1[e + 1] = p * z.y + q * z.x;
          }
        }
      } else if (together) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 z = turns[c0 + e];
          const float p = y0[e], q = y1[e];
          y0[e] = p * z.x - q * z.y, y1[e] = p * z.y + q * z.x;
        }
      }
      if constexpr (EIGHT) {
        if (!is_q) {
          float m = 0.f;
#pragma unroll
          for (int e = 0; e < N; ++e) m = fmaxf(m, fmaxf(finite_size(y0[e]), finite_size(y1[e])));
          m = over_lanes(m, units, most);
          const int byte = scale_byte(m);
          const float inv = inverse_scale(byte);
          int2 b0, b1;
          b0.x = packed8<true>(y0[2], y0[3], inv, packed8<false>(y0[0], y0[1], inv, 0));
          b0.y = packed8<true>(y0[6], y0[7], inv, packed8<false>(y0[4], y0[5], inv, 0));
          b1.x = packed8<true>(y1[2], y1[3], inv, packed8<false>(y1[0], y1[1], inv, 0));
          b1.y = packed8<true>(y1[6], y1[7], inv, packed8<false>(y1[4], y1[5], inv, 0));
          uint8_t* y = static_cast<uint8_t*>(s.k_cache) + (slab * 16 + slot + t0 + t) * d;
          *reinterpret_cast<int2*>(y + c0) = b0;
          *reinterpret_cast<int2*>(y + c1) = b1;
          if (k == 0) x.scales[slab * 32 + slot + t0 + t] = (uint8_t)byte;
          return;
        }
      }
      Chunk<T> o0, o1;
#pragma unroll
      for (int e = 0; e < N; ++e) o0.v[e] = static_cast<T>(y0[e]), o1.v[e] = static_cast<T>(y1[e]);
      T* y = is_q ? static_cast<T*>(s.q) + ((size_t)(row + t0 + t) * s.h_q + head) * d
                  : static_cast<T*>(s.k_cache) + (slab * 16 + slot + t0 + t) * d;
      *reinterpret_cast<uint4*>(y + c0) = __builtin_bit_cast(uint4, o0);
      *reinterpret_cast<uint4*>(y + c1) = __builtin_bit_cast(uint4, o1);
    };
    for (int t0 = 0; t0 < n; t0 += 8) {
      if (t0) load(t0);
#pragma unroll
      for (int t = 0; t < 8; ++t)
        if (t0 + t < n) one(t, t0);
    }
    return;
  }
  if (!value || !ok) return;
  const size_t slab = (size_t)id * s.h_kv + col / d;
  Chunk<T> v[16];
#pragma unroll
  for (int t = 0; t < 16; ++t) v[t] = __builtin_bit_cast(Chunk<T>, a[t]);
  if constexpr (EIGHT) {
    uint8_t* y = static_cast<uint8_t*>(s.v_cache) + (slab * d + col % d) * 16 + slot;
    float inv[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, finite_size(static_cast<float>(v[t].v[e])));
      m = over_lanes(m, d / N, most);
      const int byte = scale_byte(m);
      inv[t] = inverse_scale(byte);
      if (col % d == 0 && t < n) x.scales[slab * 32 + 16 + slot + t] = (uint8_t)byte;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      int p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        auto at8 = [&](int t) { const float f = static_cast<float>(v[t].v[e]); return fmaf(f, 0.f, f * inv[t]); };
        p[i] = __builtin_amdgcn_cvt_pk_fp8_f32(at8(4 * i), at8(4 * i + 1), 0, false);
        p[i] = __builtin_amdgcn_cvt_pk_fp8_f32(at8(4 * i + 2), at8(4 * i + 3), p[i], true);
      }
      if (n == 16) {
        *reinterpret_cast<int4*>(y + e * 16) = make_int4(p[0], p[1], p[2], p[3]);
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (t < n) y[e * 16 + t] = (uint8_t)(p[t / 4] >> (8 * (t % 4)));
      }
    }
  } else {
    T* y = static_cast<T*>(s.v_cache) + (slab * d + col % d) * 16 + slot;
    if (n < 16) {
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t < n)
#pragma unroll
          for (int e = 0; e < N; ++e) y[e * 16 + t] = v[t].v[e];
      return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
      for (int t = 0; t < 16; t += N) {
        Chunk<T> o;
#pragma unroll
        for (int i = 0; i < N; ++i) o.v[i] = v[t + i].v[e];
        *reinterpret_cast<uint4*>(y + e * 16 + t) = __builtin_bit_cast(uint4, o);
      }
  }
}

template <typename T, bool ADJACENT, bool EIGHT>
hipError_t launch(const NormSplitArgs& x, const int4* requests, hipStream_t s) {
  const RopeSplitArgs& a = x.rope;
  const int n = 16 / sizeof(T), d = a.head_dim;
  const int units = (((a.h_q + a.h_kv) * d / (2 * n) + 15) & ~15) + a.h_kv * d / n;
  const int groups = a.tokens / 16 + 2 * a.num_reqs, columns = (units + 255) / 256;
  if (a.num_reqs <= kRopeTable) {
    Passed p;
    for (int r = 0; r < a.num_reqs; ++r) p.at[r] = make_int2(requests[r].y, requests[r].w);
    p.at[a.num_reqs] = make_int2(a.tokens, 0);
    hipLaunchKernelGGL((norm_split<T, ADJACENT, EIGHT, Passed>), dim3(groups + (a.err ? 1 : 0), columns), dim3(256), 0, s, x, p);
  } else {
    hipLaunchKernelGGL((norm_split<T, ADJACENT, EIGHT, Uploaded>), dim3(groups, columns), dim3(256), 0, s, x, Uploaded{a.meta});
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_split(const NormSplitArgs& x, const int4* requests, hipStream_t s) {
  const RopeSplitArgs& a = x.rope;
  if (a.tokens <= 0 && !a.err) return hipSuccess;  // with an error word one workgroup clears that
  if (x.scales) return a.adjacent ? launch<__bf16, true, true>(x, requests, s) : launch<__bf16, false, true>(x, requests, s);
  if (a.dtype == DUET_BF16)
    return a.adjacent ? launch<__bf16, true, false>(x, requests, s) : launch<__bf16, false, false>(x, requests, s);
  return a.adjacent ? launch<float, true, false>(x, requests, s) : launch<float, false, false>(x, requests, s);
}

}  // namespace duet
