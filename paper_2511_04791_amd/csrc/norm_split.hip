// The QKV split with a norm of each head and the position rotation on the way, into pages of the projection's type or
// into 8-bit ones.
//
// A head's row x of a query or key becomes y = x w / sqrt(mean(x^2) + eps), in 32 bits, then its pairs turn as in
// rope_split.hip; values are copied.  8-bit pages hold e4m3 values times a power of two that the d values of a token's
// head share: the smallest that brings the largest of them to 448, e4m3's largest, so the exponent follows from the bits of
// the largest value and the division is exact; one rounding in all, after the rotation.
//
// Bound by memory: the projection is read once, queries and pages are written.  The rows of one request on one page go to a group of
// workgroups; a thread takes two 16-byte chunks of a head for two or four of the rows, or eight columns of values for all of them, which
// whole pages need turned around.  A head's row lies in 4 to 16 neighbouring lanes, and its sum or maximum is taken by moves inside a
// row of 16 lanes.  With all sixteen rows of queries and keys a thread, as rope_split.hip has it, a small batch waited for one chain of
// norms (five chunks on a rank, 2588 rows, into 8 bits 25 us; now 7.7) and few waves fitted (8224 rows of 64 + 2 x 8 heads 90 us; now
// 71, 4.7 TB/s; a large copy reaches 5.1).  8192 rows of 32 + 2 x 8 heads into 8 bits 39 us (4.7 TB/s); one decode row 4.5.
//
// Values are converted two of a row at a time, as the row shares the power, and turned as bytes; magnitudes of bf16 are compared
// as their bits, two in a register.  Both took a third of the instructions of a value at a time.  A page that is covered in part gets
// whole words where four slots are new, else bytes.  Requests of one row each need no search for their group.
#include <hip/hip_runtime.h>

#include <algorithm>
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

// The exponent's byte of a row whose largest finite magnitude has these upper bits (fp32's, or bf16's alone): 448 is 1.75 2^8, so the
// power is 2^(exponent - 8), or the next where the fraction is above 0.75.  At least 2^-126.
__device__ __forceinline__ int scale_byte(float m) { return max((int)((__float_as_uint(m) + 0x1fffffu) >> 23) - 8, 1); }
__device__ __forceinline__ int scale_byte_bf16(unsigned m) { return max((int)((m + 0x1fu) >> 7) - 8, 1); }
__device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)e << 23); }
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

// Values over a power of two as e4m3, two in the low or high half of `old`: rounded to even, what is not finite as NaN.
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned four8(float a, float b, float c, float d, float scale) {
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true));
}
__device__ __forceinline__ unsigned four8(unsigned ab, unsigned cd, float scale) {  // of bf16
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, ab), scale, false);
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, cd), scale, true));
}

// bf16 magnitudes are ordered as their bits.
__device__ __forceinline__ unsigned pk_max(unsigned a, unsigned b) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ unsigned largest(const uint4& x) {  // of eight, in the low half
  const unsigned m = pk_max(pk_max(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), pk_max(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ unsigned finite16(unsigned x) {  // two magnitudes, what is not finite as 0
  const unsigned lo = x & 0x7fffu, hi = x >> 16 & 0x7fffu;
  return (lo < 0x7f80u ? lo : 0) | (hi < 0x7f80u ? hi : 0) << 16;
}
__device__ __forceinline__ unsigned largest_finite(const uint4& x) {
  return largest(make_uint4(finite16(x.x), finite16(x.y), finite16(x.z), finite16(x.w)));
}
template <int CTRL>
__device__ __forceinline__ unsigned moved_bits(unsigned x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ unsigned pk_max_over_lanes(unsigned x, int lanes) {  // 8 or 16 of them, as over_lanes
  x = pk_max(x, moved_bits<0xB1>(x));
  x = pk_max(x, moved_bits<0x4E>(x));
  x = pk_max(x, moved_bits<0x141>(x));
  return lanes >= 16 ? pk_max(x, moved_bits<0x140>(x)) : x;
}

// The workgroups of a group next to each other, so that rows are read from one end to the other: 8224 rows of 64 + 2 x 8 heads 71 us, 78
// with the groups next to each other; 8192 rows of 32 + 2 x 8 into 8 bits 41 against 46.
constexpr int kGridY = 32768;
dim3 grid_of(int columns, int groups) { return dim3(columns, std::min(groups, kGridY), (groups + kGridY - 1) / kGridY); }

template <typename T, bool ADJACENT, bool EIGHT, int kRows, typename Table>
__global__ __launch_bounds__(256, EIGHT ? 4 : 3) void norm_split(NormSplitArgs x, Table requests) {
  constexpr int N = Chunk<T>::N;
  constexpr bool kPassed = std::is_same<Table, Passed>::value;
  __shared__ float2 turn[16][kMaxPairs];
  const RopeSplitArgs& s = x.rope;
  const int d = s.head_dim, pairs = s.rot_dim / 2, tid = threadIdx.x;
  int group = blockIdx.z * kGridY + blockIdx.y;
  if (group >= x.groups) return;
  if (kPassed && s.err) {
    if (group == 0) {
      if constexpr (kPassed)
        if (blockIdx.x == 0) check_pages(s, requests, reinterpret_cast<int2*>(turn));
      return;
    }
    --group;
  }
  int r = group;  // one row a request: one group each
  Group at;
  if (x.single) {
    const Request q = requests[r];
    at = Group{q.row, q.cached, 1, q.cached >> 4};
  } else {
    r = uniform(find_request(s.num_reqs, [&](int i) { return first_group(requests.row(i), i) <= group; }));
    at = group_of(requests[r], r, group);
  }
  const int n = at.rows, pos = at.pos, row = at.row, slot = pos & 15;
  if (n <= 0) return;
  const int id = s.page_table[(size_t)r * s.max_pages + at.page];
  const bool ok = page_ok(id, s.num_phys_pages);
  if (!kPassed && !ok && blockIdx.x == 0 && tid == 0) atomicOr(s.err, 1);
  // A thread's unit: of queries and keys two chunks of kRows rows, neighbours in the row first; after those of all the page's
  // rows, and from a multiple of 16 on, so that a head's lie in one row of lanes, eight columns of values, all rows.
  const int units = d / (2 * N), nqk = s.h_q + s.h_kv, width = (nqk + s.h_kv) * d;
  const int qk_units = nqk * units, v_units = (qk_units * x.parts + 15) & ~15, u = blockIdx.x * 256 + tid;
  const T* src = static_cast<const T*>(s.qkv) + (size_t)row * width;
  const bool qk = u < qk_units * x.parts;
  const int part = u / qk_units, unit = u - part * qk_units, t0 = kRows * part;
  const int head = unit / units, k = unit - head * units;
  const bool together = !ADJACENT && k < pairs / N;
  const int from = ADJACENT || together ? 0 : s.rot_dim - pairs, half = ADJACENT ? d / 2 : together ? pairs : (d - s.rot_dim) / 2;
  const int c0 = from + k * N, c1 = c0 + half;
  const int col = (u - v_units) * N;
  const bool value = !qk && col >= 0 && col < s.h_kv * d;
  const bool there = qk && t0 < n;
  uint4 a[16];
  if (there && n == 1) {
    a[0] = *reinterpret_cast<const uint4*>(src + head * d + c0);
    a[kRows] = *reinterpret_cast<const uint4*>(src + head * d + c1);
  } else if (there) {
    const T* y = src + (size_t)t0 * width + head * d;
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const T* z = y + (size_t)min(t, n - 1 - t0) * width;
      a[t] = *reinterpret_cast<const uint4*>(z + c0);
      a[kRows + t] = *reinterpret_cast<const uint4*>(z + c1);
    }
  } else if (value && n == 1) {
    a[0] = *reinterpret_cast<const uint4*>(src + nqk * d + col);
  } else if (value) {
#pragma unroll
    for (int t = 0; t < 16; ++t)  // by the page's slots
      a[t] = *reinterpret_cast<const uint4*>(src + (size_t)max(0, min(t - slot, n - 1)) * width + nqk * d + col);
  }
  // The sines of the rows that the workgroup's units of queries and keys have.
  const int first_row = kRows * (int)(blockIdx.x * 256 / qk_units);
  const int last_row = min(n, kRows * (min((int)blockIdx.x * 256 + 255, qk_units * x.parts - 1) / qk_units + 1));
  for (int i = tid + first_row * pairs; i < last_row * pairs; i += 256) {
    const int t = i / pairs, pair = i - t * pairs;
    const int p = s.positions ? s.positions[(size_t)s.pair_axis[pair] * s.tokens + row + t] : pos + t;
    turn[t][pair] = cos_sin_of(p * s.turns[pair]);
  }
  __syncthreads();
  if (qk) {
    const bool is_q = head < s.h_q;
    if (!there || (!is_q && !ok)) return;
    const T* w = static_cast<const T*>(is_q ? x.wq : x.wk);
    Chunk<T> w0, w1;
    if (w) {
      w0 = *reinterpret_cast<const Chunk<T>*>(w + c0);
      w1 = *reinterpret_cast<const Chunk<T>*>(w + c1);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) w0.v[e] = w1.v[e] = static_cast<T>(1.f);
    }
    const size_t slab = (size_t)id * s.h_kv + head - s.h_q;
    const float mean = 1.f / d;  // d is 64 or 128: exact
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      if (t0 + t >= n) break;
      __builtin_amdgcn_sched_barrier(0);  // a row at a time: the registers of all four together leave room for fewer waves
      const Chunk<T> v0 = __builtin_bit_cast(Chunk<T>, a[t]), v1 = __builtin_bit_cast(Chunk<T>, a[kRows + t]);
      float y0[N], y1[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y0[e] = static_cast<float>(v0.v[e]), y1[e] = static_cast<float>(v1.v[e]);
      if (x.norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) sum = fmaf(y0[e], y0[e], fmaf(y1[e], y1[e], sum));
        sum = over_lanes(sum, units, add);
        const float inv = __builtin_amdgcn_rsqf(fmaf(sum, mean, x.eps));
#pragma unroll
        for (int e = 0; e < N; ++e) y0[e] *= inv * static_cast<float>(w0.v[e]), y1[e] *= inv * static_cast<float>(w1.v[e]);
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
      const int token = slot + t0 + t;
      if (EIGHT && !is_q) {
        if constexpr (EIGHT) {
          float m = 0.f;
#pragma unroll
          for (int e = 0; e < N; ++e) m = fmaxf(m, fmaxf(fabsf(y0[e]), fabsf(y1[e])));
          if (__any(m == INFINITY)) {
            m = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) m = fmaxf(m, fmaxf(finite_size(y0[e]), finite_size(y1[e])));
          }
          m = over_lanes(m, units, most);
          const int byte = scale_byte(m);
          const float scale = power(byte);
          const uint2 b0 = make_uint2(four8(y0[0], y0[1], y0[2], y0[3], scale), four8(y0[4], y0[5], y0[6], y0[7], scale));
          const uint2 b1 = make_uint2(four8(y1[0], y1[1], y1[2], y1[3], scale), four8(y1[4], y1[5], y1[6], y1[7], scale));
          uint8_t* y = static_cast<uint8_t*>(s.k_cache) + (slab * 16 + token) * d;
          *reinterpret_cast<uint2*>(y + c0) = b0;
          *reinterpret_cast<uint2*>(y + c1) = b1;
          if (k == 0) x.scales[slab * 32 + token] = (uint8_t)byte;
        }
      } else {
        Chunk<T> o0, o1;
#pragma unroll
        for (int e = 0; e < N; ++e) o0.v[e] = static_cast<T>(y0[e]), o1.v[e] = static_cast<T>(y1[e]);
        T* y = is_q ? static_cast<T*>(s.q) + ((size_t)(row + t0 + t) * s.h_q + head) * d
                    : static_cast<T*>(s.k_cache) + (slab * 16 + token) * d;
        *reinterpret_cast<uint4*>(y + c0) = __builtin_bit_cast(uint4, o0);
        *reinterpret_cast<uint4*>(y + c1) = __builtin_bit_cast(uint4, o1);
      }
    }
    return;
  }
  if (!value || !ok) return;
  const size_t slab = (size_t)id * s.h_kv + col / d;
  if constexpr (EIGHT) {
    uint8_t* y = static_cast<uint8_t*>(s.v_cache) + (slab * d + col % d) * 16;
    uint8_t* bytes = x.scales + slab * 32 + 16;
    const bool first = col % d == 0;
    if (n == 1) {
      y += slot;
      bytes += slot;
      unsigned m = largest(a[0]);
      if (__any(m >= 0x7f80u)) m = largest_finite(a[0]);
      const int byte = scale_byte_bf16(pk_max_over_lanes(m, d / N));
      const unsigned w[2] = {four8(a[0].x, a[0].y, power(byte)), four8(a[0].z, a[0].w, power(byte))};
#pragma unroll
      for (int e = 0; e < N; ++e) y[e * 16] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
      if (first) *bytes = (uint8_t)byte;
      return;
    }
    // The rows' exponents, two rows a register.
    unsigned m[8], any = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      m[t] = largest(a[2 * t]) | largest(a[2 * t + 1]) << 16;
      any = pk_max(any, m[t]);
    }
    if (__any((any & 0xffffu) >= 0x7f80u || any >> 16 >= 0x7f80u)) {
#pragma unroll
      for (int t = 0; t < 8; ++t) m[t] = largest_finite(a[2 * t]) | largest_finite(a[2 * t + 1]) << 16;
    }
    unsigned e4[4];  // the bytes of four rows
    unsigned out[N][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int byte[4];
#pragma unroll
      for (int t = 0; t < 4; t += 2) {
        const unsigned both = pk_max_over_lanes(m[2 * i + t / 2], d / N);
        byte[t] = scale_byte_bf16(both & 0xffffu);
        byte[t + 1] = scale_byte_bf16(both >> 16);
      }
      e4[i] = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
      // Four rows of four columns in a register each, turned into a column's four rows each.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unsigned w[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint4 v = a[4 * i + t];
          w[t] = four8(h ? v.z : v.x, h ? v.w : v.y, power(byte[t]));
        }
        const unsigned lo01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
        const unsigned lo23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
        out[4 * h][i] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
        out[4 * h + 1][i] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
        out[4 * h + 2][i] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
        out[4 * h + 3][i] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
      }
    }
    if (n == 16) {
#pragma unroll
      for (int e = 0; e < N; ++e) *reinterpret_cast<uint4*>(y + e * 16) = make_uint4(out[e][0], out[e][1], out[e][2], out[e][3]);
      if (first) *reinterpret_cast<uint4*>(bytes) = make_uint4(e4[0], e4[1], e4[2], e4[3]);
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * i >= slot && 4 * i + 4 <= slot + n) {
#pragma unroll
        for (int e = 0; e < N; ++e) *reinterpret_cast<unsigned*>(y + e * 16 + 4 * i) = out[e][i];
        if (first) *reinterpret_cast<unsigned*>(bytes + 4 * i) = e4[i];
        continue;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (4 * i + t < slot || 4 * i + t >= slot + n) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e * 16 + 4 * i + t] = (uint8_t)(out[e][i] >> (8 * t));
        if (first) bytes[4 * i + t] = (uint8_t)(e4[i] >> (8 * t));
      }
    }
  } else {
    T* y = static_cast<T*>(s.v_cache) + (slab * d + col % d) * 16;
    if (n == 1) {
      const Chunk<T> v = __builtin_bit_cast(Chunk<T>, a[0]);
#pragma unroll
      for (int e = 0; e < N; ++e) y[e * 16 + slot] = v.v[e];
      return;
    }
    Chunk<T> v[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] = __builtin_bit_cast(Chunk<T>, a[t]);
#pragma unroll
    for (int t = 0; t < 16; t += N) {  // N slots of a column are 16 bytes
      if (t >= slot && t + N <= slot + n) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          Chunk<T> o;
#pragma unroll
          for (int i = 0; i < N; ++i) o.v[i] = v[t + i].v[e];
          *reinterpret_cast<uint4*>(y + e * 16 + t) = __builtin_bit_cast(uint4, o);
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (t + i < slot || t + i >= slot + n) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e * 16 + t + i] = v[t + i].v[e];
      }
    }
  }
}

// kRows rows of queries and keys a thread: into 8 bits two, else four, or two where that leaves fewer than four workgroups a CU.  us with
// 2 / 4: 8224 rows of 64 + 2 x 8 heads, bf16, 72.9 / 70.7; 8192 rows of 32 + 2 x 8 into 8 bits 39.0 / 41.5; 2588 rows of 8 + 2 x 1 into 8
// bits 7.6 / 11.1 (one row 8.3, eight 13.1).
template <typename T, bool ADJACENT, bool EIGHT, int kRows>
hipError_t launch_rows(NormSplitArgs x, int groups, int longest, const int4* requests, hipStream_t s) {
  const RopeSplitArgs& a = x.rope;
  const int n = 16 / sizeof(T), d = a.head_dim;
  x.parts = (std::min(longest, 16) + kRows - 1) / kRows;
  const int units = (((a.h_q + a.h_kv) * d / (2 * n) * x.parts + 15) & ~15) + a.h_kv * d / n;
  const int columns = (units + 255) / 256;
  const bool passed = a.num_reqs <= kRopeTable;
  x.groups = groups + (passed && a.err ? 1 : 0);  // the first clears the error word
  if (passed) {
    Passed p;
    for (int r = 0; r < a.num_reqs; ++r) p.at[r] = make_int2(requests[r].y, requests[r].w);
    p.at[a.num_reqs] = make_int2(a.tokens, 0);
    hipLaunchKernelGGL((norm_split<T, ADJACENT, EIGHT, kRows, Passed>), grid_of(columns, x.groups), dim3(256), 0, s, x, p);
  } else {
    hipLaunchKernelGGL((norm_split<T, ADJACENT, EIGHT, kRows, Uploaded>), grid_of(columns, x.groups), dim3(256), 0, s, x, Uploaded{a.meta});
  }
  return hipGetLastError();
}
template <typename T, bool ADJACENT, bool EIGHT>
hipError_t launch(NormSplitArgs x, const int4* requests, hipStream_t s) {
  const RopeSplitArgs& a = x.rope;
  int longest = 0;
  for (int r = 0; r < a.num_reqs; ++r) longest = std::max(longest, requests[r].z);
  x.single = longest == 1;
  const int groups = x.single ? a.num_reqs : a.tokens / 16 + 2 * a.num_reqs;
  const long long threads = (long long)groups * (a.h_q + a.h_kv) * a.head_dim * (int)sizeof(T) / 32 * ((std::min(longest, 16) + 3) / 4);
  if constexpr (!EIGHT)
    if (threads >= 4 * 256 * 256) return launch_rows<T, ADJACENT, EIGHT, 4>(x, groups, longest, requests, s);
  return launch_rows<T, ADJACENT, EIGHT, 2>(x, groups, longest, requests, s);
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
