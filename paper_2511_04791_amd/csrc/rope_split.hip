// The QKV split with the position rotation on the way (rotary position embedding): the query and key
// rows of the projection are turned by their token's position, keys and values enter the paged cache.
//
// A pair (a, b) of a head's row turns by t = p f: a' = a cos t - b sin t, b' = a sin t + b cos t, with p the
// position of the token on the pair's axis and f the pair's frequency.  Dimensions past rot_dim and
// values are copied.  p f / 2 pi is formed in 64 bits (at position 100000 the product alone would lose
// 2^-8 of a radian in 32) and brought within an eighth of a turn of a quarter there; sine, cosine and the
// rotation are 32-bit, with one rounding to the stored type.
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
  switch ((int)(quarter - 4.0 * floor(0.25 * quarter))) {
    case 0: return make_float2(c, s);
    case 1: return make_float2(-s, c);
    case 2: return make_float2(-c, -s);
    default: return make_float2(s, -c);
  }
}

// One workgroup per row, a thread per column.
template <typename T>
__global__ __launch_bounds__(256) void rope_split(RopeSplitArgs s) {
  const int row = blockIdx.x, d = s.head_dim, nq = s.h_q * d, nk = s.h_kv * d, half = s.rot_dim / 2;
  const int r = uniform(find_request(s.num_reqs, [&](int x) { return s.meta[x].y <= row; }));
  const int4 m = s.meta[r];
  const int pos = m.w + row - m.y, slot = pos & 15;
  const int id = s.page_table[(size_t)r * s.max_pages + (pos >> 4)];
  const bool ok = page_ok(id, s.num_phys_pages);
  if (!ok && threadIdx.x == 0) atomicOr(s.err, 1);
  const T* x = static_cast<const T*>(s.qkv) + (size_t)row * (nq + 2 * nk);
  for (int col = threadIdx.x; col < nq + 2 * nk; col += 256) {
    const int e = col % d;
    T y = x[col];
    if (col < nq + nk && e < s.rot_dim) {
      const int pair = s.adjacent ? e / 2 : e % half;
      const bool first = s.adjacent ? e % 2 == 0 : e < half;
      const int step = s.adjacent ? 1 : half;
      const int p = s.positions ? s.positions[(size_t)s.pair_axis[pair] * s.tokens + row] : pos;
      const float2 t = cos_sin_of(p * s.turns[pair]);
      const float a = static_cast<float>(x[first ? col : col - step]), b = static_cast<float>(x[first ? col + step : col]);
      y = static_cast<T>(first ? a * t.x - b * t.y : a * t.y + b * t.x);
    }
    if (col < nq) {
      static_cast<T*>(s.q)[(size_t)row * nq + col] = y;
    } else if (ok) {
      const int head = (col - nq) / d % s.h_kv;
      if (col < nq + nk) static_cast<T*>(s.k_cache)[(((size_t)id * s.h_kv + head) * 16 + slot) * d + e] = y;
      else static_cast<T*>(s.v_cache)[(((size_t)id * s.h_kv + head) * d + e) * 16 + slot] = y;
    }
  }
}

}  // namespace

hipError_t launch_rope_split(const RopeSplitArgs& a, hipStream_t s) {
  if (a.tokens <= 0) return hipSuccess;
  if (a.dtype == DUET_BF16) hipLaunchKernelGGL(rope_split<__bf16>, dim3(a.tokens), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rope_split<float>, dim3(a.tokens), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace duet
