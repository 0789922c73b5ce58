// Pages of the 8-bit cache read back into bf16 pages: a value is e4m3 times its token's power of two, which bf16 holds exactly
// (four significant bits), past its largest as infinity, under its smallest normal one rounded.
//
// Bound by memory: 2 d + 2 bytes of a token and head read, 4 d written.  A workgroup takes a logical page of a request, all
// heads; a thread 16 bytes at a time: 16 values of a key's row, or the 16 tokens of a dimension of values.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "cache_ops.h"
#include "wave_ops.h"

namespace duet {
namespace {

struct PassedPages {
  int2 at[kRopeTable + 1];
  __device__ __forceinline__ int2 operator[](int r) const { return at[r]; }
};
struct UploadedPages {
  const int2* at;
  __device__ __forceinline__ int2 operator[](int r) const { return at[r]; }
};

__device__ __forceinline__ float power(int byte) { return __uint_as_float((unsigned)byte << 23); }

template <typename Table>
__global__ __launch_bounds__(256) void cache8_read(Cache8ReadArgs a, Table reqs) {
  const int group = blockIdx.x;
  const int r = uniform(find_request(a.num_reqs, [&](int i) { return reqs[i].x <= group; }));
  const int2 at = reqs[r];
  const int page = group - at.x, n = min(16, at.y - 16 * page);
  if (n <= 0) return;
  const int id = a.table[(size_t)r * a.max_pages + page], to = a.out_table[(size_t)r * a.out_max_pages + page];
  if (!page_ok(id, a.pages) || !page_ok(to, a.out_pages)) {
    if (a.err && threadIdx.x == 0) atomicOr(a.err, 1);
    return;
  }
  const int d = a.head_dim, all = a.h_kv * 2 * d;  // 16-byte pieces
  for (int u = threadIdx.x; u < all; u += 256) {
    const int head = u / (2 * d), i = u - head * 2 * d;
    const bool key = i < d;
    const int piece = key ? i : i - d;
    const size_t from = (size_t)id * a.h_kv + head, slab = (size_t)to * a.h_kv + head;
    const uint4 x = *reinterpret_cast<const uint4*>((key ? a.k : a.v) + from * 16 * d + piece * 16);
    const uint8_t* scales = a.scales + from * 32;
    const unsigned w[4] = {x.x, x.y, x.z, x.w};
    float f[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], true);
      f[4 * j] = lo[0], f[4 * j + 1] = lo[1], f[4 * j + 2] = hi[0], f[4 * j + 3] = hi[1];
    }
    const int token = piece / (d / 16);
    if (key) {
      if (token >= n) continue;
      const float scale = power(scales[token]);
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] *= scale;
    } else {
      const uint4 b = *reinterpret_cast<const uint4*>(scales + 16);
      const unsigned e[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] *= power(e[j / 4] >> (8 * (j % 4)) & 255);
    }
    struct Row {
      __bf16 v[16];
    } o;
#pragma unroll
    for (int j = 0; j < 16; ++j) o.v[j] = static_cast<__bf16>(f[j]);
    __bf16* y = (key ? a.k_out : a.v_out) + slab * 16 * d + piece * 16;
    if (key || n == 16) {
      struct Two {
        uint4 v[2];
      };
      const Two t = __builtin_bit_cast(Two, o);
      reinterpret_cast<uint4*>(y)[0] = t.v[0];
      reinterpret_cast<uint4*>(y)[1] = t.v[1];
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j < n) y[j] = o.v[j];
    }
  }
}

}  // namespace

hipError_t launch_cache8_read(const Cache8ReadArgs& a, const int2* reqs, hipStream_t s) {
  if (a.groups <= 0) return hipSuccess;
  if (reqs) {
    PassedPages p;
    for (int r = 0; r <= a.num_reqs; ++r) p.at[r] = reqs[r];
    hipLaunchKernelGGL((cache8_read<PassedPages>), dim3(a.groups), dim3(256), 0, s, a, p);
  } else {
    hipLaunchKernelGGL((cache8_read<UploadedPages>), dim3(a.groups), dim3(256), 0, s, a, UploadedPages{a.reqs});
  }
  return hipGetLastError();
}

}  // namespace duet
