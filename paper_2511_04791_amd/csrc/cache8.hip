// Pages of the 8-bit cache read back into bf16 pages: a value is e4m3 times its token's power of two, which bf16 holds exactly
// (four significant bits), past its largest as infinity, under its smallest normal one rounded.
//
// Bound by memory: 2 d + 2 bytes of a token and head read, 4 d written.  A workgroup takes a part of a logical page of a request; a
// thread's piece is 8 bytes in and 16 out, so that neighbours write neighbouring chunks: 8 values of a key's row, or 8 tokens of a
// dimension of values.  Its four pieces' loads go out together.
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

template <int kPieces, typename Table>
__global__ __launch_bounds__(256) void cache8_read(Cache8ReadArgs a, Table reqs) {
  const int group = blockIdx.x;
  const int r = uniform(find_request(a.num_reqs, [&](int i) { return reqs[i].x <= group; }));
  const int2 at = reqs[r];
  const int page = group - at.x, n = min(16, at.y - 16 * page);
  if (n <= 0) return;
  const int id = a.table[(size_t)r * a.max_pages + page], to = a.out_table[(size_t)r * a.out_max_pages + page];
  if (!page_ok(id, a.pages) || !page_ok(to, a.out_pages)) {
    if (a.err && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(a.err, 1);
    return;
  }
  const int d = a.head_dim, all = a.h_kv * 4 * d;
  uint2 x[kPieces], e[kPieces];
  auto piece = [&](int i) { return (int)(blockIdx.y * kPieces + i) * 256 + (int)threadIdx.x; };
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int u = min(piece(i), all - 1), head = u / (4 * d), w = u - head * 4 * d;  // 2 d pieces of keys, then of values
    const bool key = w < 2 * d;
    const int at8 = (key ? w : w - 2 * d) * 8;
    const size_t from = (size_t)id * a.h_kv + head;
    x[i] = *reinterpret_cast<const uint2*>((key ? a.k : a.v) + from * 16 * d + at8);
    const uint8_t* scales = a.scales + from * 32;
    if (key) e[i].x = scales[at8 / d];
    else e[i] = *reinterpret_cast<const uint2*>(scales + 16 + (at8 & 8));
  }
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    if (piece(i) >= all) break;
    const int u = piece(i), head = u / (4 * d), w = u - head * 4 * d;
    const bool key = w < 2 * d;
    const int at8 = (key ? w : w - 2 * d) * 8;
    const int token = key ? at8 / d : at8 & 8;
    if (token >= n) continue;
    float f[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(j ? x[i].y : x[i].x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(j ? x[i].y : x[i].x, true);
      f[4 * j] = lo[0], f[4 * j + 1] = lo[1], f[4 * j + 2] = hi[0], f[4 * j + 3] = hi[1];
    }
    struct Row {
      __bf16 v[8];
    } o;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned byte = key ? e[i].x : (j < 4 ? e[i].x : e[i].y) >> (8 * (j % 4)) & 255;
      o.v[j] = static_cast<__bf16>(f[j] * power(byte));
    }
    __bf16* y = (key ? a.k_out : a.v_out) + ((size_t)to * a.h_kv + head) * 16 * d + at8;
    if (key || token + 8 <= n) {
      *reinterpret_cast<uint4*>(y) = __builtin_bit_cast(uint4, o);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (token + j < n) y[j] = o.v[j];
    }
  }
}

// Two pieces a thread where four would leave fewer than four workgroups a CU: one prompt of 100 tokens, 8 heads, 3.9 us against 5.2;
// 32768 tokens 53.8 against 48.3 (202 MB, 4.2 TB/s; a large copy reaches 5.1), with eight 48.2.  Pieces of 16 bytes in and 32 out, whose
// stores leave every other chunk to the next, took 66; a page's workgroups next to each other the same 48.
template <int P, typename Table>
void launch_pieces(const Cache8ReadArgs& a, const Table& t, hipStream_t s) {
  const dim3 grid(a.groups, (a.h_kv * 4 * a.head_dim + 256 * P - 1) / (256 * P));
  hipLaunchKernelGGL((cache8_read<P, Table>), grid, dim3(256), 0, s, a, t);
}
template <typename Table>
hipError_t launch(const Cache8ReadArgs& a, const Table& t, hipStream_t s) {
  if ((long long)a.groups * a.h_kv * a.head_dim < 4 * 256 * 256) launch_pieces<2>(a, t, s);
  else launch_pieces<4>(a, t, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache8_read(const Cache8ReadArgs& a, const int2* reqs, hipStream_t s) {
  if (a.groups <= 0) return hipSuccess;
  if (reqs) {
    PassedPages p;
    for (int r = 0; r <= a.num_reqs; ++r) p.at[r] = reqs[r];
    return launch(a, p, s);
  }
  return launch(a, UploadedPages{a.reqs}, s);
}

}  // namespace duet
