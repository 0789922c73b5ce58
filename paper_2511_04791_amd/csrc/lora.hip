// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale_a B_a (A_a x[t]),  a the adapter of token t's request.
// Two kernels: h = scale_a A_a x in fp32 into the workspace, then out = base + B_a h with one rounding.
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "wave_ops.h"

namespace duet {
namespace {

__device__ __forceinline__ int4 request_of(const LoraArgs& s, int row) {
  return s.reqs[uniform(find_request(s.num_reqs, [&](int x) { return s.reqs[x].y <= row; }))];
}

// One workgroup per row, a wave per rank.
__global__ __launch_bounds__(256) void lora_down(LoraArgs s) {
  const int row = blockIdx.x, lane = threadIdx.x & 63, a = request_of(s, row).x;
  if (a < 0) return;
  const __bf16* x = s.x + (size_t)row * s.ldx;
  for (int r = threadIdx.x >> 6; r < s.rank; r += 4) {
    const __bf16* w = s.a + ((size_t)a * s.rank + r) * s.d_in;
    float sum = 0.f;
    for (int i = lane; i < s.d_in; i += 64) sum += static_cast<float>(x[i]) * static_cast<float>(w[i]);
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
    if (lane == 0) s.h[(size_t)row * s.rank + r] = sum * (s.scale ? s.scale[a] : 1.f);
  }
}

// One workgroup per row, a thread per column.
__global__ __launch_bounds__(256) void lora_up(LoraArgs s) {
  const int row = blockIdx.x, a = request_of(s, row).x;
  const float* h = s.h + (size_t)row * s.rank;
  for (int c = threadIdx.x; c < s.d_out; c += 256) {
    const __bf16 base = s.base[(size_t)row * s.ldb + c];
    float sum = static_cast<float>(base);
    if (a >= 0)
      for (int r = 0; r < s.rank; ++r) sum += h[r] * static_cast<float>(s.b[((size_t)a * s.d_out + c) * s.rank + r]);
    s.out[(size_t)row * s.ldo + c] = a >= 0 ? static_cast<__bf16>(sum) : base;
  }
}

}  // namespace

hipError_t launch_lora(const LoraArgs& a, hipStream_t s) {
  if (a.tokens <= 0) return hipSuccess;
  hipLaunchKernelGGL(lora_down, dim3(a.tokens), dim3(256), 0, s, a);
  hipLaunchKernelGGL(lora_up, dim3(a.tokens), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace duet
