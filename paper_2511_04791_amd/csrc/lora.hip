// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale_a B_a (A_a x[t]),  a the adapter of token t's request.
// Two kernels: h = A_a x in fp32 parts into the workspace, then out = base + scale_a B_a h with one rounding to bf16.
// Both are bound by memory: x, base and out pass once, the adapters are a few MB.
//
// Rows of one adapter, wherever in the batch they stand, are taken in tiles of up to kTileRows, so its weights are
// read once a tile and a decode batch of a few adapters costs a few tiles.  Matrix products run on 16x16x32 MFMAs
// with the adapter's side as the first operand: a lane's four results are then neighbours of one row.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"
#include "wave_ops.h"

namespace duet {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRowTiles = kLoraTileRows / 16;
constexpr int kUnit = 64;  // input columns of a wave's step: 128 bytes of each row

__device__ __forceinline__ bf16x8 load8(const __bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }

// h of a tile over the columns of one part: four waves take its 64-column units in turn, each all of the tile's
// rows and ranks, and are summed through LDS in a fixed order.  NT: 16-rank tiles.
template <int NT>
__global__ __launch_bounds__(256) void lora_down(LoraArgs s) {
  __shared__ f32x4 sums[2][kRowTiles * NT][64];
  const LoraTile tile = s.tiles[blockIdx.x];
  if (tile.adapter < 0) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int units = (s.d_in + kUnit - 1) / kUnit;
  const int u1 = (int)((long long)units * (blockIdx.y + 1) / s.parts);
  const int row_tiles = (tile.count + 15) / 16;
  const __bf16* x[kRowTiles];
#pragma unroll
  for (int t = 0; t < kRowTiles; ++t) x[t] = s.x + s.rows[tile.first + min(16 * t + m, tile.count - 1)] * s.ldx + 8 * g;
  const __bf16* w[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) w[n] = s.a + ((size_t)tile.adapter * s.rank + min(16 * n + m, s.rank - 1)) * s.d_in + 8 * g;
  f32x4 acc[kRowTiles][NT] = {};
  for (int u = (int)((long long)units * blockIdx.y / s.parts) + wave; u < u1; u += 4) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int k = u * kUnit + 32 * half;
      const bool in = k + 8 * g < s.d_in;  // d_in is a multiple of 8
      bf16x8 wv[NT], xv[kRowTiles];
#pragma unroll
      for (int n = 0; n < NT; ++n) wv[n] = in ? load8(w[n] + k) : zero8();
#pragma unroll
      for (int t = 0; t < kRowTiles; ++t) xv[t] = in && t < row_tiles ? load8(x[t] + k) : zero8();
#pragma unroll
      for (int t = 0; t < kRowTiles; ++t)
        if (t < row_tiles)
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[n], xv[t], acc[t][n], 0, 0, 0);
    }
  }
  auto put = [&](int b) {
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (t < row_tiles) sums[b][t * NT + n][lane] = acc[t][n];
  };
  auto add = [&](int b) {
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (t < row_tiles) acc[t][n] += sums[b][t * NT + n][lane];
  };
  if (wave >= 2) put(wave - 2);
  __syncthreads();
  if (wave < 2) add(wave);
  __syncthreads();
  if (wave == 1) put(0);
  __syncthreads();
  if (wave) return;
  add(0);
  float* h = s.h + ((size_t)blockIdx.y * s.tokens + tile.first) * s.rank;
#pragma unroll
  for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (16 * t + m < tile.count && 16 * n + 4 * g < s.rank)
        *reinterpret_cast<f32x4*>(h + (size_t)(16 * t + m) * s.rank + 16 * n + 4 * g) = acc[t][n];
}

// out of a tile, 64 columns a wave at a time.  h is summed over its parts, scaled and held in LDS as two bf16 (its
// value and what that leaves out: 16 bits together), side by side along the product's axis: [h_hi | h_lo] times
// [B | B].  The 16 columns of an MFMA are taken in fours out of 32, so that two MFMAs give a lane eight neighbours.
__global__ __launch_bounds__(256) void lora_up(LoraArgs s) {
  extern __shared__ __align__(16) __bf16 hs[];  // [kLoraTileRows][stride]
  const LoraTile tile = s.tiles[blockIdx.x];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int chunks = s.rank / 8, steps = (2 * chunks + 3) / 4, stride = steps * 32 + 8;
  const int row_tiles = (tile.count + 15) / 16;
  if (tile.adapter >= 0) {
    const float scale = s.scale ? s.scale[tile.adapter] : 1.f;
    for (int i = threadIdx.x; i < row_tiles * 16 * steps * 32; i += 256) {
      const int row = i / (steps * 32), c = i % (steps * 32);
      if (c < s.rank) {
        float h = 0.f;
        if (row < tile.count)
          for (int p = 0; p < s.parts; ++p) h += s.h[((size_t)p * s.tokens + tile.first + row) * s.rank + c];
        h *= scale;
        const __bf16 hi = static_cast<__bf16>(h);
        hs[row * stride + c] = hi;
        hs[row * stride + s.rank + c] = static_cast<__bf16>(__builtin_isfinite(h) ? h - static_cast<float>(hi) : 0.f);
      } else if (c >= 2 * s.rank) {
        hs[row * stride + c] = static_cast<__bf16>(0.f);
      }
    }
  }
  __syncthreads();
  long long row[kRowTiles];
#pragma unroll
  for (int t = 0; t < kRowTiles; ++t) row[t] = s.rows[tile.first + min(16 * t + m, tile.count - 1)];
  const __bf16* w = s.b + (size_t)max(tile.adapter, 0) * s.d_out * s.rank;
  for (int c0 = (blockIdx.y * 4 + wave) * 64; c0 < s.d_out; c0 += gridDim.y * 256) {
    bf16x8 base[kRowTiles][2];
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int c = c0 + 32 * p + 8 * g;
        if (16 * t + m < tile.count && c < s.d_out) base[t][p] = load8(s.base + row[t] * s.ldb + c);
      }
    f32x4 acc[kRowTiles][4] = {};
    if (tile.adapter >= 0) {
      for (int st = 0; st < steps; ++st) {
        const int q = 4 * st + g;
        bf16x8 wv[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int c = c0 + 32 * (n / 2) + 8 * (m / 4) + 4 * (n % 2) + m % 4;
          wv[n] = q < 2 * chunks && c < s.d_out ? load8(w + (size_t)c * s.rank + 8 * (q < chunks ? q : q - chunks)) : zero8();
        }
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t)
          if (t < row_tiles) {
            const bf16x8 hv = load8(hs + (16 * t + m) * stride + 8 * q);
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[n], hv, acc[t][n], 0, 0, 0);
          }
      }
    }
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int c = c0 + 32 * p + 8 * g;
        if (16 * t + m >= tile.count || c >= s.d_out) continue;
        bf16x8 o = base[t][p];
        if (tile.adapter >= 0)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            o[e] = static_cast<__bf16>(static_cast<float>(base[t][p][e]) + acc[t][2 * p + e / 4][e % 4]);
        *reinterpret_cast<bf16x8*>(s.out + row[t] * s.ldo + c) = o;
      }
  }
}

}  // namespace

int lora_parts(int tokens, int d_in) {
  const int tiles = (tokens + kLoraTileRows - 1) / kLoraTileRows, units = (d_in + kUnit - 1) / kUnit;
  return std::max(1, std::min({16, 512 / std::max(tiles, 1), (units + 3) / 4}));
}

hipError_t launch_lora(const LoraArgs& a, hipStream_t s) {
  if (a.n_tiles <= 0) return hipSuccess;
  const dim3 down(a.n_tiles, a.parts), block(256);
  if (a.rank <= 16) hipLaunchKernelGGL(lora_down<1>, down, block, 0, s, a);
  else if (a.rank <= 32) hipLaunchKernelGGL(lora_down<2>, down, block, 0, s, a);
  else if (a.rank <= 64) hipLaunchKernelGGL(lora_down<4>, down, block, 0, s, a);
  else hipLaunchKernelGGL(lora_down<8>, down, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int steps = (a.rank / 4 + 3) / 4;
  const int blocks = (a.d_out + 255) / 256;
  const dim3 up(a.n_tiles, std::max(1, std::min(blocks, 2048 / a.n_tiles)));
  hipLaunchKernelGGL(lora_up, up, block, kLoraTileRows * (steps * 32 + 8) * sizeof(__bf16), s, a);
  return hipGetLastError();
}

}  // namespace duet
