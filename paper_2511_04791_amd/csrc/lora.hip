// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale_a B_a (A_a x[t]),  a the adapter of token t's request.
// Two kernels: h = scale_a A_a x into the workspace, then out = base + B_a h with one rounding to bf16.
// Both are bound by memory: x, base and out pass once, the adapters are a few MB.
//
// Few rows and tiles (kLoraPassedRows, kLoraPassedTiles) travel with the launches' arguments and the second kernel adds the
// parts of h itself; otherwise they are uploaded, with the counters by which the last part to finish does: a third launch, which
// the host and the GPU pay for (64 rows of 16 adapters, 4096 to 6144 columns, rank 16: 20.5 us a call with it, 14.9 without).
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
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRowTiles = kLoraTileRows / 16;

__device__ __forceinline__ bf16x8 load8(const __bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }

// Four values that another workgroup, on whatever XCD, reads or wrote within the launch: device-scope accesses go
// past the XCD's L2, without the write-back and invalidation of all of it that a device-scope fence costs.
__device__ __forceinline__ void store_shared(float* p, f32x4 v) {
  const ulonglong2 u = __builtin_bit_cast(ulonglong2, v);
  unsigned long long* q = reinterpret_cast<unsigned long long*>(p);
  __hip_atomic_store(q, u.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(q + 1, u.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4 load_shared(const float* p) {
  const unsigned long long* q = reinterpret_cast<const unsigned long long*>(p);
  return __builtin_bit_cast(f32x4, make_ulonglong2(__hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                                                   __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
}

// The tiles and rows as the kernels read them.
struct Uploaded {
  static constexpr bool kPassed = false;
  const LoraTile* tiles;
  const int32_t* rows;
  __device__ __forceinline__ LoraTile tile(int i) const { return tiles[i]; }
  __device__ __forceinline__ int row(int i) const { return rows[i]; }
};
struct Passed {
  static constexpr bool kPassed = true;
  LoraTile tiles[kLoraPassedTiles];
  int32_t rows[kLoraPassedRows];
  __device__ __forceinline__ LoraTile tile(int i) const { return tiles[i]; }
  __device__ __forceinline__ int row(int i) const { return rows[i]; }
};

// h and what its rounding to bf16 leaves out (16 bits together).
__device__ __forceinline__ void split(float h, __bf16* hi, __bf16* lo) {
  *hi = static_cast<__bf16>(h);
  *lo = static_cast<__bf16>(__builtin_isfinite(h) ? h - static_cast<float>(*hi) : 0.f);
}

// Partial sums of h of a tile's 16 RT rows over the columns of one part: four waves take its units of kUnit columns in
// turn, each all of the rows and ranks (NT 16-rank tiles), and are summed through LDS in a fixed order.  A unit's
// loads are issued ahead of the products of the one before it.
template <int NT, int RT, typename Lists>
__device__ __forceinline__ void down_part(const LoraArgs& s, const Lists& lists, const LoraTile& tile, f32x4 (*sums)[kRowTiles * NT][64]) {
  constexpr int kHalves = NT == 8 ? 1 : 2, kUnit = 32 * kHalves;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int units = (s.d_in + kUnit - 1) / kUnit;
  const int u0 = (int)((long long)units * blockIdx.y / s.parts) + wave;
  const int u1 = (int)((long long)units * (blockIdx.y + 1) / s.parts);
  const __bf16 *x[RT], *w[NT];
#pragma unroll
  for (int t = 0; t < RT; ++t) x[t] = s.x + lists.row(tile.first + min(16 * t + m, tile.count - 1)) * s.ldx + 8 * g;
#pragma unroll
  for (int n = 0; n < NT; ++n) w[n] = s.a + ((size_t)tile.adapter * s.rank + min(16 * n + m, s.rank - 1)) * s.d_in + 8 * g;
  struct Unit {
    bf16x8 w[kHalves][NT], x[kHalves][RT];
  };
  f32x4 acc[RT][NT] = {};
  auto load = [&](int u, Unit& f) {
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
#pragma unroll
      for (int n = 0; n < NT; ++n) f.w[half][n] = load8(w[n] + u * kUnit + 32 * half);
#pragma unroll
      for (int t = 0; t < RT; ++t) f.x[half][t] = load8(x[t] + u * kUnit + 32 * half);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](const Unit& f) {
#pragma unroll
    for (int half = 0; half < kHalves; ++half)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.w[half][n], f.x[half][t], acc[t][n], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  const int whole = min(u1, s.d_in / kUnit);  // the last unit may be cut off, at a multiple of 8 columns
  if (u0 < whole) {
    const int n = (whole - u0 + 3) / 4;
    Unit even, odd;
    load(u0, even);
    for (int i = 0; i + 2 <= n; i += 2) {
      load(u0 + 4 * (i + 1), odd);
      multiply(even);
      load(u0 + 4 * min(i + 2, n - 1), even);
      multiply(odd);
    }
    if (n & 1) multiply(even);
  }
  if (whole < u1 && (whole - u0) % 4 == 0) {
    Unit cut;
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
      const int k = whole * kUnit + 32 * half;
      const bool in = k + 8 * g < s.d_in;
#pragma unroll
      for (int n = 0; n < NT; ++n) cut.w[half][n] = in ? load8(w[n] + k) : zero8();
#pragma unroll
      for (int t = 0; t < RT; ++t) cut.x[half][t] = in ? load8(x[t] + k) : zero8();
    }
    multiply(cut);
  }
  auto put = [&](int b) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n) sums[b][t * NT + n][lane] = acc[t][n];
  };
  auto add = [&](int b) {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[t][n] += sums[b][t * NT + n][lane];
  };
  if (wave >= 2) put(wave - 2);
  __syncthreads();
  if (wave < 2) add(wave);
  __syncthreads();
  if (wave == 1) put(0);
  __syncthreads();
  if (wave) return;
  add(0);
  float* part = s.part + ((size_t)blockIdx.y * s.tokens + tile.first) * s.rank;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (16 * t + m < tile.count && 16 * n + 4 * g < s.rank) {
        float* to = part + (size_t)(16 * t + m) * s.rank + 16 * n + 4 * g;
        if (Lists::kPassed) *reinterpret_cast<f32x4*>(to) = acc[t][n];
        else store_shared(to, acc[t][n]);
      }
}

// The part of a tile that finishes last adds all of them in their order and writes h for the second kernel: scaled, as
// two bf16 (its value and what that leaves out, 16 bits together).
template <int NT, typename Lists>
__global__ __launch_bounds__(256) void lora_down(LoraArgs s, Lists lists) {
  __shared__ f32x4 sums[2][kRowTiles * NT][64];
  __shared__ int last;
  const LoraTile tile = lists.tile(blockIdx.x);
  if (tile.adapter < 0) return;
  if (tile.count > 32) down_part<NT, 4>(s, lists, tile, sums);
  else if (tile.count > 16) down_part<NT, 2>(s, lists, tile, sums);
  else down_part<NT, 1>(s, lists, tile, sums);
  if (Lists::kPassed) return;
  if (threadIdx.x < 64) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's stores have completed
    if (threadIdx.x == 0) last = atomicAdd(s.done + blockIdx.x, 1) == s.parts - 1;
  }
  __syncthreads();
  if (!last) return;
  const float scale = s.scale ? s.scale[tile.adapter] : 1.f;
  const size_t step = (size_t)s.tokens * s.rank, at = (size_t)tile.first * s.rank;
  for (int i = threadIdx.x; i < tile.count * s.rank / 4; i += 256) {
    f32x4 v[kLoraMaxParts];
#pragma unroll
    for (int p = 0; p < kLoraMaxParts; ++p) v[p] = load_shared(s.part + min(p, s.parts - 1) * step + at + 4 * i);
    f32x4 h = v[0];
#pragma unroll
    for (int p = 1; p < kLoraMaxParts; ++p)
      if (p < s.parts) h += v[p];
    h *= scale;
    bf16x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      __bf16 a, b;
      split(h[e], &a, &b);
      hi[e] = a, lo[e] = b;
    }
    __bf16* to = s.h + (size_t)(tile.first + 4 * i / s.rank) * 2 * s.rank + 4 * i % s.rank;
    *reinterpret_cast<bf16x4*>(to) = hi;
    *reinterpret_cast<bf16x4*>(to + s.rank) = lo;
  }
}

// out of 16 RT rows of a tile from row0 on, 64 columns at a time, every col_step-th from col0 on.  Ranks up to 16 (STEPS 0)
// take h's two halves and B twice along one MFMA, [h_hi | h_lo] times [B | B]; others STEPS times 32 ranks, B for both
// halves.  The 16 columns of an MFMA are taken in fours out of 32, so that two MFMAs give a lane eight neighbours.  The next
// columns' base is read ahead of the products.
template <int STEPS, int RT, typename Lists>
__device__ __forceinline__ void up_rows(const LoraArgs& s, const Lists& lists, const LoraTile& tile, int row0, int col0, int col_step) {
  constexpr int kSteps = STEPS ? STEPS : 1, kParts = STEPS ? 2 : 1;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, chunks = s.rank / 8;
  const bool some = tile.adapter >= 0;
  if (col0 >= s.d_out) return;
  const __bf16* base[RT];
  int index[RT];
  __bf16* out[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int i = tile.first + min(row0 + 16 * t + m, tile.count - 1);
    const long long row = lists.row(i);
    index[t] = i;
    base[t] = s.base + row * s.ldb;
    out[t] = s.out + row * s.ldo;
  }
  auto read = [&](int c0, bf16x8 (*v)[2]) {  // past the last column: the last eight again
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) v[t][p] = load8(base[t] + min(c0 + 32 * p + 8 * g, s.d_out - 8));
  };
  bf16x8 now[RT][2], next[RT][2];
  read(col0, now);
  bf16x8 hv[kSteps][kParts][RT];
  if (some) {
    const float scale = Lists::kPassed && s.scale ? s.scale[tile.adapter] : 1.f;
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int q = 4 * st + g;
        if (q >= (STEPS ? chunks : 2 * chunks)) {
#pragma unroll
          for (int p = 0; p < kParts; ++p) hv[st][p][t] = zero8();
        } else if (!Lists::kPassed) {
#pragma unroll
          for (int p = 0; p < kParts; ++p) hv[st][p][t] = load8(s.h + ((size_t)index[t] * 2 + p) * s.rank + 8 * q);
        } else {  // the parts of h, in their order
          const bool low = !STEPS && q >= chunks;
          const float* part = s.part + (size_t)index[t] * s.rank + 8 * (low ? q - chunks : q);
          const size_t step = (size_t)s.tokens * s.rank;
          f32x4 h[2] = {};
          for (int p = 0; p < s.parts; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) h[i] += *reinterpret_cast<const f32x4*>(part + p * step + 4 * i);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 hi, lo;
            split(h[e / 4][e % 4] * scale, &hi, &lo);
            hv[st][0][t][e] = low ? lo : hi;
            if (kParts == 2) hv[st][kParts - 1][t][e] = lo;
          }
        }
      }
  }
  const __bf16* w = s.b + (size_t)max(tile.adapter, 0) * s.d_out * s.rank;
  for (int c0 = col0; c0 < s.d_out; c0 += col_step) {
    f32x4 acc[RT][4] = {};
    if (some) {
      bf16x8 wv[kSteps][4];
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int q = 4 * st + g, c = min(c0 + 32 * (n / 2) + 8 * (m / 4) + 4 * (n % 2) + m % 4, s.d_out - 1);
          const __bf16* wc = w + (size_t)c * s.rank;
          if (STEPS) wv[st][n] = q < chunks ? load8(wc + 8 * q) : zero8();
          else wv[st][n] = q < 2 * chunks ? load8(wc + 8 * (q < chunks ? q : q - chunks)) : zero8();
        }
      read(c0 + col_step, next);
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n)
              acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[st][n], hv[st][p][t], acc[t][n], 0, 0, 0);
    } else {
      read(c0 + col_step, next);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        bf16x8 o = now[t][p];
        if (some)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            o[e] = static_cast<__bf16>(static_cast<float>(o[e]) + acc[t][2 * p + e / 4][e % 4]);
        const int c = c0 + 32 * p + 8 * g;
        if (row0 + 16 * t + m < tile.count && c < s.d_out) *reinterpret_cast<bf16x8*>(out[t] + c) = o;
        now[t][p] = next[t][p];
      }
  }
}

// A wave takes 32 rows of a tile: two waves the rows of one that holds more, so two 64-column blocks at a time for the
// workgroup, else four.
template <int STEPS, typename Lists>
__global__ __launch_bounds__(256) void lora_up(LoraArgs s, Lists lists) {
  const LoraTile tile = lists.tile(blockIdx.x);
  const int wave = threadIdx.x >> 6;
  if (tile.count > 32) up_rows<STEPS, 2>(s, lists, tile, 32 * (wave & 1), (blockIdx.y * 2 + (wave >> 1)) * 64, gridDim.y * 128);
  else if (tile.count > 16) up_rows<STEPS, 2>(s, lists, tile, 0, (blockIdx.y * 4 + wave) * 64, gridDim.y * 256);
  else up_rows<STEPS, 1>(s, lists, tile, 0, (blockIdx.y * 4 + wave) * 64, gridDim.y * 256);
}

}  // namespace

int lora_parts(int tokens, int d_in) {
  const int tiles = std::max(1, (tokens + kLoraTileRows - 1) / kLoraTileRows), units = (d_in + 63) / 64;
  return std::max(1, std::min({kLoraMaxParts, (160 + tiles - 1) / tiles, (units + 3) / 4}));
}

namespace {
template <typename Lists>
hipError_t launch(const LoraArgs& a, const Lists& lists, hipStream_t s) {
  const dim3 down(a.n_tiles, a.parts), block(256);
  if (a.rank <= 16) hipLaunchKernelGGL((lora_down<1, Lists>), down, block, 0, s, a, lists);
  else if (a.rank <= 32) hipLaunchKernelGGL((lora_down<2, Lists>), down, block, 0, s, a, lists);
  else if (a.rank <= 64) hipLaunchKernelGGL((lora_down<4, Lists>), down, block, 0, s, a, lists);
  else hipLaunchKernelGGL((lora_down<8, Lists>), down, block, 0, s, a, lists);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = (a.d_out + 127) / 128;
  const dim3 up(a.n_tiles, std::max(1, std::min(blocks, 2048 / a.n_tiles)));
  if (a.rank <= 16) hipLaunchKernelGGL((lora_up<0, Lists>), up, block, 0, s, a, lists);
  else if (a.rank <= 32) hipLaunchKernelGGL((lora_up<1, Lists>), up, block, 0, s, a, lists);
  else if (a.rank <= 64) hipLaunchKernelGGL((lora_up<2, Lists>), up, block, 0, s, a, lists);
  else hipLaunchKernelGGL((lora_up<4, Lists>), up, block, 0, s, a, lists);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_lora(const LoraArgs& a, hipStream_t s) {
  return a.n_tiles > 0 ? launch(a, Uploaded{a.tiles, a.rows}, s) : hipSuccess;
}

hipError_t launch_lora_passed(const LoraArgs& a, const LoraTile* tiles, const int32_t* rows, int n_rows, hipStream_t s) {
  if (a.n_tiles <= 0) return hipSuccess;
  Passed p;
  std::copy(tiles, tiles + a.n_tiles, p.tiles);
  std::copy(rows, rows + n_rows, p.rows);
  return launch(a, p, s);
}

}  // namespace duet
