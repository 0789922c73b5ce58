// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale_a B_a (A_a x[t]),  a the adapter of token t's request.
// Two kernels: h = A_a x in fp32 parts into the workspace, then out = base + scale_a B_a h, scale_a h as two bf16 (2^-17 of it
// off at most), sums in fp32, rounded to bf16 once.
// Both are bound by memory: x, base and out pass once, the adapters are a few MB.  us of the two: 64 rows, 4096 to 6144 columns,
// rank 16, 4.1 + 6.1 (latency); 2112 rows, 4096 to 28672, rank 16, 8 + 56 (4.4 TB/s); 6298 rows, 14336 to 4096, rank 64, 47 + 29
// (3.9 TB/s of x, and of base and out; the first has 500 workgroups for 256 CUs, which read A again for each tile: 364 MB in all,
// of which 224 come from past the L2).  64 and 2112 rows, 4096 to 6144, rank 128: 7 + 19 and 14 + 30.
//
// The lists of up to kLoraPassedTiles tiles travel with the launches' arguments; longer ones are uploaded, a launch of its own
// (64 rows of 16 adapters, 4096 to 6144 columns, rank 16: 20.5 us a call with it, 14.9 without).
//
// Rows of one adapter, wherever in the batch they stand, are taken in tiles of up to kTileRows, so its weights are
// read once a tile and a decode batch of a few adapters costs a few tiles.  Matrix products run on 16x16x32 MFMAs
// with the adapter's side as the first operand: a lane's four results are then neighbours of one row.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "serving_ops.h"
#include "wave_ops.h"

namespace duet {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRowTiles = kLoraTileRows / 16;

__device__ __forceinline__ bf16x8 load8(const __bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }

// The tiles and rows as the kernels read them.
struct Uploaded {
  const LoraTile* tiles;
  const int32_t* rows;
  __device__ __forceinline__ LoraTile tile(int i) const { return tiles[i]; }
  __device__ __forceinline__ int row(const LoraTile& t, int i) const { return t.rows >= 0 ? t.rows + i : rows[~t.rows + i]; }
};
struct Passed {
  LoraTile tiles[kLoraPassedTiles];
  int32_t rows[kLoraPassedRows];
  __device__ __forceinline__ LoraTile tile(int i) const { return tiles[i]; }
  __device__ __forceinline__ int row(const LoraTile& t, int i) const { return t.rows >= 0 ? t.rows + i : rows[~t.rows + i]; }
};

// h and what its rounding to bf16 leaves out (16 bits together).  Finite values that would round to infinity are bf16's
// largest and the rest; nothing is left of an infinity.
__device__ __forceinline__ void split(float h, __bf16* hi, __bf16* lo) {
  constexpr float kMost = 0x1.fep127f;
  float r = static_cast<float>(static_cast<__bf16>(h));
  if (__builtin_isinf(r) && !__builtin_isinf(h)) r = __builtin_copysignf(kMost, h);
  *hi = static_cast<__bf16>(r);
  *lo = static_cast<__bf16>(__builtin_isfinite(r) ? h - r : 0.f);
}

// Partial sums of h of a tile's 16 RT rows over the columns of one part: four waves take its units of kUnit columns in
// turn, each all of the rows and ranks (NT 16-rank tiles), and are summed through LDS in a fixed order.
//
// An MFMA operand wants a row a lane, and a load of that shape costs the address unit 82 cycles (neighbouring lanes lie in
// different rows); a load whose neighbours lie in one row costs 19.  So a unit's rows are loaded 64 or 128 bytes by
// neighbours, put into the wave's part of LDS and read from there in the operands' shape, a row's 16-byte chunks in an order
// by which the 16 lanes of a read meet all banks.  us of 6298 rows of 14336 columns, rank 64: 67 without this.
template <int NT>
struct Down {
  static constexpr int kHalves = NT == 8 ? 1 : 2, kUnit = 32 * kHalves;
  static constexpr int kChunks = 4 * kHalves, kLoadRows = 64 / kChunks;  // of a unit's row, of one load
  static constexpr int kLoads = (kLoraTileRows + 16 * NT) / kLoadRows;   // of a unit, at most
  static constexpr int kLds = 4 * kLoads > 2 * kRowTiles * NT ? 4 * kLoads : 2 * kRowTiles * NT;  // KB
};
template <int NT, int RT, typename Lists>
__device__ __forceinline__ void down_part(const LoraArgs& s, const Lists& lists, const LoraTile& tile, uint4* lds) {
  using D = Down<NT>;
  constexpr int kHalves = D::kHalves, kUnit = D::kUnit, C = D::kChunks, R = D::kLoadRows;
  constexpr int kXLoads = 16 * RT / R, kWLoads = 16 * NT / R;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int units = (s.d_in + kUnit - 1) / kUnit;
  const int u0 = (int)((long long)units * blockIdx.y / s.parts) + wave;
  const int u1 = (int)((long long)units * (blockIdx.y + 1) / s.parts);
  uint4* const own = lds + wave * D::kLoads * 64;
  // The chunk c of row i of a tile lies at place c ^ order(i) of the row.
  auto order = [](int i) { return C == 8 ? (i >> 1) & 7 : (i >> 2) & 3; };
  const __bf16 *x[kXLoads], *w[kWLoads];
  int chunk[2];  // loads of even and odd index
#pragma unroll
  for (int l = 0; l < 2; ++l) chunk[l] = lane % C ^ order(l * R + lane / C);
#pragma unroll
  for (int l = 0; l < kXLoads; ++l)
    x[l] = s.x + lists.row(tile, min(l * R + lane / C, tile.count - 1)) * s.ldx + 8 * chunk[l & 1];
#pragma unroll
  for (int l = 0; l < kWLoads; ++l)
    w[l] = s.a + ((size_t)tile.adapter * s.rank + min(l * R + lane / C, s.rank - 1)) * s.d_in + 8 * chunk[l & 1];
  struct Unit {
    uint4 x[kXLoads], w[kWLoads];
  };
  f32x4 acc[RT][NT] = {};
  auto load = [&](int u, Unit& f) {
#pragma unroll
    for (int l = 0; l < kXLoads; ++l) f.x[l] = *reinterpret_cast<const uint4*>(x[l] + u * kUnit);
#pragma unroll
    for (int l = 0; l < kWLoads; ++l) f.w[l] = *reinterpret_cast<const uint4*>(w[l] + u * kUnit);
  };
  auto place = [&](const Unit& f) {
#pragma unroll
    for (int l = 0; l < kXLoads; ++l) own[l * 64 + lane] = f.x[l];
#pragma unroll
    for (int l = 0; l < kWLoads; ++l) own[(kXLoads + l) * 64 + lane] = f.w[l];
  };
  auto multiply = [&] {
#pragma unroll
    for (int half = 0; half < kHalves; ++half) {
      const uint4* at = own + m * C + ((4 * half + g) ^ order(m));
      bf16x8 wv[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) wv[n] = __builtin_bit_cast(bf16x8, at[(RT + n) * 16 * C]);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const bf16x8 xv = __builtin_bit_cast(bf16x8, at[t * 16 * C]);
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[n], xv, acc[t][n], 0, 0, 0);
      }
    }
  };
  const int whole = min(u1, s.d_in / kUnit);  // the last unit may be cut off, at a multiple of 8 columns
  Unit f;
  if (u0 < whole) {
    load(u0, f);
    for (int u = u0; u < whole; u += 4) {
      place(f);
      load(u + 4 < whole ? u + 4 : u0, f);
      __builtin_amdgcn_sched_barrier(0);
      multiply();
    }
  }
  if (whole < u1 && (whole - u0) % 4 == 0) {
#pragma unroll
    for (int l = 0; l < kXLoads; ++l) f.x[l] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int l = 0; l < kWLoads; ++l) f.w[l] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int odd = 0; odd < 2; ++odd)
      if (whole * kUnit + 8 * chunk[odd] < s.d_in) {
#pragma unroll
        for (int l = odd; l < kXLoads; l += 2) f.x[l] = *reinterpret_cast<const uint4*>(x[l] + whole * kUnit);
#pragma unroll
        for (int l = odd; l < kWLoads; l += 2) f.w[l] = *reinterpret_cast<const uint4*>(w[l] + whole * kUnit);
      }
    place(f);
    multiply();
  }
  __syncthreads();
  f32x4(*sums)[RT * NT][64] = reinterpret_cast<f32x4(*)[RT * NT][64]>(lds);
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
      if (16 * t + m < tile.count && 16 * n + 4 * g < s.rank)
        *reinterpret_cast<f32x4*>(part + (size_t)(16 * t + m) * s.rank + 16 * n + 4 * g) = acc[t][n];
}

template <int NT, typename Lists>
__global__ __launch_bounds__(256) void lora_down(LoraArgs s, Lists lists) {
  __shared__ uint4 lds[Down<NT>::kLds * 64];
  const LoraTile tile = lists.tile(blockIdx.x);
  if (tile.adapter < 0) return;
  if (tile.count > 32) down_part<NT, 4>(s, lists, tile, lds);
  else if (tile.count > 16) down_part<NT, 2>(s, lists, tile, lds);
  else down_part<NT, 1>(s, lists, tile, lds);
}

// h of the i-th of the tiles' rows for STEPS times 32 ranks (0: up to 16): the sum of its parts in their order, scaled, as its
// value in bf16 and what that leaves out (16 bits together), in an MFMA operand's shape.
template <int STEPS>
struct H {
  static constexpr int kSteps = STEPS ? STEPS : 1;
  bf16x8 high[kSteps], low[kSteps];
};
template <int STEPS>
__device__ __forceinline__ H<STEPS> h_of(const LoraArgs& s, const LoraTile& tile, int i) {
  const int g = (threadIdx.x & 63) >> 4, chunks = s.rank / 8;
  const float scale = s.scale ? s.scale[tile.adapter] : 1.f;
  H<STEPS> h;
#pragma unroll
  for (int st = 0; st < H<STEPS>::kSteps; ++st) {
    const int q = 4 * st + g;
    if (q >= chunks) {
      h.high[st] = h.low[st] = zero8();
    } else {
      const float* part = s.part + (size_t)i * s.rank + 8 * q;
      const size_t step = (size_t)s.tokens * s.rank;
      f32x4 sum[2] = {};
      for (int p = 0; p < s.parts; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) sum[k] += *reinterpret_cast<const f32x4*>(part + p * step + 4 * k);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 high, low;
        split(sum[e / 4][e % 4] * scale, &high, &low);
        h.high[st][e] = high;
        h.low[st][e] = low;
      }
    }
  }
  return h;
}

// The sum over h's low parts, as a finite number.  One that is not has an infinite or NaN weight in it, or weights so large that a
// high part's product is infinite (2^8 times the low part's and more, of up to 128).  The high parts then give the infinity or NaN
// that is B h's, where a low part, zero or of the other sign, would have made NaN of an infinity.  A median with a NaN is the
// smallest of the others.
__device__ __forceinline__ f32x4 finite(f32x4 v) {
  constexpr float kMost = 0x1.fffffep127f;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_fmed3f(v[i], -kMost, kMost);
  return v;
}

// out of a tile of up to 16 rows, 64 columns a wave at a time, every col_step-th from col0 on.  The 16 columns of an MFMA are
// taken in fours out of 32, so that two MFMAs give a lane eight neighbours.  The next columns' base is read ahead of the
// products.
template <int STEPS, typename Lists>
__device__ __forceinline__ void up_few(const LoraArgs& s, const Lists& lists, const LoraTile& tile, int col0, int col_step) {
  constexpr int kSteps = H<STEPS>::kSteps;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, chunks = s.rank / 8;
  const bool some = tile.adapter >= 0;
  if (col0 >= s.d_out) return;
  const int i = min(m, tile.count - 1);
  const long long row = lists.row(tile, i);
  const __bf16* base = s.base + row * s.ldb;
  __bf16* out = s.out + row * s.ldo;
  auto read = [&](int c0, bf16x8* v) {  // past the last column: the last eight again
#pragma unroll
    for (int p = 0; p < 2; ++p) v[p] = load8(base + min(c0 + 32 * p + 8 * g, s.d_out - 8));
  };
  bf16x8 now[2], next[2];
  read(col0, now);
  H<STEPS> h;
  if (some) h = h_of<STEPS>(s, tile, tile.first + i);
  const __bf16* w = s.b + (size_t)max(tile.adapter, 0) * s.d_out * s.rank;
  for (int c0 = col0; c0 < s.d_out; c0 += col_step) {
    f32x4 acc[4] = {};
    if (some) {
      bf16x8 wv[kSteps][4];
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int q = 4 * st + g, c = min(c0 + 32 * (n / 2) + 8 * (m / 4) + 4 * (n % 2) + m % 4, s.d_out - 1);
          wv[st][n] = q < chunks ? load8(w + (size_t)c * s.rank + 8 * q) : zero8();
        }
      read(c0 + col_step, next);
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[st][n], h.low[st], acc[n], 0, 0, 0);
#pragma unroll
      for (int n = 0; n < 4; ++n) acc[n] = finite(acc[n]);
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[st][n], h.high[st], acc[n], 0, 0, 0);
    } else {
      read(c0 + col_step, next);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      bf16x8 o = now[p];
      if (some)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = static_cast<__bf16>(static_cast<float>(o[e]) + acc[2 * p + e / 4][e % 4]);
      const int c = c0 + 32 * p + 8 * g;
      if (m < tile.count && c < s.d_out) *reinterpret_cast<bf16x8*>(out + c) = o;
      now[p] = next[p];
    }
  }
}

// out of a larger tile, a wave 16 rows and the workgroup 128 columns at a time, every `ways`-th from the way-th on.  h is the first
// operand here: with the columns of MFMA n taken as 8 j + n, lane j has eight neighbours of a row after eight MFMAs, and the 16
// lanes of a row 256 bytes.  B's columns, which the waves share, go through LDS, eight of them and 16 bytes apart, so that
// those 16 lanes meet all banks.  The next columns' base and B are read ahead of the products.
template <int STEPS>
constexpr int kMostRank = STEPS ? 32 * STEPS : 16;
template <int STEPS, typename Lists>
__device__ __forceinline__ void up_many(const LoraArgs& s, const Lists& lists, const LoraTile& tile, int way, int ways,
                                        uint4* lds) {
  constexpr int kSteps = H<STEPS>::kSteps, kUnits = 128 * kMostRank<STEPS> / 8 / 256;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, j = lane & 15, g = lane >> 4, chunks = s.rank / 8;
  const bool some = tile.adapter >= 0, rows = 16 * wave < tile.count;
  const __bf16* base[4];
  __bf16* out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long row = lists.row(tile, min(16 * wave + 4 * g + i, tile.count - 1));
    base[i] = s.base + row * s.ldb;
    out[i] = s.out + row * s.ldo;
  }
  const __bf16* w = s.b + (size_t)max(tile.adapter, 0) * s.d_out * s.rank;
  // This thread's 16-byte units of 128 columns of B, which lie one after the other, and their places.
  int place[kUnits];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) place[k] = k * 256 + tid + (k * 256 + tid) / (8 * chunks);
  bf16x8 b[kUnits], now[4], next[4];
  auto read = [&](int c0, bf16x8* v) {  // past the last column: the last eight again
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load8(base[i] + min(c0 + 8 * j, s.d_out - 8));
  };
  auto read_b = [&](int c0) {
    const int left = (min(c0 + 128, s.d_out) - c0) * chunks;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) b[k] = k * 256 + tid < left ? load8(w + (size_t)c0 * s.rank + 8 * (k * 256 + tid)) : zero8();
  };
  const int step = 128 * ways;
  int c0 = 128 * way;
  if (c0 >= s.d_out) return;
  if (rows) read(c0, now);
  if (some) read_b(c0);
  H<STEPS> h;
  if (some) h = h_of<STEPS>(s, tile, tile.first + min(16 * wave + j, tile.count - 1));
  for (; c0 < s.d_out; c0 += step) {
    f32x4 acc[8] = {};
    if (some) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kUnits; ++k)
        if (k * 256 + tid < 128 * chunks) lds[place[k]] = __builtin_bit_cast(uint4, b[k]);
      __syncthreads();
      if (c0 + step < s.d_out) read_b(c0 + step);
    }
    if (!rows) continue;
    read(c0 + step, next);
    if (some) {
      const uint4* own = lds + j * (8 * chunks + 1);
      const bool partial = chunks < 4 * kSteps;  // zeros past the rank's end
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        bf16x8 wv[kSteps];
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const int q = 4 * st + g;
          wv[st] = __builtin_bit_cast(bf16x8, own[n * chunks + min(q, chunks - 1)]);
          if (partial && q >= chunks) wv[st] = zero8();
        }
#pragma unroll
        for (int st = 0; st < kSteps; ++st) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h.low[st], wv[st], acc[n], 0, 0, 0);
        acc[n] = finite(acc[n]);
#pragma unroll
        for (int st = 0; st < kSteps; ++st) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h.high[st], wv[st], acc[n], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 o = now[i];
      if (some)
#pragma unroll
        for (int n = 0; n < 8; ++n) o[n] = static_cast<__bf16>(static_cast<float>(o[n]) + acc[n][i]);
      if (16 * wave + 4 * g + i < tile.count && c0 + 8 * j < s.d_out) *reinterpret_cast<bf16x8*>(out[i] + c0 + 8 * j) = o;
      now[i] = next[i];
    }
  }
}

template <int STEPS, typename Lists>
__global__ __launch_bounds__(256) void lora_up(LoraArgs s, Lists lists) {
  __shared__ uint4 lds[128 * kMostRank<STEPS> / 8 + 16];
  const LoraTile tile = lists.tile(blockIdx.x);
  if (tile.count > 16) up_many<STEPS>(s, lists, tile, blockIdx.y, gridDim.y, lds);
  else up_few<STEPS>(s, lists, tile, (blockIdx.y * 4 + (threadIdx.x >> 6)) * 64, gridDim.y * 256);
}

}  // namespace

int lora_most_parts(int tokens, int d_in) {
  const int tiles = std::max(1, (tokens + kLoraTileRows - 1) / kLoraTileRows), units = (d_in + 63) / 64;
  return std::max(1, std::min({kLoraMaxParts, 2048 / tiles, (units + 3) / 4}));
}

int lora_parts(int tiles, int most) {
  int best = 1;
  double least = 1e9;
  for (int p = 1; p <= most; ++p) {
    const double cost = (double)((tiles * (long long)p + 255) / 256) / p + 0.01 * p;
    if (cost < least) least = cost, best = p;
  }
  return best;
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
  // Workgroups a tile: some 512 in all (us with 256 / 512 / 1024 / 3000: 41 tiles of 28672 columns, rank 16, 59 / 53 / 57 / 53; 100
  // of 4096, rank 64, 37 / 25 / 30 / 30).
  const int blocks = (a.d_out + 127) / 128;
  const dim3 up(a.n_tiles, std::max(1, std::min(blocks, 512 / a.n_tiles)));
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
