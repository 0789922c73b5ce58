// Device code for prefixes that many query rows share (attn_shared.hip says what it computes).
//
// Eight waves of 32 rows on 32x32x16 matrix instructions, S^T = K Q^T and O^T += V^T P^T, with the operand orders of the prefill kernel
// (attn_prefill.hip): its tile loads, swizzles and softmax without the causal mask, over a run of whole pages.  A tile of 64 keys
// takes 1.4 us with one wave of rows a SIMD, 1.8 to 2.1 with two.  Measured slower: 64 rows a wave on four waves, also with the matrix instructions of one
// half of the rows between the exponentials of the other (100 and 103 against 84 us for 512 rows after 32768 tokens), and one wave of a
// SIMD half a step behind the other (93).
#pragma once

#include <hip/hip_runtime.h>

#include "attn_prefill_device.h"
#include "cache_ops.h"
#include "wave_ops.h"

namespace duet {
namespace shared {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A row's reference lies kLift above its largest score, and moves when a score passes that one by kSlack, all in powers of two.  So
// weights are at most 2^(kSlack - kLift), and the sums of a run, of up to 2^14 tokens, stay finite over bf16's largest values.  Weights
// under 2^-102 of the largest become 0.
constexpr float kLift = 24.f, kSlack = 8.f;

__device__ __forceinline__ float power(unsigned word, int byte) {
  return __uint_as_float((word >> (8 * byte) & 255u) << 23);
}

// A denominator with the mark of a bad page.
__device__ __forceinline__ float marked(float l, bool bad) {
  return __uint_as_float((__float_as_uint(l) & 0x7fffffffu) | (bad ? 0x80000000u : 0u));
}

// A request's first slot and slots; the prefixes' members.
__device__ __forceinline__ int2 slots_of(const SharedTables& tab, int r) { return tab.slots[r]; }
template <int R, int P>
__device__ __forceinline__ int2 slots_of(const SharedPassed<R, P>& tab, int r) { return make_int2(tab.slots[r], tab.slots[r + 1] - tab.slots[r]); }
template <int R>
__device__ __forceinline__ int2 slots_of(const SharedSlots<R>& tab, int r) { return make_int2(tab.slots[r], tab.slots[r + 1] - tab.slots[r]); }
template <int R>
__device__ __forceinline__ int2 slots_of(const SharedPlain<R>& tab, int r) { return make_int2(tab.first[r], tab.first[r + 1] - tab.first[r]); }
__device__ __forceinline__ int listed(const SharedTables& tab, int i) { return tab.list[i]; }
template <int R, int P>
__device__ __forceinline__ int listed(const SharedPassed<R, P>& tab, int i) { return tab.list[i / 4] >> (i % 4 * 8) & 255; }
template <int R>
__device__ __forceinline__ int listed(const SharedPlain<R>&, int i) { return i; }

constexpr int kWideThreads = 512, kWideWaves = 8;
constexpr int kTile = 64;  // keys of a tile: four pages

// LDS: a ring of tiles, K as [64 keys][d] and V as V^T [d][64 keys] in bf16, then the run's page ids.
template <int D, bool EIGHT>
struct WideLds {
  static constexpr int kStages = EIGHT ? 2 : 4;
  static constexpr int kStageElems = 2 * kTile * D;
  static constexpr size_t kTileBytes = (size_t)kStages * kStageElems * 2;
  static constexpr size_t kBytes = kTileBytes + kWidePages * sizeof(int);
};

// Up to 256 rows of a run, 32 a wave, with kv head j.  The run is of whole pages.
template <int D, bool EIGHT, typename Table>
__device__ __forceinline__ void wide_item(const SharedArgs& a, const Table& tab, const SharedRun& e, int j, __bf16* const lds) {
  using L = WideLds<D, EIGHT>;
  using namespace prefill;
  constexpr int NK = D / 16, NO = D / 32, KCH = D / 8, VCH = kTile / 8, S = L::kStages;
  constexpr int kB = EIGHT ? 1 : 2;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, hh = lane >> 5;
  const int g = a.group, rows = e.members * g, n_pages = e.tokens / 16, n_tiles = (n_pages + 3) >> 2;
  const int row = e.row0 + 32 * wave + (lane & 31);
  const bool active = wave < e.waves && e.row0 + 32 * wave < rows;  // the wave has rows
  const bool row_ok = active && row < rows;
  const int member = row_ok ? listed(tab, e.member0 + row / g) : 0, head = j * g + (row_ok ? row % g : 0);

  bf16x8 qf[NK];
  {
    const __bf16* q = a.q + ((size_t)member * a.h_q + head) * D + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
      const uint4 u = row_ok ? *reinterpret_cast<const uint4*>(q + 16 * ks) : make_uint4(0, 0, 0, 0);
      qf[ks] = __builtin_bit_cast(bf16x8, u);
    }
  }
  // The run's page ids, -1 for those outside the pool and past the end (up to a whole tile).
  int* const ids = reinterpret_cast<int*>(reinterpret_cast<char*>(lds) + L::kTileBytes);
  const int* prow = a.table + (size_t)e.table_row * a.max_pages + e.page0;
  bool bad = false;
  for (int p = tid; p < 4 * n_tiles; p += kWideThreads) {
    const int id = p < n_pages ? prow[p] : -1;
    const bool ok = page_ok(id, a.pages);
    bad |= p < n_pages && !ok;
    ids[p] = ok ? id : -1;
  }
  bad = uniform(__syncthreads_or(bad));
  // Which of a tile's pages count.  All of most: the ids are read again only where some do not, since waiting for them would mean
  // waiting for the operands read before.
  auto page_mask = [&](int t) {
    if (!bad && (t + 1 < n_tiles || n_pages % 4 == 0)) return 15;
    const int4 v = *reinterpret_cast<const int4*>(ids + 4 * t);
    return uniform((v.x >= 0 ? 1 : 0) | (v.y >= 0 ? 2 : 0) | (v.z >= 0 ? 4 : 0) | (v.w >= 0 ? 8 : 0));
  };

  constexpr size_t kSlab = 16 * D * kB;
  const char* kbase = static_cast<const char*>(a.k) + (size_t)j * kSlab;
  const char* vbase = static_cast<const char*>(a.v) + (size_t)j * kSlab;
  const size_t page_stride = (size_t)a.h_kv * kSlab;

  // bf16: direct loads into the ring, blocks of 1 KiB, S - 1 tiles ahead.
  constexpr int KB = kTile * D * 2 / 1024, BPW = KB / kWideWaves;
  int k_pi[BPW], k_off[BPW], v_pi[BPW], v_off[BPW];
  if constexpr (!EIGHT) {
#pragma unroll
    for (int b = 0; b < BPW; ++b) {
      const int blk = wave + kWideWaves * b, krow = (64 / KCH) * blk + lane / KCH;
      const int kc = (lane % KCH) ^ (kswz(krow) & (KCH - 1));
      k_pi[b] = krow >> 4;
      k_off[b] = (krow & 15) * (D * 2) + kc * 16;
      const int vrow = 8 * blk + lane / 8, vc = (lane % 8) ^ (vswz(vrow) & (VCH - 1));
      v_pi[b] = vc >> 1;
      v_off[b] = vrow * 32 + (vc & 1) * 16;
    }
  }
  auto issue = [&](int t) {
    __bf16* kdst = lds + (t % S) * L::kStageElems;
    __bf16* vdst = kdst + kTile * D;
#pragma unroll
    for (int b = 0; b < BPW; ++b) {
      const int blk = wave + kWideWaves * b;
      const int kid = max(ids[4 * t + k_pi[b]], 0), vid = max(ids[4 * t + v_pi[b]], 0);
      load_lds16(kbase + (size_t)uniform(kid) * page_stride + k_off[b], kdst + blk * 512);
      load_lds16(vbase + (size_t)(unsigned)vid * page_stride + v_off[b], vdst + blk * 512);
    }
  };
  auto wait_tiles = [&](int later) {
    constexpr int L1 = 2 * BPW, L2 = 4 * BPW;
    if (later >= 2) __builtin_amdgcn_s_waitcnt((L2 & 15) | ((L2 >> 4) << 14) | 0x0F70);
    else if (later == 1) __builtin_amdgcn_s_waitcnt((L1 & 15) | ((L1 >> 4) << 14) | 0x0F70);
    else __builtin_amdgcn_s_waitcnt(0x0F70);
  };
  // Values of pages that do not count are zeroed in LDS: their weights are 0, and 0 times NaN is NaN.
  auto publish = [&](int t, int later) {
    wait_tiles(later);
    __builtin_amdgcn_s_barrier();
    const int mask = page_mask(t);
    if (mask != 15) {
      __bf16* vs = lds + (t % S) * L::kStageElems + kTile * D;
      for (int x = tid; x < D * VCH; x += kWideThreads) {
        const int vrow = x / VCH, sc = x % VCH, c = sc ^ (vswz(vrow) & (VCH - 1));
        if (!(mask >> (c >> 1) & 1)) *reinterpret_cast<uint4*>(vs + vrow * kTile + sc * 8) = make_uint4(0, 0, 0, 0);
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);
      __builtin_amdgcn_s_barrier();
    }
  };

  // 8-bit: 16 bytes of keys and of values a thread go through registers and are widened and scaled once for all waves: exact in
  // bf16, as duet_cache8_read gives them.
  constexpr int kPieces = kTile * D / 16;  // of keys, and of values
  const bool mover = tid < kPieces;
  const int krow8 = tid / (D / 16), kc8 = tid % (D / 16), vrow8 = tid / 4, vp8 = tid % 4;
  struct Raw {
    uint4 k, v, ve;
    unsigned ke;
    bool vok;
  };
  auto fetch = [&](int t) {
    Raw r;
    if (!mover) return r;
    const int kid = ids[4 * t + krow8 / 16], vid = ids[4 * t + vp8];
    r.vok = vid >= 0;
    const size_t kslab = (size_t)max(kid, 0) * a.h_kv + j, vslab = (size_t)max(vid, 0) * a.h_kv + j;
    r.k = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.k) + kslab * kSlab + (krow8 & 15) * D + kc8 * 16);
    r.v = *reinterpret_cast<const uint4*>(static_cast<const char*>(a.v) + vslab * kSlab + vrow8 * 16);
    r.ke = a.scales[kslab * 32 + (krow8 & 15)];
    r.ve = *reinterpret_cast<const uint4*>(a.scales + vslab * 32 + 16);
    return r;
  };
  auto put = [&](int t, const Raw& r) {
    if (!mover) return;
    __bf16* ks = lds + (t % S) * L::kStageElems;
    __bf16* vs = ks + kTile * D;
    union Row {
      bf16x2 p[8];
      uint4 u[2];
    } x;
    const unsigned w[4] = {r.k.x, r.k.y, r.k.z, r.k.w};
    const float scale = __uint_as_float(r.ke << 23);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      x.p[2 * n] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[n], scale, false);
      x.p[2 * n + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[n], scale, true);
    }
    const int kx = kswz(krow8) & (KCH - 1);
    *reinterpret_cast<uint4*>(ks + krow8 * D + ((2 * kc8) ^ kx) * 8) = x.u[0];
    *reinterpret_cast<uint4*>(ks + krow8 * D + ((2 * kc8 + 1) ^ kx) * 8) = x.u[1];
    const unsigned vw[4] = {r.v.x, r.v.y, r.v.z, r.v.w}, ew[4] = {r.ve.x, r.ve.y, r.ve.z, r.ve.w};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(vw[n], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(vw[n], true);
      x.p[2 * n] = bf16x2{static_cast<__bf16>(lo[0] * power(ew[n], 0)), static_cast<__bf16>(lo[1] * power(ew[n], 1))};
      x.p[2 * n + 1] = bf16x2{static_cast<__bf16>(hi[0] * power(ew[n], 2)), static_cast<__bf16>(hi[1] * power(ew[n], 3))};
    }
    if (!r.vok) x.u[0] = x.u[1] = make_uint4(0, 0, 0, 0);
    const int vx = vswz(vrow8) & (VCH - 1);
    *reinterpret_cast<uint4*>(vs + vrow8 * kTile + ((2 * vp8) ^ vx) * 8) = x.u[0];
    *reinterpret_cast<uint4*>(vs + vrow8 * kTile + ((2 * vp8 + 1) ^ vx) * 8) = x.u[1];
  };

  f32x16 oacc[NO];
#pragma unroll
  for (int n = 0; n < NO; ++n)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[n][v] = 0.f;
  float m_ref = -INFINITY, m_sub = 0.f, l_run = 0.f;
  auto compute = [&](int t) {
    const __bf16* ks = lds + (t % S) * L::kStageElems;
    const __bf16* vs = ks + kTile * D;
    bf16x8 kf[2][NK];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      const int kr = 32 * nb + swap_bits23(lane & 31);
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
        kf[nb][kk] = *reinterpret_cast<const bf16x8*>(ks + kr * D + ((2 * kk + hh) ^ (kswz(kr) & (KCH - 1))) * 8);
    }
    f32x16 sacc[2];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v) sacc[nb][v] = 0.f;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) sacc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[nb][kk], qf[kk], sacc[nb], 0, 0, 0);
    bf16x8 vf[NO][4];
#pragma unroll
    for (int n = 0; n < NO; ++n) {
      const int vr = 32 * n + (lane & 31);
#pragma unroll
      for (int k2 = 0; k2 < 4; ++k2)
        vf[n][k2] = *reinterpret_cast<const bf16x8*>(vs + vr * kTile + ((2 * k2 + hh) ^ (vswz(vr) & (VCH - 1))) * 8);
    }
    __builtin_amdgcn_s_setprio(0);
    const int mask = page_mask(t);
    if (mask != 15) {  // register v of half nb is of page 2 nb + v / 8
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!(mask >> (2 * nb + (v >> 3)) & 1)) sacc[nb][v] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sacc[nb][v]);
    mx = pair_max(mx) * a.scale_log2;
    if (__any(mx > m_ref + (kSlack - kLift))) {
      const float to = fmaxf(m_ref, mx + kLift), alpha = to == -INFINITY ? 1.f : fast_exp2(m_ref - to);
      m_ref = to;
      m_sub = to == -INFINITY ? 0.f : to;
      l_run *= alpha;
#pragma unroll
      for (int n = 0; n < NO; ++n) oacc[n] *= alpha;
    }
    bf16x8 pb[4];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        pb[2 * nb + (v >> 3)][v & 7] = static_cast<__bf16>(fast_exp2(__builtin_fmaf(sacc[nb][v], a.scale_log2, -m_sub)));
    const bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
    for (int k2 = 0; k2 < 4; ++k2)
#pragma unroll
      for (int x = 0; x < 4; ++x) l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[k2][2 * x], pb[k2][2 * x + 1]}, ones, l_run, false);
#pragma unroll
    for (int n = 0; n < NO; ++n)
#pragma unroll
      for (int k2 = 0; k2 < 4; ++k2) oacc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n][k2], pb[k2], oacc[n], 0, 0, 0);
  };

  if constexpr (EIGHT) {
    const Raw first = fetch(0);
    Raw next = first;
    if (n_tiles > 1) next = fetch(1);
    put(0, first);
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
      // Tile t + 1 was loaded during the step before, t + 2 is during this one.
      if (t + 1 < n_tiles) put(t + 1, next);
      if (t + 2 < n_tiles) next = fetch(t + 2);
      if (active) compute(t);
      __syncthreads();
    }
  } else {
    for (int t = 0; t < S - 1 && t < n_tiles; ++t) issue(t);
    publish(0, min(n_tiles - 1, S - 2));
    __builtin_amdgcn_s_waitcnt(0x0F70);  // the queries are here too, so that no step waits for them and all tiles
    for (int t = 0; t < n_tiles; ++t) {
      if (t + S - 1 < n_tiles) issue(t + S - 1);
      if (active) compute(t);
      if (t + 1 < n_tiles) publish(t + 1, min(n_tiles - 1, t + S - 1) - (t + 1));
    }
  }
  if (!row_ok) return;
  const size_t at = (size_t)(slots_of(tab, member).x + e.slot) * a.h_q + head;
  float* o = a.acc + at * D + 4 * hh;
#pragma unroll
  for (int n = 0; n < NO; ++n)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *reinterpret_cast<f32x4*>(o + 32 * n + 2 * v) = f32x4{oacc[n][v], oacc[n][v + 1], oacc[n][v + 2], oacc[n][v + 3]};
  const float total = pair_sum(l_run);
  if (hh == 0) a.ml[at] = make_float2(m_ref, marked(total, bad));
}

}  // namespace shared
}  // namespace duet
