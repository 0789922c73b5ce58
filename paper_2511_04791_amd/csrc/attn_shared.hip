// Decode attention over a paged cache, bf16 or 8-bit, for requests that may share the pages of a prefix.
//
// A request's output is softmax(q K^T / sqrt(d)) V over its keys.  The keys are cut into runs; a run gives each query row an
// unnormalised output, a reference maximum m and a denominator l, and a row's runs are joined by their exp(m).  A shared
// prefix is cut once and attended by the rows of every member, so its pages are read once for all of them, and a page
// that one request holds alone is attended by the g heads of its group.
//
// A wave takes an item: a run (split), a kv head and up to 16 or 64 query rows, and walks the run 64 keys at a time.
//   S^T [tokens x rows] = K Q^T and O^T [dims x rows] += V^T P^T on 16x16x32 matrix instructions.
// The tokens of S^T's rows are chosen so that a lane of quad y (16 lanes) gets all 16 tokens of the step's page y: instruction
// p takes tokens 4 p .. 4 p + 3 of each of the four pages.  P^T is then already the operand of the second product, and a
// lane's values are whole rows of a dim-major page: 16 bytes a load for 8-bit pages as for bf16 ones.
// 8-bit values become bf16 exactly; a key's power of two multiplies its scores, a value's its probability.
#include <hip/hip_runtime.h>

#include "attn_shared_wide.h"
#include "cache_ops.h"
#include "wave_ops.h"

namespace duet {
namespace {

using namespace shared;

__device__ __forceinline__ bf16x8 widened(uint2 x) {
  union {
    bf16x2 p[4];
    bf16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.x, 1.f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.x, 1.f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.y, 1.f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.y, 1.f, true);
  return u.v;
}
// The first n of 16 values of 8 or 16 bits, the others zero.
__device__ __forceinline__ unsigned first_bytes(unsigned x, int n) {  // of 4
  return n >= 4 ? x : n <= 0 ? 0u : x & ((1u << (8 * n)) - 1);
}
__device__ __forceinline__ uint4 first_bytes(uint4 x, int n) {  // of 16
  return make_uint4(first_bytes(x.x, n), first_bytes(x.y, n - 4), first_bytes(x.z, n - 8), first_bytes(x.w, n - 12));
}

template <int D, bool EIGHT, int MT>
__global__ __launch_bounds__(256) void shared_partial(SharedArgs a, const SharedEntry* entries, int n_entries, int n_items) {
  constexpr int kB = EIGHT ? 1 : 2;           // bytes of a value
  constexpr int kLoads = D * kB / 64;         // 16-byte loads of a key's row by four lanes
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int item = uniform(4 * blockIdx.x + (threadIdx.x >> 6));
  if (item >= n_items) return;
  const SharedEntry e = entries[uniform(find_request(n_entries, [&](int i) { return entries[i].first_item <= item; }))];
  const int g = a.group, rows = e.members * g, blocks = (rows + 16 * MT - 1) / (16 * MT);
  // Row blocks of one run and head next to each other, then heads, then runs.
  const int i = item - e.first_item, block = i % blocks, j = i / blocks % a.h_kv, split = i / blocks / a.h_kv;
  const int page0 = e.page0 + split * e.split_pages;
  const int n_tok = min(e.tokens - 16 * split * e.split_pages, 16 * e.split_pages);
  const int n_pages = (n_tok + 15) >> 4;
  const int* prow = a.table + (size_t)e.table_row * a.max_pages + page0;

  int head_row[MT];  // request * h_q + head of the tile's row `col`, or -1
  bf16x8 qf[MT][D / 32];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = (block * MT + m) * 16 + col;
    head_row[m] = row < rows ? a.list[e.member0 + row / g] * a.h_q + j * g + row % g : -1;
    const __bf16* q = a.q + (size_t)max(head_row[m], 0) * D;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      // The dimensions of contraction step ks that this quad holds, as the keys' loads give them.
      const int dim = EIGHT ? 64 * (ks / 2) + 16 * quad + 8 * (ks % 2) : 32 * ks + 8 * quad;
      const uint4 u = head_row[m] >= 0 ? *reinterpret_cast<const uint4*>(q + dim) : make_uint4(0, 0, 0, 0);
      qf[m][ks] = __builtin_bit_cast(bf16x8, u);
    }
  }
  f32x4 acc[MT][D / 16];
  float l[MT], m_ref[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    l[m] = 0.f, m_ref[m] = -INFINITY;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool bad = false;
  for (int p0 = 0; p0 < n_pages; p0 += 4) {
    const int kpage = p0 + (col >> 2), vpage = p0 + quad;
    const int kid = prow[min(kpage, n_pages - 1)], vid = prow[min(vpage, n_pages - 1)];
    const bool kok = page_ok(kid, a.pages), vok = page_ok(vid, a.pages);
    bad |= !vok;
    const size_t kslab = (size_t)(kok ? kid : 0) * a.h_kv + j, vslab = (size_t)(vok ? vid : 0) * a.h_kv + j;
    const char* kp = static_cast<const char*>(a.k) + kslab * 16 * D * kB + (col & 3) * D * kB + quad * 16;
    const char* vp = static_cast<const char*>(a.v) + vslab * 16 * D * kB + col * 16 * kB;
    // Tokens of page `vpage` that count.
    const int nv = vok ? max(0, min(16, n_tok - 16 * vpage)) : 0;
    uint4 kr[4][kLoads], vr[D / 16][kB];
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int s = 0; s < kLoads; ++s) kr[p][s] = *reinterpret_cast<const uint4*>(kp + 4 * p * D * kB + 64 * s);
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
#pragma unroll
      for (int h = 0; h < kB; ++h) vr[n][h] = *reinterpret_cast<const uint4*>(vp + n * 256 * kB + 16 * h);
    uint4 ke = make_uint4(0, 0, 0, 0), ve = ke;
    if constexpr (EIGHT) {
      ke = *reinterpret_cast<const uint4*>(a.scales + vslab * 32);
      ve = *reinterpret_cast<const uint4*>(a.scales + vslab * 32 + 16);
    }
    const bool part = __any(nv < 16);
    if (part) {
      ve = first_bytes(ve, nv);
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        if constexpr (EIGHT) {
          vr[n][0] = first_bytes(vr[n][0], nv);
        } else {
          vr[n][0] = first_bytes(vr[n][0], 2 * nv);
          vr[n][kB - 1] = first_bytes(vr[n][kB - 1], 2 * nv - 16);
        }
      }
    }
    bf16x8 kf[4][D / 32];
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int s = 0; s < kLoads; ++s) {
        if constexpr (EIGHT) {
          kf[p][2 * s] = widened(make_uint2(kr[p][s].x, kr[p][s].y));
          kf[p][2 * s + 1] = widened(make_uint2(kr[p][s].z, kr[p][s].w));
        } else {
          kf[p][s] = __builtin_bit_cast(bf16x8, kr[p][s]);
        }
      }
    float kscale[16], vscale[16];
    const unsigned kw[4] = {ke.x, ke.y, ke.z, ke.w}, vw[4] = {ve.x, ve.y, ve.z, ve.w};
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      kscale[t] = EIGHT ? power(kw[t / 4], t % 4) * a.scale_log2 : a.scale_log2;
      vscale[t] = EIGHT ? power(vw[t / 4], t % 4) : 1.f;
    }
    bf16x8 pf[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float sc[16];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[p][ks], qf[m][ks], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[4 * p + i] = s[i] * kscale[4 * p + i];
      }
      if (part) {
#pragma unroll
        for (int t = 0; t < 16; ++t) sc[t] = t < nv ? sc[t] : -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int t = 1; t < 16; ++t) mx = fmaxf(mx, sc[t]);
      mx = max_rows(mx);
      if (__any(mx > m_ref[m] + kSlack)) {
        const float to = fmaxf(m_ref[m], mx);
        const float alpha = to == -INFINITY ? 1.f : fast_exp2(m_ref[m] - to);
        m_ref[m] = to;
        l[m] *= alpha;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) acc[m][n] *= alpha;
      }
      const float sub = m_ref[m] == -INFINITY ? 0.f : m_ref[m];  // no key yet that counts: every weight is 0
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        // The denominator sums the probabilities as the second product takes them.
        const __bf16 w = static_cast<__bf16>(fast_exp2(sc[t] - sub));
        l[m] += static_cast<float>(w);
        pf[m][t / 8][t % 8] = EIGHT ? static_cast<__bf16>(static_cast<float>(w) * vscale[t]) : w;
      }
    }
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 vf;
        if constexpr (EIGHT) vf = widened(h ? make_uint2(vr[n][0].z, vr[n][0].w) : make_uint2(vr[n][0].x, vr[n][0].y));
        else vf = __builtin_bit_cast(bf16x8, vr[n][h % kB]);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[m][h], acc[m][n], 0, 0, 0);
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const float total = sum_rows(l[m]);
    if (head_row[m] < 0) continue;
    const int r = head_row[m] / a.h_q;
    const size_t at = (size_t)(a.slots[r].x + e.slot_off + split) * a.h_q + (head_row[m] - r * a.h_q);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) *reinterpret_cast<f32x4*>(a.acc + at * D + 16 * n + 4 * quad) = acc[m][n];
    if (quad == 0) a.ml[at] = make_float2(m_ref[m], total);
  }
  if (__any(bad) && lane == 0) atomicOr(a.err, 1);
}

template <int D, bool EIGHT>
__global__ __launch_bounds__(kWideThreads, 1) void shared_wide(SharedArgs a) {
  extern __shared__ __attribute__((aligned(16))) __bf16 lds[];
  const int item = blockIdx.x;
  const SharedEntry e = a.entries[uniform(find_request(a.n_wide, [&](int i) { return a.entries[i].first_item <= item; }))];
  wide_item<D, EIGHT>(a, e, item - e.first_item, lds);
}

// Joins the runs of one (request, query head): W waves, each every W-th run, eight loads in flight.
template <int D, int W>
__global__ __launch_bounds__(256) void shared_merge(SharedArgs a) {
  constexpr int E = D / 64;
  __shared__ float part[W > 1 ? W : 1][D + 2];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), w = wave % W;
  const int pair = (blockIdx.x * 4 + wave) / W;
  if (pair >= a.num_reqs * a.h_q) return;  // the whole workgroup where W is 4
  const int r = pair / a.h_q;
  const int2 at = a.slots[r];
  const size_t first = (size_t)at.x * a.h_q + pair - r * a.h_q;
  float top = -INFINITY, den = 0.f, num[E] = {};
  for (int s0 = w; s0 < at.y; s0 += 8 * W) {
    float2 ml[8];
    float x[8][E];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = min(s0 + u * W, at.y - 1);
      const size_t row = first + (size_t)s * a.h_q;
      ml[u] = a.ml[row];
      if (s0 + u * W >= at.y) ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int i = 0; i < E; ++i) x[u][i] = a.acc[row * D + 64 * i + lane];
    }
    float to = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) to = fmaxf(to, ml[u].x);
    if (to == -INFINITY) continue;  // runs without a key that counts
    const float f = fast_exp2(top - to);
    top = to;
    den *= f;
#pragma unroll
    for (int i = 0; i < E; ++i) num[i] *= f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float wgt = fast_exp2(ml[u].x - to);
      if (s0 + u * W >= at.y) break;
      den += wgt * ml[u].y;
#pragma unroll
      for (int i = 0; i < E; ++i) num[i] += wgt * x[u][i];
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int i = 0; i < E; ++i) part[w][64 * i + lane] = num[i];
    if (lane == 0) part[w][D] = top, part[w][D + 1] = den;
    __syncthreads();
    if (w) return;
    float to = -INFINITY;
#pragma unroll
    for (int u = 0; u < W; ++u) to = fmaxf(to, part[u][D]);
    den = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) num[i] = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float wgt = to == -INFINITY ? 0.f : fast_exp2(part[u][D] - to);
      den += wgt * part[u][D + 1];
#pragma unroll
      for (int i = 0; i < E; ++i) num[i] += wgt * part[u][64 * i + lane];
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) a.out[(size_t)pair * D + 64 * i + lane] = static_cast<__bf16>(num[i] / den);
}

template <int D, bool EIGHT>
hipError_t launch(const SharedArgs& a, hipStream_t s) {
  if (a.wide_items) {
    constexpr size_t kBytes = WideLds<D, EIGHT>::kBytes;
    static const hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void*>(&shared_wide<D, EIGHT>),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
    if (set != hipSuccess) return set;
    hipLaunchKernelGGL((shared_wide<D, EIGHT>), dim3(a.wide_items), dim3(kWideThreads), kBytes, s, a);
  }
  if (a.narrow_items)
    hipLaunchKernelGGL((shared_partial<D, EIGHT, kNarrowRows / 16>), dim3((a.narrow_items + 3) / 4), dim3(256), 0, s, a,
                       a.entries + a.n_wide, a.n_narrow, a.narrow_items);
  const int pairs = a.num_reqs * a.h_q;
  if (a.max_slots > 16) hipLaunchKernelGGL((shared_merge<D, 4>), dim3(pairs), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((shared_merge<D, 1>), dim3((pairs + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared(const SharedArgs& a, hipStream_t s) {
  if (a.num_reqs == 0) return hipSuccess;
  if (a.scales) return a.head_dim == 128 ? launch<128, true>(a, s) : launch<64, true>(a, s);
  return a.head_dim == 128 ? launch<128, false>(a, s) : launch<64, false>(a, s);
}

}  // namespace duet
