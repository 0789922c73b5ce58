// Decode attention over a paged cache, bf16 or 8-bit, for requests that may share the pages of a prefix.
//
// A request's output is softmax(q K^T / sqrt(d)) V over its keys.  The keys are cut into runs; a run gives each query row an
// unnormalised output, a reference m (kLift above its largest score) and a denominator l, and a row's runs are joined by their
// exp(m).  A shared prefix is cut once and attended by the rows of every member, so its pages are read once for all of them, and
// a page that one request holds alone is attended by the g heads of its group.
//
// Up to 16 rows: a wave, or a team of four that shares a run, walks it 64 keys at a time.
//   S^T [tokens x rows] = K Q^T and O^T [dims x rows] += V^T P^T on 16x16x32 matrix instructions.
// The tokens of S^T's rows are chosen so that a lane of quad y (16 lanes) gets all 16 tokens of the step's page y: instruction
// p takes tokens 4 p .. 4 p + 3 of each of the four pages.  P^T is then already the operand of the second product, and a
// lane's values are whole rows of a dim-major page: 16 bytes a load for 8-bit pages as for bf16 ones.
// 8-bit values become bf16 exactly; a key's power of two multiplies its scores, a value's its probability.  Probabilities are rounded to
// bf16, the second product's operands, and the denominator sums them as rounded: 256 requests of 512 to 8192 tokens are off by 0.0020 of
// the results' size, 0.0017 of it their own rounding.
// Bound by memory: 256 requests of 512 to 8192 tokens, 8 kv heads, 8-bit: 264 us, 5.5 TB/s.  A step's loads go out during the step
// before; two teams fit a CU.  A wave's runs of more than 32 pages are slower than a team's (100 pages: 301 us).
//
// More rows (attn_shared_wide.h): a workgroup takes up to 256 of them and brings tiles of 64 keys through LDS, bound by the matrix
// cores, the exponentials and the LDS reads alike: 512 rows a kv head after 131072 tokens 947 TFLOP/s over bf16, 919 over 8-bit pages.
// Both kinds run in one launch, those of many rows on fewer CUs than there are: 64 requests of 64 / 8 heads after 32768 shared tokens with
// 200 to 1000 of their own take 86 and 41 us one after the other, 103 together.
//
// The runs' states are joined by a second launch; where every request has one run, results go straight out.  What the kernels know
// of the batch travels with their launches up to 256 requests and 32 prefixes: an upload is a launch of 4.5 us of its own.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

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

// What a wave has of its rows: lane (quad, col) holds row `col`, dims 16 n + 4 quad .. + 3 of the output.
template <int D>
struct Rows {
  f32x4 acc[D / 16];
  float l, m;
};

// The wave's steps of a run: pages first, first + 1 .. + 3, then `stride` pages on.  Whether a page lay outside the pool.
// (Loaded values are masked as they enter the product, not in place: modified in a branch, they were given registers of other values
// by the compiler.)
template <int D, bool EIGHT>
__device__ __forceinline__ bool walk(const SharedArgs& a, const int* prow, int n_tok, int j, int first, int stride,
                                     const bf16x8 (&qf)[D / 32], Rows<D>& o) {
  constexpr int kB = EIGHT ? 1 : 2;           // bytes of a value
  constexpr int kLoads = D * kB / 64;         // 16-byte loads of a key's row by four lanes
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int n_pages = (n_tok + 15) >> 4;
  o.l = 0.f, o.m = -INFINITY;
#pragma unroll
  for (int n = 0; n < D / 16; ++n) o.acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  bool bad = false;
  int kid = 0, vid = 0;
  auto ids = [&](int p0) {
    kid = prow[min(p0 + (col >> 2), n_pages - 1)];
    vid = prow[min(p0 + quad, n_pages - 1)];
  };
  uint4 kr[4][kLoads], vr[D / 16][kB], ke = make_uint4(0, 0, 0, 0), ve = ke;
  size_t vslab = 0;
  bool vok = false;
  auto load_k = [&] {
    const bool kok = page_ok(kid, a.pages);
    const size_t kslab = (size_t)(kok ? kid : 0) * a.h_kv + j;
    const char* kp = static_cast<const char*>(a.k) + kslab * 16 * D * kB + (col & 3) * D * kB + quad * 16;
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int s = 0; s < kLoads; ++s) kr[p][s] = *reinterpret_cast<const uint4*>(kp + 4 * p * D * kB + 64 * s);
    vok = page_ok(vid, a.pages);
    bad |= !vok;
    vslab = (size_t)(vok ? vid : 0) * a.h_kv + j;
    if constexpr (EIGHT) ke = *reinterpret_cast<const uint4*>(a.scales + vslab * 32);
  };
  auto load_v = [&] {
    const char* vp = static_cast<const char*>(a.v) + vslab * 16 * D * kB + col * 16 * kB;
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
#pragma unroll
      for (int h = 0; h < kB; ++h) vr[n][h] = *reinterpret_cast<const uint4*>(vp + n * 256 * kB + 16 * h);
    if constexpr (EIGHT) ve = *reinterpret_cast<const uint4*>(a.scales + vslab * 32 + 16);
  };
  // A step's keys are loaded once the step before has its scores, its values once that has its product; page ids a step earlier.
  if (first >= n_pages) return false;
  ids(first);
  load_k();
  load_v();
  ids(first + stride);
  for (int p0 = first;; p0 += stride) {
    const int vpage = p0 + quad;
    // Tokens of page `vpage` that count.
    const int nv = vok ? max(0, min(16, n_tok - 16 * vpage)) : 0;
    const bool part = __any(nv < 16);
    // Scores S^T: the lane's are the 16 tokens of page `vpage` for row `col`.
    float sc[16];
    const unsigned kw[4] = {ke.x, ke.y, ke.z, ke.w};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if constexpr (EIGHT) {
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(make_uint2(kr[p][i].x, kr[p][i].y)), qf[2 * i], s, 0, 0, 0);
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(make_uint2(kr[p][i].z, kr[p][i].w)), qf[2 * i + 1], s, 0, 0, 0);
        } else {
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[p][i]), qf[i], s, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[4 * p + i] = s[i] * (EIGHT ? power(kw[p], i) * a.scale_log2 : a.scale_log2);
    }
    const bool more = p0 + stride < n_pages;
    if (more) {
      load_k();
      ids(p0 + 2 * stride);
    }
    if (part) {
#pragma unroll
      for (int t = 0; t < 16; ++t) sc[t] = t < nv ? sc[t] : -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int t = 1; t < 16; ++t) mx = fmaxf(mx, sc[t]);
    mx = max_rows(mx);
    if (__any(mx > o.m + (kSlack - kLift))) {
      const float to = fmaxf(o.m, mx + kLift);
      const float alpha = to == -INFINITY ? 1.f : fast_exp2(o.m - to);
      o.m = to;
      o.l *= alpha;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) o.acc[n] *= alpha;
    }
    const float sub = o.m == -INFINITY ? 0.f : o.m;  // no key yet that counts: every weight is 0
    // The denominator sums the probabilities as the second product takes them.
    const bf16x2 ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
    const uint4 vx = part ? first_bytes(ve, nv) : ve;
    const unsigned vw[4] = {vx.x, vx.y, vx.z, vx.w};
    bf16x8 pf[2];
#pragma unroll
    for (int t = 0; t < 16; t += 2) {
      const bf16x2 w = {static_cast<__bf16>(fast_exp2(sc[t] - sub)), static_cast<__bf16>(fast_exp2(sc[t + 1] - sub))};
      o.l = __builtin_amdgcn_fdot2_f32_bf16(w, ones, o.l, false);
      if constexpr (EIGHT) {
        // Times a power of two: the upper halves of the products are exact down to 2^-126, a value's 2^-93 at a weight of 1.
        const unsigned b = __builtin_bit_cast(unsigned, w);
        const unsigned x = __float_as_uint(__uint_as_float(b << 16) * power(vw[t / 4], t % 4));
        const unsigned y = __float_as_uint(__uint_as_float(b & 0xffff0000u) * power(vw[t / 4], t % 4 + 1));
        const bf16x2 z = __builtin_bit_cast(bf16x2, highs(x, y));
        pf[t / 8][t % 8] = z[0], pf[t / 8][t % 8 + 1] = z[1];
      } else {
        pf[t / 8][t % 8] = w[0], pf[t / 8][t % 8 + 1] = w[1];
      }
    }
    // Values that do not count are zeroed: their weights are 0, and 0 times NaN is NaN.
    auto product = [&](auto masked) {
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 v = vr[n][h % kB];
          if constexpr (decltype(masked)::value) v = first_bytes(v, EIGHT ? nv : 2 * nv - 16 * h);
          bf16x8 vf;
          if constexpr (EIGHT) vf = widened(h ? make_uint2(v.z, v.w) : make_uint2(v.x, v.y));
          else vf = __builtin_bit_cast(bf16x8, v);
          o.acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[h], o.acc[n], 0, 0, 0);
        }
    };
    if (part) product(std::true_type{});
    else product(std::false_type{});
    if (!more) break;
    load_v();
  }
  o.l = sum_rows(o.l);
  return __any(bad);
}

template <typename Table>
constexpr bool kIsPlain = false;
template <int R>
constexpr bool kIsPlain<SharedPlain<R>> = true;

// Item `item` of the runs of one kind (0: many rows, 1: teams, 2: lone waves): its part of a run.
__device__ __forceinline__ SharedRun run_of(const SharedArgs& a, const SharedTables& tab, int kind, int item) {
  const int first = kind == 0 ? 0 : kind == 1 ? a.n_wide : a.n_wide + a.n_team, n = kind == 0 ? a.n_wide : kind == 1 ? a.n_team : a.n_lone;
  return tab.runs[first + min(item / a.h_kv, n - 1)];
}
template <int R, int P>
__device__ __forceinline__ SharedRun run_of(const SharedArgs& a, const SharedPassed<R, P>& tab, int kind, int item) {
  int part = item / a.h_kv;
  if (kind == 0 || part < tab.parts[kind - 1]) {
    const int first = tab.kind[kind];
    const typename SharedPassed<R, P>::Prefix x =
        tab.prefixes[first + uniform(find_request(tab.kind[kind + 1] - first, [&](int i) { return tab.prefixes[first + i].first <= part; }))];
    // The blocks of rows of one part next to each other, so that its tiles are in their XCD's L2.
    const int members = x.members >> 16, member0 = x.members & 65535, split = x.split_pages, rows = members * a.group;
    const int blocks = kind ? narrow_blocks(rows) : wide_blocks(rows), waves = kind ? 0 : wide_waves(rows);
    part -= x.first;
    const int row0 = part % blocks * (kind ? kNarrowRows : 32 * waves);
    part /= blocks;
    return SharedRun{listed(tab, member0), part * split, min(x.tokens - 16 * part * split, 16 * split), part, member0, members, row0, waves};
  }
  part -= tab.parts[kind - 1];
  const int first = tab.owners[kind - 1];
  const typename SharedPassed<R, P>::Own x =
      tab.own[first + uniform(find_request(tab.owners[kind] - first, [&](int i) { return (int)(tab.own[first + i].at & 65535) <= part; }))];
  const int r = x.at >> 16 & 255, of = x.at >> 24;
  part -= x.at & 65535;
  int page0 = 0, slot = tab.slots[r] + part;
  if (of < P) {
    const int split = tab.prefixes[of].split_pages;
    page0 = tab.prefixes[of].tokens >> 4;
    slot += (page0 + split - 1) / split;
  }
  return SharedRun{r, page0 + part * tab.split_pages, min(x.tokens - 16 * part * tab.split_pages, 16 * tab.split_pages), slot, r, 1, 0, 0};
}
template <int R>
__device__ __forceinline__ SharedRun run_of(const SharedArgs& a, const SharedPlain<R>& tab, int, int item) {
  const int slot = item / a.h_kv, r = uniform(find_request(a.num_reqs, [&](int i) { return tab.first[i] <= slot; }));
  const int part = slot - tab.first[r];
  return SharedRun{r, part * tab.split_pages, min(tab.tokens[r] - 16 * part * tab.split_pages, 16 * tab.split_pages), slot, r, 1, 0, 0};
}

// The error word of a launch that nothing cleared it for: a workgroup checks every page id that the others read, 16 lanes a request.
// (All lanes on one request after another: 52 us for 256 requests of 16 to 100 tokens.)
template <int R>
__device__ void check_pages(const SharedArgs& a, const SharedPlain<R>& tab) {
  bool bad = false;
  for (int r = threadIdx.x / 16; r < a.num_reqs; r += blockDim.x / 16) {
    const int* row = a.table + (size_t)r * a.max_pages;
    for (int p = threadIdx.x % 16; p < (tab.tokens[r] + 15) >> 4; p += 16) bad |= !page_ok(row[p], a.pages);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *a.err = bad;
}

template <int D>
constexpr int team_floats(int rows) { return kTeamWaves * rows * (D + 4); }  // LDS; rows start on different banks

// Runs of up to 16 rows, by a workgroup of W waves: `block` counts the workgroups of such runs, teams first, then lone waves.
template <int D, bool EIGHT, int W, typename Table>
__device__ __forceinline__ void narrow_items(const SharedArgs& a, const Table& tab, int block, float* lds) {
  constexpr int kTeams = W / kTeamWaves;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4, wave = uniform(threadIdx.x >> 6);
  constexpr bool kChecked = kIsPlain<Table>;  // direct: the error word is another workgroup's
  const bool direct = a.direct;
  const int team_blocks = (a.team_items + kTeams - 1) / kTeams;
  const bool team = block < team_blocks;
  const int item = team ? block * kTeams + wave / kTeamWaves : (block - team_blocks) * W + wave;
  const bool has = item < (team ? a.team_items : a.lone_items);
  if (!team && !has) return;
  const SharedRun e = run_of(a, tab, team ? 1 : 2, has ? item : 0);
  const int g = a.group, rows = min(kNarrowRows, e.members * g - e.row0), j = (has ? item : 0) % a.h_kv;
  // A row as request * h_q + head.  A request alone is its row of the page table.
  auto head_of = [&](int row) {
    row += e.row0;
    return (e.members == 1 ? e.table_row : listed(tab, e.member0 + row / g)) * a.h_q + j * g + row % g;
  };
  const int head_row = col < rows ? head_of(col) : -1;
  bf16x8 qf[D / 32];
  {
    const __bf16* q = a.q + (size_t)max(head_row, 0) * D;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      // The dimensions of contraction step ks that this quad holds, as the keys' loads give them.
      const int dim = EIGHT ? 64 * (ks / 2) + 16 * quad + 8 * (ks % 2) : 32 * ks + 8 * quad;
      const uint4 u = head_row >= 0 ? *reinterpret_cast<const uint4*>(q + dim) : make_uint4(0, 0, 0, 0);
      qf[ks] = __builtin_bit_cast(bf16x8, u);
    }
  }
  auto state = [&](int head_row) {  // where the row's state goes
    const int r = head_row / a.h_q;
    return (size_t)(e.members == 1 ? e.slot : slots_of(tab, r).x + e.slot) * a.h_q + (head_row - r * a.h_q);
  };
  Rows<D> o;
  const int member = wave % kTeamWaves;  // of its team
  const int* prow = a.table + (size_t)e.table_row * a.max_pages + e.page0;
  bool bad = walk<D, EIGHT>(a, prow, has ? e.tokens : 0, j, team ? 4 * member : 0, team ? 4 * kTeamWaves : 4, qf, o);
  if (!team) {
    if (!kChecked && direct && bad && lane == 0) atomicOr(a.err, 1);
    if (head_row < 0) return;
    if (direct) {
      __bf16* y = a.out + (size_t)head_row * D + 4 * quad;
      const float inv = 1.f / o.l;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[16 * n + i] = static_cast<__bf16>(o.acc[n][i] * inv);
      return;
    }
    const size_t at = state(head_row);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) *reinterpret_cast<f32x4*>(a.acc + at * D + 16 * n + 4 * quad) = o.acc[n];
    if (quad == 0) a.ml[at] = make_float2(o.m, marked(o.l, bad));
    return;
  }
  // The team's four states are joined through LDS.
  float* const part = lds + wave / kTeamWaves * team_floats<D>(kNarrowRows);
  float* mine = part + (member * rows + col) * (D + 4);
  if (col < rows) {
#pragma unroll
    for (int n = 0; n < D / 16; ++n) *reinterpret_cast<f32x4*>(mine + 16 * n + 4 * quad) = o.acc[n];
    if (quad == 0) mine[D] = o.m, mine[D + 1] = o.l;
  }
  bad = __syncthreads_or(bad);
  if (!kChecked && direct && bad && threadIdx.x == 0) atomicOr(a.err, 1);
  if (!has) return;
  for (int x = 4 * (64 * member + lane); x < rows * D; x += 4 * 64 * kTeamWaves) {
    const int row = x / D, dim = x % D;
    const float* p = part + row * (D + 4);
    float m[kTeamWaves], to = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < kTeamWaves; ++w) m[w] = p[w * rows * (D + 4) + D], to = fmaxf(to, m[w]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kTeamWaves; ++w) {
      const float f = m[w] == -INFINITY ? 0.f : fast_exp2(m[w] - to);
      l += f * p[w * rows * (D + 4) + D + 1];
      sum += f * *reinterpret_cast<const f32x4*>(p + w * rows * (D + 4) + dim);
    }
    const int to_row = head_of(row);
    if (direct) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      const float inv = 1.f / l;
      *reinterpret_cast<bf16x4*>(a.out + (size_t)to_row * D + dim) =
          bf16x4{static_cast<__bf16>(sum[0] * inv), static_cast<__bf16>(sum[1] * inv), static_cast<__bf16>(sum[2] * inv),
                 static_cast<__bf16>(sum[3] * inv)};
    } else {
      const size_t at = state(to_row);
      *reinterpret_cast<f32x4*>(a.acc + at * D + dim) = sum;
      if (dim == 0) a.ml[at] = make_float2(to, marked(l, bad));
    }
  }
}

template <int D, bool EIGHT, typename Table>
__global__ __launch_bounds__(64 * kTeamWaves) void shared_narrow(SharedArgs a, Table tab) {
  extern __shared__ __attribute__((aligned(16))) float part[];
  if constexpr (kIsPlain<Table>) {
    if (a.direct) {
      if (blockIdx.x == 0) check_pages(a, tab);
      else narrow_items<D, EIGHT, kTeamWaves>(a, tab, blockIdx.x - 1, part);
      return;
    }
  }
  if (!a.direct && blockIdx.x == 0 && threadIdx.x == 0) *a.err = 0;  // the join sets it
  narrow_items<D, EIGHT, kTeamWaves>(a, tab, blockIdx.x, part);
}

// Runs of many rows first, then those of few: the one is bound by the matrix cores, the other by memory.
template <int D, bool EIGHT, typename Table>
__global__ __launch_bounds__(kWideThreads, 1) void shared_mixed(SharedArgs a, Table tab) {
  extern __shared__ __attribute__((aligned(16))) __bf16 lds[];
  const int item = blockIdx.x;
  if (item == 0 && threadIdx.x == 0) *a.err = 0;  // the join sets it
  if (item >= a.wide_items) {
    narrow_items<D, EIGHT, kWideWaves>(a, tab, item - a.wide_items, reinterpret_cast<float*>(lds));
    return;
  }
  wide_item<D, EIGHT>(a, tab, run_of(a, tab, 0, item), item % a.h_kv, lds);
}

// Joins the runs of one (request, query head): W waves, each every W-th run, eight loads in flight.
template <int D, int W, typename Table>
__global__ __launch_bounds__(64 * (W > 4 ? W : 4)) void shared_merge(SharedArgs a, Table tab) {
  constexpr int E = D / 64;
  __shared__ float part[W > 1 ? W : 1][D + 2];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), w = wave % W;
  const int pair = W >= 4 ? (int)blockIdx.x : (int)(blockIdx.x * 4 + wave) / W;
  if (pair >= a.num_reqs * a.h_q) return;  // the whole workgroup where W is not 1
  const int r = pair / a.h_q;
  const int2 at = slots_of(tab, r);
  const size_t first = (size_t)at.x * a.h_q + pair - r * a.h_q;
  float top = -INFINITY, den = 0.f, num[E] = {};
  const float lift = at.y > 1 ? 32 - __builtin_clz(at.y - 1) : 0;  // weights of at most 1 / slots: the sum is no larger than a run's
  bool bad = false;
  for (int s0 = w; s0 < at.y; s0 += 8 * W) {
    float2 ml[8];
    float x[8][E];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = min(s0 + u * W, at.y - 1);
      const size_t row = first + (size_t)s * a.h_q;
      ml[u] = a.ml[row];
#pragma unroll
      for (int i = 0; i < E; ++i) x[u][i] = a.acc[row * D + 64 * i + lane];
    }
    float to = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      bad |= __float_as_uint(ml[u].y) >> 31;
      ml[u].y = fabsf(ml[u].y);
      to = fmaxf(to, ml[u].x);
    }
    // Runs without a key that counts weigh 0, and a NaN among their denominators stays.
    const float ref = to == -INFINITY ? 0.f : to, f = fast_exp2(top - ref), sub = ref + lift;
    top = to;
    den *= f;
#pragma unroll
    for (int i = 0; i < E; ++i) num[i] *= f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool there = s0 + u * W < at.y;  // selected, not branched on: the loads stay together
      const float wgt = fast_exp2(ml[u].x - sub);
      den += there ? wgt * ml[u].y : 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) num[i] += there ? wgt * x[u][i] : 0.f;
    }
  }
  if (bad && lane == 0) atomicOr(a.err, 1);
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

// Waves for each (request, query head) so that a round or two of loads is enough where there are few of them (us of 32 with 16 runs: one
// wave 4.3, four 3.4; of 4096 with 13: 7.2 against 9.4), within the 2^32 threads that a grid may have.
template <int D, typename Table>
void launch_merge(const SharedArgs& a, const Table& tab, hipStream_t s) {
  const int pairs = a.num_reqs * a.h_q;
  if (a.max_slots > 64 && pairs <= 1 << 21) hipLaunchKernelGGL((shared_merge<D, 16, Table>), dim3(pairs), dim3(1024), 0, s, a, tab);
  else if (a.max_slots > (pairs < 1024 ? 8 : 16) && pairs <= 1 << 23) hipLaunchKernelGGL((shared_merge<D, 4, Table>), dim3(pairs), dim3(256), 0, s, a, tab);
  else hipLaunchKernelGGL((shared_merge<D, 1, Table>), dim3((pairs + 3) / 4), dim3(256), 0, s, a, tab);
}

template <int D, typename Table>
void join(const SharedArgs& a, const Table& tab, hipStream_t s) {
  launch_merge<D>(a, tab, s);
}
template <int D, int R, int P>
void join(const SharedArgs& a, const SharedPassed<R, P>& tab, hipStream_t s) {  // the slots are all that it reads
  SharedSlots<R> slots;
  std::copy(tab.slots, tab.slots + a.num_reqs + 1, slots.slots);
  launch_merge<D>(a, slots, s);
}

template <int D, bool EIGHT, typename Table>
hipError_t launch(const SharedArgs& a, const Table& tab, hipStream_t s) {
  constexpr bool kPlain = kIsPlain<Table>;
  auto blocks = [&](int waves) {
    return (a.team_items + waves / kTeamWaves - 1) / (waves / kTeamWaves) + (a.lone_items + waves - 1) / waves;
  };
  bool wide = false;
  if constexpr (!kPlain) {
    if (a.wide_items) {
      wide = true;
      constexpr size_t kBytes = std::max(WideLds<D, EIGHT>::kBytes, 2 * team_floats<D>(kNarrowRows) * sizeof(float));
      static const hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void*>(&shared_mixed<D, EIGHT, Table>),
                                                        hipFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
      if (set != hipSuccess) return set;
      hipLaunchKernelGGL((shared_mixed<D, EIGHT, Table>), dim3(a.wide_items + blocks(kWideWaves)), dim3(kWideThreads), kBytes, s, a, tab);
    }
  }
  if (!wide)
    hipLaunchKernelGGL((shared_narrow<D, EIGHT, Table>), dim3(blocks(kTeamWaves) + (kPlain && a.direct ? 1 : 0)),
                       dim3(64 * kTeamWaves), team_floats<D>(kIsPlain<Table> ? a.group : kNarrowRows) * sizeof(float), s, a, tab);
  if (a.direct) return hipGetLastError();
  join<D>(a, tab, s);
  return hipGetLastError();
}
template <typename Table>
hipError_t launch(const SharedArgs& a, const Table& t, hipStream_t s) {
  if (a.scales) return a.head_dim == 128 ? launch<128, true>(a, t, s) : launch<64, true>(a, t, s);
  return a.head_dim == 128 ? launch<128, false>(a, t, s) : launch<64, false>(a, t, s);
}

SharedPassed<kSharedFew, kSharedFewPrefixes> few(const SharedArgs& a, const SharedPassedAll& t) {
  SharedPassed<kSharedFew, kSharedFewPrefixes> f;
  for (int i = 0; i < t.kind[3]; ++i) f.prefixes[i] = {t.prefixes[i].tokens, t.prefixes[i].first, t.prefixes[i].split_pages, t.prefixes[i].members};
  for (int i = 0; i < t.owners[2]; ++i) f.own[i] = {t.own[i].tokens, t.own[i].at};
  std::copy(t.slots, t.slots + a.num_reqs + 1, f.slots);
  std::copy(t.list, t.list + kSharedFew / 4, f.list);
  std::copy(t.kind, t.kind + 4, f.kind);
  std::copy(t.owners, t.owners + 3, f.owners);
  f.split_pages = t.split_pages;
  std::copy(t.parts, t.parts + 2, f.parts);
  return f;
}
SharedPlain<kSharedFew> few(const SharedArgs& a, const SharedPlainAll& t) {
  SharedPlain<kSharedFew> f;
  std::copy(t.first, t.first + a.num_reqs + 1, f.first);
  std::copy(t.tokens, t.tokens + a.num_reqs, f.tokens);
  f.split_pages = t.split_pages;
  return f;
}

}  // namespace

hipError_t launch_shared(const SharedArgs& a, const SharedTables& tables, const SharedPassedAll* passed, const SharedPlainAll* plain,
                         hipStream_t s) {
  if (a.num_reqs == 0) return hipSuccess;
  if (plain) return passed_tables(a.num_reqs, 0) == kSharedFew ? launch(a, few(a, *plain), s) : launch(a, *plain, s);
  if (passed) return passed_tables(a.num_reqs, passed->kind[3]) == kSharedFew ? launch(a, few(a, *passed), s) : launch(a, *passed, s);
  return launch(a, tables, s);
}

}  // namespace duet
