// Device code that the splits with a position rotation share (internal): sines, the requests' page groups, the check of page ids.
#pragma once

#include <hip/hip_runtime.h>

#include "serving_ops.h"
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
  const int q = (int)(quarter - 4.0 * floor(0.25 * quarter));
  const float x = q & 1 ? s : c, y = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y);
}

// The requests as the kernel reads them: first row, rows, cached tokens.
struct Request {
  int row, rows, cached;
};
struct Uploaded {
  const int4* meta;
  __device__ __forceinline__ int row(int r) const { return meta[r].y; }
  __device__ __forceinline__ Request operator[](int r) const { return Request{meta[r].y, meta[r].z, meta[r].w}; }
};
struct Passed {
  int2 at[kRopeTable + 1];  // (first row, cached tokens); the rows' end after the last
  __device__ __forceinline__ int row(int r) const { return at[r].x; }
  __device__ __forceinline__ Request operator[](int r) const { return Request{at[r].x, at[r + 1].x - at[r].x, at[r].y}; }
};
__device__ __forceinline__ int first_group(int row, int r) { return (row >> 4) + 2 * r; }

// The group's page of its request: where its rows start and how many they are (0 or less: past the last page).
struct Group {
  int row, pos, rows, page;
};
__device__ __forceinline__ Group group_of(const Request& q, int r, int group) {
  const int page = (q.cached >> 4) + group - first_group(q.row, r);
  const int pos = max(q.cached, 16 * page);
  return Group{q.row + pos - q.cached, pos, min(q.cached + q.rows, 16 * page + 16) - pos, page};
}

template <typename T>
struct Chunk {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};

constexpr int kMaxPairs = 64;

// Whether any page id of the batch lies outside the pool, into the error word; one workgroup.
__device__ void check_pages(const RopeSplitArgs& s, const Passed& requests, int2* at) {
  for (int i = threadIdx.x; i <= s.num_reqs; i += 256) at[i] = requests.at[i];
  __syncthreads();
  bool bad = false;
  const int groups = s.tokens / 16 + 2 * s.num_reqs;
  for (int g = threadIdx.x; g < groups; g += 256) {
    int r = 0, end = s.num_reqs;
    while (end - r > 1) {
      const int mid = (r + end) / 2;
      if (first_group(at[mid].x, mid) <= g) r = mid;
      else end = mid;
    }
    const Group group = group_of(Request{at[r].x, at[r + 1].x - at[r].x, at[r].y}, r, g);
    if (group.rows > 0) bad |= !page_ok(s.page_table[(size_t)r * s.max_pages + group.page], s.num_phys_pages);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *s.err = bad;
}

}  // namespace
}  // namespace duet
