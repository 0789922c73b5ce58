// Launch interface of the operators around the 8-bit cache and shared prefixes (internal).
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "serving_ops.h"

namespace duet {

// The rotating QKV split with a norm of each head before the rotation, into pages of the projection's type or 8-bit
// ones (norm_split.hip).  rope.rot_dim 0: nothing turns.  For 8-bit pages k_cache and v_cache hold bytes.
struct NormSplitArgs {
  RopeSplitArgs rope;
  const void *wq, *wk;  // [d] of rope.dtype, or null: ones
  float eps;
  int32_t norm;         // heads are normalised
  uint8_t* scales;      // [P, h_kv, 2, 16] of 8-bit pages, else null
  int32_t parts, single;  // parts of a page's rows; every request has one row (the launch sets both)
};
hipError_t launch_norm_split(const NormSplitArgs& a, const int4* requests, hipStream_t s);

// Requests' pages out of the 8-bit cache into bf16 pages (cache8.hip).
struct Cache8ReadArgs {
  const uint8_t *k, *v, *scales;
  const int32_t *table, *out_table;
  __bf16 *k_out, *v_out;
  const int2* reqs;  // [R + 1] (pages of the requests before it, tokens), uploaded; not used for up to kRopeTable requests
  long long pages, out_pages;
  int32_t* err;      // may be null for up to kRopeTable requests
  int32_t num_reqs, max_pages, out_max_pages, h_kv, head_dim, groups;
};
hipError_t launch_cache8_read(const Cache8ReadArgs& a, const int2* reqs, hipStream_t s);

// Decode attention over runs of pages that one or several requests share (attn_shared.hip).  An entry is a run and the
// query rows that attend it: of `members` requests, listed from list[member0] on, the g heads of each kv head.
struct SharedEntry {
  int32_t first_item;  // items (split, kv head, row block) of its kind's entries before it
  int32_t member0, members;
  int32_t table_row, page0, tokens;  // the run: pages from page0 of a row of the page table
  int32_t split_pages;
  int32_t slot_off;    // split s of member r is slot first_slot[r] + slot_off + s
};
// What of the batch the kernels read: entries of many rows (wide), of at most kNarrowRows rows in runs that a team of waves
// takes, and of so few pages that a wave takes them alone; the members' requests; (first slot, slots) of each request.
constexpr int kSharedPassed = 64;  // up to this many entries and requests travel with the launches
struct SharedTables {
  const SharedEntry* entries;
  const int32_t* list;
  const int2* slots;
};
struct SharedPassed {
  SharedEntry entries[kSharedPassed];
  int32_t list[2 * kSharedPassed];
  int2 slots[kSharedPassed];
};
struct SharedArgs {
  const __bf16* q;  // [R, h_q, d]
  const void *k, *v;
  const uint8_t* scales;  // null: bf16 pages
  const int32_t* table;
  long long pages;
  __bf16* out;
  float* acc;                  // [slots, h_q, d] unnormalised outputs
  float2* ml;                  // [slots, h_q] (reference maximum in base-2 units, denominator; the latter's sign bit: a bad page)
  int32_t* err;
  int32_t num_reqs, max_pages, h_q, h_kv, group, head_dim;
  int32_t n_wide, n_team, n_lone, wide_items, team_items, lone_items;
  int32_t max_slots;  // of a request
  int32_t direct;     // one slot each and no wide entry: the results go straight to out, and err is clear beforehand
  float scale_log2;
};
constexpr int kWideRows = 256, kNarrowRows = 16;
constexpr int kWidePages = 1024;  // most pages of a wide split
constexpr int kTeamWaves = 4;
// passed: on the host, or null (then `tables` is in device memory).
hipError_t launch_shared(const SharedArgs& a, const SharedTables& tables, const SharedPassed* passed, hipStream_t s);

}  // namespace duet
