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
  int32_t parts, single, groups;  // parts of a page's rows; every request has one row; groups of workgroups (the launch sets them)
};
hipError_t launch_norm_split(const NormSplitArgs& a, const int4* requests, hipStream_t s);

// Requests' pages out of the 8-bit cache into bf16 pages (cache8.hip).
struct Cache8ReadArgs {
  const uint8_t *k, *v, *scales;
  const int32_t *table, *out_table;
  __bf16 *k_out, *v_out;
  const int2* reqs;  // [R] (pages of the requests before it, tokens), uploaded with the workspace; not used without one
  long long pages, out_pages;
  int32_t* err;      // the workspace's, else null
  int32_t num_reqs, max_pages, out_max_pages, h_kv, head_dim, groups;
};
// reqs: where there is no workspace, [R + 1] on the host, for up to kRopeTable requests.
hipError_t launch_cache8_read(const Cache8ReadArgs& a, const int2* reqs, hipStream_t s);

// Decode attention over runs of pages that one or several requests share (attn_shared.hip).  A run is attended by the query
// rows of its members, requests listed from list[member0] on: of each the g heads of a kv head.  A workgroup, a team of its waves or
// a wave takes a run (or a part of it and of its rows) and a kv head, heads next to each other.
struct SharedRun {
  int32_t table_row, page0, tokens;  // pages from page0 of a row of the page table
  int32_t slot;      // where the rows' states go: of one member, else counted from each member's first slot
  int32_t member0, members;
  int32_t row0, waves;  // the first row; of many rows: a workgroup's waves with rows
};
// A run before it is cut: part s is of split_pages pages and goes to slot + s.
struct SharedEntry {
  SharedRun run;
  int32_t first_item, split_pages;  // items (part, block of rows, head) of its kind's entries before it
};
constexpr int kWideRows = 256, kNarrowRows = 16;
constexpr int kWidePages = 1024;  // most pages of a part of a run of many rows
constexpr int kTeamWaves = 4;
inline __host__ __device__ int narrow_blocks(int rows) { return (rows + kNarrowRows - 1) / kNarrowRows; }
inline __host__ __device__ int wide_blocks(int rows) { return (rows + kWideRows - 1) / kWideRows; }
inline __host__ __device__ int wide_waves(int rows) {  // of a workgroup, where the blocks share the rows evenly
  return ((rows + 31) / 32 + wide_blocks(rows) - 1) / wide_blocks(rows);
}

// What of the batch the kernels read, in one of three ways: runs of many rows (wide) come first, then those of at most kNarrowRows
// rows that a team of waves takes, and those of so few pages that a wave takes them alone.
struct SharedTables {  // in device memory, every part of a run listed
  const SharedRun* runs;
  const int32_t* list;
  const int2* slots;  // [R] (first slot, slots)
};
// Tables that travel with the launches: for up to 256 requests, and for up to 32, since 4 KB of arguments cost the host 1 us a launch
// more (a call of one request 12.5 us against 12.0).  Uploaded ones cost a call some 4 us (256 / 257 requests of 100 tokens 22.2 / 25.9,
// behind five prefixes of 4000 tokens 77.2 / 81.6), and the host 0.03 us a request (1024 requests 50 to 80 us a call, under their kernels'
// 80 to 1480).
constexpr int kSharedPassed = 256, kSharedPrefixes = 32, kSharedFew = 32, kSharedFewPrefixes = 8;
// Words throughout: of arrays of bytes and of words with one index the compiler made scalar loads whose base was odd, which drop its
// low bits.
template <int R, int P>
struct SharedPassed {  // up to R requests, P prefixes and 65535 slots
  struct Prefix {
    int32_t tokens, first;      // first: items before its, of one kv head and its kind
    uint32_t split_pages;
    uint32_t members;           // the first of its members in the list, and from bit 16 on how many they are
  } prefixes[P];  // by their kind
  struct Own {                  // a request's tokens behind its prefix
    int32_t tokens;
    uint32_t at;                // parts before its, of its kind; from bit 16 on the request, from bit 24 its prefix or 255
  } own[R];         // those that teams take, then lone waves
  int32_t slots[R + 1];         // the requests' first ones, their end after the last
  uint32_t list[R / 4];         // the prefixes' members, a byte each
  int32_t kind[4], owners[3];   // where the kinds' prefixes and requests start
  int32_t split_pages;          // of the requests' own runs
  int32_t parts[2];             // of the prefixes that teams and lone waves take, with their blocks of rows
};
template <int R>
struct SharedSlots {
  int32_t slots[R + 1];
};
template <int R>
struct SharedPlain {  // up to R requests that share nothing, all of them taken by teams or all by lone waves
  int32_t first[R + 1];  // the requests' first slots, the slots' end after the last
  int32_t tokens[R];
  int32_t split_pages;
};
constexpr int kSharedCheckedPages = 8192;  // page ids that a workgroup beside the others checks

struct SharedArgs {
  const __bf16* q;  // [R, h_q, d]
  const void *k, *v;
  const uint8_t* scales;  // null: bf16 pages
  const int32_t* table;
  long long pages;
  __bf16* out;
  float* acc;                  // [slots, h_q, d] unnormalised outputs
  float2* ml;                  // [slots, h_q] (reference in base-2 units, denominator; the latter's sign bit: a bad page)
  int32_t* err;
  int32_t num_reqs, max_pages, h_q, h_kv, group, head_dim;
  int32_t n_wide, n_team, n_lone;  // runs (of SharedTables)
  int32_t wide_items, team_items, lone_items;
  int32_t max_slots;  // of a request
  int32_t direct;     // one slot each and no run of many rows: the results go straight to out
  float scale_log2;
};
using SharedPassedAll = SharedPassed<kSharedPassed, kSharedPrefixes>;
using SharedPlainAll = SharedPlain<kSharedPassed>;
static_assert(sizeof(SharedArgs) + sizeof(SharedPassedAll) <= 4096, "arguments of a launch");
inline int passed_tables(int num_reqs, int prefixes) {  // requests of the smallest tables that hold so many
  return num_reqs <= kSharedFew && prefixes <= kSharedFewPrefixes ? kSharedFew : kSharedPassed;
}
// On the host one of plain and passed, or neither (then what `tables` names is in device memory).
hipError_t launch_shared(const SharedArgs& a, const SharedTables& tables, const SharedPassedAll* passed, const SharedPlainAll* plain,
                         hipStream_t s);

}  // namespace duet
