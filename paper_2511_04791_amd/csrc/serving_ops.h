// Launch interface of the token-level operators of a served model (internal): the rotating QKV split, adapters, sampling.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "duet.h"

namespace duet {

// The QKV split with the position rotation on the way (rope_split.hip), bf16 or fp32.
struct RopeSplitArgs {
  const void* qkv;         // [T, (h_q + 2 h_kv) d]
  void* q;                 // [T, h_q, d]
  void* k_cache;           // [P, h_kv, 16, d]
  void* v_cache;           // [P, h_kv, d, 16]
  const int4* meta;        // [R] (kind, q_start, q_len, cached_len), uploaded; not used for up to kRopeTable requests
  const int32_t* page_table;
  const int32_t* positions;  // [axes, T], or null: the tokens' places in the cache
  long long num_phys_pages;
  int32_t* err;            // may be null for up to kRopeTable requests
  int32_t num_reqs, max_pages, h_q, h_kv, head_dim, dtype, tokens;
  int32_t rot_dim, adjacent;
  double turns[64];        // turns per position of each pair (frequency / 2 pi)
  uint8_t pair_axis[64];
};
constexpr int kRopeTable = DUET_ROPE_NO_WORKSPACE;
hipError_t launch_rope_split(const RopeSplitArgs& a, const int4* requests, hipStream_t s);  // requests: the batch, on the host

// out = base + scale_a B_a (A_a x) of each token's adapter a (lora.hip).  The rows are taken by adapter in tiles; row i of a
// tile is rows + i, or entry ~rows + i of a list where the tile's rows do not follow each other.
constexpr int kLoraTileRows = 64;
struct LoraTile {
  int32_t adapter, first, count, rows;  // -1: none; the tiles' rows before this one; its rows
};
struct LoraArgs {
  const __bf16 *x, *base, *a, *b;  // x [T, d_in], base [T, d_out], a [N, rank, d_in], b [N, d_out, rank]
  __bf16* out;                     // [T, d_out]
  const float* scale;              // [N], or null: 1
  float* part;                     // [parts, T, rank], rows in the tiles' order
  const LoraTile* tiles;
  const int32_t* rows;             // the list
  long long ldx, ldb, ldo;
  int32_t n_tiles, parts, tokens, rank, d_in, d_out;
};
// Parts of the input's columns, each a workgroup a tile.  A CU pulls at most some 30 GB/s of its own from memory, so the 256 CUs'
// largest share counts, and a little for each part; at least four 64-column units a part.  us of the down product with
// 1 / 2 / 4 / 5 / 6 / 8 parts: 17 tiles of a few rows, 4096 columns, rank 16, 8.0 / 5.4 / 4.5 / . / 4.5 / 4.0; 41 tiles (2112 rows)
// 20 / 14 / 11 / . / 11 / 12; 100 tiles (6298 rows) of 14336 columns, rank 64, 82 / 56 / 59 / 53 / 73 / 69.
constexpr int kLoraMaxParts = 8;
int lora_most_parts(int tokens, int d_in);
int lora_parts(int tiles, int most);
hipError_t launch_lora(const LoraArgs& a, hipStream_t s);
// The same with the lists on the host: a.tiles and a.rows are not used.
constexpr int kLoraPassedTiles = 128, kLoraPassedRows = 256;
hipError_t launch_lora_passed(const LoraArgs& a, const LoraTile* tiles, const int32_t* rows, int n_rows, hipStream_t s);

// One token from each row of logits (sample.hip); the parameters' arrays may be null.
struct SampleArgs {
  const void* logits;  // [rows, vocab]
  long long row_stride;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* ids;
  float* probs;  // may be null
  int32_t dtype, rows, vocab;
};
constexpr int kMaxVocab = 1 << 18;
size_t sample_workspace(int rows, int vocab);  // bytes, on 16; may be 0
hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s);

}  // namespace duet
