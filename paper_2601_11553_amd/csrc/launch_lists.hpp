// What the host hands to the kernels of packed_attention.hip and kv_fork.hip.
#pragma once

#include "percache_internal.hpp"

namespace pc {
namespace packed {
constexpr int kWide = 0, kNarrow = 1;      // kinds of items
constexpr int kWideRows = 256, kNarrowRows = 32;

// A workgroup's work, for every kv head: rows() stacked rows from head rem0 of token i0 of a request on, over n_cached cached tiles from tile tile0 of
// chunk entry ent on, then over the fresh tiles [f0, f1).
struct Item {
  int32_t row0, T, i0, n_cached, ent, tile0, f0, f1;
  int32_t slot0, used0;     // entry ent: a workgroup's first tiles are asked for before its entries are there
  int32_t part;             // first row of its partial results, -1: it is the block's only partition
  uint16_t rem0, rows_kind; // rows * 2 + kind
  __host__ __device__ int rows() const { return rows_kind >> 1; }
  __host__ __device__ int kind() const { return rows_kind & 1; }
};
constexpr int kItemWords = sizeof(Item) / 4;
struct Merge { int32_t row0, i0, rem0, rows, part, n; };   // partition p of the block has its partial rows from part + p * rows on
constexpr int kMergeWords = sizeof(Merge) / 4;

struct Args {
  const __bf16 *q, *k, *v;   // [heads][N][D]
  const __bf16 *k16, *v16;
  const uint8_t *k8, *v8;
  const float *k_scale, *v_scale;
  const int32_t *words;      // items, merges, chunk entries (slot, used length > 0)
  __bf16 *out;               // [N][Hq * D]
  float *lse;                // [Hq][N] or null
  float *part_o, *part_ml;   // [part_rows of every kv head][D], [...][2]
  long N, part_rows;
  int merges_at, ents_at, n_ents, Hq, Hkv, C, n_slots16;
  unsigned per_group;        // 2^32 / G, rounded up: x / G = the upper half of x times it for the small x of a block
  float scale_log2e;
};

// Lists that fit a launch's arguments are read from there: no launch in front that copies them.
constexpr int kArgWords = (4096 - (int)sizeof(Args)) / 4;
struct ArgsAndWords {
  Args a;
  int32_t words[kArgWords];
};

}  // namespace packed

namespace fork {
constexpr int kMoves = 240;   // moves of a launch (its arguments are at most 4096 bytes)
struct Move { int32_t src, dst, len; };   // slots of one store; dst -1: src into the registers; src -1: from them
struct Moves {
  Move m[kMoves];
  uint16_t start[kMoves + 1];   // moves start[p] .. start[p + 1] depend on each other
};

}  // namespace fork
}  // namespace pc
