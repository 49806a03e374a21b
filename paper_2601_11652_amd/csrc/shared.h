// Batches whose requests share prefixes: the planned batch and the launchers of its kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace wisp {

constexpr int kTile = 32;              // query rows, and tokens, of a matrix product's tile

// Rows that read one run of tokens: a group's rows and the prefix that they share (its table the first
// request's), or a request's rows and the tokens of its own.  Row j sees the tokens up to ctx + j.
// Every kv head has the same work: lists are of one, and a launch's workgroups are item x kv head.
struct SharedItem {                    // up to four row tiles of a segment over tokens t0 .. t1 - 1
  int32_t table, t0, t1, ctx;
  int32_t row0, nrow, tile0, tiles;    // the segment's first row and rows; first row tile, row tiles
  int32_t part, step, pad[2];          // kv head 0's first partial result (a tile each), those of a head; -1: none
};
// The partial results of a bundle of row tiles (four of a segment's, the last one's rest) lie [part][kv head][row tile]
// from tile `at` on, a tile in the order of the accumulators.  A row has those of its own segment's
// bundle, and of its group's; one in all was written as it was computed.
struct SharedBundle {
  int32_t at, parts, tiles, row;       // row: in a SharedRow, the flat row in it
};
struct SharedRow {                     // of a row of the batch: where head 0 of a kv head lies
  SharedBundle own, pre;               // in the request's segment, in its group's (no parts: there is none)
  int32_t own_next, pre_next;          // the bundles behind them, in which the last heads of a row may lie
};

// Column sums of a segment's probabilities: tokens t0 .. t1 - 1 (a block of them; of one stage of rows some
// blocks), flat rows r0 .. r1 - 1
struct MassItem {
  int32_t table, t0, t1, ctx;
  int32_t row0, nrow, req, r0;         // req: the request whose rows these are, -1: a group's
  int32_t r1, part, step, pad;         // kv head 0's partial sums, those of a head; -1: the only ones
};
struct MassJoin {                      // a token block whose sums have several parts
  int32_t table, t0, t1, ctx;
  int32_t part, parts, step, pad;
};

constexpr int kBundle = 4;             // row tiles of a workgroup
constexpr int kMassBlock = 4 * kTile;  // tokens of a workgroup: a tile a wave
constexpr int kMassTiles = 512;        // row tiles of an item at most
constexpr int kSharedMaxItems = 1 << 22;

struct SharedPlan {                    // a wisp_shared_batch
  uint64_t magic;
  const int32_t *page_table;
  char *ws;
  int32_t device, dtype, nq, nkv, hd, rows, B;
  int32_t pt_stride, n_items, n_parts, joined, n_mass, n_mass_join, pad;
  // byte offsets in the workspace; w_row: a row's request
  uint64_t w_items, w_bundles, w_row, w_join, w_mass, w_mass_join, w_po, w_pml, w_pm, total;
};

struct SharedCache {                   // one layer's pools
  const void *k, *v;
  int n_blocks;
};

void shared_attention(const SharedPlan &p, const SharedCache &c, const void *q, void *out, float *lse, int *err, hipStream_t s);
void shared_mass(const SharedPlan &p, const SharedCache &c, const void *q, const float *lse, const int32_t *count, float decay,
                 const float *prev, float *mass, int *err, hipStream_t s);
// workgroups that a CU holds
int shared_wgs_per_cu(int dtype, int hd);
int mass_wgs_per_cu(int dtype, int hd);
int mass_stage_tiles(int dtype, int hd);   // row tiles that the weights' kernel has at a time

}  // namespace wisp
