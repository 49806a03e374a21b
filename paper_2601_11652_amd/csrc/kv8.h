// The 8-bit KV cache (e4m3 codes, one fp32 scale for K and one for V per page and kv head): page
// layout, the planned batch and the launchers of its append and attention kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace wisp {

// ---------------------------------------------------------------------------------------
// page layout: 16 slots x hd codes of one block and kv head.  Both orders give every lane of
// the attention kernel 16 consecutive bytes per load: for K the same 8 dims of two slots 4
// apart (one in each of the two products over a page pair), for V the same 8 slots of two dims
// 16 apart (one in each of two blocks of output dims).
// ---------------------------------------------------------------------------------------
__host__ __device__ inline int k8_page_off(int slot, int e) {
  return (((e >> 5) * 4 + ((e & 31) >> 3)) * 8 + (slot >> 3) * 4 + (slot & 3)) * 16 + ((slot >> 2) & 1) * 8 + (e & 7);
}
__host__ __device__ inline int v8_page_off(int slot, int e) {
  return ((e >> 5) * 2 + (slot >> 3)) * 256 + (e & 15) * 16 + ((e >> 4) & 1) * 8 + (slot & 7);
}

constexpr float kE4m3Max = 448.f;

// ---------------------------------------------------------------------------------------
// the planned batch
// ---------------------------------------------------------------------------------------
struct Kv8Unit {    // a page that gets new rows: `held` valid slots before, then `rows` new ones
  int32_t req, page, row, held_rows;   // page: index in the request's table; held | rows << 8
};
struct Kv8Item {    // attention of up to four row groups over tokens t0 .. t1 - 1 of their request
  int32_t req, t0, t1, ctx;
  int32_t row0, nrow, groups, part;    // first row and rows of the request; kv8_pack; first partial, -1: none
};
struct Kv8Group {   // the partials of one row group, `stride` apart, combined in order
  int32_t row0, nrow, rbg, part, n_parts, stride, pad[2];
};
// an item's first row group and their number
inline int32_t kv8_pack(int first, int n) { return first | (n - 1) << 24; }
__host__ __device__ inline int kv8_first(int32_t g) { return g & 0xFFFFFF; }
__host__ __device__ inline int kv8_groups(int32_t g) { return (g >> 24) + 1; }

constexpr int kKv8MaxItems = 1 << 22;  // work items of one batch

struct Kv8Plan {    // a wisp_kv8_batch
  uint64_t magic;
  const int32_t *page_table;
  char *ws;
  int32_t device, dtype, nq, nkv, hd, rows, B;
  int32_t pt_stride, n_units, n_items, n_shares, n_groups, rb, n_parts, stream, n_wide;
  // byte offsets in the workspace
  uint64_t w_units, w_items, w_first, w_groups, w_pos, w_cs, w_po, w_pml, total;
};

struct Kv8Cache {   // one layer's pools
  uint8_t *k, *v;
  float *scale;     // [n_blocks][n_kv][2]
  int n_blocks;
};

// The projection's output, rows x (nq + 2 nkv) heads: of the model's type with row stride ld
// (splits = 0), or `splits` fp32 partial results, `stride` elements apart, to be added in order
struct QkvRows {
  const void *p;
  int64_t ld, stride;
  int splits;
};

void kv8_append(const Kv8Plan &p, const Kv8Cache &c, const QkvRows &src, void *q, int *err, hipStream_t s);
// out: rows x nq * hd, row-major, or in the fragment order of a projection's input (packed, bf16)
void kv8_attention(const Kv8Plan &p, const Kv8Cache &c, const void *q, void *out, bool packed, int *err, hipStream_t s);

}  // namespace wisp
