// Host side of the 8-bit KV cache's plan, shared by its own entry points and the step's.
#pragma once
#include <vector>

#include "../../include/wisp.h"
#include "kv8.h"

namespace wisp {

struct Kv8Build {
  Kv8Plan p{};
  std::vector<int32_t> host;      // the arrays that the device needs; the i_ are places in it
  size_t i_units = 0, i_items = 0, i_first = 0, i_groups = 0, i_pos = 0;
  size_t po_bytes = 0, pml_bytes = 0, cs_bytes = 0;
};
// the plan of a checked model and batch, not yet placed in a workspace
wisp_status kv8_build(Kv8Build &b, const wisp_model *m, const wisp_batch_desc *d);
// places it: `host` at byte desc of ws, partial results and the rotation table from scratch on
void kv8_place(Kv8Build &b, char *ws, size_t desc, size_t scratch);
// checks a cache and takes its pointers
wisp_status kv8_cache(Kv8Cache &c, const wisp_kv8 *kv);

}  // namespace wisp
