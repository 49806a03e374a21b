// C ABI of the operators on batches whose requests share prefixes (declared in include/wisp.h): the plan of a
// batch and the calls that run on it.
#include <algorithm>
#include <climits>
#include <cstring>
#include <numeric>
#include <queue>

#include "api.h"
#include "host_guard.h"
#include "kernels.h"
#include "shared.h"

using namespace wisp;

namespace {

constexpr uint64_t kMagic = 0x31646572616873ull;   // a planned wisp_shared_batch
constexpr int32_t kAll = 1 << 30;                   // ctx of a group's segment: its rows see every token

struct Segment {
  int32_t table, t0, t1, ctx, row0, nrow, req;      // as in the items; req: -1 for a group's
  int32_t tiles, parts, at;                         // row tiles; parts of the tokens; first partial result
};

struct Build {
  SharedPlan p{};
  std::vector<int32_t> host;
  size_t i_items = 0, i_row = 0, i_join = 0, i_mass = 0, i_mass_join = 0;
  int64_t mass_parts = 0;                           // floats
};

template <typename V>
size_t put(std::vector<int32_t> &host, const std::vector<V> &v) {
  const size_t at = host.size();
  host.resize(at + (v.size() * (sizeof(V) / 4) + 63) / 64 * 64, 0);
  if (!v.empty()) std::memcpy(&host[at], v.data(), v.size() * sizeof(V));
  return at;
}

wisp_status too_many(int64_t n) {
  return fail(WISP_E_UNSUPPORTED, "the batch needs %lld work items (at most %d)", (long long)n, kSharedMaxItems);
}

wisp_status segments_of(std::vector<Segment> &segs, std::vector<SharedJoin> &joins, std::vector<int32_t> &pre_seg,
                        const wisp_batch_desc *d, int32_t n_groups, const int32_t *size, const int32_t *prefix) {
  if (n_groups < 0) return fail(WISP_E_INVALID, "n_groups < 0");
  if (n_groups > 0 && (!size || !prefix)) return fail(WISP_E_INVALID, "group_size / prefix_len is NULL");
  int32_t row = 0, i = 0;
  auto rows_of = [&](int32_t r) { return (d->prefill_len ? d->prefill_len[r] : 0) + d->gamma[r] + 1; };
  const int32_t groups = n_groups > 0 ? n_groups : d->B;
  for (int32_t g = 0; g < groups; ++g) {
    const int32_t n = n_groups > 0 ? size[g] : 1, pre = n_groups > 0 ? prefix[g] : 0;
    if (n < 1 || n > d->B - i) return fail(WISP_E_INVALID, "group_size[%d] = %d: the sizes must be positive and add up to B", g, n);
    if (pre < 0 || pre % WISP_PAGE) return fail(WISP_E_INVALID, "prefix_len[%d] = %d: not a number of whole pages", g, pre);
    for (int32_t r = i; r < i + n; ++r)
      if (d->ctx_len[r] < pre) return fail(WISP_E_INVALID, "request %d has %d cached tokens, its group shares %d", r, d->ctx_len[r], pre);
    const bool together = n > 1 && pre > 0;
    const int32_t shared = together ? (int32_t)segs.size() : -1, first = row;
    if (together) segs.push_back(Segment{i, 0, pre, kAll, row, 0, -1, 0, 0, 0});
    for (int32_t r = i; r < i + n; ++r) {
      const int32_t nrow = rows_of(r), ctx = d->ctx_len[r];
      SharedJoin j{};
      j.row0 = row;
      j.pre_row = row - first;
      joins.push_back(j);
      pre_seg.push_back(shared);
      segs.push_back(Segment{r, together ? pre : 0, ctx + nrow, ctx, row, nrow, r, 0, 0, 0});
      row += nrow;
    }
    if (together) segs[shared].nrow = row - first;
    i += n;
  }
  if (i != d->B) return fail(WISP_E_INVALID, "the group sizes add up to %d, B is %d", i, d->B);
  return WISP_OK;
}

// Row tiles go in bundles of four, one a wave; one or two that are left share their tokens among four waves.
// What a workgroup's pass over 32 tokens (a turn) costs, by the bundle's tiles, what starting and ending an
// item does, and a row tile's partial result, written and read again; in ns.
constexpr int64_t kTurnCost[5] = {0, 700, 800, 450, 450}, kStartCost = 4000, kPartCost = 1500;

struct Tokens {                                     // of a segment, in tiles
  int64_t tiles, full, rest;                        // and its bundles: of four row tiles; the row tiles left
  int64_t turns(int row_tiles) const { return row_tiles > 2 ? tiles : (tiles * row_tiles + 3) / 4; }
  int64_t cost(int row_tiles) const { return turns(row_tiles) * kTurnCost[row_tiles]; }
};
Tokens tokens_of(const Segment &s) { return Tokens{(s.t1 - s.t0 + kTile - 1) / kTile, s.tiles / 4, s.tiles % 4}; }
// parts of a segment's tokens, for items of at most about `share`
int32_t parts_of(const Segment &s, int64_t share) {
  const Tokens t = tokens_of(s);
  const int most = t.full ? 4 : (int)t.rest;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(t.turns(most), (t.cost(most) + share - 1) / share));
}
// When the last workgroup ends, the longest items first, and what the join adds
int64_t time_of(const std::vector<Segment> &segs, int64_t share, int64_t slots) {
  std::vector<int64_t> cost;
  int64_t joined = 0;
  for (const Segment &s : segs) {
    const Tokens t = tokens_of(s);
    const int64_t n = parts_of(s, share);
    for (int64_t x = 0; x < n; ++x) {
      cost.insert(cost.end(), t.full, kStartCost + (t.cost(4) + n - 1) / n);
      if (t.rest) cost.push_back(kStartCost + (t.cost((int)t.rest) + n - 1) / n);
    }
    if (n > 1) joined += n * s.tiles;
  }
  std::sort(cost.begin(), cost.end(), std::greater<int64_t>());
  std::priority_queue<int64_t, std::vector<int64_t>, std::greater<int64_t>> ends;
  int64_t last = 0;
  for (int64_t c : cost) {
    int64_t at = 0;
    if ((int64_t)ends.size() == slots) {
      at = ends.top();
      ends.pop();
    }
    ends.push(at + c);
    last = std::max(last, at + c);
  }
  return last + joined * kPartCost / slots;
}

wisp_status plan_attention(Build &b, std::vector<Segment> &segs, std::vector<SharedJoin> &joins, const std::vector<int32_t> &pre_seg, int G) {
  SharedPlan &p = b.p;
  // every kv head has its part of the workgroups that run at once
  const int64_t slots = std::max<int64_t>(1, (int64_t)device_cus() * shared_wgs_per_cu(p.dtype, p.hd) / p.nkv);
  int64_t total = 0, bundles = 0;
  for (Segment &s : segs) {
    s.tiles = (int32_t)(((int64_t)s.nrow * G + kTile - 1) / kTile);
    const Tokens t = tokens_of(s);
    total += t.full * t.cost(4) + t.cost((int)t.rest);
    bundles += t.full + (t.rest > 0);
  }
  if (bundles > kSharedMaxItems / p.nkv) return too_many(bundles * p.nkv);
  // Items of an equal share of the work leave a last round of few, smaller ones more to start and to join: the
  // best of some sizes.  With many more bundles than workgroups the rounds are short by themselves.
  int64_t share = std::max<int64_t>(total / slots + 1, kStartCost);
  if (bundles < 8 * slots) {
    int64_t best = INT64_MAX, at = share;
    for (int64_t f = 3; f <= 16; ++f) {
      const int64_t c = std::max<int64_t>(share * f / 12, 1), t = time_of(segs, c, slots);
      if (t < best) {
        best = t;
        at = c;
      }
    }
    share = at;
  }
  std::vector<SharedItem> items;
  std::vector<int64_t> cost;
  int64_t tiles_at = 0, n_items = 0;
  for (Segment &s : segs) {
    const int64_t n = tokens_of(s).tiles;
    s.parts = parts_of(s, share);
    const bool alone = s.parts == 1 && s.req >= 0 && pre_seg[s.req] < 0;
    s.at = (int32_t)tiles_at;
    if (!alone) tiles_at += (int64_t)s.tiles * s.parts * p.nkv;
    n_items += (int64_t)((s.tiles + 3) / 4) * s.parts;
    if (n_items > kSharedMaxItems / p.nkv || tiles_at > INT32_MAX) return too_many(n_items * p.nkv);
    for (int32_t x = 0; x < s.parts; ++x) {
      const int32_t from = (int32_t)(n * x / s.parts), to = (int32_t)(n * (x + 1) / s.parts);
      for (int32_t k = 0; k < s.tiles; k += 4) {
        const int32_t m = std::min(4, s.tiles - k);
        items.push_back(SharedItem{s.table, s.t0 + from * kTile, std::min(s.t1, s.t0 + to * kTile), s.ctx, s.row0, s.nrow, k, m,
                                   alone ? -1 : (int32_t)(s.at + (int64_t)x * p.nkv * s.tiles + k), s.tiles, {0, 0}});
        cost.push_back(kTurnCost[m] * (m > 2 ? to - from : ((to - from) * m + 3) / 4));
      }
    }
    if (s.req >= 0) {
      SharedJoin &j = joins[s.req];
      j.own_at = s.at;
      j.own = s.parts;
      j.own_tiles = s.tiles;
      j.pre_row *= G;
      if (!alone) p.joined = 1;
    }
  }
  for (size_t r = 0; r < joins.size(); ++r)
    if (pre_seg[r] >= 0) {
      const Segment &s = segs[pre_seg[r]];
      joins[r].pre_at = s.at;
      joins[r].pre = s.parts;
      joins[r].pre_tiles = s.tiles;
    }
  // the longest first: the last ones to start are short
  std::vector<int32_t> order(items.size());
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return cost[x] > cost[y]; });
  std::vector<SharedItem> sorted;
  sorted.reserve(items.size());
  for (int32_t x : order) sorted.push_back(items[x]);
  p.n_items = (int32_t)sorted.size();
  p.n_parts = (int32_t)tiles_at;
  b.i_items = put(b.host, sorted);
  return WISP_OK;
}

// A token block's sums over its rows, in parts where there are few blocks for many rows
wisp_status plan_mass(Build &b, const std::vector<Segment> &segs, int G) {
  SharedPlan &p = b.p;
  constexpr int64_t kShort = 16;                    // row tiles that are not worth a part
  const int64_t slots = (int64_t)device_cus() * 2;
  int64_t total = 0, blocks = 0;
  auto first_row = [&](const Segment &s, int64_t t0) {   // of those that see token t0
    return s.req < 0 ? 0 : std::max<int64_t>(0, (t0 - s.ctx) * G) / kTile * kTile;
  };
  for (const Segment &s : segs) blocks += (s.t1 - s.t0 + kMassBlock - 1) / kMassBlock;
  if (blocks > kSharedMaxItems / p.nkv) return too_many(blocks * p.nkv);
  for (const Segment &s : segs)
    for (int64_t t = s.t0; t < s.t1; t += kMassBlock) total += ((int64_t)s.nrow * G - first_row(s, t) + kTile - 1) / kTile;
  // three items for a workgroup that runs at once: the last ones to end are short
  const int64_t share = std::max<int64_t>(total * p.nkv / (3 * slots), kShort);
  std::vector<MassItem> items;
  std::vector<MassJoin> joins;
  for (const Segment &s : segs)
    for (int64_t t = s.t0; t < s.t1; t += kMassBlock) {
      const int64_t r0 = first_row(s, t), rows = (int64_t)s.nrow * G, n = (rows - r0 + kTile - 1) / kTile;
      const int64_t parts = std::max<int64_t>(1, n / share);
      const int32_t t1 = (int32_t)std::min<int64_t>(s.t1, t + kMassBlock);
      if ((int64_t)items.size() + parts > kSharedMaxItems / p.nkv || b.mass_parts + parts * p.nkv * kMassBlock > INT32_MAX)
        return too_many(((int64_t)items.size() + parts) * p.nkv);
      for (int64_t x = 0; x < parts; ++x)
        items.push_back(MassItem{s.table, (int32_t)t, t1, s.ctx, s.row0, s.nrow, s.req, (int32_t)(r0 + n * x / parts * kTile),
                                 (int32_t)std::min(rows, r0 + n * (x + 1) / parts * kTile),
                                 parts > 1 ? (int32_t)(b.mass_parts + x * kMassBlock) : -1, (int32_t)(parts * kMassBlock), 0});
      if (parts > 1) {
        joins.push_back(MassJoin{s.table, (int32_t)t, t1, s.ctx, (int32_t)b.mass_parts, (int32_t)parts, (int32_t)(parts * kMassBlock), 0});
        b.mass_parts += parts * p.nkv * kMassBlock;
      }
    }
  std::stable_sort(items.begin(), items.end(), [](const MassItem &x, const MassItem &y) { return x.r1 - x.r0 > y.r1 - y.r0; });
  p.n_mass = (int32_t)items.size();
  p.n_mass_join = (int32_t)joins.size();
  b.i_mass = put(b.host, items);
  b.i_mass_join = put(b.host, joins);
  return WISP_OK;
}

wisp_status shared_build(Build &b, const wisp_model *m, const wisp_batch_desc *d, int32_t n_groups, const int32_t *size, const int32_t *prefix) {
  SharedPlan &p = b.p;
  wisp_status st;
  p.magic = kMagic;
  p.page_table = d->kv_page_table;
  p.pt_stride = d->pt_stride;
  p.dtype = m->dtype;
  p.nq = m->n_q_heads;
  p.nkv = m->n_kv_heads;
  p.hd = m->head_dim;
  p.B = d->B;
  const int G = p.nq / p.nkv;
  if (G > 64) return fail(WISP_E_UNSUPPORTED, "GQA group > 64");
  std::vector<Segment> segs;
  std::vector<SharedJoin> joins;
  std::vector<int32_t> pre_seg, row;
  if ((st = segments_of(segs, joins, pre_seg, d, n_groups, size, prefix)) != WISP_OK) return st;
  for (const Segment &s : segs)
    if (s.req >= 0)
      for (int32_t j = 0; j < s.nrow; ++j) {
        row.push_back(s.req);
        row.push_back(j);
      }
  p.rows = (int32_t)(row.size() / 2);
  if ((st = plan_attention(b, segs, joins, pre_seg, G)) != WISP_OK || (st = plan_mass(b, segs, G)) != WISP_OK) return st;
  b.i_row = put(b.host, row);
  b.i_join = put(b.host, joins);
  const size_t desc = 256;
  p.w_items = desc + b.i_items * 4;
  p.w_row = desc + b.i_row * 4;
  p.w_join = desc + b.i_join * 4;
  p.w_mass = desc + b.i_mass * 4;
  p.w_mass_join = desc + b.i_mass_join * 4;
  p.w_po = align256(desc + b.host.size() * 4);
  p.w_pml = p.w_po + align256((size_t)p.n_parts * kTile * p.hd * 4);
  p.w_pm = p.w_pml + align256((size_t)p.n_parts * kTile * 8);
  p.total = p.w_pm + align256((size_t)b.mass_parts * 4);
  return WISP_OK;
}

static_assert(sizeof(SharedPlan) <= sizeof(wisp_shared_batch), "wisp_shared_batch holds a plan");

wisp_status planned(SharedPlan &p, const wisp_shared_batch *batch) {
  if (!batch) return fail(WISP_E_INVALID, "batch is NULL");
  std::memcpy(&p, batch, sizeof(p));
  if (p.magic != kMagic) return fail(WISP_E_INVALID, "the batch has not been planned (wisp_shared_plan)");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(WISP_E_HIP, "hipGetDevice failed");
  if (dev != p.device) return fail(WISP_E_INVALID, "the batch was planned on device %d, the current one is %d", p.device, dev);
  return WISP_OK;
}

wisp_status cache_of(SharedCache &c, const wisp_kv *kv) {
  if (!kv || !kv->k_pool || !kv->v_pool) return fail(WISP_E_INVALID, "KV pools are NULL");
  if (kv->page_size != WISP_PAGE) return fail(WISP_E_UNSUPPORTED, "page_size must be %d", WISP_PAGE);
  if (kv->n_blocks <= 0) return fail(WISP_E_INVALID, "n_blocks must be positive");
  if (((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool) & 15) return fail(WISP_E_INVALID, "KV pools must be 16-byte aligned");
  c = SharedCache{kv->k_pool, kv->v_pool, kv->n_blocks};
  return WISP_OK;
}

}  // namespace

extern "C" {

size_t wisp_shared_workspace_size(const wisp_model *model, const wisp_batch_desc *desc, int32_t n_groups, const int32_t *group_size,
                                  const int32_t *prefix_len) {
  return guarded_size([&]() -> size_t {
    if (check_model(model, false) != WISP_OK || check_desc(desc, false, true) != WISP_OK) return 0;
    Build b;
    if (shared_build(b, model, desc, n_groups, group_size, prefix_len) != WISP_OK) return 0;
    return b.p.total;
  });
}

wisp_status wisp_shared_plan(const wisp_model *model, const wisp_batch_desc *desc, int32_t n_groups, const int32_t *group_size,
                             const int32_t *prefix_len, void *workspace, size_t workspace_bytes, wisp_shared_batch *batch, void *stream) {
  return guarded("wisp_shared_plan", [&]() -> wisp_status {
    wisp_status st;
    if (!batch) return fail(WISP_E_INVALID, "batch is NULL");
    std::memset(batch, 0, sizeof(*batch));
    if ((st = check_model(model, false)) != WISP_OK) return st;
    if ((st = check_desc(desc, true, true)) != WISP_OK) return st;
    Build b;
    if ((st = shared_build(b, model, desc, n_groups, group_size, prefix_len)) != WISP_OK) return st;
    if (desc->B > 0) {
      if (!workspace) return fail(WISP_E_INVALID, "NULL workspace");
      if ((uintptr_t)workspace & 255) return fail(WISP_E_INVALID, "workspace must be 256-byte aligned");
      if (workspace_bytes < b.p.total)
        return fail(WISP_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, (size_t)b.p.total);
      b.p.ws = static_cast<char *>(workspace);
      const hipStream_t s = (hipStream_t)stream;
      hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
      if (hipStreamIsCapturing(s, &cap) != hipSuccess) return fail(WISP_E_HIP, "stream query failed");
      st = cap == hipStreamCaptureStatusNone ? upload_ints(b.host, b.p.ws + 256, s) : upload_ints_by_arguments(b.host, b.p.ws + 256, s);
      if (st != WISP_OK) return st;
    }
    if (hipGetDevice(&b.p.device) != hipSuccess) return fail(WISP_E_HIP, "hipGetDevice failed");
    std::memcpy(batch, &b.p, sizeof(b.p));
    return WISP_OK;
  });
}

wisp_status wisp_attention_shared(const wisp_shared_batch *batch, const wisp_kv *kv, const void *q, void *out, float *lse, void *stream) {
  return guarded("wisp_attention_shared", [&]() -> wisp_status {
    wisp_status st;
    SharedPlan p;
    if ((st = planned(p, batch)) != WISP_OK) return st;
    if (p.B == 0) return WISP_OK;
    SharedCache c;
    if ((st = cache_of(c, kv)) != WISP_OK) return st;
    if (!q || !out) return fail(WISP_E_INVALID, "NULL q / out");
    if (((uintptr_t)q | (uintptr_t)out) & 15) return fail(WISP_E_INVALID, "q and out must be 16-byte aligned");
    shared_attention(p, c, q, out, lse, reinterpret_cast<int *>(p.ws), (hipStream_t)stream);
    return hip_check("attention launch");
  });
}

wisp_status wisp_attention_mass(const wisp_shared_batch *batch, const wisp_kv *kv, const void *q, const float *lse, const int32_t *count,
                                float decay, const float *prev, float *mass, void *stream) {
  return guarded("wisp_attention_mass", [&]() -> wisp_status {
    wisp_status st;
    SharedPlan p;
    if ((st = planned(p, batch)) != WISP_OK) return st;
    if (p.B == 0) return WISP_OK;
    SharedCache c;
    if ((st = cache_of(c, kv)) != WISP_OK) return st;
    if (!q || !lse || !mass) return fail(WISP_E_INVALID, "NULL q / lse / mass");
    if ((uintptr_t)q & 15) return fail(WISP_E_INVALID, "q must be 16-byte aligned");
    shared_mass(p, c, q, lse, count, decay, prev, mass, reinterpret_cast<int *>(p.ws), (hipStream_t)stream);
    return hip_check("weights launch");
  });
}

}  // extern "C"
