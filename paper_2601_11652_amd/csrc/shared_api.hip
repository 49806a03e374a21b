// C ABI of the operators on batches whose requests share prefixes (declared in include/wisp.h): the plan of a
// batch and the calls that run on it.
#include <algorithm>
#include <climits>
#include <cstring>
#include <map>
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
  int32_t tiles, bundle0;                           // row tiles; the first of its bundles
};

struct RowAt {                                      // a row's segment and its row there, and its group's (-1: none)
  int32_t own, own_row, pre, pre_row;
};

struct Build {
  SharedPlan p{};
  std::vector<int32_t> host;
  size_t i_items = 0, i_bundles = 0, i_row = 0, i_join = 0, i_mass = 0, i_mass_join = 0;
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

wisp_status segments_of(std::vector<Segment> &segs, std::vector<RowAt> &joins, std::vector<int32_t> &pre_seg,
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
    if (together) segs.push_back(Segment{i, 0, pre, kAll, row, 0, -1, 0, 0});
    for (int32_t r = i; r < i + n; ++r) {
      const int32_t nrow = rows_of(r), ctx = d->ctx_len[r];
      for (int32_t x = 0; x < nrow; ++x) joins.push_back(RowAt{(int32_t)segs.size(), x, shared, row - first + x});   // of segments, yet
      pre_seg.push_back(shared);
      segs.push_back(Segment{r, together ? pre : 0, ctx + nrow, ctx, row, nrow, r, 0, 0});
      row += nrow;
    }
    if (together) segs[shared].nrow = row - first;
    i += n;
  }
  if (i != d->B) return fail(WISP_E_INVALID, "the group sizes add up to %d, B is %d", i, d->B);
  return WISP_OK;
}

// Row tiles of a segment go in bundles of four, one a wave; of a bundle of one or two the four waves share the tokens.
// In ns, as measured with two workgroups a CU: what starting and ending an item costs, a row tile's partial result, written
// and read again, the least that a piece is cut to, and a pass over 32 tokens (a turn) by the bundle's row tiles.  (With
// starts of 2500 or 7000, or turns a fifth shorter or longer, seven batches of twelve change by less than 2%, the others by
// up to 25% either way.)
constexpr int64_t kStartCost = 3500, kPartCost = 1500, kLeast = 2500;
int64_t turn_cost(int dtype, int hd, int tiles) {
  if (dtype != WISP_BF16) return (int64_t)hd * 27 * shared_wgs_per_cu(dtype, hd);   // its products
  return (tiles > 2 ? 900 : 1200) * (hd + 64) / 192;
}

struct Bundle {
  int32_t seg, tile0, tiles, tokens;                // first row tile, row tiles; token tiles up to its last row's limit
  int64_t turns, turn;                              // and the cost of one
  bool joined;                                      // its rows have other results to be joined with
};
struct Piece {                                      // turns from .. to - 1 of a bundle, a bundle's in order
  int32_t bundle;
  int64_t from, to;
};
int64_t cost_of(const std::vector<Bundle> &bundles, const Piece &x) { return kStartCost + (x.to - x.from) * bundles[x.bundle].turn; }

// Bundles longer than `share` (a start and the least of any, or more) are laid one behind another over shares of that
// length and cut at their borders; the others stay whole.
std::vector<Piece> pieces_of(const std::vector<Bundle> &bundles, int64_t share) {
  std::vector<Piece> pieces;
  int64_t room = share;
  for (size_t k = 0; k < bundles.size(); ++k) {
    const Bundle &u = bundles[k];
    const int64_t least = std::max<int64_t>(1, (kLeast + u.turn / 2) / u.turn);
    int64_t at = 0;
    while (kStartCost + (u.turns - at) * u.turn > (at ? room : share)) {
      int64_t n = (room - kStartCost) / u.turn;
      if (n >= u.turns - at) break;
      if (n >= least) {
        n = std::min(n, std::max<int64_t>(u.turns - at - least, 1));
        pieces.push_back(Piece{(int32_t)k, at, at + n});
        at += n;
      }
      room = share;
    }
    pieces.push_back(Piece{(int32_t)k, at, u.turns});
    if (at) room -= cost_of(bundles, pieces.back());
  }
  return pieces;
}
// When the last workgroup ends, the longest pieces first, and what the join adds
int64_t time_of(const std::vector<Bundle> &bundles, const std::vector<Piece> &pieces, int64_t slots) {
  std::vector<int64_t> cost;
  int64_t joined = 0;
  for (const Piece &x : pieces) {
    const Bundle &u = bundles[x.bundle];
    cost.push_back(cost_of(bundles, x));
    if (u.joined || x.to - x.from < u.turns) joined += u.tiles;
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

wisp_status plan_attention(Build &b, std::vector<Segment> &segs, std::vector<RowAt> &joins, const std::vector<int32_t> &pre_seg, int G) {
  SharedPlan &p = b.p;
  int64_t count = 0;
  for (Segment &s : segs) {
    s.tiles = (int32_t)(((int64_t)s.nrow * G + kTile - 1) / kTile);
    count += (s.tiles + kBundle - 1) / kBundle;
  }
  if (count > kSharedMaxItems / p.nkv) return too_many(count * p.nkv);
  std::vector<Bundle> bundles;
  int64_t total = 0, longest = 0;
  for (size_t k = 0; k < segs.size(); ++k) {
    Segment &s = segs[k];
    s.bundle0 = (int32_t)bundles.size();
    for (int32_t t = 0; t < s.tiles; t += kBundle) {
      Bundle u{};
      u.seg = (int32_t)k;
      u.tile0 = t;
      u.tiles = std::min(kBundle, s.tiles - t);
      const int64_t last = std::min<int64_t>((int64_t)s.nrow * G, (int64_t)(t + u.tiles) * kTile) - 1;
      u.tokens = (int32_t)((std::min<int64_t>(s.t1, s.ctx + last / G + 1) - s.t0 + kTile - 1) / kTile);
      u.turns = u.tiles > 2 ? u.tokens : (u.tokens * (int64_t)u.tiles + 3) / 4;
      u.turn = turn_cost(p.dtype, p.hd, u.tiles);
      longest = std::max(longest, u.turn);
      u.joined = s.req < 0 || pre_seg[s.req] >= 0;
      total += kStartCost + u.turns * u.turn;
      bundles.push_back(u);
    }
  }
  // Every kv head has its part of the workgroups that run at once.  Equal shares of the work, or longer ones, of which
  // fewer bundles are cut, or shorter ones, of which the last round is shorter: the best by the costs above.  With many
  // more bundles than workgroups none is cut.
  const int64_t slots = std::max<int64_t>(1, (int64_t)device_cus() * shared_wgs_per_cu(p.dtype, p.hd) / p.nkv);
  std::vector<Piece> pieces;
  if ((int64_t)bundles.size() < 8 * slots) {
    int64_t best = INT64_MAX;
    for (int64_t f : {40, 50, 60, 70, 80, 90, 100, 110, 125, 150, 200, 300}) {
      const int64_t share = std::max(total / slots * f / 100, kStartCost + kLeast + longest);
      std::vector<Piece> x = pieces_of(bundles, share);
      const int64_t t = time_of(bundles, x, slots);
      if (t < best) {
        best = t;
        pieces.swap(x);
      }
    }
  } else {
    pieces = pieces_of(bundles, INT64_MAX);
  }
  if ((int64_t)pieces.size() > kSharedMaxItems / p.nkv) return too_many((int64_t)pieces.size() * p.nkv);
  std::vector<SharedItem> items;
  std::vector<SharedBundle> table;
  std::vector<SharedRow> rows;
  int64_t at = 0;
  for (size_t k = 0; k < pieces.size();) {
    const Bundle &u = bundles[pieces[k].bundle];
    const Segment &s = segs[u.seg];
    int32_t n = 0;
    while (k + n < pieces.size() && pieces[k + n].bundle == pieces[k].bundle) ++n;
    const bool alone = n == 1 && !u.joined;
    if (at + (int64_t)n * p.nkv * u.tiles > INT32_MAX) return too_many(at);
    for (int32_t x = 0; x < n; ++x) {
      const Piece &y = pieces[k + x];
      auto token = [&](int64_t turn) {              // of a turn's first tile; the waves that share tokens take 4 / tiles of them
        const int64_t tile = u.tiles > 2 ? turn : turn * 4 / u.tiles;
        return (int32_t)std::min<int64_t>((int64_t)u.tokens * kTile, tile * kTile);
      };
      items.push_back(SharedItem{s.table, s.t0 + token(y.from), std::min(s.t1, s.t0 + token(y.to)), s.ctx, s.row0, s.nrow, u.tile0, u.tiles,
                                 alone ? -1 : (int32_t)(at + (int64_t)x * p.nkv * u.tiles), u.tiles, {0, 0}});
    }
    table.push_back(SharedBundle{(int32_t)at, n, u.tiles, 0});
    if (!alone) {
      at += (int64_t)n * p.nkv * u.tiles;
      p.joined = 1;
    }
    k += n;
  }
  if (p.joined)
    for (RowAt &j : joins) {
      auto place = [&](int32_t seg, int32_t row, int32_t &next) {
        if (seg < 0) return SharedBundle{0, 0, 0, 0};
        const int32_t f = row * G, k = segs[seg].bundle0 + f / (kBundle * kTile);
        next = std::min(k + 1, (int32_t)table.size() - 1);
        SharedBundle x = table[k];
        x.row = f % (kBundle * kTile);
        return x;
      };
      SharedRow r{};
      r.own = place(j.own, j.own_row, r.own_next);
      r.pre = place(j.pre, j.pre_row, r.pre_next);
      rows.push_back(r);
    }
  // the longest first: the last ones to start are short
  std::vector<int32_t> order(items.size());
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return cost_of(bundles, pieces[x]) > cost_of(bundles, pieces[y]); });
  std::vector<SharedItem> sorted;
  sorted.reserve(items.size());
  for (int32_t x : order) sorted.push_back(items[x]);
  p.n_items = (int32_t)sorted.size();
  p.n_parts = (int32_t)at;
  b.i_items = put(b.host, sorted);
  b.i_bundles = put(b.host, table);
  b.i_join = put(b.host, rows);
  return WISP_OK;
}

// A token block's sums over its rows, in parts where that ends sooner (sixteen row tiles in one item: 24 us; in parts of 4,
// 13).  In ns: an item's start and end, one of its row tiles, the parts and their sum.
constexpr int64_t kMassStart = 4000, kMassTile = 900, kMassJoin = 8000, kMassSpan = 4;

wisp_status plan_mass(Build &b, const std::vector<Segment> &segs, int G) {
  SharedPlan &p = b.p;
  const int64_t slots = (int64_t)device_cus() * mass_wgs_per_cu(p.dtype, p.hd);
  int64_t blocks = 0;
  auto first_row = [&](const Segment &s, int64_t t0) {   // of those that see token t0
    return s.req < 0 ? 0 : std::max<int64_t>(0, (t0 - s.ctx) * G) / kTile * kTile;
  };
  for (const Segment &s : segs) blocks += (s.t1 - s.t0 + kMassBlock - 1) / kMassBlock;
  if (blocks > kSharedMaxItems / p.nkv) return too_many(blocks * p.nkv);
  std::map<int64_t, int64_t> sizes;                      // row tiles of a block; blocks
  for (const Segment &s : segs)
    for (int64_t t = s.t0; t < s.t1; t += kMassBlock) ++sizes[((int64_t)s.nrow * G - first_row(s, t) + kTile - 1) / kTile];
  int64_t share = kMassTiles, best = INT64_MAX;
  for (int64_t c : {4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 256, kMassTiles}) {
    int64_t sum = 0, longest = 0;
    bool cut = false;
    for (auto [n, count] : sizes) {
      const int64_t parts = std::max<int64_t>(1, n / c);
      sum += count * (parts * kMassStart + n * kMassTile);
      longest = std::max(longest, kMassStart + (n + parts - 1) / parts * kMassTile);
      cut |= parts > 1;
    }
    const int64_t t = std::max(longest, sum * p.nkv / slots) + (cut ? kMassJoin : 0);
    if (t < best) {
      best = t;
      share = c;
    }
  }
  // Blocks of one stage of rows go several to an item, where there are more than run at once: half of an item's time is what
  // comes before and after its rows (32 sessions on a document: 21.4 us, one by one 22.4)
  const int64_t stage = mass_stage_tiles(p.dtype, p.hd);
  int64_t short_blocks = 0;
  for (auto [n, count] : sizes) short_blocks += n <= stage ? count : 0;
  const int64_t span = std::min<int64_t>(std::max<int64_t>(short_blocks * p.nkv / slots, 1), kMassSpan);
  std::vector<MassItem> items;
  std::vector<MassJoin> joins;
  for (const Segment &s : segs)
    for (int64_t t = s.t0, next; t < s.t1; t = next) {
      const int64_t r0 = first_row(s, t), rows = (int64_t)s.nrow * G, n = (rows - r0 + kTile - 1) / kTile;
      const int64_t parts = std::max<int64_t>({1, n / share, (n + kMassTiles - 1) / kMassTiles});
      next = t + (n <= stage ? span : 1) * kMassBlock;
      const int32_t t1 = (int32_t)std::min<int64_t>(s.t1, next);
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
  auto size_of = [](const MassItem &x) { return (int64_t)(x.r1 - x.r0) * (x.t1 - x.t0); };
  std::stable_sort(items.begin(), items.end(), [&](const MassItem &x, const MassItem &y) { return size_of(x) > size_of(y); });
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
  if (p.nkv > 65535 || (int64_t)p.nq * p.hd > 1 << 22)   // a grid's second index; 64 rows' places in 32 bits
    return fail(WISP_E_UNSUPPORTED, "more than 65535 kv heads, or n_q_heads x head_dim above 2^22");
  std::vector<Segment> segs;
  std::vector<RowAt> joins;
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
  const size_t desc = 256;
  p.w_items = desc + b.i_items * 4;
  p.w_bundles = desc + b.i_bundles * 4;
  p.w_row = desc + b.i_row * 4;
  p.w_join = desc + b.i_join * 4;
  p.w_mass = desc + b.i_mass * 4;
  p.w_mass_join = desc + b.i_mass_join * 4;
  p.w_po = align256(desc + b.host.size() * 4);
  p.w_pml = p.w_po + align256((size_t)p.n_parts * kTile * p.hd * 4);
  p.w_pm = p.w_pml + align256((size_t)p.n_parts * kTile * 16);
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
