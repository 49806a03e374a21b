// C ABI of the operators on the 8-bit KV cache (declared in include/wisp.h): the plan of a batch
// (pages that get rows, attention items, rotation table) and the calls that run on it.
#include <algorithm>
#include <cstring>
#include <numeric>
#include <queue>

#include "api.h"
#include "host_guard.h"
#include "kernels.h"
#include "kv8_plan.h"

using namespace wisp;

namespace {

constexpr uint64_t kMagic = 0x31387670736977ull;   // a planned wisp_kv8_batch

size_t take(std::vector<int32_t> &host, size_t ints) {
  const size_t at = host.size();
  host.resize(at + (ints + 63) / 64 * 64, 0);
  return at;
}

template <typename V>
size_t put(std::vector<int32_t> &host, const std::vector<V> &v) {
  const size_t at = take(host, v.size() * (sizeof(V) / 4));
  if (!v.empty()) std::memcpy(&host[at], v.data(), v.size() * sizeof(V));
  return at;
}

struct Bundle {
  int32_t req, first, groups, tokens;   // row groups; tokens: up to its last row's causal limit
  int64_t pairs, pair, cost;            // page pairs, the cost of one, of all
};
struct Piece {                          // page pairs from .. to - 1 of a bundle, in a share; a bundle's in order
  int32_t bundle, share;
  int64_t from, to;
};

// The cost of a page pair in quarters of a wave's turn: one row group's pairs are spread over four
// waves; two groups have two waves each but share what is read, three or four one.  Starting
// an item takes as long as two turns of four waves (15 thousand cycles, a turn 7).  128 requests of
// 0.25-32k: 331 us; with pairs of 4, 4 and 7 405, of 4, 8 and 16 338, without the cost of an item 338; 32 of
// 0.5-2k 25.3, 27.4, 24.8 and 28.1; 16 of 4-32k on 64 query heads 86, 104, 88 and 89; 128 of 0.3-1.2k 38.9,
// 38.7, 39.0 and 52.4.
// kWide: of a pair that the waves convert together (two prompts of 1500-2000 rows beside 10 requests 79.7 us;
// 9: 77.8, 14: 79.7; one of 100 beside 3 11.9, 13.5 and 13.2; one of 4096 172 with all).
constexpr int64_t kPair[5] = {0, 4, 7, 14, 14}, kStart = 64, kWide = 12;
constexpr int64_t kTurn = 32;           // cost of a turn
// Where both workgroups of a CU are there, the older one's waves go first: percent of the work that
// the older half of the shares takes (128 requests of 0.25-32k: 331 us; 50 %: 356, 60 %: 355; 66 of 2k 55.7,
// 57.2 and 61.0; 64 of 1-6k on 64 query heads 112, 115 and 117; but a prompt of 4096 rows 172, 168 and 186,
// one of 3000 beside 40 requests 115, 108 and 117).
constexpr int64_t kOld = 55;
int64_t grain_of(const Bundle &u) { return u.groups == 1 ? 8 : u.groups == 2 ? 4 : 2; }   // pairs of a turn

// Shares of equal cost, the bundles one after another: one that a share's border cuts becomes several
// pieces.  Short shares are whole turns of all four waves.
std::vector<Piece> by_borders(const std::vector<Bundle> &bundles, int64_t shares, int64_t size, int64_t total) {
  const int64_t half = shares / 2, snap = size / 16;   // a cut this close to the bundle's edge is left out
  auto border = [&](int64_t s) {                       // cost before share s
    if (size < 8 * kTurn) return s * size;
    return s <= half ? total * kOld / 100 * s / std::max<int64_t>(1, half)
                     : total * kOld / 100 + total * (100 - kOld) / 100 * (s - half) / (shares - half);
  };
  std::vector<Piece> pieces;
  pieces.reserve(bundles.size() + shares);
  int64_t at = 0, share = 0;                           // cost before this bundle
  for (size_t k = 0; k < bundles.size(); ++k) {
    const Bundle &u = bundles[k];
    const int64_t grain = grain_of(u), unit = u.pair * grain;
    int64_t done = 0;
    for (; share + 1 < shares; ++share) {
      const int64_t b = border(share + 1);
      if (b >= at + u.cost - snap) break;
      const int64_t cut = (std::max<int64_t>(b - at - kStart, 0) + unit / 2) / unit * grain;   // pairs before it
      if (cut > done && cut < u.pairs && b > at + snap) {
        pieces.push_back(Piece{(int32_t)k, (int32_t)share, done, cut});
        done = cut;
      }
    }
    pieces.push_back(Piece{(int32_t)k, (int32_t)share, done, u.pairs});
    at += u.cost;
  }
  return pieces;
}

// Whole bundles, the longest first, each to the share that ends first with it.  `end`: when the last
// share ends, in the cost of a share at the mean speed.
std::vector<Piece> by_length(const std::vector<Bundle> &bundles, int64_t shares, int64_t &end) {
  std::vector<Piece> pieces;
  for (size_t k = 0; k < bundles.size(); ++k) pieces.push_back(Piece{(int32_t)k, 0, 0, bundles[k].pairs});
  std::vector<int32_t> order(bundles.size());
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return bundles[x].cost > bundles[y].cost; });
  using End = std::pair<int64_t, int32_t>;             // when a share ends, the share
  std::priority_queue<End, std::vector<End>, std::greater<End>> ends;
  for (int32_t s = 0; s < shares; ++s) ends.push({0, s});
  end = 0;
  for (int32_t k : order) {
    const int32_t s = ends.top().second;
    const int64_t e = ends.top().first + bundles[k].cost * (s < shares / 2 ? 100 - kOld : kOld);
    ends.pop();
    ends.push({e, s});
    pieces[k].share = s;
    end = std::max(end, e);
  }
  end = end * 100 / (2 * kOld * (100 - kOld));
  return pieces;
}

// A kv head's work in at most `shares` shares (how many: on return).
std::vector<Piece> shares_of(const std::vector<Bundle> &bundles, int64_t &shares) {
  int64_t total = 0;
  for (const Bundle &u : bundles) total += u.cost;
  int64_t size = (total + shares - 1) / shares;
  if (size < 8 * kTurn) size = std::max<int64_t>(1, (size + kTurn - 1) / kTurn) * kTurn;
  shares = std::max<int64_t>(1, (total + size - 1) / size);
  std::vector<Piece> pieces = by_borders(bundles, shares, size, total);
  // Cut bundles start twice, write what they have per row group and wait for its join: shares of whole
  // ones may end that much later.  128 requests of 0.3-1.2k tokens: 47.2 us cut, 38.9 whole; 66 of 2k 56
  // and 61; 256 of 1-4k 207 and 191; 64 of 1-6k on 64 query heads 112 and 245; two prompts of 1500-2000 rows
  // beside 10 requests 113 and 80, six of them 215 and 202, one of 4096 181 and 172.  The rule takes the
  // better side of each.  Short shares are cut: whole bundles would leave CUs idle.
  if (size >= 8 * kTurn) {
    int64_t end = 0, groups = 0;
    for (const Bundle &u : bundles) groups += u.groups;
    std::vector<Piece> whole = by_length(bundles, shares, end);
    if (end <= size + 180 + 40 * groups / (int64_t)bundles.size()) pieces.swap(whole);
  }
  return pieces;
}

}  // namespace

wisp_status wisp::kv8_build(Kv8Build &b, const wisp_model *m, const wisp_batch_desc *d) {
  Kv8Plan &p = b.p;
  p.magic = kMagic;
  p.page_table = d->kv_page_table;
  p.pt_stride = d->pt_stride;
  p.dtype = m->dtype;
  p.nq = m->n_q_heads;
  p.nkv = m->n_kv_heads;
  p.hd = m->head_dim;
  p.B = d->B;
  const int G = p.nq / p.nkv;
  std::vector<Kv8Unit> units;
  std::vector<int32_t> pos, nrow(p.B), row0(p.B);
  int most = 0;
  for (int i = 0; i < p.B; ++i) {
    row0[i] = (int32_t)pos.size();
    nrow[i] = (d->prefill_len ? d->prefill_len[i] : 0) + d->gamma[i] + 1;
    most = std::max(most, nrow[i]);
    const int c = d->ctx_len[i], end = c + nrow[i];
    for (int t = c; t < end; ++t) pos.push_back(t);
    for (int pg = c / kPage; pg * kPage < end; ++pg) {
      const int first = std::max(c, pg * kPage), last = std::min(end, (pg + 1) * kPage);
      units.push_back(Kv8Unit{i, pg, row0[i] + first - c, (first - pg * kPage) | (last - first) << 8});
    }
  }
  p.rows = (int32_t)pos.size();
  p.n_units = (int32_t)units.size();

  // Row groups of 32 rows, of 16 where no request has more (and for fp32, whose three parts fill
  // the registers); up to four of a request make a bundle that runs together.
  p.rb = p.dtype == WISP_BF16 && (int64_t)most * G > 16 ? 2 : 1;
  const int R = 16 * p.rb;
  std::vector<Bundle> bundles;
  int64_t bytes = 0;
  int64_t n_bundles = 0;
  for (int i = 0; i < p.B; ++i) {
    bytes += 2 * ((int64_t)d->ctx_len[i] + nrow[i]) * p.nkv * p.hd;
    n_bundles += (((int64_t)nrow[i] * G + R - 1) / R + 3) / 4;
  }
  // Items carry a row group's index in 24 bits, and the kernels count a request's rows x G in 32: both
  // hold for every batch of at most kKv8MaxItems bundles x kv heads.
  auto too_many = [&](int64_t n) {
    return fail(WISP_E_UNSUPPORTED, "the batch needs %lld attention work items (at most %d)", (long long)n, kKv8MaxItems);
  };
  if (n_bundles > kKv8MaxItems / p.nkv) return too_many(n_bundles * p.nkv);
  // the append's threads, in one launch and counted in 32 bits
  if (2 * p.hd * ((int64_t)p.n_units * p.nkv + 1) + (int64_t)p.rows * (p.hd / 16) * ((p.nq + 1) / 2) > UINT32_MAX)
    return fail(WISP_E_UNSUPPORTED, "rows x heads beyond one append's 2^32 threads");
  p.stream = bytes > (256 << 20);                      // more than the last-level cache holds
  for (int i = 0; i < p.B; ++i) {
    const int64_t groups = ((int64_t)nrow[i] * G + R - 1) / R, nb = (groups + 3) / 4;
    for (int64_t k = 0; k < nb; ++k) {
      const int64_t f = k * groups / nb, e = (k + 1) * groups / nb;
      const int32_t T = d->ctx_len[i] + (int32_t)((std::min<int64_t>((int64_t)nrow[i] * G, e * R) - 1) / G) + 1;
      const int64_t pairs = (T + 31) / 32;
      const int64_t pair = kPair[e - f];
      bundles.push_back(Bundle{i, (int32_t)f, (int32_t)(e - f), T, pairs, pair, kStart + pairs * pair});
    }
  }
  // Every kv head's work, the same for all, in shares, one for each workgroup (two per CU).  Bundles of
  // three and four row groups run apart (the attention's wide items) where they are half of the work
  // or more, each set with its part of the workgroups: a prompt of 4096 rows 185 us together, 172
  // apart, one of 500 beside 3 decoding requests 23.7 and 21.6, one of 3000 beside 40 116 and 115, six of
  // 1500-2000 224 and 202; of less than half, 128 requests of 0.25-32k and up to 17 rows, 331 and 357.
  const int64_t wgs = (int64_t)device_cus() * 2, most_shares = std::max<int64_t>(1, wgs / p.nkv);
  if (n_bundles + most_shares > kKv8MaxItems / p.nkv) return too_many((n_bundles + most_shares) * p.nkv);
  int64_t cost[2] = {0, 0};
  for (const Bundle &u : bundles) cost[u.groups > 2] += u.cost;
  const bool apart = p.rb == 2 && cost[1] >= cost[0];
  std::vector<Bundle> sets[2];
  cost[0] = cost[1] = 0;
  for (Bundle u : bundles) {
    const int w = apart && u.groups > 2;
    if (w) u.pair = kWide;
    u.cost = kStart + u.pairs * u.pair;
    cost[w] += u.cost;
    sets[w].push_back(u);
  }
  std::vector<Kv8Item> items;
  std::vector<Kv8Group> groups;
  std::vector<int32_t> first;
  p.n_parts = 0;
  for (int w = 0; w < 2; ++w) {
    if (sets[w].empty()) continue;
    int64_t shares = most_shares;
    if (cost[1 - w] > 0)
      shares = std::max<int64_t>(1, std::min(most_shares - 1, (2 * most_shares * cost[w] + cost[0] + cost[1]) / (2 * (cost[0] + cost[1]))));
    const std::vector<Piece> pieces = shares_of(sets[w], shares);
    (w ? p.n_wide : p.n_shares) = (int32_t)shares;
    std::vector<int32_t> next(shares + 1, 0);            // where a share's items start, then its next item
    for (const Piece &x : pieces) ++next[x.share + 1];
    next[0] = (int32_t)items.size();
    std::partial_sum(next.begin(), next.end(), next.begin());
    first.insert(first.end(), next.begin(), next.end());
    items.resize(items.size() + pieces.size());
    for (size_t k = 0; k < pieces.size();) {
      const Bundle &u = sets[w][pieces[k].bundle];
      int32_t n = 0;                                     // its pieces
      while (k + n < pieces.size() && pieces[k + n].bundle == pieces[k].bundle) ++n;
      for (int32_t x = 0; x < n; ++x) {
        const Piece &y = pieces[k + x];
        items[next[y.share]++] = Kv8Item{u.req, (int32_t)(32 * y.from), (int32_t)std::min<int64_t>(u.tokens, 32 * y.to),
                                         d->ctx_len[u.req], row0[u.req], nrow[u.req], kv8_pack(u.first, u.groups),
                                         n > 1 ? p.n_parts + x * u.groups : -1};
      }
      if (n > 1) {
        for (int32_t g = 0; g < u.groups; ++g)
          groups.push_back(Kv8Group{row0[u.req], nrow[u.req], u.first + g, p.n_parts + g, n, u.groups, {0, 0}});
        p.n_parts += n * u.groups;
      }
      k += n;
    }
  }
  p.n_items = (int32_t)items.size();
  p.n_groups = (int32_t)groups.size();
  b.i_first = put(b.host, first);

  b.i_units = put(b.host, units);
  b.i_items = put(b.host, items);
  b.i_groups = put(b.host, groups);
  b.i_pos = put(b.host, pos);
  const size_t slots_of_parts = (size_t)p.n_parts * p.nkv * R;
  b.po_bytes = align256(slots_of_parts * p.hd * 4);
  b.pml_bytes = align256(slots_of_parts * 2 * 4);
  b.cs_bytes = align256((size_t)p.rows * p.hd * 4);
  return WISP_OK;
}

void wisp::kv8_place(Kv8Build &b, char *ws, size_t desc, size_t scratch) {
  Kv8Plan &p = b.p;
  p.ws = ws;
  p.w_units = desc + b.i_units * 4;
  p.w_items = desc + b.i_items * 4;
  p.w_first = desc + b.i_first * 4;
  p.w_groups = desc + b.i_groups * 4;
  p.w_pos = desc + b.i_pos * 4;
  p.w_po = scratch;
  p.w_pml = p.w_po + b.po_bytes;
  p.w_cs = p.w_pml + b.pml_bytes;
  p.total = p.w_cs + b.cs_bytes;
}

wisp_status wisp::kv8_cache(Kv8Cache &c, const wisp_kv8 *kv) {
  if (!kv || !kv->k_pool || !kv->v_pool || !kv->scale) return fail(WISP_E_INVALID, "8-bit KV pools or scales are NULL");
  if (kv->page_size != WISP_PAGE) return fail(WISP_E_UNSUPPORTED, "page_size must be %d", WISP_PAGE);
  if (kv->n_blocks <= 0) return fail(WISP_E_INVALID, "n_blocks must be positive");
  if ((((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool) & 15) || ((uintptr_t)kv->scale & 7))
    return fail(WISP_E_INVALID, "8-bit KV pools must be 16-byte aligned, their scales 8-byte");
  c = Kv8Cache{static_cast<uint8_t *>(kv->k_pool), static_cast<uint8_t *>(kv->v_pool), kv->scale, kv->n_blocks};
  return WISP_OK;
}

namespace {

static_assert(sizeof(Kv8Plan) <= sizeof(wisp_kv8_batch), "wisp_kv8_batch holds a plan");

wisp_status planned(Kv8Plan &p, const wisp_kv8_batch *batch) {
  if (!batch) return fail(WISP_E_INVALID, "batch is NULL");
  std::memcpy(&p, batch, sizeof(p));
  if (p.magic != kMagic) return fail(WISP_E_INVALID, "the batch has not been planned (wisp_kv8_plan)");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(WISP_E_HIP, "hipGetDevice failed");
  if (dev != p.device) return fail(WISP_E_INVALID, "the batch was planned on device %d, the current one is %d", p.device, dev);
  return WISP_OK;
}

size_t own_size(Kv8Build &b) {
  kv8_place(b, nullptr, 256, align256(256 + b.host.size() * 4));
  return b.p.total;
}

}  // namespace

extern "C" {

size_t wisp_kv8_workspace_size(const wisp_model *model, const wisp_batch_desc *desc) {
  return guarded_size([&]() -> size_t {
    if (check_model(model, false) != WISP_OK || check_desc(desc, false, true) != WISP_OK) return 0;
    Kv8Build b;
    if (kv8_build(b, model, desc) != WISP_OK) return 0;
    return own_size(b);
  });
}

wisp_status wisp_kv8_plan(const wisp_model *model, const wisp_batch_desc *desc, void *workspace, size_t workspace_bytes,
                          wisp_kv8_batch *batch, void *stream) {
  return guarded("wisp_kv8_plan", [&]() -> wisp_status {
    wisp_status st;
    if (!batch) return fail(WISP_E_INVALID, "batch is NULL");
    std::memset(batch, 0, sizeof(*batch));
    if ((st = check_model(model, false)) != WISP_OK) return st;
    if ((st = check_desc(desc, true, true)) != WISP_OK) return st;
    Kv8Build b;
    if ((st = kv8_build(b, model, desc)) != WISP_OK) return st;
    if (hipGetDevice(&b.p.device) != hipSuccess) return fail(WISP_E_HIP, "hipGetDevice failed");
    const size_t need = own_size(b);
    if (desc->B > 0) {
      if (!workspace) return fail(WISP_E_INVALID, "NULL workspace");
      if ((uintptr_t)workspace & 255) return fail(WISP_E_INVALID, "workspace must be 256-byte aligned");
      if (workspace_bytes < need)
        return fail(WISP_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, need);
      char *ws = static_cast<char *>(workspace);
      kv8_place(b, ws, 256, align256(256 + b.host.size() * 4));
      const hipStream_t s = (hipStream_t)stream;
      hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
      if (hipStreamIsCapturing(s, &cap) != hipSuccess) return fail(WISP_E_HIP, "stream query failed");
      st = cap == hipStreamCaptureStatusNone ? upload_ints(b.host, ws + 256, s) : upload_ints_by_arguments(b.host, ws + 256, s);
      if (st != WISP_OK) return st;
      StepDesc sd{};
      sd.row_pos = reinterpret_cast<const int32_t *>(ws + b.p.w_pos);
      rope_table(sd, reinterpret_cast<float *>(ws + b.p.w_cs), b.p.rows, b.p.hd, model->rope_base, s);
      if ((st = hip_check("plan launch")) != WISP_OK) return st;
    }
    std::memcpy(batch, &b.p, sizeof(b.p));
    return WISP_OK;
  });
}

wisp_status wisp_kv8_append(const wisp_kv8_batch *batch, const wisp_kv8 *kv, const void *qkv, int64_t qkv_ld, void *q,
                            void *stream) {
  return guarded("wisp_kv8_append", [&]() -> wisp_status {
    wisp_status st;
    Kv8Plan p;
    if ((st = planned(p, batch)) != WISP_OK) return st;
    if (p.B == 0) return WISP_OK;
    Kv8Cache c;
    if ((st = kv8_cache(c, kv)) != WISP_OK) return st;
    if (!qkv || !q) return fail(WISP_E_INVALID, "NULL qkv / q");
    const int64_t es = p.dtype == WISP_BF16 ? 2 : 4;
    if (qkv_ld < (int64_t)(p.nq + 2 * p.nkv) * p.hd) return fail(WISP_E_INVALID, "qkv_ld shorter than a row");
    if ((((uintptr_t)qkv | (uintptr_t)q) & 15) || qkv_ld * es % 16)
      return fail(WISP_E_INVALID, "qkv, its rows and q must be 16-byte aligned");
    kv8_append(p, c, QkvRows{qkv, qkv_ld, 0, 0}, q, reinterpret_cast<int *>(p.ws), (hipStream_t)stream);
    return hip_check("append launch");
  });
}

wisp_status wisp_attention_kv8(const wisp_kv8_batch *batch, const wisp_kv8 *kv, const void *q, void *out, void *stream) {
  return guarded("wisp_attention_kv8", [&]() -> wisp_status {
    wisp_status st;
    Kv8Plan p;
    if ((st = planned(p, batch)) != WISP_OK) return st;
    if (p.B == 0) return WISP_OK;
    Kv8Cache c;
    if ((st = kv8_cache(c, kv)) != WISP_OK) return st;
    if (!q || !out) return fail(WISP_E_INVALID, "NULL q / out");
    if (((uintptr_t)q | (uintptr_t)out) & 15) return fail(WISP_E_INVALID, "q and out must be 16-byte aligned");
    kv8_attention(p, c, q, out, false, reinterpret_cast<int *>(p.ws), (hipStream_t)stream);
    return hip_check("attention launch");
  });
}

}  // extern "C"
