// Eviction from the paged KV cache: of each request and kv head the tokens of greatest weight stay, with the
// first and the last ones, and move together; a kept key is rotated from its old position to its new one.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "api.h"
#include "host_guard.h"
#include "kernels.h"

namespace wisp {

namespace {

struct EvictReq {                      // a request, the longest first
  int32_t req, ctx, keep, sink;
  int32_t recent, start, pad[2];       // start: of its tokens in a head's list
};

// Requests travel as arguments where they fit: a launch's 4 KB hold 256 bytes of the runtime's, the angles and what else stands
// below.  (40 requests of 500 tokens: 38.9 us, with an upload first 44.4; few requests are not slower for the larger block.)
constexpr int kArgumentBytes = 4096 - 256, kAngles = 128, kFew = (kArgumentBytes - kAngles * 8 - 96) / 32;
struct EvictArgs {
  const EvictReq *reqs;                // NULL: few
  const int32_t *table, *to;
  void *k, *v;
  float *mass;
  int32_t *kept;
  int *err;
  int64_t total;                       // kept tokens of all requests
  int stride, to_stride, n_blocks, nkv, runs;
  EvictReq few[kFew];
};

// the request of a workgroup, in scalar registers
__device__ __forceinline__ EvictReq request_of(const EvictArgs &a, int i) {
  EvictReq r = a.reqs ? a.reqs[i] : a.few[i];
  int32_t v[sizeof(r) / 4];
  __builtin_memcpy(v, &r, sizeof(r));
#pragma unroll
  for (int x = 0; x < (int)(sizeof(r) / 4); ++x) v[x] = __builtin_amdgcn_readfirstlane(v[x]);
  __builtin_memcpy(&r, v, sizeof(r));
  return r;
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kSelectHeld = 16, kSelectBins = 2048;

// floats in the order of their values as unsigned integers, -0 as 0, NaN below everything
__device__ __forceinline__ uint32_t key_of(float f) {
  if (f != f) return 0u;
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which tokens stay: a workgroup for each layer, kv head and request, a wave for a run of tokens.  A radix
// selection finds the least key that stays and how many of that key do (the first ones): 11 bits (a float's
// exponent and two more), 11 and 10; then the tokens are listed in order.  HELD: the keys stay in registers, where the sixteen of
// a thread are enough; else they are read again in each of five passes, without loads ahead (one request of 16384 tokens to choose
// from, back to half: 68 us for the whole call, of 16385 90, of 32768 160; 32 such requests: 722, 752 and 1488).
// Bound by latency: two loads that depend on each other, and 14 barriers.
template <bool HELD>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kSelectBins];
  __shared__ int more[kSelectWaves], same[kSelectWaves];
  __shared__ uint32_t sh_key;
  __shared__ int sh_left;
  const EvictReq r = request_of(a, blockIdx.x);
  const int kvh = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t *pt = a.table + (int64_t)r.req * a.stride;
  const float *mass = a.mass + (int64_t)layer * a.n_blocks * a.nkv * kPage;
  int32_t *kept = a.kept + ((int64_t)layer * a.nkv + kvh) * a.total + r.start;
  if (r.keep == r.ctx) {
    for (int t = tid; t < r.keep; t += kSelectThreads) kept[t] = t;
    return;
  }
  const int n = r.ctx - r.sink - r.recent;             // tokens to choose from
  const int steps = (n + kSelectThreads - 1) / kSelectThreads, x0 = wave * steps * 64 + lane;   // a wave's run, 64 a step
  auto token = [&](int i) __attribute__((always_inline)) { return r.sink + min(x0 + 64 * i, n - 1); };
  bool bad = false;
  auto key = [&](int i, int b) __attribute__((always_inline)) {
    bad |= b < 0 || b >= a.n_blocks;
    return key_of(mass[((int64_t)min(max(b, 0), a.n_blocks - 1) * a.nkv + kvh) * kPage + (token(i) & 15)]);
  };
  uint32_t held[HELD ? kSelectHeld : 1];
  if constexpr (HELD) {
    int b[kSelectHeld];
#pragma unroll
    for (int i = 0; i < kSelectHeld; ++i) b[i] = i < steps ? pt[token(i) >> 4] : 0;
#pragma unroll
    for (int i = 0; i < kSelectHeld; ++i) held[i] = i < steps ? key(i, b[i]) : 0;
  }
  // f(key, whether there is one) for each of this lane's tokens, in order
  auto each = [&](auto &&f) __attribute__((always_inline)) {
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i)
        if (i < steps) f(held[i], x0 + 64 * i < n, i);
    } else {
      for (int i = 0; i < steps; ++i) f(key(i, pt[token(i) >> 4]), x0 + 64 * i < n, i);
    }
  };
  uint32_t found = 0;
  int left = r.keep - r.sink - r.recent;               // tokens with the key's bits so far that stay
  auto digit = [&](int shift, int bits, uint32_t above) __attribute__((always_inline)) {
    if (left == 0) return;
    for (int x = tid; x < kSelectBins; x += kSelectThreads) hist[x] = 0;
    __syncthreads();
    each([&](uint32_t k, bool on, int) __attribute__((always_inline)) {
      if (on && (k & above) == found) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // the digit at which the count from the top reaches `left`: two digits a thread
    const int top = kSelectBins - 1 - 2 * tid;
    const int c0 = hist[top], c1 = hist[top - 1];
    int before = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o);
      before += lane >= o ? v : 0;
    }
    if (lane == 63) more[wave] = before;
    __syncthreads();
    before -= c0 + c1;
    for (int w = 0; w < wave; ++w) before += more[w];
    if (before < left && before + c0 + c1 >= left) {
      const bool second = before + c0 < left;
      sh_key = found | (uint32_t)(top - second) << shift;
      sh_left = left - before - (second ? c0 : 0);
    }
    __syncthreads();
    found = sh_key;
    left = sh_left;
  };
  digit(21, 11, 0u);
  digit(10, 11, ~0u << 21);
  digit(0, 10, ~0u << 10);
  if (left == 0) found = UINT_MAX;                      // none of the middle stays (no key is above)
  // first the runs' numbers of tokens, then their places
  int m = 0, s = 0;
  each([&](uint32_t k, bool on, int) __attribute__((always_inline)) {
    m += __popcll(__builtin_amdgcn_ballot_w64(on && k > found));
    s += __popcll(__builtin_amdgcn_ballot_w64(on && k == found));
  });
  __syncthreads();
  if (lane == 0) {
    more[wave] = m;
    same[wave] = s;
  }
  __syncthreads();
  m = 0;                                                // tokens listed before this one's, with the key and above it
  s = 0;
  for (int w = 0; w < wave; ++w) {
    m += more[w];
    s += same[w];
  }
  const unsigned long long below = (1ull << lane) - 1;
  each([&](uint32_t k, bool on, int i) __attribute__((always_inline)) {
    const unsigned long long gt = __builtin_amdgcn_ballot_w64(on && k > found), eq = __builtin_amdgcn_ballot_w64(on && k == found);
    const int e = s + __popcll(eq & below), place = r.sink + m + __popcll(gt & below) + min(e, left);
    if (on && (k > found || (k == found && e < left))) kept[place] = r.sink + x0 + 64 * i;
    m += __popcll(gt);
    s += __popcll(eq);
  });
  if (bad) flag_error(a.err, kErrBlock);
  for (int t = tid; t < r.sink; t += kSelectThreads) kept[t] = t;
  for (int t = tid; t < r.recent; t += kSelectThreads) kept[r.keep - r.recent + t] = r.ctx - r.recent + t;
}

// Moves the kept tokens of a layer, kv head and request: a workgroup for 8 dims of K with the 8 that turn with
// them and for 16 dims of V, its `runs` waves for 64 tokens each a turn.  All sources of a turn are read before
// its slots are written; those of later turns lie past them, as a token never moves up.  So a cache is compacted
// in its own pages.  What a turn's tokens are is looked up while the turn before runs, their positions two turns
// ahead.
//
// A page holds V by dims, eight slots of one in a row: the half pages that have kept tokens are read whole into LDS, from
// where each new slot takes its own (read one by one from memory, at 2 bytes a lane, the cache's ports were the bound: 32
// requests of 2-8k tokens back to half, two layers, 496 us; put in order as they come, 435).
//
// Bound by HBM where there are many tokens: memory comes in lines of 128 bytes, which hold 8 slots of K or V, and
// almost each has a token that stays.  That call reads 1306 MB (all of its old pages) and writes 617 in 403 us, 4.77
// TB/s; a copy reaches 4.85.  kv heads are neighbours in the grid, one to an XCD: as its second index, 4% more.
// A few requests are bound by latency: 2000 of 8000 tokens, one layer, 18 us.
struct MoveArgs {
  EvictArgs e;
  double freq[kAngles];                // turns of a position's angle, of each dim below HD / 2
};
static_assert(sizeof(EvictReq) == 32 && sizeof(MoveArgs) <= kArgumentBytes, "a launch's arguments");
// Where a token lies: page of its kv head x 16 + slot; kStill: there it stays; kNone (kStill among its bits): there is none
constexpr uint32_t kStill = 1u << 31, kNone = ~0u;
constexpr int kHalves = 32;            // half pages of bf16 in a wave's LDS, 256 bytes each

template <typename T, int HD>
__global__ __launch_bounds__(1024) void evict_move_kernel(MoveArgs m) {
  constexpr int OCT = HD / 16, VEC = 8 * (int)sizeof(T) / 16;       // 16-byte pieces of eight elements
  constexpr int PAGE = kPage * HD, IN = kHalves / VEC;              // half pages that LDS holds at a time
  const EvictArgs &a = m.e;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, tid = threadIdx.x;
  const int tokens = 64 * a.runs;                       // of a turn
  uint32_t *codes = reinterpret_cast<uint32_t *>(smem);              // [2][tokens]
  int *places = reinterpret_cast<int *>(smem) + 2 * tokens;          // [2][tokens]
  uint32_t *halves = reinterpret_cast<uint32_t *>(places + 2 * tokens);   // [2][runs][64]: the half pages of a run's tokens: page x 2 + half
  uint16_t *sources = reinterpret_cast<uint16_t *>(halves + 2 * tokens);   // [2][tokens]: a token's half page, of its run's, x 8 + slot there
  int *news = reinterpret_cast<int *>(sources + 2 * tokens), *n_halves = news + 2 * tokens / 16;   // [2][tokens / 16]; [2][runs]
  // this wave's half pages of V, 16 dims of 8 slots each
  uint4 *raw = reinterpret_cast<uint4 *>(smem + ((2 * tokens * 14 + 10 * a.runs * 4 + 15) & ~15)) + wave * kHalves * 16;
  const int rest = blockIdx.x / a.nkv;
  const EvictReq r = request_of(a, rest / OCT);
  const int oct = rest % OCT, t0 = wave * 64, kvh = blockIdx.x - rest * a.nkv, layer = blockIdx.z;
  const int32_t *pt = a.table + (int64_t)r.req * a.stride, *to = a.to + (int64_t)r.req * a.to_stride;
  const int32_t *kept = a.kept + ((int64_t)layer * a.nkv + kvh) * a.total + r.start;
  const int64_t layer_at = (int64_t)layer * a.n_blocks * a.nkv * PAGE;
  // this lane's slot of K, in the order of the new page, and its octet's place there
  const int ks = (lane % 8 / 4) * 8 + lane % 16 / 8 * 4 + lane % 4;
  T *kp = static_cast<T *>(a.k) + layer_at + k_page_off(0, 8 * oct);
  const int partner = k_page_off(0, 8 * oct + HD / 2) - k_page_off(0, 8 * oct);
  // of V: dim lane % 16 of the octets' block, slots 8 (lane / 16 % 2) .. of pages lane / 32 and 2 more
  T *vp = static_cast<T *>(a.v) + layer_at + v_page_off(0, 16 * oct + lane % 16);
  const int v_half = lane / 16 % 2;

  const int turns = (r.keep + tokens - 1) / tokens;
  auto position = [&](int x) __attribute__((always_inline)) { return x * tokens + tid < r.keep ? kept[x * tokens + tid] : -1; };
  int pos = position(0), blk = pos >= 0 ? pt[pos >> 4] : 0, new_page = pos >= 0 ? to[tid >> 4] : -1;
  float *mass = a.mass + (int64_t)layer * a.n_blocks * a.nkv * kPage;
  const bool weighs = oct == 0;                         // with one workgroup the weights move too
  float weight = 0.f, moving = 0.f;
  int put_to = -1, put_next = -1;                      // the new place (a page of the head), if it is another one
  auto list = [&](int x) __attribute__((always_inline)) {
    const int at = (x & 1) * tokens + tid, b = min(max(blk, 0), a.n_blocks - 1);
    if (pos >= 0 && (blk != b || new_page < 0 || new_page >= a.n_blocks)) flag_error(a.err, kErrBlock);
    put_next = pos >= 0 && new_page >= 0 && new_page < a.n_blocks && (pos != x * tokens + tid || b != new_page) ? new_page * a.nkv + kvh : -1;
    if (weighs && put_next >= 0) weight = mass[((int64_t)b * a.nkv + kvh) * kPage + (pos & 15)];
    codes[at] = pos < 0 ? kNone : (uint32_t)(b * a.nkv + kvh) << 4 | (pos & 15) | (pos == x * tokens + tid && b == new_page ? kStill : 0);
    places[at] = pos;
    // the first of a half page's tokens: they are in order
    const int before = __shfl_up(pos, 1);
    const bool first = pos >= 0 && (lane == 0 || before >> 3 != pos >> 3);
    const unsigned long long all = __builtin_amdgcn_ballot_w64(first);
    const int in_run = __popcll(all & ((2ull << lane) - 1)) - 1;
    if (first) halves[(at & ~63) + in_run] = (uint32_t)(b * a.nkv + kvh) << 1 | (pos >> 3 & 1);
    sources[at] = pos < 0 ? 0 : in_run << 3 | (pos & 7);
    if (lane == 0) n_halves[at >> 6] = __popcll(all);
    if (tid % 16 == 0) news[((x & 1) * tokens + tid) / 16] = new_page >= 0 && new_page < a.n_blocks ? new_page * a.nkv + kvh : -1;
  };
  list(0);
  moving = weight;
  put_to = put_next;
  pos = position(1);
  __syncthreads();
  for (int x = 0; x < turns; ++x) {
    const int at = (x & 1) * tokens + t0, d0 = x * tokens + t0;
    const uint32_t ck = codes[at + (lane & ~15) + ks];
    const int delta = d0 + (lane & ~15) + ks - places[at + (lane & ~15) + ks], kd = news[(at + lane) / 16];
    uint32_t cv[2][8];
    int vd[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int from = at + 32 * y + 16 * (lane / 32) + 8 * v_half;
      __builtin_memcpy(cv[y], __builtin_assume_aligned(&codes[from], 32), 32);
      vd[y] = news[from / 16];
    }
    T moved[2][8] = {};                                 // V in its new order
    // the lookups of the next turn
    int after = -1;
    if (x + 1 < turns) {
      blk = pos >= 0 ? pt[pos >> 4] : 0;
      new_page = pos >= 0 ? to[((x + 1) * tokens + tid) >> 4] : -1;
      after = position(x + 2);
    }
    // of no token: the pool's first one, not used
    uint4 lo[VEC], hi[VEC];
    {
      const uint32_t c = ck == kNone ? 0 : ck & ~kStill;
      const T *from = kp + (int64_t)(c >> 4) * PAGE + k_page_off(c & 15, 0);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        lo[v] = ld16(reinterpret_cast<const char *>(from) + 16 * v);
        hi[v] = ld16(reinterpret_cast<const char *>(from + partner) + 16 * v);
      }
    }
    {
      const uint32_t *half = halves + at;
      const int n = __builtin_amdgcn_readfirstlane(n_halves[at >> 6]);
      for (int h0 = 0; h0 < n; h0 += IN) {
        uint4 w[IN / 4][VEC];
#pragma unroll
        for (int i = 0; i < IN / 4; ++i) {
          const uint32_t c = half[min(h0 + 4 * i + lane / 16, n - 1)];
          const T *from = vp + (int64_t)(c >> 1) * PAGE + (c & 1) * 128;
#pragma unroll
          for (int v = 0; v < VEC; ++v) w[i][v] = ld16(reinterpret_cast<const char *>(from) + 16 * v);
        }
#pragma unroll
        for (int i = 0; i < IN / 4; ++i)
#pragma unroll
          for (int v = 0; v < VEC; ++v) raw[((4 * i + lane / 16) * 16 + lane % 16) * VEC + v] = w[i][v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int from = (int)sources[at + 32 * y + 16 * (lane / 32) + 8 * v_half + e] - 8 * h0;
            const T got = reinterpret_cast<const T *>(raw)[(min(max(from >> 3, 0), IN - 1) * 16 + lane % 16) * 8 + (from & 7)];
            moved[y][e] = (uint32_t)from < 8 * IN ? got : moved[y][e];
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (x + 1 < turns) {
      list(x + 1);
      pos = after;
    }
    // every load of the turn has returned, to every wave
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    if (weighs && put_to >= 0) mass[(int64_t)put_to * kPage + (tid & 15)] = moving;
    moving = weight;
    put_to = put_next;
    if (!(ck & kStill) && kd >= 0) {
      if (delta != 0) {
        uint32_t wl[4 * VEC], wh[4 * VEC];
        __builtin_memcpy(wl, lo, sizeof(wl));
        __builtin_memcpy(wh, hi, sizeof(wh));
        float l[8], h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // the angle in turns, its whole ones taken off in 64 bits; sine and cosine of it are within 2.2 x 2^-24
          const double turn = (double)delta * m.freq[8 * oct + e];
          const float f = (float)(turn - __builtin_rint(turn)), c = __builtin_amdgcn_cosf(f), n = __builtin_amdgcn_sinf(f);
          float p, q;
          if constexpr (sizeof(T) == 2) {
            p = e & 1 ? __uint_as_float(wl[e / 2] & 0xFFFF0000u) : __uint_as_float(wl[e / 2] << 16);
            q = e & 1 ? __uint_as_float(wh[e / 2] & 0xFFFF0000u) : __uint_as_float(wh[e / 2] << 16);
          } else {
            p = __uint_as_float(wl[e]);
            q = __uint_as_float(wh[e]);
          }
          l[e] = __builtin_fmaf(p, c, -(q * n));
          h[e] = __builtin_fmaf(q, c, p * n);
        }
        if constexpr (sizeof(T) == 2) {
          lo[0] = make_uint4(pack2bf_rne(l[0], l[1]), pack2bf_rne(l[2], l[3]), pack2bf_rne(l[4], l[5]), pack2bf_rne(l[6], l[7]));
          hi[0] = make_uint4(pack2bf_rne(h[0], h[1]), pack2bf_rne(h[2], h[3]), pack2bf_rne(h[4], h[5]), pack2bf_rne(h[6], h[7]));
        } else {
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            lo[v] = make_uint4(__float_as_uint(l[4 * v]), __float_as_uint(l[4 * v + 1]), __float_as_uint(l[4 * v + 2]), __float_as_uint(l[4 * v + 3]));
            hi[v] = make_uint4(__float_as_uint(h[4 * v]), __float_as_uint(h[4 * v + 1]), __float_as_uint(h[4 * v + 2]), __float_as_uint(h[4 * v + 3]));
          }
        }
      }
      T *put = kp + (int64_t)kd * PAGE + k_page_off(ks, 0);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(put) + 16 * v) = lo[v];
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(put + partner) + 16 * v) = hi[v];
      }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      if (vd[y] < 0) continue;
      T *put = vp + (int64_t)vd[y] * PAGE + 128 * v_half;
      uint32_t some = 0, all = kStill;                  // slots that are not written: of tokens that stay, and of none
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        some |= cv[y][e];
        all &= cv[y][e];
      }
      if (all) continue;
      if (!(some & kStill)) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) __builtin_memcpy(reinterpret_cast<char *>(put) + 16 * v, reinterpret_cast<const char *>(moved[y]) + 16 * v, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(cv[y][e] & kStill)) put[e] = moved[y][e];
      }
    }
  }
}

struct Evict {
  std::vector<EvictReq> reqs;
  int64_t total = 0;
  int32_t most = 0;                     // tokens that a request's are chosen from
};

wisp_status check_evict(Evict &e, const wisp_model *m, const wisp_batch_desc *d, const int32_t *keep, const int32_t *sink,
                        const int32_t *recent) {
  for (int i = 0; i < d->B; ++i) {
    const int32_t ctx = d->ctx_len[i], s = sink ? sink[i] : 0, t = recent ? recent[i] : 0;
    if (keep[i] < 0 || s < 0 || t < 0) return fail(WISP_E_INVALID, "request %d: keep, sink or recent < 0", i);
    if (keep[i] < ctx && (int64_t)s + t > keep[i])
      return fail(WISP_E_INVALID, "request %d: sink %d + recent %d beyond keep %d", i, s, t, keep[i]);
    EvictReq r{};
    r.req = i;
    r.ctx = ctx;
    r.keep = std::min(keep[i], ctx);
    r.sink = r.keep == ctx ? 0 : s;
    r.recent = r.keep == ctx ? 0 : t;
    if (e.total + r.keep > INT32_MAX) return fail(WISP_E_UNSUPPORTED, "more than 2^31 - 1 kept tokens");
    r.start = (int32_t)e.total;
    e.total += r.keep;
    if (r.keep < ctx) e.most = std::max(e.most, ctx - r.sink - r.recent);
    if (r.keep > 0) e.reqs.push_back(r);
  }
  std::stable_sort(e.reqs.begin(), e.reqs.end(), [](const EvictReq &x, const EvictReq &y) { return x.ctx > y.ctx; });
  return WISP_OK;
}

wisp_status check_evict_desc(const wisp_batch_desc *d) {
  if (!d) return fail(WISP_E_INVALID, "batch descriptor is NULL");
  if (d->B < 0) return fail(WISP_E_INVALID, "B < 0");
  if (d->B == 0) return WISP_OK;
  if (!d->ctx_len) return fail(WISP_E_INVALID, "ctx_len is NULL");
  for (int i = 0; i < d->B; ++i)
    if (d->ctx_len[i] < 0 || d->ctx_len[i] > INT32_MAX / 2) return fail(WISP_E_INVALID, "ctx_len[%d] = %d", i, d->ctx_len[i]);
  return WISP_OK;
}

size_t evict_bytes(int64_t B) { return 256 + align256((size_t)B * sizeof(EvictReq)); }

}  // namespace

}  // namespace wisp

using namespace wisp;

extern "C" {

size_t wisp_kv_evict_workspace_size(const wisp_model *model, const wisp_batch_desc *desc) {
  return guarded_size([&]() -> size_t {
    if (check_model(model, false) != WISP_OK || check_evict_desc(desc) != WISP_OK) return 0;
    return evict_bytes(desc->B);
  });
}

wisp_status wisp_kv_evict(const wisp_model *model, const wisp_kv *kv, const wisp_batch_desc *desc, const int32_t *keep,
                          const int32_t *sink, const int32_t *recent, const int32_t *to_table, int32_t to_stride, float *mass,
                          int32_t *kept, void *workspace, size_t workspace_bytes, void *stream) {
  return guarded("wisp_kv_evict", [&]() -> wisp_status {
    wisp_status st;
    if ((st = check_model(model, false)) != WISP_OK || (st = check_evict_desc(desc)) != WISP_OK) return st;
    if (desc->B == 0) return WISP_OK;
    if (!kv || !kv->k_pool || !kv->v_pool) return fail(WISP_E_INVALID, "KV pools are NULL");
    if (kv->page_size != WISP_PAGE) return fail(WISP_E_UNSUPPORTED, "page_size must be %d", WISP_PAGE);
    if (kv->n_blocks <= 0) return fail(WISP_E_INVALID, "n_blocks must be positive");
    if (((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool) & 15) return fail(WISP_E_INVALID, "KV pools must be 16-byte aligned");
    if (!keep || !mass) return fail(WISP_E_INVALID, "NULL keep / mass");
    if (!desc->kv_page_table) return fail(WISP_E_INVALID, "kv_page_table is NULL");
    Evict e;
    if ((st = check_evict(e, model, desc, keep, sink, recent)) != WISP_OK) return st;
    if (!kept && e.total > 0) return fail(WISP_E_INVALID, "kept is NULL");
    const int32_t stride = to_table ? to_stride : desc->pt_stride;
    for (const EvictReq &r : e.reqs) {
      if ((int64_t)desc->pt_stride * WISP_PAGE < r.ctx)
        return fail(WISP_E_CAPACITY, "request %d has %d tokens but the page table holds %d", r.req, r.ctx, desc->pt_stride * WISP_PAGE);
      if ((int64_t)stride * WISP_PAGE < r.keep)
        return fail(WISP_E_CAPACITY, "request %d keeps %d tokens but its new pages hold %d", r.req, r.keep, stride * WISP_PAGE);
    }
    if ((int64_t)kv->n_blocks * model->n_kv_heads >= 1 << 27) return fail(WISP_E_UNSUPPORTED, "n_blocks x n_kv_heads of 2^27 or more");
    const int oct = model->head_dim / 16;
    if ((int64_t)e.reqs.size() * model->n_kv_heads * oct >= 1 << 22)   // a launch's threads fit in 32 bits
      return fail(WISP_E_UNSUPPORTED, "requests x n_kv_heads x head_dim / 16 of 2^22 or more");
    if (model->n_layers > 65535 || model->n_kv_heads > 65535) return fail(WISP_E_UNSUPPORTED, "more than 65535 layers or kv heads");
    if (!workspace) return fail(WISP_E_INVALID, "NULL workspace");
    if ((uintptr_t)workspace & 255) return fail(WISP_E_INVALID, "workspace must be 256-byte aligned");
    if (workspace_bytes < evict_bytes(desc->B))
      return fail(WISP_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, evict_bytes(desc->B));
    if (e.reqs.empty()) return WISP_OK;
    char *ws = static_cast<char *>(workspace);
    const hipStream_t s = (hipStream_t)stream;
    EvictArgs a{};
    if (e.reqs.size() <= kFew) {
      std::copy(e.reqs.begin(), e.reqs.end(), a.few);
    } else {
      std::vector<int32_t> host(e.reqs.size() * (sizeof(EvictReq) / 4));
      std::memcpy(host.data(), e.reqs.data(), host.size() * 4);
      hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
      if (hipStreamIsCapturing(s, &cap) != hipSuccess) return fail(WISP_E_HIP, "stream query failed");
      st = cap == hipStreamCaptureStatusNone ? upload_ints(host, ws + 256, s) : upload_ints_by_arguments(host, ws + 256, s);
      if (st != WISP_OK) return st;
      a.reqs = reinterpret_cast<const EvictReq *>(ws + 256);
    }
    a.table = desc->kv_page_table;
    a.to = to_table ? to_table : desc->kv_page_table;
    a.k = kv->k_pool;
    a.v = kv->v_pool;
    a.mass = mass;
    a.kept = kept;
    a.err = reinterpret_cast<int *>(ws);
    a.total = e.total;
    a.stride = desc->pt_stride;
    a.to_stride = stride;
    a.n_blocks = kv->n_blocks;
    a.nkv = model->n_kv_heads;
    const int n = (int)e.reqs.size();
    launch(e.most <= kSelectHeld * kSelectThreads ? evict_select_kernel<true> : evict_select_kernel<false>,
           dim3(n, a.nkv, model->n_layers), kSelectThreads, 0, s, a);
    // Waves, of 64 tokens of a turn: a request's turns wait for one another.  32 requests of 2-8k tokens back to half,
    // two layers (4096 workgroups), 425 us with 8 waves, some 1% and 6% more with 4 and 16; one of 8000 back to a quarter (64
    // workgroups) a fifth more with 8 than the 33 with 16, a small fp32 model's 12 requests (384) a tenth.
    const int most_waves = (int64_t)n * a.nkv * model->n_layers * oct < 2 * device_cus() ? 16 : 8;
    int most_kept = 0;
    for (const EvictReq &r : e.reqs) most_kept = std::max(most_kept, r.keep);
    a.runs = std::max(1, std::min(most_waves, (most_kept + 63) / 64));
    MoveArgs move{a, {}};
    for (int i = 0; i < model->head_dim / 2; ++i)
      move.freq[i] = std::pow((double)model->rope_base, -2.0 * i / model->head_dim) / (2 * 3.14159265358979323846);
    const uint32_t shm = ((2 * 64 * a.runs * 14 + 10 * a.runs * 4 + 15) & ~15) + (uint32_t)a.runs * kHalves * 256;
    auto go = [&](auto kernel) {
      launch(kernel, dim3((unsigned)n * oct * a.nkv, 1, model->n_layers), 64 * a.runs, shm, s, move);
    };
    if (model->dtype == WISP_BF16) {
      if (model->head_dim == 128) go(evict_move_kernel<uint16_t, 128>);
      else go(evict_move_kernel<uint16_t, 64>);
    } else {
      switch (model->head_dim) {
        case 32: go(evict_move_kernel<float, 32>); break;
        case 64: go(evict_move_kernel<float, 64>); break;
        case 96: go(evict_move_kernel<float, 96>); break;
        case 128: go(evict_move_kernel<float, 128>); break;
        case 160: go(evict_move_kernel<float, 160>); break;
        case 192: go(evict_move_kernel<float, 192>); break;
        case 224: go(evict_move_kernel<float, 224>); break;
        default: go(evict_move_kernel<float, 256>);
      }
    }
    return hip_check("eviction launch");
  });
}

}  // extern "C"
