// Eviction from the paged KV cache: of each request and kv head the tokens of greatest weight stay, with the
// first and the last ones, and move together; a kept key is rotated from its old position to its new one.
#include <algorithm>
#include <climits>
#include <cstring>
#include <numeric>

#include "api.h"
#include "host_guard.h"
#include "kernels.h"

namespace wisp {

namespace {

struct EvictReq {                      // a request, the longest first
  int32_t req, ctx, keep, sink;
  int32_t recent, start, pad[2];       // start: of its tokens in a head's list
};

struct EvictArgs {
  const EvictReq *reqs;
  const int32_t *table, *to;
  void *k, *v;
  float *mass;
  int32_t *kept;
  int *err;
  int64_t total;                       // kept tokens of all requests
  int stride, to_stride, n_blocks, nkv, slices;
  double base;                         // rope_base
};

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kSelectKeys = 16384;

// floats in the order of their values as unsigned integers, -0 as 0, NaN below everything
__device__ __forceinline__ uint32_t key_of(float f) {
  if (f != f) return 0u;
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which tokens stay: a workgroup for each layer, kv head and request.  A radix selection, 8 bits a
// pass, finds the least key that stays and how many of that key do (the first ones); then the tokens
// are listed in order, and their weights move.
template <bool LDS>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t keys[LDS ? kSelectKeys : 1];
  __shared__ uint32_t hist[256];
  __shared__ int more[kSelectWaves], same[kSelectWaves];
  __shared__ uint32_t sh_key;
  __shared__ int sh_left;
  const EvictReq r = a.reqs[blockIdx.x];
  const int kvh = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t *pt = a.table + (int64_t)r.req * a.stride, *to = a.to + (int64_t)r.req * a.to_stride;
  float *mass = a.mass + (int64_t)layer * a.n_blocks * a.nkv * kPage;
  int32_t *kept = a.kept + ((int64_t)layer * a.nkv + kvh) * a.total + r.start;
  auto at = [&](int b, int t) { return ((int64_t)min(max(b, 0), a.n_blocks - 1) * a.nkv + kvh) * kPage + (t & 15); };
  for (int x = tid; x < (r.ctx + 15) / 16; x += kSelectThreads)
    if (pt[x] < 0 || pt[x] >= a.n_blocks) flag_error(a.err, kErrBlock);
  for (int x = tid; x < (r.keep + 15) / 16; x += kSelectThreads)
    if (to[x] < 0 || to[x] >= a.n_blocks) flag_error(a.err, kErrBlock);

  if (r.keep == r.ctx) {
    for (int t = tid; t < r.keep; t += kSelectThreads) kept[t] = t;
  } else {
    const int n = r.ctx - r.sink - r.recent;           // tokens to choose from
    auto key = [&](int x) { return LDS ? keys[x] : key_of(mass[at(pt[(r.sink + x) >> 4], r.sink + x)]); };
    if constexpr (LDS) {
      for (int x = tid; x < n; x += kSelectThreads) keys[x] = key_of(mass[at(pt[(r.sink + x) >> 4], r.sink + x)]);
      __syncthreads();
    }
    uint32_t found = 0;
    int left = r.keep - r.sink - r.recent;             // tokens with the key's bits so far that stay
    for (int shift = 24; shift >= 0 && left > 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int x = tid; x < n; x += kSelectThreads) {
        const uint32_t k = key(x);
        if (shift == 24 || (k >> (shift + 8)) == (found >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {
        // the digit at which the count from the top reaches `left`: four digits a lane
        int c[4], sum = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) sum += c[x] = hist[255 - 4 * lane - x];
        int before = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int v = __shfl_up(before, o);
          before += lane >= o ? v : 0;
        }
        before -= sum;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (before < left && before + c[x] >= left) {
            sh_key = found | (uint32_t)(255 - 4 * lane - x) << shift;
            sh_left = left - before;
          }
          before += c[x];
        }
      }
      __syncthreads();
      found = sh_key;
      left = sh_left;
    }
    if (left == 0) found = UINT_MAX;                    // none of the middle stays (no key is above)
    // each wave lists a run of tokens: first their number, then their places
    const int run = (n + kSelectThreads - 1) / kSelectThreads * 64, x0 = wave * run, x1 = min(n, x0 + run);
    int m = 0, s = 0;
    for (int x = x0 + lane; x - lane < x1; x += 64) {
      const uint32_t k = x < x1 ? key(x) : 0;
      m += __popcll(__builtin_amdgcn_ballot_w64(x < x1 && k > found));
      s += __popcll(__builtin_amdgcn_ballot_w64(x < x1 && k == found));
    }
    if (lane == 0) {
      more[wave] = m;
      same[wave] = s;
    }
    __syncthreads();
    m = 0;                                              // tokens listed before this one's, with the key and above it
    s = 0;
    for (int w = 0; w < wave; ++w) {
      m += more[w];
      s += same[w];
    }
    const unsigned long long below = (1ull << lane) - 1;
    for (int x = x0 + lane; x - lane < x1; x += 64) {
      const uint32_t k = x < x1 ? key(x) : 0;
      const unsigned long long gt = __builtin_amdgcn_ballot_w64(x < x1 && k > found), eq = __builtin_amdgcn_ballot_w64(x < x1 && k == found);
      const int e = s + __popcll(eq & below), place = r.sink + m + __popcll(gt & below) + min(e, left);
      if (x < x1 && (k > found || (k == found && e < left))) kept[place] = r.sink + x;
      m += __popcll(gt);
      s += __popcll(eq);
    }
    for (int t = tid; t < r.sink; t += kSelectThreads) kept[t] = t;
    for (int t = tid; t < r.recent; t += kSelectThreads) kept[r.keep - r.recent + t] = r.ctx - r.recent + t;
  }
  __syncthreads();
  // the weights: a token never moves up, so those still to be read lie past those written
  for (int d0 = 0; d0 < r.keep; d0 += kSelectThreads) {
    const int d = d0 + tid;
    float w = 0.f;
    int64_t dst = -1;
    if (d < r.keep) {
      const int t = kept[d], b = to[d >> 4];
      w = mass[at(pt[t >> 4], t)];
      if (b >= 0 && b < a.n_blocks) dst = at(b, d);
    }
    __syncthreads();
    if (dst >= 0) mass[dst] = w;
  }
}

// Moves the kept tokens of a layer, kv head and request: dims in slices, a workgroup each, which takes the new
// pages in order, some at a time.  All sources of a turn are read before its slots are written; those of
// later turns lie past them, as a token never moves up.  So a cache can be compacted in its own pages.
constexpr int kMoveThreads = 256;

// cos and sin of 2 pi x
__device__ __forceinline__ void turn_of(double x, float &c, float &s) {
  const float f = (float)(x - __builtin_rint(x));
  s = sinpif(2.0f * f);
  c = cospif(2.0f * f);
}

template <typename T, int HD>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a) {
  constexpr int OCT = HD / 16;                          // octets of dims that turn with the octet HD / 2 above; blocks of 16 dims of V
  constexpr int PAGES = 16;                             // of a turn
  struct Src {
    int blk, pos;
  };
  __shared__ Src src[PAGES * kPage];
  __shared__ int dst[PAGES];
  const EvictReq r = a.reqs[blockIdx.x / a.slices];
  const int slice = blockIdx.x % a.slices, kvh = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
  const int o0 = OCT * slice / a.slices, no = OCT * (slice + 1) / a.slices - o0;
  const int32_t *pt = a.table + (int64_t)r.req * a.stride, *to = a.to + (int64_t)r.req * a.to_stride;
  const int32_t *kept = a.kept + ((int64_t)layer * a.nkv + kvh) * a.total + r.start;
  T *kp = static_cast<T *>(a.k) + (int64_t)layer * a.n_blocks * a.nkv * (kPage * HD);
  T *vp = static_cast<T *>(a.v) + (int64_t)layer * a.n_blocks * a.nkv * (kPage * HD);
  auto page = [&](int b) { return ((int64_t)b * a.nkv + kvh) * (kPage * HD); };
  const int pages = (r.keep + 15) / 16;
  const int per_turn = min(PAGES, max(1, kMoveThreads / (16 * no)));   // pages: a thread one K unit at most, two of V
  // K: a slot's octet and its partner, in the order of the new page; the turns of a position's angle
  const int kx = tid % 16, ko = o0 + tid / 16 % no, kpg = tid / (16 * no);
  const int ks = (kx % 8 / 4) * 8 + kx / 8 * 4 + kx % 4;
  double freq[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) freq[e] = exp2(-2.0 * (8 * ko + e) / HD * log2(a.base)) * 0.15915494309189533577;
  for (int p0 = 0; p0 < pages; p0 += per_turn) {
    const int n = min(per_turn, pages - p0);
    __syncthreads();                                    // the list before has been read
    for (int x = tid; x < n * kPage; x += kMoveThreads) {
      const int d = p0 * kPage + x;
      Src s{-1, -1};
      if (d < r.keep) {
        s.pos = kept[d];
        s.blk = min(max(pt[s.pos >> 4], 0), a.n_blocks - 1);
      }
      src[x] = s;
    }
    if (tid < n) {
      const int b = to[p0 + tid];
      dst[tid] = b >= 0 && b < a.n_blocks ? b : -1;
    }
    __syncthreads();
    float lo[8], hi[8];
    Src sk{-1, -1};
    if (kpg < n) sk = src[kpg * kPage + ks];
    if (sk.pos >= 0) {
      const T *from = kp + page(sk.blk);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (sizeof(T) == 2) {
          lo[e] = bf2f(from[k_page_off(sk.pos & 15, 8 * ko) + e]);
          hi[e] = bf2f(from[k_page_off(sk.pos & 15, 8 * ko + HD / 2) + e]);
        } else {
          lo[e] = from[k_page_off(sk.pos & 15, 8 * ko) + e];
          hi[e] = from[k_page_off(sk.pos & 15, 8 * ko + HD / 2) + e];
        }
      }
    }
    // V: a dim of eight slots
    T val[2][8];
    bool full[2], moved[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int u = tid + y * kMoveThreads, vx = u % 32, vo = o0 + u / 32 % no, vpg = u / (32 * no);
      full[y] = true;
      moved[y] = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        val[y][e] = 0;
        Src s{-1, -1};
        if (vpg < n) s = src[vpg * kPage + vx / 16 * 8 + e];
        if (s.pos >= 0) {
          val[y][e] = vp[page(s.blk) + v_page_off(s.pos & 15, 16 * vo + vx % 16)];
          moved[y] |= s.pos != (p0 + vpg) * kPage + vx / 16 * 8 + e || s.blk != dst[vpg];
        } else {
          full[y] = false;
        }
      }
    }
    __syncthreads();
    if (sk.pos >= 0 && dst[kpg] >= 0) {
      const int d = (p0 + kpg) * kPage + ks;
      if (d != sk.pos || sk.blk != dst[kpg]) {
        T *put = kp + page(dst[kpg]);
        if (d != sk.pos) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float c, s;
            turn_of((double)(d - sk.pos) * freq[e], c, s);
            const float x = lo[e], y = hi[e];
            lo[e] = __builtin_fmaf(x, c, -(y * s));
            hi[e] = __builtin_fmaf(y, c, x * s);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (sizeof(T) == 2) {
            put[k_page_off(ks, 8 * ko) + e] = __builtin_bit_cast(uint16_t, (__bf16)lo[e]);
            put[k_page_off(ks, 8 * ko + HD / 2) + e] = __builtin_bit_cast(uint16_t, (__bf16)hi[e]);
          } else {
            put[k_page_off(ks, 8 * ko) + e] = lo[e];
            put[k_page_off(ks, 8 * ko + HD / 2) + e] = hi[e];
          }
        }
      }
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int u = tid + y * kMoveThreads, vx = u % 32, vo = o0 + u / 32 % no, vpg = u / (32 * no);
      if (vpg >= n || !moved[y] || dst[vpg] < 0) continue;
      T *put = vp + page(dst[vpg]) + v_page_off(vx / 16 * 8, 16 * vo + vx % 16);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (full[y] || src[vpg * kPage + vx / 16 * 8 + e].pos >= 0) put[e] = val[y][e];
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
    if (model->n_layers > 65535 || model->n_kv_heads > 65535) return fail(WISP_E_UNSUPPORTED, "more than 65535 layers or kv heads");
    if (!workspace) return fail(WISP_E_INVALID, "NULL workspace");
    if ((uintptr_t)workspace & 255) return fail(WISP_E_INVALID, "workspace must be 256-byte aligned");
    if (workspace_bytes < evict_bytes(desc->B))
      return fail(WISP_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, evict_bytes(desc->B));
    if (e.reqs.empty()) return WISP_OK;
    char *ws = static_cast<char *>(workspace);
    const hipStream_t s = (hipStream_t)stream;
    std::vector<int32_t> host(e.reqs.size() * (sizeof(EvictReq) / 4));
    std::memcpy(host.data(), e.reqs.data(), host.size() * 4);
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &cap) != hipSuccess) return fail(WISP_E_HIP, "stream query failed");
    st = cap == hipStreamCaptureStatusNone ? upload_ints(host, ws + 256, s) : upload_ints_by_arguments(host, ws + 256, s);
    if (st != WISP_OK) return st;
    EvictArgs a{};
    a.reqs = reinterpret_cast<const EvictReq *>(ws + 256);
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
    a.base = model->rope_base;
    const int n = (int)e.reqs.size();
    launch(e.most <= kSelectKeys ? evict_select_kernel<true> : evict_select_kernel<false>, dim3(n, a.nkv, model->n_layers),
           kSelectThreads, 0, s, a);
    const int64_t units = (int64_t)n * a.nkv * model->n_layers, wgs = 4 * (int64_t)device_cus();
    a.slices = 1;
    while (a.slices < model->head_dim / 16 && units * a.slices < wgs) a.slices *= 2;
    a.slices = std::min(a.slices, model->head_dim / 16);
    auto go = [&](auto kernel) { launch(kernel, dim3((unsigned)n * a.slices, a.nkv, model->n_layers), kMoveThreads, 0, s, a); };
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
