// What a server tells about the tokens of its answer (the rows that wisp_verify scored): the log
// probability of each given token, the entropy of its distribution and the most probable tokens.
// Declared in include/wisp.h.
//
// One pass over the logits: a workgroup holds a chunk of a row in registers, takes its maximum m
// and the sums s = sum e^((x - m) / T) and c = sum (x - m) e^((x - m) / T), x - m formed first, so that
// large logits lose nothing.  With the chunks joined, ln p(t) = (x_t - m) / T - ln s and the entropy is
// ln s - c / (s T).  For the most probable tokens the pass also leaves the largest of each group of 32
// entries: the k-th largest of those bounds the k-th largest entry from below, and only the
// few groups that reach it are read again.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "api.h"
#include "host_guard.h"
#include "kernels.h"
#include "wave_reduce.h"

using namespace wisp;

namespace {

constexpr int kChunk = 8192, kThreads = 256, kGroup = kChunk / kThreads;
constexpr int kMaxChunks = 1 << 23;   // of a launch
constexpr float kLog2e = 1.4426950408889634f;

// log2(e) / T, finite: of a T below 4.3e-39 the quotient is infinite, and its product with the
// maximum's difference, 0, would be NaN
__host__ __device__ inline float scale_of(float T) { return fminf(kLog2e / T, 3.402823466e38f); }

struct Part {   // of one chunk: the maximum, and the sums about it (0 where nothing is above -inf)
  double s, c;
  float m, pad;
};

// Entry j of thread t's group sits at entry_at(t, j) of its chunk: a group is what one thread loads
template <int W>   // consecutive entries of a load
__device__ __forceinline__ int entry_at(int t, int j) { return ((j / W) * kThreads + t) * W + j % W; }

template <typename T> __device__ __forceinline__ float logit(const T *x, int64_t i);
template <> __device__ __forceinline__ float logit<float>(const float *x, int64_t i) { return x[i]; }
template <> __device__ __forceinline__ float logit<uint16_t>(const uint16_t *x, int64_t i) { return bf2f(x[i]); }

// of the row of a workgroup; false: the row has no token, and is left as it was
__device__ __forceinline__ bool row_counts(const int32_t *tokens, int64_t row) { return !tokens || tokens[row] != -1; }

__device__ __forceinline__ Part join(const Part &a, const Part &b, float sc) {
  // about the larger maximum; a side without entries (s = 0) adds nothing, a NaN stays
  Part r;
  r.m = fmaxf(a.m, b.m);
  r.pad = 0.f;
  auto side = [&](const Part &p, double &s, double &c) {
    const double d = p.m == r.m ? 0.0 : (double)p.m - (double)r.m, w = __builtin_amdgcn_exp2f((float)d * sc);
    s = p.s == 0.0 ? 0.0 : p.s * w;
    c = p.s == 0.0 ? 0.0 : w * (p.c + d * p.s);
  };
  double s1, c1, s2, c2;
  side(a, s1, c1);
  side(b, s2, c2);
  r.s = s1 + s2;
  r.c = c1 + c2;
  return r;
}

// Grid rows x chunks, chunks fastest.  Bound by the memory where there are many fp32 rows (742 of
// 128256: 66 us for 381 MB, 5.8 TB/s).  In bf16, whose entries come twice as fast, about half of the time
// is vector instructions (12 for each place of a chunk, of 300 rows of 50021 5 to 6 of 11 us for 30 MB), the
// rest waits for loads, which a thread of one round has nothing to do beside.  A chunk is 32 entries a
// thread: with the sums about the wave's own maximum, known before the first exponential, an entry
// takes one exponential and no rescaling.
// VEC: 16-byte loads, where every row starts on 16 bytes; else one entry a load.  742 contiguous rows of
// 50257 (which start anywhere) with 8 tokens each take 40 us in fp32 and 50 in
// bf16, padded to rows of 16 bytes 36 and 31; 6 rows 10.2 and 12.9, padded 10.1 and 10.4.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void logprobs_chunk_kernel(const T *__restrict__ logits, int V, int64_t ld, int nch,
                                                                 float sc, const int32_t *__restrict__ tokens,
                                                                 Part *__restrict__ parts, float *__restrict__ gmax) {
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1;
  const int64_t row = blockIdx.x / nch;
  const int ch = blockIdx.x % nch, t = threadIdx.x;
  if (!row_counts(tokens, row)) return;
  const int base = ch * kChunk, n = min(V - base, kChunk);
  const T *x = logits + row * ld + base;
  float v[kGroup];
  if constexpr (VEC) {
    uint4 raw[kGroup / W];
    const bool whole = n == kChunk;        // every chunk but the row's last
#pragma unroll
    for (int k = 0; k < kGroup / W; ++k) {   // all loads of the thread in flight at once
      const int e = (k * kThreads + t) * W;
      if (whole || e + W <= n) raw[k] = ld16_stream(x + e);
    }
#pragma unroll
    for (int k = 0; k < kGroup / W; ++k) {
      const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if constexpr (sizeof(T) == 4) v[k * W + i] = __uint_as_float(w[i]);
        else v[k * W + i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
      }
    }
    if (!whole) {
#pragma unroll
      for (int k = 0; k < kGroup / W; ++k) {
        const int e = (k * kThreads + t) * W;
        if (e + W > n) {                   // at or past the row's end
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float f = logit(x, min(e + i, n - 1));
            v[k * W + i] = e + i < n ? f : -INFINITY;
          }
        }
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const int e = entry_at<1>(t, k);
      v[k] = e < n ? logit(x, e) : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kGroup; ++k) m = fmaxf(m, v[k]);
  // sums about the wave's maximum; in a wave of nothing but -inf about 0, where they are 0
  const float mw = wave_max(m), mc = mw == -INFINITY ? 0.f : mw;
  float s = 0.f, c = 0.f;
#pragma unroll
  for (int k = 0; k < kGroup; ++k) {
    const float d = v[k] - mc, e = __builtin_amdgcn_exp2f(d * sc);
    s += e;
    c = fmaf(fmaxf(d, -3.4e38f), e, c);   // -inf x 0 stays out; a NaN enters through e
  }
  if (gmax) gmax[(row * nch + ch) * kThreads + t] = m;
  s = wave_sum(s);
  c = wave_sum(c);
  __shared__ Part sh[kThreads / 64];
  if ((t & 63) == 0) sh[t >> 6] = Part{s, c, mw, 0.f};
  __syncthreads();
  if (t == 0) parts[row * nch + ch] = join(join(sh[0], sh[1], sc), join(sh[2], sh[3], sc), sc);
}

// order-preserving key of a float; -inf is the least
__device__ __forceinline__ uint32_t key_of(float f) {
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

constexpr int kCand = 1024, kList = 256;   // candidates, and groups of a wave, that the quick way takes

// A candidate as a number that is larger for a larger value, and of equal ones (-0 is 0) for the first
__device__ __forceinline__ uint64_t candidate(float v, int i) { return (uint64_t)key_of(v + 0.f) << 32 | (uint32_t)~i; }

// The n candidates' ranks: those below k are written out.
__device__ void write_ranked(const uint64_t *best, int n, int k, const double m, double T, double lse, int32_t *ids, float *lps) {
  for (int a = threadIdx.x; a < n; a += blockDim.x) {
    const uint64_t mine = best[a];
    int rank = 0;
    for (int o = 0; o < n; o += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) rank += o + i < n && best[o + i] > mine;
    if (rank < k) {
      const uint32_t key = (uint32_t)(mine >> 32);
      ids[rank] = (int32_t)~(uint32_t)mine;
      lps[rank] = (float)(((double)value_of(key) - m) / T - lse);
    }
  }
}

// One workgroup per row: four waves look for the most probable tokens, a fifth joins the chunks
// meanwhile (n_top = 0: alone).  N chunks at most (0: any number), so that a thread holds the group
// maxima that it needs: those of its own groups, one a chunk.  Bound by latency (a handful of rows) or by
// starting a workgroup for each: everything that depends on no other load is asked for first, and a
// wave reads its own groups again, so that two barriers are enough (five of them, and the join in
// every wave: 6 rows of 128256 with 5 tokens each 7.5 us, so 6.4; 742 rows with 20 15.1 and 13.7).
template <typename T, int W, int N>
__global__ __launch_bounds__(kThreads + 64) void logprobs_row_kernel(const T *__restrict__ logits, int V, int64_t ld, int nch,
                                                               float temperature, const int32_t *__restrict__ tokens,
                                                               const Part *__restrict__ parts, const float *__restrict__ gmax,
                                                               int top, float *__restrict__ logprob,
                                                               float *__restrict__ entropy, int32_t *__restrict__ top_ids,
                                                               float *__restrict__ top_lps, int *__restrict__ err) {
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63;
  const int tok = tokens ? tokens[row] : -1;
  if (tokens && tok == -1) return;
  const T *x = logits + row * ld;
  const float *gm = gmax + row * nch * kThreads;
  int32_t *ids = top_ids + row * top;
  float *lps = top_lps + row * top;
  __shared__ float sh_max[kThreads];
  __shared__ uint64_t best[kCand];
  __shared__ int32_t sh_group[kThreads / 64][kList];
  __shared__ int sh_n;
  __shared__ bool sh_many;
  __shared__ float sh_m;
  __shared__ double sh_lse;
  const bool search = t + 64 < (int)blockDim.x;
  if (!search) {
    // the chunks joined: a lane's in order, then the lanes
    const bool tok_ok = tok >= 0 && tok < V;
    const float xt = tok_ok ? logit(x, tok) : 0.f;
    const float sc = scale_of(temperature);
    float m = -INFINITY;
    double s = 0.0, cs = 0.0;
    for (int c = lane; c < nch; c += 64) {
      const Part p = parts[row * nch + c];
      const float hi = fmaxf(m, p.m);
      const double d0 = m == hi ? 0.0 : (double)m - hi, d1 = p.m == hi ? 0.0 : (double)p.m - hi;
      const float w0 = __builtin_amdgcn_exp2f((float)d0 * sc), w1 = __builtin_amdgcn_exp2f((float)d1 * sc);
      // a side without entries adds nothing, a NaN stays
      cs = (s == 0.0 ? 0.0 : w0 * (cs + d0 * s)) + (p.s == 0.0 ? 0.0 : w1 * (p.c + d1 * p.s));
      s = (s == 0.0 ? 0.0 : w0 * s) + (p.s == 0.0 ? 0.0 : w1 * p.s);
      m = hi;
    }
    const float mw = wave_max(m);
    {
      const double d = m == mw ? 0.0 : (double)m - mw;
      const float w = __builtin_amdgcn_exp2f((float)d * sc);
      cs = s == 0.0 ? 0.0 : w * (cs + d * s);
      s = s == 0.0 ? 0.0 : w * s;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      s += __shfl_xor(s, o);
      cs += __shfl_xor(cs, o);
    }
    const double lse = log(s);
    const bool none = s == 0.0;                // every logit is -inf
    if (lane == 0) {
      if (tokens && !tok_ok) flag_error(err, kErrToken);
      if (logprob) {
        logprob[row] = !tok_ok || s != s                ? NAN
                       : none || xt == -INFINITY ? -INFINITY
                                                 : (float)(((double)xt - mw) / temperature - lse);
      }
      if (entropy) entropy[row] = none ? 0.f : (float)(lse - cs / s / temperature);
      sh_m = mw;
      sh_lse = lse;
    }
    if (lane < top) {                          // places that no entry fills
      ids[lane] = -1;
      lps[lane] = s != s ? NAN : -INFINITY;
    }
    if (top == 0) return;                      // there is no other wave
  }
  float gv[N ? N : 1];
  if (search) {
    float mine = -INFINITY;
    if constexpr (N > 0) {
#pragma unroll
      for (int c = 0; c < N; ++c) gv[c] = c < nch ? gm[c * kThreads + t] : -INFINITY;
#pragma unroll
      for (int c = 0; c < N; ++c) mine = fmaxf(mine, gv[c]);
    } else {
      for (int c = 0; c < nch; ++c) mine = fmaxf(mine, gm[c * kThreads + t]);
    }
    sh_max[t] = mine;
    if (t == 0) {
      sh_n = 0;
      sh_many = false;
    }
  }
  __syncthreads();
  if (search) {
    // A bound that at least `top` entries reach: the top-th largest of 64 maxima, each of four threads'
    // groups.  Their keys' last six bits give way to the lane, so that all differ.
    static_assert(WISP_TOP_MAX <= 64, "a bound from 64 maxima; a wave fills the places");
    const float most = fmaxf(fmaxf(sh_max[lane], sh_max[lane + 64]), fmaxf(sh_max[lane + 128], sh_max[lane + 192]));
    const uint32_t key = key_of(most + 0.f) & ~63u;
    const uint32_t mine = key | lane;
    int rank = 0;
#pragma unroll
    for (int o = 0; o < 64; ++o) rank += (uint32_t)__builtin_amdgcn_readlane(mine, o) > mine;
    const uint32_t tau = __builtin_amdgcn_readlane(key, __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == top - 1)));
    auto reaches = [&](float v) { return v > -INFINITY && key_of(v + 0.f) >= tau; };
    // the wave's groups that do
    int32_t *list = sh_group[t >> 6];
    int ng = 0;
    auto note = [&](float v, int c) {
      const bool in = reaches(v);
      const uint64_t mask = __builtin_amdgcn_ballot_w64(in);
      const int at = ng + __popcll(mask & ((1ull << lane) - 1));
      if (in && at < kList) list[at] = c * kThreads + t;
      ng += __popcll(mask);
    };
    if constexpr (N > 0) {
#pragma unroll
      for (int c = 0; c < N; ++c) note(gv[c], c);
    } else {
      for (int c = 0; c < nch; ++c) note(gm[c * kThreads + t], c);
    }
    if (ng > kList) {
      if (lane == 0) sh_many = true;
    } else {
      constexpr int P = kGroup / W;            // loads of a group
      for (int u0 = 0; u0 < ng * P; u0 += 64) {
        const int u = min(u0 + lane, ng * P - 1), g = list[u / P];
        const int e0 = g / kThreads * kChunk + entry_at<W>(g % kThreads, u % P * W);
        float v[W];
        if (W > 1 && e0 + W <= V) {
          const uint4 r = ld16(x + e0);
          const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
          for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i % 4]);
            else v[i] = __uint_as_float(i & 1 ? w[i / 2 % 4] & 0xFFFF0000u : w[i / 2 % 4] << 16);
          }
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i) v[i] = e0 + i < V ? logit(x, e0 + i) : -INFINITY;
        }
        uint64_t mask[W];
        int n = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          mask[i] = __builtin_amdgcn_ballot_w64(u0 + lane < ng * P && reaches(v[i]));
          n += __popcll(mask[i]);
        }
        if (n == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh_n, n);   // the order does not matter: candidates are ranked
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const int to = at + __popcll(mask[i] & ((1ull << lane) - 1));
          if ((mask[i] >> lane & 1) && to < kCand) best[to] = candidate(v[i], e0 + i);
          at += __popcll(mask[i]);
        }
      }
    }
  }
  __syncthreads();
  if (!sh_many && sh_n <= kCand) {
    write_ranked(best, sh_n, top, sh_m, temperature, sh_lse, ids, lps);
    return;
  }

  // Too many reach the bound (a mask's lowest value in most places, say): the top-th largest
  // key by four passes over its bytes, then one pass in order for what is above it and for the
  // first that equal it.
  __shared__ uint32_t hist[256];
  __shared__ uint32_t sh_prefix, sh_left;
  uint32_t prefix = 0, left = top;               // keys wanted among those with this prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (search) hist[t] = 0;
    __syncthreads();
    for (int e = search ? t : INT32_MAX; e < (V + 63) / 64 * 64; e += kThreads) {   // whole waves
      const float v = e < V ? logit(x, e) : -INFINITY;
      const uint32_t key = key_of(v + 0.f);
      const bool in = e < V && v > -INFINITY && (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8));
      const int bin = key >> shift & 255;
      uint64_t todo = __builtin_amdgcn_ballot_w64(in);
      if (todo == 0) continue;
      const int lead = __builtin_ctzll(todo), one = __shfl(bin, lead);
      const uint64_t same = __builtin_amdgcn_ballot_w64(in && bin == one);   // equal values: one count
      if ((t & 63) == lead) atomicAdd(&hist[one], (uint32_t)__popcll(same));
      if (in && bin != one) atomicAdd(&hist[bin], 1u);
    }
    __syncthreads();
    if (t == 0) {
      uint32_t seen = 0;
      int b = 255;
      while (b > 0 && seen + hist[b] < left) seen += hist[b--];
      sh_prefix = prefix | (uint32_t)b << shift;
      sh_left = left - min(seen, left);
    }
    __syncthreads();
    prefix = sh_prefix;
    left = sh_left;
  }
  // fewer entries than places: the key ends at the smallest there is, and all are taken
  if (t == 0) sh_n = 0;
  __shared__ uint32_t sh_count[kThreads / 64];
  uint32_t equal_before = 0;
  __syncthreads();
  for (int e0 = 0; e0 < V; e0 += kThreads) {
    const int e = e0 + t;
    const bool in = search && e < V;
    const float v = in ? logit(x, e) : -INFINITY;
    const uint32_t key = key_of(v + 0.f);
    const bool here = in && v > -INFINITY;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(here && key == prefix);
    if (search && (t & 63) == 0) sh_count[t >> 6] = __popcll(eq);
    __syncthreads();
    uint32_t at = equal_before + __popcll(eq & ((1ull << (t & 63)) - 1));
    for (int w = 0; w < kThreads / 64; ++w) at += w < (t >> 6) ? sh_count[w] : 0;
    if (here && (key > prefix || (key == prefix && at < left))) {
      const int k = atomicAdd(&sh_n, 1);
      if (k < kCand) best[k] = candidate(v, e);
    }
    for (int w = 0; w < kThreads / 64; ++w) equal_before += sh_count[w];
    __syncthreads();
  }
  write_ranked(best, min(sh_n, kCand), top, sh_m, temperature, sh_lse, ids, lps);
}

int chunks_of(int32_t vocab) { return (int)(((int64_t)vocab + kChunk - 1) / kChunk); }

}  // namespace

extern "C" size_t wisp_token_logprobs_workspace_size(int32_t rows, int32_t vocab, int32_t n_top) {
  if (rows < 0 || vocab < 1 || n_top < 0 || n_top > WISP_TOP_MAX) return 0;
  const size_t n = (size_t)rows * chunks_of(vocab);
  return 256 + align256(n * sizeof(Part)) + (n_top ? align256(n * kThreads * 4) : 0);
}

extern "C" wisp_status wisp_token_logprobs(const void *logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t ld,
                                           float temperature, const int32_t *tokens, int32_t n_top, float *logprob,
                                           float *entropy, int32_t *top_tokens, float *top_logprobs, void *workspace,
                                           size_t workspace_bytes, void *stream) {
  return guarded("wisp_token_logprobs", [&]() -> wisp_status {
    if (rows < 0 || vocab < 1 || ld < vocab) return fail(WISP_E_INVALID, "rows < 0, vocab < 1 or ld < vocab");
    if (!(temperature > 0.f) || isinf(temperature)) return fail(WISP_E_INVALID, "temperature must be finite and > 0");
    if (n_top < 0 || n_top > WISP_TOP_MAX) return fail(WISP_E_INVALID, "n_top = %d outside 0..%d", n_top, WISP_TOP_MAX);
    if (dtype != WISP_F32 && dtype != WISP_BF16) return fail(WISP_E_UNSUPPORTED, "dtype %d", dtype);
    if (logprob && !tokens) return fail(WISP_E_INVALID, "logprob without tokens");
    if (n_top > 0 && (!top_tokens || !top_logprobs)) return fail(WISP_E_INVALID, "NULL top_tokens / top_logprobs");
    if (vocab > 1 << 30) return fail(WISP_E_UNSUPPORTED, "vocab > 2^30");
    if (rows == 0) return WISP_OK;
    const int nch = chunks_of(vocab);
    if ((int64_t)rows * nch > INT32_MAX) return fail(WISP_E_UNSUPPORTED, "more than 2^31 - 1 chunks of 8192 logits in one call");
    if (!logits || !workspace) return fail(WISP_E_INVALID, "NULL logits / workspace");
    if ((uintptr_t)workspace & 15) return fail(WISP_E_INVALID, "workspace must be 16-byte aligned");
    if ((uintptr_t)logits & (dtype == WISP_F32 ? 3 : 1)) return fail(WISP_E_INVALID, "logits not aligned to their type");
    const size_t need = wisp_token_logprobs_workspace_size(rows, vocab, n_top);
    if (workspace_bytes < need) return fail(WISP_E_WORKSPACE, "workspace %zu bytes < %zu needed", workspace_bytes, need);
    char *ws = static_cast<char *>(workspace);
    Part *parts = reinterpret_cast<Part *>(ws + 256);
    float *gmax = n_top ? reinterpret_cast<float *>(ws + 256 + align256((size_t)rows * nch * sizeof(Part))) : nullptr;
    int *err = reinterpret_cast<int *>(ws);
    const hipStream_t s = (hipStream_t)stream;
    const float sc = scale_of(temperature);
    // a launch has less than 2^32 threads: this many rows each (at least 64)
    const int32_t step = kMaxChunks / nch;
    auto go = [&](auto *x, auto chunk, auto row) {
      for (int64_t r = 0; r < rows; r += step) {
        const uint32_t n = (uint32_t)std::min<int64_t>(step, rows - r);
        const int32_t *tok = tokens ? tokens + r : nullptr;
        Part *p = parts + r * nch;
        float *g = gmax ? gmax + r * nch * kThreads : nullptr;
        launch(chunk, n * nch, kThreads, 0, s, x + r * ld, (int)vocab, ld, nch, sc, tok, p, g);
        launch(row, n, n_top ? kThreads + 64 : 64, 0, s, x + r * ld, (int)vocab, ld, nch, temperature, tok, (const Part *)p,
               (const float *)g, (int)n_top, logprob ? logprob + r : nullptr, entropy ? entropy + r : nullptr,
               n_top ? top_tokens + r * n_top : nullptr, n_top ? top_logprobs + r * n_top : nullptr, err);
      }
    };
    // the row kernel that holds the chunks' group maxima (V <= 131072: 16, twice that: 32)
    auto rows_of = [&](auto *x, auto w) {
      using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
      constexpr int W = decltype(w)::value;
      return nch <= 16 ? logprobs_row_kernel<T, W, 16> : nch <= 32 ? logprobs_row_kernel<T, W, 32> : logprobs_row_kernel<T, W, 0>;
    };
    using One = std::integral_constant<int, 1>;
    const int es = dtype == WISP_F32 ? 4 : 2;
    const bool vec = ((uintptr_t)logits & 15) == 0 && (rows == 1 || ld * es % 16 == 0);   // every row starts on 16 bytes
    if (dtype == WISP_F32) {
      const float *x = static_cast<const float *>(logits);
      vec ? go(x, logprobs_chunk_kernel<float, true>, rows_of(x, std::integral_constant<int, 4>{}))
          : go(x, logprobs_chunk_kernel<float, false>, rows_of(x, One{}));
    } else {
      const uint16_t *x = static_cast<const uint16_t *>(logits);
      vec ? go(x, logprobs_chunk_kernel<uint16_t, true>, rows_of(x, std::integral_constant<int, 8>{}))
          : go(x, logprobs_chunk_kernel<uint16_t, false>, rows_of(x, One{}));
    }
    return hip_check("wisp_token_logprobs");
  });
}
