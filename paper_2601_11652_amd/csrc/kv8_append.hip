// Append to the 8-bit KV cache (Sec. 4.5's in-place KV update, on e4m3 pages): the rotary
// embedding of the new rows' Q and K, Q written for the attention, K and V quantised into their
// pages.
//
// A page's value is code x scale, one scale for its K and one for its V of a kv head.  A page
// that gets new rows gets the scale 2^k with the smallest k for which every valid value of the
// page, old or new, is at most 448 x 2^k: a power of two moves the codes of the slots that were
// there by whole exponents, so a page filled in many steps is not rounded again and again (a
// code loses bits only where it falls below e4m3's smallest normal).  New values are rounded
// once, from fp32 to e4m3, nearest even.
#include <type_traits>

#include "kernels.h"
#include "kv8.h"
#include "wave_reduce.h"

namespace wisp {

namespace {

// 8 or 2 consecutive columns of a row, read once; S = 0: stored as T, else S fp32 partials (a bound
// above 4).  bf16 words are kept as they come: widening them is the use that waits for the load.
template <typename T, int S>
struct Cols {
  static constexpr bool kWords = S == 0 && std::is_same<T, uint16_t>::value;
  static constexpr int kPer = kWords ? 2 : 1;   // values per word
  using Word = std::conditional_t<kWords, uint32_t, float>;

  template <int N>
  static __device__ __forceinline__ void load(const QkvRows &src, int64_t row, int col, Word *w) {
    if constexpr (kWords) {
      const uint16_t *p = reinterpret_cast<const uint16_t *>(src.p) + row * src.ld + col;
      if constexpr (N == 8) {
        const uint4 x = ld16_stream(p);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
      } else {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
      }
    } else {
      constexpr int MAX = S == 0 ? 1 : S;
      const float *p = reinterpret_cast<const float *>(src.p) + row * src.ld + col;
#pragma unroll
      for (int z = 0; z < MAX; ++z) {
        const float *pz = p + (MAX <= 4 ? z : min(z, src.splits - 1)) * src.stride;
        float x[N];
        if constexpr (N == 8) {
          const float4 a = *reinterpret_cast<const float4 *>(pz), b = *reinterpret_cast<const float4 *>(pz + 4);
          x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
          x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
          const float2 a = *reinterpret_cast<const float2 *>(pz);
          x[0] = a.x; x[1] = a.y;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = z == 0 ? x[e] : MAX <= 4 || z < src.splits ? w[e] + x[e] : w[e];
      }
    }
  }
  static __device__ __forceinline__ float value(const Word *w, int e) {
    if constexpr (kWords) return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    else return w[e];
  }
};

__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack2bf_rne(v[0], v[1]), pack2bf_rne(v[2], v[3]), pack2bf_rne(v[4], v[5]), pack2bf_rne(v[6], v[7]));
}

// (cos, sin) of 8 consecutive dims of a row
struct Angles {
  float4 t[4];
  __device__ __forceinline__ void load(const float2 *__restrict__ cs) {
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = reinterpret_cast<const float4 *>(cs)[e];
  }
  // (x_i, x_{i + hd/2}) rotated by the angle of dim i
  __device__ __forceinline__ void rotate8(float (&lo)[8], float (&hi)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float c = e & 1 ? t[e / 2].z : t[e / 2].x, s = e & 1 ? t[e / 2].w : t[e / 2].y;
      const float a = lo[e], b = hi[e];
      lo[e] = a * c - b * s;
      hi[e] = b * c + a * s;
    }
  }
};

typedef float float2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode8(uint2 w, float scale, float (&v)[8]) {
  const uint32_t x[2] = {w.x, w.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], true);
    v[4 * i] = a.x * scale;
    v[4 * i + 1] = a.y * scale;
    v[4 * i + 2] = b.x * scale;
    v[4 * i + 3] = b.y * scale;
  }
}
// nearest even; |v| * inv <= 448
__device__ __forceinline__ uint2 encode8(const float (&v)[8], float inv) {
  int x[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
    x[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, x[i], true);
  }
  return make_uint2(x[0], x[1]);
}

// exponent k of the scale for a largest magnitude `most`, 0 for a page of zeros.  448 = 1.75 x 2^8.
// At least -100 (smaller values round towards 0), so that the attention's probabilities x scale
// stay normal in bf16.
__device__ __forceinline__ int scale_exp(float most) {
  const uint32_t b = __float_as_uint(most);
  if (b == 0) return 0;
  const int k = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFF) > 0x600000);
  return max(-100, k);
}
__device__ __forceinline__ float exp2i(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// a magnitude that the cache holds: at most 448 x 2^100 (infinity and NaN are not), so that the
// probabilities x scale stay finite
__device__ __forceinline__ bool holds(float v) { return v <= kE4m3Max * 1.2676506002282294e30f; }
// largest magnitude of both; a NaN stays
__device__ __forceinline__ float most_of(float m, float a, float b) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, fabsf(a)), fabsf(b));
}

constexpr uint32_t kNan4 = 0x7F7F7F7Fu;   // four e4m3 NaN

constexpr int kQHeads = 2;   // q heads of a thread

// Two kinds of workgroups, interleaved over the grid in one even pattern.  A page's chain of loads
// (unit, page table, old codes) would leave the memory idle by itself: all pages first, 12538 rows of
// 32 + 2 x 8 heads of 128 take 58.5 us, interleaved 55.9 (283 MB, 5.1 TB/s: a copy's rate, so the
// memory bounds it; 32 requests of 2 to 9 rows 4.6 us, the chain's latency).
// One page of one kv head, 2 * hd threads: the first hd hold K, thread (slot, i) the dims 8i .. 8i + 7
// and their rotation partners; the others V, thread (half, p) the dims 2p, 2p + 1 of 8 slots: each
// thread's values make whole 8-byte pieces of the page.  Or Q, a thread 8 + 8 dims of kQHeads heads of
// one row (the same rows 54.6 us with 1 head, 59.6 with 4; 64 query heads 88.9 with 1, 92.7 with 2; but 3600
// rows 16.7 and 16.0, 256 requests 14.4 and 13.5).  Q is stored through the caches: past them this
// kernel took 47 us, but the attention that reads Q next 11 us more.
template <typename T, int S>
__global__ __launch_bounds__(512) void kv8_append_kernel(const Kv8Unit *__restrict__ units,
                                                         const int32_t *__restrict__ page_table, int pt_stride,
                                                         const float2 *__restrict__ cs, QkvRows src, T *__restrict__ q,
                                                         uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                                                         float2 *__restrict__ scales, int n_blocks, int rows, int nq,
                                                         int nkv, int hd, uint32_t q_share, int *__restrict__ err) {
  using C = Cols<T, S>;
  const int tid = threadIdx.x, half = hd / 2;
  // workgroup b is Q's next one where floor(b q_share / 2^32) steps up
  const uint32_t q_at = __umulhi(blockIdx.x, q_share);
  if (__umulhi(blockIdx.x + 1, q_share) > q_at) {
    const int per = half / 8, groups = (nq + kQHeads - 1) / kQHeads;   // threads of a head; of a row: per * groups
    const uint32_t t = q_at * blockDim.x + tid, per_row = per * groups;
    const int64_t row = t / per_row;
    if (row >= rows) return;
    const int u = t % per_row, i = (u % per) * 8, h0 = u / per;
    typename C::Word w[kQHeads][16 / C::kPer];
    Angles turn;
    turn.load(cs + row * half + i);
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
      const int h = min(h0 + k * groups, nq - 1);
      C::template load<8>(src, row, h * hd + i, w[k]);
      C::template load<8>(src, row, h * hd + half + i, w[k] + 8 / C::kPer);
    }
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
      const int h = h0 + k * groups;
      if (h >= nq) break;
      float lo[8], hi[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = C::value(w[k], e);
        hi[e] = C::value(w[k], 8 + e);
      }
      turn.rotate8(lo, hi);
      T *o = q + (row * nq + h) * hd + i;
      store8(o, lo);
      store8(o + half, hi);
    }
    return;
  }
  __shared__ uint32_t sh_bad[8], sh_most[2];   // 512 threads
  const int page_block = blockIdx.x - q_at, unit = (uint32_t)page_block / nkv, kvh = (uint32_t)page_block % nkv;
  const Kv8Unit un = units[unit];
  const int blk = page_table[(int64_t)un.req * pt_stride + un.page];
  const int held = un.held_rows & 255, filled = held + (un.held_rows >> 8);
  if (tid < 2) sh_most[tid] = 0;
  const bool is_k = tid < hd;
  // K: slot, dims i .. i + 7 (a) and half + i .. (b); V: dims i (a) and i + 1 (b) of slots slot .. slot + 7
  const uint32_t u = is_k ? tid : tid - hd, per = is_k ? half / 8 : half, at = u / per;
  const int slot = is_k ? at : at * 8, i = (u - at * per) * (is_k ? 8 : 2);
  const int col = (nq + kvh + (is_k ? 0 : nkv)) * hd + i;
  // The new rows, asked for before the page's place in the pool is known.  Slots without a new row
  // take the nearest one's: no branch stands between these loads, and none waits for another.
  typename C::Word raw[16 / C::kPer];
  Angles turn;
  auto row_of = [&](int sl) { return (int64_t)un.row + min(max(sl - held, 0), filled - held - 1); };
  if (is_k) {
    turn.load(cs + row_of(slot) * half + i);
    C::template load<8>(src, row_of(slot), col, raw);
    C::template load<8>(src, row_of(slot), col + half, raw + 8 / C::kPer);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) C::template load<2>(src, row_of(slot + e), col, raw + 2 * e / C::kPer);
  }
  if (blk < 0 || blk >= n_blocks) {
    if (tid == 0) flag_error(err, kErrBlock);
    return;
  }
  const int64_t page = (int64_t)blk * nkv + kvh;
  uint8_t *pg = (is_k ? k_pool : v_pool) + page * (kPage * hd);
  const int at_a = is_k ? k8_page_off(slot, i) : v8_page_off(slot, i);
  const int at_b = is_k ? k8_page_off(slot, half + i) : v8_page_off(slot, i + 1);
  uint2 ca{}, cb{};
  float old = 1.f;
  // what is there: the old slots' values; for V also the codes past the last row, which stay
  if (is_k ? slot < held : slot < held || filled < slot + 8) {
    ca = *reinterpret_cast<const uint2 *>(pg + at_a);
    cb = *reinterpret_cast<const uint2 *>(pg + at_b);
    const float2 sc = scales[page];
    old = is_k ? sc.x : sc.y;
  }
  float a[8], b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float k0 = C::value(raw, e), k1 = C::value(raw, 8 + e);
    const float v0 = C::value(raw, 2 * e), v1 = C::value(raw, 2 * e + 1);
    a[e] = is_k ? k0 : v0;
    b[e] = is_k ? k1 : v1;
  }
  if (slot < held) {
    float oa[8], ob[8];
    decode8(ca, old, oa);
    decode8(cb, old, ob);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((is_k ? slot : slot + e) < held) {
        a[e] = oa[e];
        b[e] = ob[e];
      }
  }
  uint32_t bad = 0;   // slots with a new value that the cache does not hold
  if (is_k) {
    if (slot >= held) {
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = most_of(m, a[e], b[e]);
      turn.rotate8(a, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) m = most_of(m, a[e], b[e]);
      bad = holds(m) || slot >= filled ? 0u : 1u << slot;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      bad |= holds(most_of(0.f, a[e], b[e])) || slot + e < held || slot + e >= filled ? 0u : 1u << (slot + e);
  }
  uint32_t wave_bad = 0;
  for (uint64_t m = __ballot(bad != 0); m != 0; m &= m - 1) wave_bad |= __builtin_amdgcn_readlane(bad, __builtin_ctzll(m));
  if ((tid & 63) == 0) sh_bad[tid >> 6] = wave_bad;
  __syncthreads();   // also sh_most, and everyone has read the old scales
  bad = 0;
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) bad |= sh_bad[w];
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int sl = is_k ? slot : slot + e;
    // an old NaN (kept from an earlier row) does not count: fmaxf passes it over
    const float m = fmaxf(fabsf(a[e]), fabsf(b[e]));
    most = fmaxf(most, sl < filled && !(bad >> sl & 1) ? m : 0.f);
  }
  most = half_wave_max(most);   // hd is a multiple of 32: a half wave holds K or V only
  if ((tid & 31) == 0) atomicMax(&sh_most[is_k ? 0 : 1], __float_as_uint(most));
  __syncthreads();
  const int kk = scale_exp(__uint_as_float(sh_most[0])), kv = scale_exp(__uint_as_float(sh_most[1]));
  const float inv = exp2i(-(is_k ? kk : kv));
  if (tid == 0) scales[page] = make_float2(exp2i(kk), exp2i(kv));
  if (is_k) {
    if (slot >= filled) return;
    uint2 na = encode8(a, inv), nb = encode8(b, inv);
    if (bad >> slot & 1) na = nb = make_uint2(kNan4, kNan4);
    *reinterpret_cast<uint2 *>(pg + at_a) = na;
    *reinterpret_cast<uint2 *>(pg + at_b) = nb;
  } else {
    if (slot >= filled) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (bad >> (slot + e) & 1) a[e] = b[e] = 0.f;
    uint2 na = encode8(a, inv), nb = encode8(b, inv);
    const int n = min(8, filled - slot);             // slots past the last row keep their codes
    const uint64_t keep = n == 8 ? 0ull : ~0ull << (8 * n);
    auto mix = [&](uint2 x, uint2 o) {
      const uint64_t w = ((uint64_t)x.y << 32 | x.x), z = ((uint64_t)o.y << 32 | o.x);
      const uint64_t r = (w & ~keep) | (z & keep);
      return make_uint2((uint32_t)r, (uint32_t)(r >> 32));
    };
    *reinterpret_cast<uint2 *>(pg + at_a) = mix(na, ca);
    *reinterpret_cast<uint2 *>(pg + at_b) = mix(nb, cb);
  }
}

template <typename T>
void append(const Kv8Plan &p, const Kv8Cache &c, const QkvRows &src, T *q, int *err, hipStream_t s) {
  const Kv8Unit *units = reinterpret_cast<const Kv8Unit *>(p.ws + p.w_units);
  const float2 *cs = reinterpret_cast<const float2 *>(p.ws + p.w_cs);
  const int threads = 2 * p.hd;
  const int64_t per_row = (int64_t)p.hd / 16 * ((p.nq + kQHeads - 1) / kQHeads);
  const int64_t q_blocks = (p.rows * per_row + threads - 1) / threads, blocks = (int64_t)p.n_units * p.nkv + q_blocks;
  // rounded up: with blocks < 2^31 (wisp_kv8_plan) the error stays below one step, and the last step is whole
  const uint32_t q_share = (uint32_t)((((uint64_t)q_blocks << 32) + blocks - 1) / blocks);
  auto go = [&](auto kernel) {
    launch(kernel, (uint32_t)blocks, threads, 0, s, units, p.page_table, p.pt_stride, cs, src, q, c.k, c.v,
           reinterpret_cast<float2 *>(c.scale), c.n_blocks, p.rows, p.nq, p.nkv, p.hd, q_share, err);
  };
  if (src.splits == 0) go(kv8_append_kernel<T, 0>);
  else if (src.splits == 1) go(kv8_append_kernel<T, 1>);
  else if (src.splits == 2) go(kv8_append_kernel<T, 2>);
  else if (src.splits <= 4) src.splits == 3 ? go(kv8_append_kernel<T, 3>) : go(kv8_append_kernel<T, 4>);
  else src.splits <= 8 ? go(kv8_append_kernel<T, 8>) : go(kv8_append_kernel<T, 16>);
}

}  // namespace

void kv8_append(const Kv8Plan &p, const Kv8Cache &c, const QkvRows &src, void *q, int *err, hipStream_t s) {
  if (p.rows == 0) return;
  if (p.dtype == 1) append(p, c, src, static_cast<uint16_t *>(q), err, s);
  else append(p, c, src, static_cast<float *>(q), err, s);
}

}  // namespace wisp
