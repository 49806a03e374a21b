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

// 8 or 2 consecutive columns of a row; S = 0: stored as T, else S fp32 partials (a bound above 4)
template <typename T, int S, int N>
__device__ __forceinline__ void load_cols(const QkvRows &src, int64_t row, int col, float (&v)[N]) {
  if constexpr (S == 0 && std::is_same<T, uint16_t>::value) {
    const uint16_t *p = reinterpret_cast<const uint16_t *>(src.p) + row * src.ld + col;
    uint32_t w[N / 2];
    if constexpr (N == 8) {
      const uint4 x = ld16(p);
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
      w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  } else {
    constexpr int MAX = S == 0 ? 1 : S;
    const float *p = reinterpret_cast<const float *>(src.p) + row * src.ld + col;
#pragma unroll
    for (int z = 0; z < MAX; ++z) {
      const float *pz = p + (MAX <= 4 ? z : min(z, src.splits - 1)) * src.stride;
      float w[N];
      if constexpr (N == 8) {
        const float4 a = *reinterpret_cast<const float4 *>(pz), b = *reinterpret_cast<const float4 *>(pz + 4);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
      } else {
        const float2 a = *reinterpret_cast<const float2 *>(pz);
        w[0] = a.x; w[1] = a.y;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = z == 0 ? w[e] : MAX <= 4 || z < src.splits ? v[e] + w[e] : v[e];
    }
  }
}

__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack2bf_rne(v[0], v[1]), pack2bf_rne(v[2], v[3]), pack2bf_rne(v[4], v[5]), pack2bf_rne(v[6], v[7]));
}

// (x_i, x_{i + hd/2}) rotated by the angle of dim i; cs: (cos, sin) of 8 consecutive dims
__device__ __forceinline__ void rotate8(float (&lo)[8], float (&hi)[8], const float2 *__restrict__ cs) {
  float4 t[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) t[e] = reinterpret_cast<const float4 *>(cs)[e];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = e & 1 ? t[e / 2].z : t[e / 2].x, s = e & 1 ? t[e / 2].w : t[e / 2].y;
    const float a = lo[e], b = hi[e];
    lo[e] = a * c - b * s;
    hi[e] = b * c + a * s;
  }
}

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

// a value that the cache holds: at most 448 x 2^100 (infinities and NaN are not), so that the
// probabilities x scale stay finite
__device__ __forceinline__ bool holds(float v) { return fabsf(v) <= kE4m3Max * 1.2676506002282294e30f; }

constexpr uint32_t kNan4 = 0x7F7F7F7Fu;   // four e4m3 NaN

constexpr int kQHeads = 4;   // q heads of a thread

// Workgroups 0 .. n_units * nkv - 1: one page of one kv head, 2 * hd threads.  The first hd hold
// K, thread (slot, i) the dims 8i .. 8i + 7 and their rotation partners; the others V, thread
// (half, p) the dims 2p, 2p + 1 of 8 slots: each thread's values make whole 8-byte pieces of the
// page.  The other workgroups: Q, a thread 8 + 8 dims of kQHeads heads of one row.
template <typename T, int S>
__global__ __launch_bounds__(512) void kv8_append_kernel(const Kv8Unit *__restrict__ units, int n_units,
                                                         const int32_t *__restrict__ page_table, int pt_stride,
                                                         const float2 *__restrict__ cs, QkvRows src, T *__restrict__ q,
                                                         uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                                                         float2 *__restrict__ scales, int n_blocks, int rows, int nq,
                                                         int nkv, int hd, int *__restrict__ err) {
  const int tid = threadIdx.x, half = hd / 2;
  if ((int)blockIdx.x >= n_units * nkv) {
    const int per = half / 8, groups = (nq + kQHeads - 1) / kQHeads;   // threads of a head; of a row: per * groups
    const uint32_t t = (blockIdx.x - n_units * nkv) * blockDim.x + tid, per_row = per * groups;
    const int64_t row = t / per_row;
    if (row >= rows) return;
    const int u = t % per_row, i = (u % per) * 8, h0 = u / per;
    float lo[kQHeads][8], hi[kQHeads][8];
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
      const int h = min(h0 + k * groups, nq - 1);
      load_cols<T, S>(src, row, h * hd + i, lo[k]);
      load_cols<T, S>(src, row, h * hd + half + i, hi[k]);
    }
#pragma unroll
    for (int k = 0; k < kQHeads; ++k) {
      const int h = h0 + k * groups;
      if (h >= nq) break;
      rotate8(lo[k], hi[k], cs + row * half + i);
      T *o = q + (row * nq + h) * hd + i;
      store8(o, lo[k]);
      store8(o + half, hi[k]);
    }
    return;
  }
  __shared__ uint32_t sh_bad, sh_most[2];
  const int unit = blockIdx.x / nkv, kvh = blockIdx.x % nkv;
  const Kv8Unit un = units[unit];
  const int blk = page_table[(int64_t)un.req * pt_stride + un.page];
  if (blk < 0 || blk >= n_blocks) {
    if (tid == 0) flag_error(err, kErrBlock);
    return;
  }
  const int held = un.held_rows & 255, filled = held + (un.held_rows >> 8);
  const int64_t page = (int64_t)blk * nkv + kvh;
  const float2 old = scales[page];
  if (tid == 0) sh_bad = 0;
  if (tid < 2) sh_most[tid] = 0;
  __syncthreads();
  const bool is_k = tid < hd;
  // K: slot, dims i .. i + 7 (a) and half + i .. (b); V: dims i (a) and i + 1 (b) of slots slot .. slot + 7
  const int u = is_k ? tid : tid - hd;
  const int slot = is_k ? u / (half / 8) : u / half * 8, i = is_k ? u % (half / 8) * 8 : u % half * 2;
  uint8_t *pg = (is_k ? k_pool : v_pool) + page * (kPage * hd);
  const int at_a = is_k ? k8_page_off(slot, i) : v8_page_off(slot, i);
  const int at_b = is_k ? k8_page_off(slot, half + i) : v8_page_off(slot, i + 1);
  float a[8], b[8];
  uint2 ca{}, cb{};
  const int col = (nq + kvh + (is_k ? 0 : nkv)) * hd + i;
  // what is there: the old slots' values; for V also the codes past the last row, which stay
  if (is_k ? slot < held : slot < held || filled < slot + 8) {
    ca = *reinterpret_cast<const uint2 *>(pg + at_a);
    cb = *reinterpret_cast<const uint2 *>(pg + at_b);
  }
  decode8(ca, is_k ? old.x : old.y, a);
  decode8(cb, is_k ? old.x : old.y, b);
  uint32_t bad = 0;   // slots with a new value that the cache does not hold
  if (is_k) {
    if (slot >= held && slot < filled) {
      const int64_t row = un.row + slot - held;
      load_cols<T, S>(src, row, col, a);
      load_cols<T, S>(src, row, col + half, b);
      bool ok = true;
#pragma unroll
      for (int e = 0; e < 8; ++e) ok = ok && holds(a[e]) && holds(b[e]);
      rotate8(a, b, cs + row * half + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) ok = ok && holds(a[e]) && holds(b[e]);
      bad = ok ? 0u : 1u << slot;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (slot + e >= held && slot + e < filled) {
        float w[2];
        load_cols<T, S>(src, un.row + slot + e - held, col, w);
        a[e] = w[0];
        b[e] = w[1];
        if (!holds(w[0]) || !holds(w[1])) bad |= 1u << (slot + e);
      }
  }
  if (bad) atomicOr(&sh_bad, bad);
  __syncthreads();
  bad = sh_bad;
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int sl = is_k ? slot : slot + e;
    const bool counts = sl < filled && !(bad >> sl & 1);
    // an old NaN (kept from an earlier row) does not count either: fmaxf passes it over
    if (counts) most = fmaxf(most, fmaxf(fabsf(a[e]), fabsf(b[e])));
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
  const int64_t blocks = (int64_t)p.n_units * p.nkv + (p.rows * per_row + threads - 1) / threads;
  auto go = [&](auto kernel) {
    launch(kernel, (uint32_t)blocks, threads, 0, s, units, p.n_units, p.page_table, p.pt_stride, cs, src, q, c.k, c.v,
           reinterpret_cast<float2 *>(c.scale), c.n_blocks, p.rows, p.nq, p.nkv, p.hd, err);
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
