// Ragged multi-query causal attention over the 8-bit paged KV cache: the attention of Sec. 4.5's
// batched one-step verification on e4m3 pages with one K and one V scale per page and kv head.
//
// A workgroup of four waves runs a share of one kv head's work, items one after another: an item is
// up to four row groups (16 RB of a request's rows x query heads each) over a range of the request's
// tokens.  One row group's tokens are split over the four waves, two row groups have two waves
// each, three or four one each: waves that share tokens read the same lines at the same time, and
// bundles of three and four that run apart (wide_items) also convert their codes together.  Per
// page pair (32 tokens) a wave computes S^T = K Q^T and O^T += V^T P^T with 16x16x32 matrix products in
// bf16, which holds every e4m3 value exactly: the codes are converted between load and product,
// the K scale multiplies the scores and the V scale the probabilities (a lane's eight tokens of
// a pair lie in one page, so each is one factor per lane).  Every query row stays in one lane column
// (lane % 16), so the online softmax needs two cross-row steps, and the probabilities leave the
// first product in the order that the second consumes.  The waves of a row group are joined
// through LDS, the parts of a context that several items share by a second kernel.
//
// Bound by the memory for long contexts (128 requests of 0.25-32k tokens, 32 + 8 heads of 128: 1.73 GB in
// 328 us, 5.3 TB/s), by vector instructions for prompts (4096 rows: 172 us in a row of calls, 0.81 PFLOP/s,
// 192 by itself: two instructions of softmax, half a conversion and two of addresses, scales and
// rescaling for each product), by latency for few requests (one of 1300 tokens: 8 us and 3 for the join).
//
// A bf16 model's probabilities are rounded to bf16 (2^-8 of each at most) for the second product, as those
// over a bf16 cache are: in one part that product takes half a prompt's matrix instructions, in two
// two thirds.  The sum that divides adds the same rounded values.  Against 64 bits the results are off by
// 1.7e-3 to 1.9e-3 of their size, of which the output's own rounding makes 1.7e-3.
//
// An fp32 model's queries and probabilities enter the products as three bf16 parts each (8 bits
// of the significand per part: 24 in all), so its results are fp32's.
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "kv8.h"

namespace wisp {

namespace {

// Eight codes x 2^EXP in bf16 (exact)
template <int EXP = 0>
__device__ __forceinline__ bf16x8_t to_bf16(uint32_t lo, uint32_t hi) {
  constexpr float scale = EXP >= 0 ? 1 << EXP : 1.f / (1 << -EXP);
  union {
    bf16x2_t h[4];
    bf16x8_t v;
  } u;
  u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}
// V's codes enter the second product x 2^-12, and the results leave it x 2^12: a probability of up to 2^8
// (the reference lags behind the maximum) x a scale of 2^100 x 448 overflowed fp32 after 2^11
// tokens; so 2^23 may follow, and at scales of 2^-100 a sum still has 24 bits above fp32's least.
constexpr int kVDown = -12;
constexpr float kVUp = 4096.f;
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// a barrier that orders LDS only: the loads ahead and the results' stores stay in flight
// (__syncthreads waits for them too: 4 us at the end of every item)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// x, its value unknown to the compiler: what is computed from it at the end of an item stays there
// (hoisted out of the loop over items, such offsets filled the registers that the codes ahead need)
__device__ __forceinline__ int opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The larger of two scores, as their median with the largest float: fmaxf quiets its operands
// first, an instruction for each.  A NaN is passed over; of two, what comes out does not matter, as
// their row's result is NaN.
__device__ __forceinline__ float max2(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, 3.402823466e38f); }

// block ids, read through the scalar cache: nothing writes them while a kernel runs
typedef const int32_t __attribute__((address_space(4))) ids_t;

__device__ __forceinline__ uint4 as_uint4(bf16x8_t v) { return __builtin_bit_cast(uint4, v); }

struct Kv8Args {
  const Kv8Item *items;
  const int32_t *wide_first;   // as first, of the workgroups before wide_blocks, which run wide items
  int wide_blocks;
  const int32_t *first;   // share s runs items first[s] .. first[s + 1] - 1
  const int32_t *page_table;
  const uint8_t *k, *v;
  const float2 *scale;
  const void *q;
  void *out;
  float *part_o, *part_ml;
  int *err;
  int pt_stride, n_blocks, nq, nkv, out_K;
  float c_log2;   // log2(e) / sqrt(head_dim)
  bool packed;
};

// Magnitude of a score in base 2 up to which its maximum's rounding moves a probability by less than bf16's
constexpr float kFarScore = 65536.f;

// The online softmax of a quad: its scores s (without K's scale; [row block][pair][half of its pages'
// slots]) to probabilities x V's scale, in the order that the second product consumes.  Scales of the
// lane's pages: ks K's in base 2, lv log2 of V's, vi its inverse.
template <int RB, int MB, int NP>
__device__ __forceinline__ void softmax(floatx4 (&s)[RB][2][2], const float (&ks)[2], const float (&lv)[2],
                                        const float (&vi)[2], float (&m_run)[RB], float (&l_run)[RB], floatx4 (&o)[RB][MB],
                                        uint4 (&pb)[NP][RB][2]) {
  constexpr bool F32 = NP > 1;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float mx[2];                       // scores in base 2
#pragma unroll
    for (int h = 0; h < 2; ++h)
      mx[h] = ks[h] * max2(max2(max2(s[rb][h][0][0], s[rb][h][0][1]), max2(s[rb][h][0][2], s[rb][h][0][3])),
                           max2(max2(s[rb][h][1][0], s[rb][h][1][1]), max2(s[rb][h][1][2], s[rb][h][1][3])));
    const float top = xor32_max(xor16_max(fmaxf(mx[0], mx[1])));
    // the running maximum rises only by more than 8: p stays below 2^8, and the accumulators
    // are rescaled on few quads; numerator and denominator share the reference
    const bool grow = top > m_run[rb] + 8.0f;
    if (__builtin_amdgcn_ballot_w64(grow)) {
      const float alpha = grow ? __builtin_amdgcn_exp2f(m_run[rb] - top) : 1.0f;
      m_run[rb] = grow ? top : m_run[rb];
      l_run[rb] *= alpha;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[rb][mb] *= alpha;
    }
    float m = m_run[rb] == -INFINITY ? 0.f : m_run[rb], k[2] = {ks[0], ks[1]};
    // m is a rounded product, s ks below an exact one: of large scores their difference would be mostly
    // m's rounding (from 2^31 on, infinite probabilities)
    if (__builtin_amdgcn_ballot_w64(fabsf(m) > kFarScore)) {
#pragma clang fp contract(off)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[rb][h][x][e] = s[rb][h][x][e] * ks[h] - m;
        k[h] = 1.f;
      }
      m = 0.f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // p x V's scale = 2^(s ks - m + log2 vs)
      const float off = lv[h] - m;
      float rs = 0.f;
      uint32_t pw[NP][4];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float f = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][h][x][e], k[h], off));
          float g = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][h][x][e + 1], k[h], off));
          if constexpr (F32) rs += f + g;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const uint32_t w = pack2bf_rne(f, g);
            pw[p][x * 2 + e / 2] = w;
            f -= low(w);
            g -= high(w);
          }
          // bf16: the sum adds the rounded values, as the second product does
          if constexpr (!F32) {
            const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
            rs = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[0][x * 2 + e / 2]), one, rs, false);
          }
        }
      l_run[rb] = __builtin_fmaf(rs, vi[h], l_run[rb]);   // this lane's tokens; the lanes are added up at the end
#pragma unroll
      for (int p = 0; p < NP; ++p) pb[p][rb][h] = make_uint4(pw[p][0], pw[p][1], pw[p][2], pw[p][3]);
    }
  }
}

// The same for bundles of three or four row groups (a prompt's, whose rows are many and whose codes are
// few), of which each wave takes one: by themselves they would all convert the same codes, 128 instructions
// beside 64 matrix products a quad.  Here each converts a quarter of a quad for all, through LDS, a
// quad ahead, and codes are asked for two quads ahead; the queries are in registers.  Bound by vector
// instructions as before, with 96 fewer a quad: a prompt of 4096 rows takes 185 us without and 172
// with it, one of 100 rows beside three requests 14.8 and 11.9.
template <int HD>
__device__ __forceinline__ void wide_items(const Kv8Args &a, uint4 *smem, float2 (*sh_ml)[32]) {
  constexpr int RB = 2, ROWS = 16 * RB, KC = HD / 32, MB = HD / 16, LDJ = HD + 4;
  constexpr int kBuf = 2 * KC * 2 * 64;                // 16-byte operands of a quad's K, or V
  constexpr int NV = KC / 2;                           // 16-byte loads of a wave, of each
  uint4(*kv)[2][kBuf] = reinterpret_cast<uint4(*)[2][kBuf]>(smem);   // [buffer][K, V]: pair, chunk, half, lane
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 15, lg = lane >> 4;
  const int block = blockIdx.x, kvh = block % a.nkv, G = a.nq / a.nkv;
  const int k_off = lg * 128 + (lc & 7) * 16, v_off = (lg & 1) * 256 + lc * 16;
  const int k_end = a.wide_first[block / a.nkv + 1];
  for (int k = a.wide_first[block / a.nkv]; k < k_end; ++k) {
    const Kv8Item it = a.items[k];
    const int groups = kv8_groups(it.groups), quads = (it.t1 - it.t0 + 63) / 64, rows = it.nrow * G;
    const int lr0 = (kv8_first(it.groups) + min(wave, groups - 1)) * ROWS;
    const int open = min(it.t1, it.ctx + __builtin_amdgcn_readfirstlane(lr0 / G) + 1);   // seen by every row before it
    // (of three groups' waves the fourth computes the third once more, and writes nothing)
    // the pages of quad i; past the end the last page
    const ids_t *ids = reinterpret_cast<const ids_t *>(reinterpret_cast<uintptr_t>(a.page_table + (int64_t)it.req * a.pt_stride));
    struct Pages {
      int b[4];
    };
    auto pages_of = [&](int i) __attribute__((always_inline)) {
      Pages p;
#pragma unroll
      for (int x = 0; x < 4; ++x) p.b[x] = ids[min((it.t0 >> 4) + 4 * i + x, (it.t1 - 1) >> 4)];
      return p;
    };
    auto place = [&](int b) __attribute__((always_inline)) {
      return (int64_t)min(max(b, 0), a.n_blocks - 1) * a.nkv + kvh;
    };
    uint4 kr[NV], vr[NV];
    float2 sc[2];
    auto load_codes = [&](const Pages &p) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < NV; ++x) {
        const int h = (wave * NV + x) / KC, c = (wave * NV + x) % KC;
        const int64_t p0 = place(h ? p.b[2] : p.b[0]), p1 = place(h ? p.b[3] : p.b[1]);
        kr[x] = ld16(a.k + (lc >= 8 ? p1 : p0) * (kPage * HD) + k_off + c * 512);
        vr[x] = ld16(a.v + (lg >= 2 ? p1 : p0) * (kPage * HD) + v_off + c * 512);
      }
    };
    auto load_scales = [&](const Pages &p) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) sc[h] = a.scale[lg >= 2 ? place(p.b[2 * h + 1]) : place(p.b[2 * h])];
    };
    auto store_codes = [&](int i) __attribute__((always_inline)) {
      const int tp = it.t0 + 64 * i;
#pragma unroll
      for (int x = 0; x < NV; ++x) {
        const int h = (wave * NV + x) / KC, c = (wave * NV + x) % KC, at = (h * KC + c) * 128 + lane;
        // slots past the range may hold anything: zero probability is not enough against a NaN
        if (tp + 64 > it.t1) {
          const int in = min(max(it.t1 - (tp + 32 * h + 8 * lg), 0), 8);
          const uint32_t mlo = in >= 4 ? ~0u : (1u << (8 * in)) - 1u, mhi = in <= 4 ? 0u : in == 8 ? ~0u : (1u << (8 * (in - 4))) - 1u;
          vr[x].x &= mlo;
          vr[x].y &= mhi;
          vr[x].z &= mlo;
          vr[x].w &= mhi;
        }
        kv[i & 1][0][at] = as_uint4(to_bf16(kr[x].x, kr[x].y));
        kv[i & 1][0][at + 64] = as_uint4(to_bf16(kr[x].z, kr[x].w));
        kv[i & 1][1][at] = as_uint4(to_bf16<kVDown>(vr[x].x, vr[x].y));
        kv[i & 1][1][at + 64] = as_uint4(to_bf16<kVDown>(vr[x].z, vr[x].w));
      }
    };

    Pages p = pages_of(0);
    load_codes(p);
    load_scales(p);
    uint4 qf[RB][KC];
    int jrow[RB];
    float m_run[RB], l_run[RB];
    floatx4 o[RB][MB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int lr = min(lr0 + rb * 16 + lc, rows - 1);   // padding rows: a real one
      const uint16_t *from = reinterpret_cast<const uint16_t *>(a.q) + ((int64_t)(it.row0 + lr / G) * a.nq + kvh * G + lr % G) * HD + 8 * lg;
#pragma unroll
      for (int c = 0; c < KC; ++c) qf[rb][c] = ld16(from + 32 * c);
      jrow[rb] = lr / G;
      m_run[rb] = -INFINITY;
      l_run[rb] = 0.f;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[rb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    // block ids out of range are reported (and clamped above)
    for (int x = threadIdx.x; x <= ((it.t1 - 1) >> 4) - (it.t0 >> 4); x += 256) {
      const int b = a.page_table[(int64_t)it.req * a.pt_stride + (it.t0 >> 4) + x];
      if (b < 0 || b >= a.n_blocks) flag_error(a.err, kErrBlock);
    }
    p = pages_of(1);
    store_codes(0);
    load_codes(p);
    Pages next = pages_of(2);
    lds_barrier();
    for (int i = 0; i < quads; ++i) {
      const int tp = it.t0 + 64 * i;
      float ks[2], lv[2], vi[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        ks[h] = sc[h].x * a.c_log2;
        lv[h] = __builtin_amdgcn_logf(sc[h].y);
        vi[h] = __builtin_amdgcn_exp2f(-lv[h]);
      }
      floatx4 s[RB][2][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int h = 0; h < 2; ++h) s[rb][h][0] = s[rb][h][1] = floatx4{0.f, 0.f, 0.f, 0.f};
      // operands are read from LDS while the products before them run
      uint4 f[2][4];
      auto read4 = [&](int what, int h, int c, int to) __attribute__((always_inline)) {
        f[to][h * 2] = kv[i & 1][what][(h * KC + c) * 128 + lane];
        f[to][h * 2 + 1] = kv[i & 1][what][(h * KC + c) * 128 + 64 + lane];
      };
      read4(0, 0, 0, 0);
      read4(0, 1, 0, 0);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c + 1 < KC) {
          read4(0, 0, c + 1, (c + 1) & 1);
          read4(0, 1, c + 1, (c + 1) & 1);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              s[rb][h][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f[c & 1][h * 2 + x]), as_bf16x8(qf[rb][c]), s[rb][h][x], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      store_codes(i + 1);
      load_scales(p);
      load_codes(next);
      p = next;
      next = pages_of(i + 3);
      __builtin_amdgcn_sched_barrier(0);
      if (tp + 64 > open) {
        const int t = opaque(tp + 8 * lg);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const int lim = min(it.t1, it.ctx + jrow[rb] + 1) - t;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (32 * h + 4 * x + e >= lim) s[rb][h][x][e] = -INFINITY;
        }
      }
      uint4 pb[1][RB][2];
      softmax(s, ks, lv, vi, m_run, l_run, o, pb);
      __builtin_amdgcn_sched_barrier(0);
      read4(1, 0, 0, 0);
      read4(1, 1, 0, 0);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c + 1 < KC) {
          read4(1, 0, c + 1, (c + 1) & 1);
          read4(1, 1, c + 1, (c + 1) & 1);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              o[rb][2 * c + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f[c & 1][h * 2 + x]), as_bf16x8(pb[0][rb][h]), o[rb][2 * c + x], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
    }
    // through LDS: 8 dims of a row per thread
    {
      const int lane = opaque(threadIdx.x) & 63, lc = lane & 15, lg = lane >> 4;
      float(*jo)[LDJ] = reinterpret_cast<float(*)[LDJ]>(smem) + wave * ROWS;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float l = xor32_sum(xor16_sum(l_run[rb]));
        if (lg == 0) sh_ml[wave][rb * 16 + lc] = make_float2(m_run[rb], l);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) *reinterpret_cast<floatx4 *>(&jo[rb * 16 + lc][mb * 16 + 4 * lg]) = o[rb][mb];
      }
      lds_barrier();
      const int end = wave < groups ? min(ROWS, rows - lr0) * (HD / 8) : 0;
#pragma unroll 1
      for (int u = lane; u < end; u += 64) {
        const int r = u / (HD / 8), c0 = u % (HD / 8) * 8;
        floatx4 y = *reinterpret_cast<const floatx4 *>(&jo[r][c0]), z = *reinterpret_cast<const floatx4 *>(&jo[r][c0 + 4]);
        const float2 ml = sh_ml[wave][r];
        if (it.part >= 0) {
          const int64_t slot = ((int64_t)(it.part + wave) * a.nkv + kvh) * ROWS + r;
          float *to = a.part_o + slot * HD + c0;
          __builtin_nontemporal_store(y, reinterpret_cast<floatx4 *>(to));
          __builtin_nontemporal_store(z, reinterpret_cast<floatx4 *>(to + 4));
          if (c0 == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = ml;
          continue;
        }
        const int64_t row = it.row0 + (lr0 + r) / G, col = (int64_t)(kvh * G + (lr0 + r) % G) * HD + c0;
        const float inv = kVUp / ml.y;
        y *= inv;
        z *= inv;
        uint16_t *to = reinterpret_cast<uint16_t *>(a.out) + (a.packed ? packed_off(row, col, a.out_K) : row * a.out_K + col);
        *reinterpret_cast<uint4 *>(to) = make_uint4(pack2bf_rne(y[0], y[1]), pack2bf_rne(y[2], y[3]), pack2bf_rne(z[0], z[1]), pack2bf_rne(z[2], z[3]));
      }
    }
    lds_barrier();                                     // before the next item's codes
  }
}

template <int HD, int RB, bool F32, bool STREAM = false, bool WIDE = false>
__global__ __launch_bounds__(256, HD <= 128 ? 2 : 1) void kv8_attn_kernel(Kv8Args a) {
  constexpr int ROWS = 16 * RB;         // of a row group
  constexpr int KC = HD / 32;           // 32-wide chunks of the contraction; 16-byte loads of K and of V
  constexpr int MB = HD / 16;           // 16-wide blocks of the output dims
  constexpr int NP = F32 ? 3 : 1;       // bf16 parts of a query and of a probability
  constexpr int LDJ = HD + 4;           // a row of a wave's accumulators in LDS, in floats: 16 bytes apart in banks
  constexpr int kQueries = 4 * NP * RB * KC * 64, kJoin = 4 * ROWS * LDJ / 4;   // 16-byte units
  // the row groups' queries in operand order while an item runs, the accumulators when it ends
  constexpr int kWide = WIDE ? 4 * 2 * KC * 2 * 64 : 0;   // wide_items' two buffers
  __shared__ uint4 smem[std::max(kWide, std::max(kQueries, kJoin))];
  __shared__ float2 sh_ml[4][ROWS];
  uint4(*qs)[NP][RB][KC][64] = reinterpret_cast<uint4(*)[NP][RB][KC][64]>(smem);
  float(*jo)[ROWS][LDJ] = reinterpret_cast<float(*)[ROWS][LDJ]>(smem);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 15, lg = lane >> 4;
  if constexpr (WIDE) {
    if ((int)blockIdx.x < a.wide_blocks) return wide_items<HD>(a, smem, sh_ml);
  }
  const int block = WIDE ? blockIdx.x - a.wide_blocks : blockIdx.x;
  const int kvh = block % a.nkv;        // neighbouring workgroups, on other XCDs: other kv heads
  const int G = a.nq / a.nkv;
  int k = a.first[block / a.nkv];
  const int k_end = a.first[block / a.nkv + 1];
  if (k >= k_end) return;

  // What a wave does of an item: row group rg, tokens tok .. end - 1 in n page quads (64 tokens)
  struct Share {
    int rg, part, parts, tok, end, n;
  };
  auto share_of = [&](const Kv8Item &it) __attribute__((always_inline)) {
    Share s;
    const int groups = kv8_groups(it.groups), quads = (it.t1 - it.t0 + 63) / 64;
    s.parts = groups == 1 ? 4 : groups == 2 ? 2 : 1;
    s.rg = wave % groups;
    s.part = wave / groups;              // of three groups' waves the fourth is idle: part 1 of 1
    const int p = min(s.part, s.parts), from = quads * p / s.parts;
    const int n = p < s.parts ? quads * (p + 1) / s.parts - from : 0;
    s.tok = it.t0 + 64 * from;
    s.end = min(it.t1, s.tok + 64 * n);
    s.n = max(1, n);                     // with nothing to do one quad, all of it masked
    return s;
  };
  auto item_at = [&](int i) __attribute__((always_inline)) { return a.items[min(i, k_end - 1)]; };
  // block ids of up to 64 pages from token tok on, one per lane
  auto ids_at = [&](const Kv8Item &it, int tok) __attribute__((always_inline)) {
    return a.page_table[(int64_t)it.req * a.pt_stride + min((tok >> 4) + lane, (it.t1 - 1) >> 4)];
  };
  auto clamped = [&](int b) { return min(max(b, 0), a.n_blocks - 1); };

  // the queries of an item, by all threads: asked for, then stored in operand order (when nobody
  // reads what is there any more)
  constexpr int QN = RB * KC;            // 16-byte operands of a thread for four row groups
  struct Queries {
    uint4 w[QN][F32 ? 2 : 1];
  };
  auto load_queries = [&](const Kv8Item &it, Queries &q) __attribute__((always_inline)) {
    const int rows = it.nrow * G, count = kv8_groups(it.groups) * RB * KC * 64, tid = opaque(threadIdx.x);
#pragma unroll
    for (int x = 0; x < QN; ++x) {
      const int u = x * 256 + tid;
      q.w[x][0] = q.w[x][F32 ? 1 : 0] = make_uint4(0, 0, 0, 0);
      if (u < count) {
        const int l = u & 63, kc = (u >> 6) % KC, r16 = (u >> 6) / KC;   // 16-row block of the item
        const int lr = min(kv8_first(it.groups) * ROWS + r16 * 16 + (l & 15), rows - 1);   // padding rows: a real one
        const int64_t at = ((int64_t)(it.row0 + lr / G) * a.nq + kvh * G + lr % G) * HD + kc * 32 + 8 * (l >> 4);
        if constexpr (F32) {
          q.w[x][0] = ld16(reinterpret_cast<const float *>(a.q) + at);
          q.w[x][1] = ld16(reinterpret_cast<const float *>(a.q) + at + 4);
        } else {
          q.w[x][0] = ld16(reinterpret_cast<const uint16_t *>(a.q) + at);
        }
      }
    }
  };
  auto store_queries = [&](const Kv8Item &it, const Queries &q) __attribute__((always_inline)) {
    const int count = kv8_groups(it.groups) * RB * KC * 64, tid = opaque(threadIdx.x);
#pragma unroll
    for (int x = 0; x < QN; ++x) {
      const int u = x * 256 + tid;
      if (u < count) {
        const int l = u & 63, kc = (u >> 6) % KC, r16 = (u >> 6) / KC;
        if constexpr (F32) {
          const uint32_t in[8] = {q.w[x][0].x, q.w[x][0].y, q.w[x][0].z, q.w[x][0].w,
                                  q.w[x][1].x, q.w[x][1].y, q.w[x][1].z, q.w[x][1].w};
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(in[e]);
#pragma unroll
          for (int p = 0; p < 3; ++p) {
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              h[e] = pack2bf_rne(f[2 * e], f[2 * e + 1]);
              f[2 * e] -= low(h[e]);
              f[2 * e + 1] -= high(h[e]);
            }
            qs[r16 / RB][p % NP][r16 % RB][kc][l] = make_uint4(h[0], h[1], h[2], h[3]);
          }
        } else {
          qs[r16 / RB][0][r16 % RB][kc][l] = q.w[x][0];
        }
      }
    }
  };

  // A segment: up to 16 quads of the wave's share, whose block ids sit in the lanes (lane l its l-th
  // page).  The next segment's, of this item or the next, are asked for while it runs.
  Kv8Item it = item_at(k), nx = item_at(k + 1);
  Share sh = share_of(it);
  int tok = sh.tok, n = min(sh.n, 16), left = sh.n - n;   // first token and quads of the segment; quads after it
  int blk = ids_at(it, tok), nblk = 0;   // nblk: once they are here
  auto check = [&](int b) __attribute__((always_inline)) {
    if (b < 0 || b >= a.n_blocks) flag_error(a.err, kErrBlock);
  };
  {
    Queries q;
    load_queries(it, q);
    check(blk);
    store_queries(it, q);
  }
  lds_barrier();

  float m_run[RB], l_run[RB];
  floatx4 o[RB][MB];
  int jrow[RB];
  int open = 0;                          // tokens before it are seen by every row of the wave's group
  auto begin_item = [&]() __attribute__((always_inline)) {
    const int first = (kv8_first(it.groups) + sh.rg) * ROWS;
    open = min(sh.end, it.ctx + __builtin_amdgcn_readfirstlane(first / G) + 1);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      jrow[rb] = min((kv8_first(it.groups) + sh.rg) * ROWS + rb * 16 + lc, it.nrow * G - 1) / G;
      m_run[rb] = -INFINITY;
      l_run[rb] = 0.f;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[rb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  };
  begin_item();

  const int k_off = lg * 128 + (lc & 7) * 16, v_off = (lg & 1) * 256 + lc * 16;
  bool more = true;                      // a segment follows this one
  // The codes of quad i of this segment, or past its end the first of the next one.  With none to
  // follow every lane asks for the start of a page (one cache line): the loads are issued on every
  // path, so that the waits stay exact.
  struct Pages {
    int64_t p[4];
  };
  auto pages_of = [&](int i) __attribute__((always_inline)) {
    int b[4];
    if (i < n) {
#pragma unroll
      for (int x = 0; x < 4; ++x) b[x] = __builtin_amdgcn_readlane(blk, 4 * i + x);
    } else {
      asm volatile("" ::: "memory");     // a branch: a select would wait for the ids on either side
#pragma unroll
      for (int x = 0; x < 4; ++x) b[x] = __builtin_amdgcn_readlane(nblk, x);
    }
    Pages p;
#pragma unroll
    for (int x = 0; x < 4; ++x) p.p[x] = (int64_t)clamped(b[x]) * a.nkv + kvh;
    return p;
  };
  // STREAM, a batch larger than the last-level cache: non-temporal where no other wave reads the same
  // codes.  Pages in any order stream at 6.8 TB/s then, 6.0 otherwise; waves that share codes find
  // them in L2 only without it (of 1.77 GB 1.23 times as much was read).  128 requests of 0.25-32k: 350
  // -> 330 us; 32 requests of 0.5-2k 25.6 without and 28.3 with it.
  bool alone = STREAM && kv8_groups(it.groups) == 1, next_alone = false;
  auto load = [&](int i, const uint8_t *pool, int off, int64_t page, uint4 (&r)[KC]) __attribute__((always_inline)) {
    const uint8_t *p = pool + page * (kPage * HD) + (i < n || more ? off : 0);
    if (STREAM && (i < n ? alone : next_alone)) {
      asm volatile("" ::: "memory");     // keeps the two branches two
#pragma unroll
      for (int c = 0; c < KC; ++c) r[c] = ld16_stream(p + c * 512);
      asm volatile("" ::: "memory");
    } else {
#pragma unroll
      for (int c = 0; c < KC; ++c) r[c] = ld16(p + c * 512);
    }
  };
  uint4 kr[2][KC], vr[2][KC];            // pair h of the quad
  float2 sc[2];                          // scales of the lane's page of pair h: lane groups 0 and 1 its first
  auto load_k = [&](int i) __attribute__((always_inline)) {
    const Pages p = pages_of(i);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      load(i, a.k, k_off, lc >= 8 ? p.p[2 * h + 1] : p.p[2 * h], kr[h]);
      sc[h] = a.scale[lg >= 2 ? p.p[2 * h + 1] : p.p[2 * h]];
    }
  };
  auto load_v = [&](int i) __attribute__((always_inline)) {
    const Pages p = pages_of(i);
#pragma unroll
    for (int h = 0; h < 2; ++h) load(i, a.v, v_off, lg >= 2 ? p.p[2 * h + 1] : p.p[2 * h], vr[h]);
  };

  // One quad in three phases; each operand's registers are filled again as soon as its phase is over:
  // K is in flight during the softmax and the second product, V during the first product and the
  // softmax.
  auto step = [&](int i) __attribute__((always_inline)) {
    const int tp = tok + 64 * i;
    float ks[2], lv[2], vi[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ks[h] = sc[h].x * a.c_log2;
      lv[h] = __builtin_amdgcn_logf(sc[h].y);
      vi[h] = __builtin_amdgcn_exp2f(-lv[h]);
    }
    floatx4 s[RB][2][2];                 // [row block][pair][half of its pages' slots]
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int h = 0; h < 2; ++h) s[rb][h][0] = s[rb][h][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int p = NP - 1; p >= 0; --p) { // small parts first
        bf16x8_t qf[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) qf[rb] = as_bf16x8(qs[sh.rg][p][rb][c][lane]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8_t k0 = to_bf16(kr[h][c].x, kr[h][c].y), k1 = to_bf16(kr[h][c].z, kr[h][c].w);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            s[rb][h][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[rb], s[rb][h][0], 0, 0, 0);
            s[rb][h][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[rb], s[rb][h][1], 0, 0, 0);
          }
        }
      }
    __builtin_amdgcn_sched_barrier(0);
    load_k(i + 1);
    __builtin_amdgcn_sched_barrier(0);
    // s[rb][h][x][e]: token tp + 32 h + 8 lg + 4 x + e, query row rb * 16 + lc of the group, without K's scale
    if (tp + 64 > open) {
      const int t = opaque(tp + 8 * lg);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int lim = min(sh.end, it.ctx + jrow[rb] + 1) - t;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (32 * h + 4 * x + e >= lim) s[rb][h][x][e] = -INFINITY;
      }
    }
    uint4 pb[NP][RB][2];
    softmax(s, ks, lv, vi, m_run, l_run, o, pb);
    // slots past the range may hold anything: zero probability is not enough against a NaN
    if (tp + 64 > sh.end) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int in = min(max(sh.end - opaque(tp + 32 * h + 8 * lg), 0), 8);
        const uint32_t mlo = in >= 4 ? ~0u : (1u << (8 * in)) - 1u, mhi = in <= 4 ? 0u : in == 8 ? ~0u : (1u << (8 * (in - 4))) - 1u;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          vr[h][c].x &= mlo;
          vr[h][c].y &= mhi;
          vr[h][c].z &= mlo;
          vr[h][c].w &= mhi;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const bf16x8_t v0 = to_bf16<kVDown>(vr[h][c].x, vr[h][c].y), v1 = to_bf16<kVDown>(vr[h][c].z, vr[h][c].w);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            o[rb][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(pb[p][rb][h]), o[rb][2 * c], 0, 0, 0);
            o[rb][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(pb[p][rb][h]), o[rb][2 * c + 1], 0, 0, 0);
          }
      }
    __builtin_amdgcn_sched_barrier(0);
    load_v(i + 1);
    __builtin_amdgcn_sched_barrier(0);
  };

  // The item's end, through LDS: every wave's accumulators, then 8 dims of a row per thread, the waves
  // that share the row's group added up in order.
  auto put_result = [&]() __attribute__((always_inline)) {
    const int lane = opaque(threadIdx.x) & 63, lc = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float l = xor32_sum(xor16_sum(l_run[rb]));
      if (lg == 0) sh_ml[wave][rb * 16 + lc] = make_float2(m_run[rb], l);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) *reinterpret_cast<floatx4 *>(&jo[wave][rb * 16 + lc][mb * 16 + 4 * lg]) = o[rb][mb];
    }
  };
  auto write_result = [&]() __attribute__((always_inline)) {
    const int groups = kv8_groups(it.groups), lr0 = kv8_first(it.groups) * ROWS;
    const int end = min(groups * ROWS, it.nrow * G - lr0) * (HD / 8);
    for (int u = opaque(threadIdx.x); u < end; u += 256) {
      const int r = u / (HD / 8), c0 = u % (HD / 8) * 8, g = r / ROWS, rr = r % ROWS;
      float2 ml[4];
      float m = -INFINITY;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (p < sh.parts) {
          ml[p] = sh_ml[g + p * groups][rr];
          m = fmaxf(m, ml[p].x);
        }
      }
      float l = 0.f;
      floatx4 x{0.f, 0.f, 0.f, 0.f}, y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (p < sh.parts) {
          // a wave that saw nothing has no maximum; a NaN stays one
          const float w = ml[p].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[p].x - m);
          const float *from = &jo[g + p * groups][rr][c0];
          l += ml[p].y * w;
          x += *reinterpret_cast<const floatx4 *>(from) * w;
          y += *reinterpret_cast<const floatx4 *>(from + 4) * w;
        }
      }
      if (it.part >= 0) {                // a part of the context: not divided yet
        const int64_t slot = ((int64_t)(it.part + g) * a.nkv + kvh) * ROWS + rr;
        float *to = a.part_o + slot * HD + c0;
        __builtin_nontemporal_store(x, reinterpret_cast<floatx4 *>(to));
        __builtin_nontemporal_store(y, reinterpret_cast<floatx4 *>(to + 4));
        if (c0 == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(m, l);
        continue;
      }
      const int64_t row = it.row0 + (lr0 + r) / G, col = (int64_t)(kvh * G + (lr0 + r) % G) * HD + c0;
      const float inv = kVUp / l;
      x *= inv;
      y *= inv;
      if constexpr (F32) {
        float *to = reinterpret_cast<float *>(a.out) + row * a.out_K + col;
        *reinterpret_cast<floatx4 *>(to) = x;
        *reinterpret_cast<floatx4 *>(to + 4) = y;
      } else {
        uint16_t *to = reinterpret_cast<uint16_t *>(a.out) + (a.packed ? packed_off(row, col, a.out_K) : row * a.out_K + col);
        *reinterpret_cast<uint4 *>(to) = make_uint4(pack2bf_rne(x[0], x[1]), pack2bf_rne(x[2], x[3]), pack2bf_rne(y[0], y[1]), pack2bf_rne(y[2], y[3]));
      }
    }
  };

  load_k(0);
  load_v(0);
  __builtin_amdgcn_sched_barrier(0);
  while (true) {
    const bool same = left > 0;                          // the next segment is this item's
    more = same || k + 1 < k_end;
    const Share ns = share_of(nx);
    next_alone = same ? alone : STREAM && kv8_groups(nx.groups) == 1;
    const int ntok = same ? tok + 64 * n : ns.tok;
    const int ids = same ? ids_at(it, ntok) : ids_at(nx, ntok);   // with nothing to follow: this item's once more
    if (n == 1) {                                        // needed at once (a branch: see pages_of)
      asm volatile("" ::: "memory");
      nblk = ids;
    }
    for (int i = 0; i < n; ++i) {
      step(i);
      if (i == 0) {                                      // older than a quad's loads by now
        nblk = opaque(ids);
        check(nblk);
      }
    }
    if (same) {
      n = min(left, 16);
      left -= n;
    } else {
      lds_barrier();                                     // the queries are no longer read
      put_result();
      lds_barrier();
      write_result();
      if (!more) break;
      Queries q;
      load_queries(nx, q);
      lds_barrier();
      store_queries(nx, q);
      ++k;
      it = nx;
      nx = item_at(k + 1);
      sh = ns;
      n = min(sh.n, 16);
      left = sh.n - n;
      begin_item();
      lds_barrier();
    }
    tok = ntok;
    blk = nblk;
    alone = next_alone;
  }
}

// Joins a row group's partials in order, in rounds of kRound whose loads are all issued before the
// first is used: one thread per (row, 8 dims).  Bound by latency: a launch and two
// dependent loads (32 requests: 4.6 us).
constexpr int kRound = 8;
template <bool F32>
__global__ __launch_bounds__(256) void kv8_join_kernel(const Kv8Group *__restrict__ groups, int rows_per_group, int hd,
                                                       const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                       void *__restrict__ out, bool packed, int out_K, int nq, int nkv) {
  const int kvh = blockIdx.x % nkv, G = nq / nkv;
  const Kv8Group g = groups[blockIdx.x / nkv];
  const int ch = hd / 8, lr0 = g.rbg * rows_per_group, nr = min(rows_per_group, g.nrow * G - lr0);
  for (int u = blockIdx.y * blockDim.x + threadIdx.x; u < nr * ch; u += gridDim.y * blockDim.x) {
    const int rr = u / ch, c0 = u % ch * 8;
    float m = -INFINITY, den = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < g.n_parts; r += kRound) {
      float2 ml[kRound];
      float4 x[kRound], y[kRound];
#pragma unroll
      for (int c = 0; c < kRound; ++c) {
        ml[c] = make_float2(-INFINITY, 0.f);
        x[c] = y[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r + c < g.n_parts) {   // the same for the whole workgroup
          const int64_t slot = ((int64_t)(g.part + (r + c) * g.stride) * nkv + kvh) * rows_per_group + rr;
          ml[c] = *reinterpret_cast<const float2 *>(part_ml + slot * 2);
          x[c] = *reinterpret_cast<const float4 *>(part_o + slot * hd + c0);
          y[c] = *reinterpret_cast<const float4 *>(part_o + slot * hd + c0 + 4);
        }
      }
      float top = m;
#pragma unroll
      for (int c = 0; c < kRound; ++c) top = fmaxf(top, ml[c].x);
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      den *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= keep;
      m = top;
#pragma unroll
      for (int c = 0; c < kRound; ++c) {
        const float w = ml[c].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[c].x - m);
        den += ml[c].y * w;
        acc[0] += x[c].x * w; acc[1] += x[c].y * w; acc[2] += x[c].z * w; acc[3] += x[c].w * w;
        acc[4] += y[c].x * w; acc[5] += y[c].y * w; acc[6] += y[c].z * w; acc[7] += y[c].w * w;
      }
    }
    const float inv = kVUp / den;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= inv;
    const int64_t row = g.row0 + (lr0 + rr) / G;
    const int64_t col = (int64_t)(kvh * G + (lr0 + rr) % G) * hd + c0;
    if constexpr (F32) {
      float *p = reinterpret_cast<float *>(out) + row * out_K + col;
      *reinterpret_cast<float4 *>(p) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4 *>(p + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
    } else {
      uint16_t *p = reinterpret_cast<uint16_t *>(out) + (packed ? packed_off(row, col, out_K) : row * out_K + col);
      *reinterpret_cast<uint4 *>(p) = make_uint4(pack2bf_rne(acc[0], acc[1]), pack2bf_rne(acc[2], acc[3]),
                                                 pack2bf_rne(acc[4], acc[5]), pack2bf_rne(acc[6], acc[7]));
    }
  }
}

}  // namespace

void kv8_attention(const Kv8Plan &p, const Kv8Cache &c, const void *q, void *out, bool packed, int *err, hipStream_t s) {
  if (p.n_items == 0) return;
  Kv8Args a;
  a.items = reinterpret_cast<const Kv8Item *>(p.ws + p.w_items);
  a.first = reinterpret_cast<const int32_t *>(p.ws + p.w_first);
  a.page_table = p.page_table;
  a.k = c.k;
  a.v = c.v;
  a.scale = reinterpret_cast<const float2 *>(c.scale);
  a.q = q;
  a.out = out;
  a.part_o = reinterpret_cast<float *>(p.ws + p.w_po);
  a.part_ml = reinterpret_cast<float *>(p.ws + p.w_pml);
  a.err = err;
  a.pt_stride = p.pt_stride;
  a.n_blocks = c.n_blocks;
  a.nq = p.nq;
  a.nkv = p.nkv;
  a.out_K = p.nq * p.hd;
  a.c_log2 = 1.4426950408889634f / sqrtf((float)p.hd);
  a.packed = packed;
  const bool f32 = p.dtype == 0;
  a.wide_first = a.first + (p.n_shares > 0 ? p.n_shares + 1 : 0);
  a.wide_blocks = p.n_wide * p.nkv;
  auto go = [&](auto kernel) { launch(kernel, (uint32_t)(p.n_shares + p.n_wide) * p.nkv, 256, 0, s, a); };
  if (f32) {
    switch (p.hd) {
      case 32: go(kv8_attn_kernel<32, 1, true>); break;
      case 64: go(kv8_attn_kernel<64, 1, true>); break;
      case 96: go(kv8_attn_kernel<96, 1, true>); break;
      case 128: go(kv8_attn_kernel<128, 1, true>); break;
      case 160: go(kv8_attn_kernel<160, 1, true>); break;
      case 192: go(kv8_attn_kernel<192, 1, true>); break;
      case 224: go(kv8_attn_kernel<224, 1, true>); break;
      default: go(kv8_attn_kernel<256, 1, true>); break;
    }
  } else {
    auto of = [&](auto hd) {
      constexpr int HD = decltype(hd)::value;
      if (p.n_wide > 0) p.stream ? go(kv8_attn_kernel<HD, 2, false, true, true>) : go(kv8_attn_kernel<HD, 2, false, false, true>);
      else if (p.stream) p.rb == 1 ? go(kv8_attn_kernel<HD, 1, false, true>) : go(kv8_attn_kernel<HD, 2, false, true>);
      else p.rb == 1 ? go(kv8_attn_kernel<HD, 1, false>) : go(kv8_attn_kernel<HD, 2, false>);
    };
    p.hd == 128 ? of(std::integral_constant<int, 128>{}) : of(std::integral_constant<int, 64>{});
  }
  if (p.n_groups == 0) return;
  const int rows = 16 * p.rb, units = rows * p.hd / 8;
  const dim3 grid((uint32_t)p.n_groups * p.nkv, (units + 255) / 256);
  launch(f32 ? kv8_join_kernel<true> : kv8_join_kernel<false>, grid, 256, 0, s,
         reinterpret_cast<const Kv8Group *>(p.ws + p.w_groups), rows, p.hd, (const float *)a.part_o,
         (const float *)a.part_ml, out, packed, a.out_K, p.nq, p.nkv);
}

}  // namespace wisp
