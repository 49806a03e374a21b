// Ragged multi-query causal attention over the 8-bit paged KV cache: the attention of Sec. 4.5's
// batched one-step verification on e4m3 pages with one K and one V scale per page and kv head.
//
// A workgroup of four waves runs one item: a row group (16 RB of a request's rows x query heads of
// one kv head) over a range of the request's tokens, each wave a quarter of the range's page
// pairs.  Per pair a wave computes S^T = K Q^T and O^T += V^T P^T with 16x16x32 matrix products in
// bf16, which holds every e4m3 value exactly: the codes are converted between load and product,
// the K scale multiplies the scores and the V scale the probabilities (a lane's eight
// tokens of a pair lie in one page, so each is one factor per lane).  Every query row stays in one
// lane column (lane % 16), so the online softmax needs two cross-row steps, and the
// probabilities leave the first product in the order that the second consumes.  The waves' partial
// results are joined through LDS, those of a context cut into several items by a second kernel.
//
// An fp32 model's queries and probabilities enter the products as three bf16 parts each (8 bits
// of the significand per part: 24 in all), so its results are fp32's.
#include "kernels.h"
#include "kv8.h"

namespace wisp {

namespace {

__device__ __forceinline__ bf16x8_t to_bf16(uint32_t lo, uint32_t hi) {
  union {
    bf16x2_t h[4];
    bf16x8_t v;
  } u;
  u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return u.v;
}
__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

struct Kv8Args {
  const Kv8Item *items;
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

template <int HD, int RB, bool F32>
__global__ __launch_bounds__(256, RB <= 2 && HD <= 128 ? 2 : 1) void kv8_attn_kernel(Kv8Args a) {
  constexpr int ROWS = 16 * RB;
  constexpr int KC = HD / 32;           // 32-wide chunks of the contraction; 16-byte loads of K and of V
  constexpr int MB = HD / 16;           // 16-wide blocks of the output dims
  constexpr int NP = F32 ? 3 : 1;       // bf16 parts of a query and of a probability
  constexpr int kQBytes = NP * RB * KC * 64 * 16, kJoinBytes = 4 * RB * MB * 64 * 16;
  __shared__ __attribute__((aligned(16))) char smem[kQBytes > kJoinBytes ? kQBytes : kJoinBytes];
  __shared__ float sh_m[4][ROWS], sh_l[4][ROWS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 15, lg = lane >> 4;
  const int kvh = blockIdx.x % a.nkv;   // neighbouring workgroups (other XCDs): other kv heads
  const Kv8Item it = a.items[blockIdx.x / a.nkv];
  const int G = a.nq / a.nkv, rows = it.nrow * G;

  // this wave's page pairs, their block ids (lane l: its l-th page) and scales
  const int pairs = (it.t1 - it.t0 + 31) / 32;
  const int pa = pairs * wave / 4, n = pairs * (wave + 1) / 4 - pa;
  const int tok0 = it.t0 + 32 * pa;
  int blk = 0;
  float ks = 0.f, vs = 0.f, vs_inv = 0.f;
  if (n > 0) {
    const int pg = min((tok0 >> 4) + lane, (min(it.t1, tok0 + 32 * n) - 1) >> 4);
    blk = a.page_table[(int64_t)it.req * a.pt_stride + pg];
    if (blk < 0 || blk >= a.n_blocks) {
      flag_error(a.err, kErrBlock);
      blk = min(max(blk, 0), a.n_blocks - 1);
    }
  }

  // the row group's queries in operand order, loaded by all four waves
  uint4(*qs)[RB][KC][64] = reinterpret_cast<uint4(*)[RB][KC][64]>(smem);
  for (int u = threadIdx.x; u < RB * KC * 64; u += 256) {
    const int l = u & 63, kc = (u >> 6) % KC, rb = (u >> 6) / KC;
    const int lr = min(it.rbg * ROWS + rb * 16 + (l & 15), rows - 1);   // padding rows reuse a real row
    const int64_t at = ((int64_t)(it.row0 + lr / G) * a.nq + kvh * G + lr % G) * HD + kc * 32 + 8 * (l >> 4);
    if constexpr (F32) {
      const float *p = reinterpret_cast<const float *>(a.q) + at;
      uint32_t w[3][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = p[2 * e], y = p[2 * e + 1];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          w[k][e] = pack2bf_rne(x, y);
          x -= low(w[k][e]);
          y -= high(w[k][e]);
        }
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) qs[k][rb][kc][l] = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
    } else {
      qs[0][rb][kc][l] = ld16(reinterpret_cast<const uint16_t *>(a.q) + at);
    }
  }
  if (n > 0) {
    const float2 s2 = a.scale[(int64_t)blk * a.nkv + kvh];
    ks = s2.x * a.c_log2;
    vs = s2.y;
    vs_inv = 1.0f / vs;
  }
  __syncthreads();

  float m_run[RB], l_run[RB];
  floatx4 o[RB][MB];
  int jrow[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    jrow[rb] = min(it.rbg * ROWS + rb * 16 + lc, rows - 1) / G;
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[rb][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto lane_of = [](float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
  const int k_off = lg * 128 + (lc & 7) * 16, v_off = (lg & 1) * 256 + lc * 16;
  for (int i = 0; i < n; ++i) {
    const int tp = tok0 + 32 * i;
    const int64_t p0 = ((int64_t)__builtin_amdgcn_readlane(blk, 2 * i) * a.nkv + kvh) * (kPage * HD);
    const int64_t p1 = ((int64_t)__builtin_amdgcn_readlane(blk, 2 * i + 1) * a.nkv + kvh) * (kPage * HD);
    const uint8_t *kp = a.k + (lc >= 8 ? p1 : p0) + k_off, *vp = a.v + (lg >= 2 ? p1 : p0) + v_off;
    uint4 kr[KC], vr[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c) kr[c] = ld16_stream(kp + c * 512);
#pragma unroll
    for (int c = 0; c < KC; ++c) vr[c] = ld16_stream(vp + c * 512);
    const float ks_l = lg >= 2 ? lane_of(ks, 2 * i + 1) : lane_of(ks, 2 * i);
    const float vs_l = lg >= 2 ? lane_of(vs, 2 * i + 1) : lane_of(vs, 2 * i);
    const float vi_l = lg >= 2 ? lane_of(vs_inv, 2 * i + 1) : lane_of(vs_inv, 2 * i);
    floatx4 s[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8_t k0 = to_bf16(kr[c].x, kr[c].y), k1 = to_bf16(kr[c].z, kr[c].w);
#pragma unroll
      for (int k = NP - 1; k >= 0; --k)   // small parts first
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const bf16x8_t qf = as_bf16x8(qs[k][rb][c][lane]);
          s[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf, s[rb][0], 0, 0, 0);
          s[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf, s[rb][1], 0, 0, 0);
        }
    }
    // slots past the range may hold anything: zero probability is not enough against a NaN
    if (tp + 32 > it.t1) {
      const int left = min(max(it.t1 - (tp + 8 * lg), 0), 8);
      const uint32_t mlo = left >= 4 ? ~0u : (1u << (8 * left)) - 1u, mhi = left <= 4 ? 0u : left == 8 ? ~0u : (1u << (8 * (left - 4))) - 1u;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        vr[c].x &= mlo;
        vr[c].y &= mhi;
        vr[c].z &= mlo;
        vr[c].w &= mhi;
      }
    }
    const bool unmasked = tp + 32 <= min(it.t1, it.ctx + 1);
    uint4 pb[NP][RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      // s[rb][h][e]: token tp + 8 lg + 4 h + e, query row rb * 16 + lc of the group
#pragma unroll
      for (int h = 0; h < 2; ++h) s[rb][h] *= ks_l;
      if (!unmasked) {
        const int lim = min(it.t1, it.ctx + jrow[rb] + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tp + 8 * lg + 4 * h + e >= lim) s[rb][h][e] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3])),
                       fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
      mx = xor32_max(xor16_max(mx));
      // the running maximum (base 2) rises only by more than 8: p stays below 2^8, and the
      // accumulators are rescaled on few pairs; numerator and denominator share the reference
      const bool grow = mx > m_run[rb] + 8.0f;
      if (__builtin_amdgcn_ballot_w64(grow)) {
        const float alpha = grow ? __builtin_amdgcn_exp2f(m_run[rb] - mx) : 1.0f;
        m_run[rb] = grow ? mx : m_run[rb];
        l_run[rb] *= alpha;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o[rb][mb] *= alpha;
      }
      const float mc = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
      float rs = 0.f;
      uint32_t pw[NP][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float x = __builtin_amdgcn_exp2f(s[rb][h][e] - mc) * vs_l, y = __builtin_amdgcn_exp2f(s[rb][h][e + 1] - mc) * vs_l;
          if constexpr (F32) rs += x + y;
#pragma unroll
          for (int k = 0; k < NP; ++k) {
            const uint32_t w = pack2bf_rne(x, y);
            pw[k][h * 2 + e / 2] = w;
            x -= low(w);
            y -= high(w);
          }
          // bf16: the sum adds the rounded values, as the second product does
          if constexpr (!F32) rs += low(pw[0][h * 2 + e / 2]) + high(pw[0][h * 2 + e / 2]);
        }
      l_run[rb] += xor32_sum(xor16_sum(rs * vi_l));
#pragma unroll
      for (int k = 0; k < NP; ++k) pb[k][rb] = make_uint4(pw[k][0], pw[k][1], pw[k][2], pw[k][3]);
    }
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8_t v0 = to_bf16(vr[c].x, vr[c].y), v1 = to_bf16(vr[c].z, vr[c].w);
#pragma unroll
      for (int k = NP - 1; k >= 0; --k)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          o[rb][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(pb[k][rb]), o[rb][2 * c], 0, 0, 0);
          o[rb][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(pb[k][rb]), o[rb][2 * c + 1], 0, 0, 0);
        }
    }
  }

  // join the waves: tile t = rb * MB + mb is added up by wave t % 4, in wave order
  if (lg == 0)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      sh_m[wave][rb * 16 + lc] = m_run[rb];
      sh_l[wave][rb * 16 + lc] = l_run[rb];
    }
  __syncthreads();   // the queries are no longer read either
  floatx4(*jo)[RB * MB][64] = reinterpret_cast<floatx4(*)[RB * MB][64]>(smem);
  float m_all[RB], l_all[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = rb * 16 + lc;
    m_all[rb] = fmaxf(fmaxf(sh_m[0][r], sh_m[1][r]), fmaxf(sh_m[2][r], sh_m[3][r]));
    auto weight = [&](float m) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_all[rb]); };
    l_all[rb] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l_all[rb] += sh_l[w][r] * weight(sh_m[w][r]);
    const float mine = weight(m_run[rb]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) jo[wave][rb * MB + mb][lane] = o[rb][mb] * mine;
  }
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int lr = it.rbg * ROWS + rb * 16 + lc;
    if (lr >= rows) continue;
    const float inv = 1.0f / l_all[rb];
    const int64_t row = it.row0 + jrow[rb];
    const int head = kvh * G + lr - jrow[rb] * G;
    const int64_t slot = ((int64_t)it.part * a.nkv + kvh) * ROWS + rb * 16 + lc;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      if ((rb * MB + mb) % 4 != wave) continue;
      const int t = rb * MB + mb;
      const floatx4 x = jo[0][t][lane] + jo[1][t][lane] + (jo[2][t][lane] + jo[3][t][lane]);
      if (it.part >= 0) {
        __builtin_nontemporal_store(x, reinterpret_cast<floatx4 *>(a.part_o + slot * HD + mb * 16 + 4 * lg));
        continue;
      }
      const int64_t col = (int64_t)head * HD + mb * 16 + 4 * lg;
      if constexpr (F32) {
        *reinterpret_cast<floatx4 *>(reinterpret_cast<float *>(a.out) + row * a.out_K + col) = x * inv;
      } else {
        const int64_t at = a.packed ? packed_off(row, col, a.out_K) : row * a.out_K + col;
        *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.out) + at) =
            make_uint2(pack2bf_rne(x[0] * inv, x[1] * inv), pack2bf_rne(x[2] * inv, x[3] * inv));
      }
    }
    if (it.part >= 0 && lg == 0 && wave == 0)
      *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(m_all[rb], l_all[rb]);
  }
}

// Joins a row group's partials in order: one thread per (row, 8 dims)
template <bool F32>
__global__ __launch_bounds__(256) void kv8_join_kernel(const Kv8Group *__restrict__ groups, int rows_per_group, int hd,
                                                       const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                       void *__restrict__ out, bool packed, int out_K, int nq, int nkv) {
  const int kvh = blockIdx.x % nkv, G = nq / nkv;
  const Kv8Group g = groups[blockIdx.x / nkv];
  const int ch = hd / 8, lr0 = g.rbg * rows_per_group, nr = min(rows_per_group, g.nrow * G - lr0);
  for (int u = blockIdx.y * blockDim.x + threadIdx.x; u < nr * ch; u += gridDim.y * blockDim.x) {
    const int rr = u / ch, c0 = u % ch * 8;
    auto slot = [&](int c) { return ((int64_t)(g.part + c) * nkv + kvh) * rows_per_group + rr; };
    float m = -INFINITY;
    for (int c = 0; c < g.n_parts; ++c) m = fmaxf(m, part_ml[slot(c) * 2]);
    float den = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < g.n_parts; ++c) {
      const float2 ml = *reinterpret_cast<const float2 *>(part_ml + slot(c) * 2);
      const float4 x = *reinterpret_cast<const float4 *>(part_o + slot(c) * hd + c0);
      const float4 y = *reinterpret_cast<const float4 *>(part_o + slot(c) * hd + c0 + 4);
      const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      den += ml.y * w;
      acc[0] += x.x * w; acc[1] += x.y * w; acc[2] += x.z * w; acc[3] += x.w * w;
      acc[4] += y.x * w; acc[5] += y.y * w; acc[6] += y.z * w; acc[7] += y.w * w;
    }
    const float inv = 1.0f / den;
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
  auto go = [&](auto kernel) { launch(kernel, (uint32_t)p.n_items * p.nkv, 256, 0, s, a); };
  if (f32) {
    switch (p.hd) {
      case 32: go(kv8_attn_kernel<32, 1, true>); break;
      case 64: p.rb == 1 ? go(kv8_attn_kernel<64, 1, true>) : go(kv8_attn_kernel<64, 2, true>); break;
      case 96: go(kv8_attn_kernel<96, 1, true>); break;
      case 128: p.rb == 1 ? go(kv8_attn_kernel<128, 1, true>) : go(kv8_attn_kernel<128, 2, true>); break;
      case 160: go(kv8_attn_kernel<160, 1, true>); break;
      case 192: go(kv8_attn_kernel<192, 1, true>); break;
      case 224: go(kv8_attn_kernel<224, 1, true>); break;
      default: go(kv8_attn_kernel<256, 1, true>); break;
    }
  } else if (p.hd == 128) {
    switch (p.rb) {
      case 1: go(kv8_attn_kernel<128, 1, false>); break;
      case 2: go(kv8_attn_kernel<128, 2, false>); break;
      case 3: go(kv8_attn_kernel<128, 3, false>); break;
      default: go(kv8_attn_kernel<128, 4, false>); break;
    }
  } else {
    switch (p.rb) {
      case 1: go(kv8_attn_kernel<64, 1, false>); break;
      case 2: go(kv8_attn_kernel<64, 2, false>); break;
      case 3: go(kv8_attn_kernel<64, 3, false>); break;
      default: go(kv8_attn_kernel<64, 4, false>); break;
    }
  }
  if (p.n_groups == 0) return;
  const int rows = 16 * p.rb, units = rows * p.hd / 8;
  const dim3 grid((uint32_t)p.n_groups * p.nkv, (units + 255) / 256);
  launch(f32 ? kv8_join_kernel<true> : kv8_join_kernel<false>, grid, 256, 0, s,
         reinterpret_cast<const Kv8Group *>(p.ws + p.w_groups), rows, p.hd, (const float *)a.part_o,
         (const float *)a.part_ml, out, packed, a.out_K, p.nq, p.nkv);
}

}  // namespace wisp
