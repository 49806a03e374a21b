// Attention of a batch whose requests share prefixes: the rows of a group attend to their common tokens
// together, each request's rows to its own, and the partial results of a row are joined.
//
// A row's result over tokens A and B is that over each with its maximum m and sum l of exp(s - m):
// m = max(mA, mB), l = lA e^(mA - m) + lB e^(mB - m), o likewise; out = o / l, lse = m + ln l.  So a group's tokens are
// read once for all its rows (128 samples of a prompt: 512 rows of a kv head, that would each have read it), and
// their products have full tiles.
//
// A workgroup takes four row tiles of 32 (a wave each, K and V through LDS for all of them) or one or two (whose tokens the
// waves share) over a run of tokens.  The host cuts the runs so that the workgroups that run at once end together.
//
// Bounds.  64 requests of a 64-head model on 8192 common tokens: 134 to 136 us, 755 TFLOP/s (a large library product reaches 1203
// on this card): a turn of four waves over 32 tokens is 512 cycles of products and took 915 before the sum of rounded probabilities,
// which is 2% of the call, as the maxima, exponentials and roundings of 16 x 64 scores a wave take some 400 that the other workgroup's
// products hide in part only (matrix units busy 0.42 of the cycles, vector instructions 0.44).  Scores of the next tile beside a tile's
// exponentials: 146 -> 137 us.  Two row tiles a wave (half the LDS reads, one workgroup a CU): 167 us.
// 128 samples of a prompt of 16384 tokens: 60 us, of which a third is what starts and ends an item (5 us: the item, its
// queries and block ids, the first pages, each waiting for the one before) and 7 the join of 28 MB of partial results.  4
// requests on 1024 tokens: 13 us, latency.  With nothing shared those samples take 372 us; but 64 requests on 512 tokens take 38, and 50
// as a group, whose partial results are written and read again.
#include <algorithm>
#include <climits>

#include "../../include/wisp.h"
#include "kernels.h"
#include "shared.h"
#include "shared_tile.h"

namespace wisp {

namespace {

struct SharedArgs {
  const SharedItem *items;
  const int32_t *page_table;
  const void *k, *v, *q;
  void *out;
  float *lse, *part_o;
  float4 *part_ml;                     // maximum, sum, sum of the probabilities as they multiply V
  int *err;
  int pt_stride, n_blocks, nq, nkv;
  float scale;
};

template <typename T, int HD>
struct Geo {
  static constexpr int KB = HD / 16, MB = HD / 32;            // steps of the contraction; blocks of output dims
  static constexpr int PAGE = kPage * HD, PAGE_BYTES = PAGE * (int)sizeof(T);
  static constexpr int STAGES = PAGE_BYTES <= 4096 ? 4 : PAGE_BYTES <= 12288 ? 3 : 2;   // tiles of K and V in LDS
  static constexpr int STAGE_BYTES = 2 * 2 * PAGE_BYTES;
  static constexpr int LDJ = HD + 4;                          // a row of accumulators in LDS, in floats
  static constexpr int SMEM = std::max(STAGES * STAGE_BYTES, 4 * kTile * LDJ * 4);
  static constexpr bool AHEAD = sizeof(T) == 2 || HD <= 64;   // registers hold the operands of a tile ahead
  static constexpr int WGS = AHEAD ? 2 : 1;
};

// maximum that passes over a NaN (the row's sum holds it)
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

template <typename T, int HD>
__global__ __launch_bounds__(256, (Geo<T, HD>::WGS)) void shared_attn_kernel(SharedArgs a) {
  using G_ = Geo<T, HD>;
  constexpr int KB = G_::KB, MB = G_::MB, PAGE = G_::PAGE, STAGES = G_::STAGES, LDJ = G_::LDJ;
  __shared__ __attribute__((aligned(1024))) char smem[G_::SMEM];
  __shared__ float4 sh_ml[4][kTile];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 31, hf = lane >> 5;
  const int kvh = blockIdx.x % a.nkv;                 // neighbouring workgroups, on other XCDs: other kv heads
  const SharedItem it = a.items[blockIdx.x / a.nkv];
  const int G = a.nq / a.nkv, rows = it.nrow * G;
  const Divisor by_g(G);
  const bool wide = it.tiles > 2;                     // one tile of rows a wave; else the waves share the tokens
  const int parts = wide ? 1 : 4 / it.tiles, tile = wide ? min(wave, it.tiles - 1) : wave % it.tiles;
  const int part = wide ? 0 : wave / it.tiles;
  const int fr0 = (it.tile0 + tile) * kTile, fr = min(fr0 + lc, rows - 1);   // padding rows: a real one
  const int jr = by_g.of(fr);
  const int64_t q_at = ((int64_t)(it.row0 + jr) * a.nq + kvh * G + fr - jr * G) * HD + 8 * hf;
  Op8<T> qf[KB];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) qf[kb] = load_op(static_cast<const T *>(a.q) + q_at + 16 * kb);
  const int lim = min(it.t1, it.ctx + jr + 1);        // tokens that this lane's row sees
  const int open = min(it.t1, it.ctx + __builtin_amdgcn_readfirstlane(by_g.of(fr0)) + 1);   // that every row of the tile sees
  const float c_log2 = a.scale * kLog2e, tau = 8.0f / c_log2;
  // Sums of the probabilities, for lse, and (bf16) as they multiply V, rounded, by which the result is divided: it is then a mean of V's
  // rows, and a token with nearly all of a row gives its own, where the other sum leaves the rounding of its probability, as
  // much as that of the result once more.  1 to 2% of a call.
  float m_run = -INFINITY, l_run = 0.f, d_run = 0.f;
  floatx16 o[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mb][i] = 0.f;

  // Online softmax of a tile's scores to probabilities.  The running maximum rises only by more
  // than 2^8 in the probabilities, so the accumulators are rescaled on few tiles.
  float mc = 0.f;                                     // m_run in base 2; 0 while the row has seen nothing
  bool far = false;                                   // of some row it is so large that its rounding counts
  auto row_max = [&](const floatx16 &s) __attribute__((always_inline)) {
    float mx = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) mx = max3(mx, s[i], s[i + 1]);
    return xor32_max(fmaxf(mx, s[15]));
  };
  auto raise = [&](float mx) __attribute__((always_inline)) {
    const bool grow = mx > m_run + tau;
    if (__builtin_amdgcn_ballot_w64(grow)) {
      const float alpha = grow ? __builtin_amdgcn_exp2f((m_run - mx) * c_log2) : 1.0f;
      m_run = grow ? mx : m_run;
      l_run *= alpha;
      d_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
      mc = m_run == -INFINITY ? 0.f : m_run * c_log2;
      far = __builtin_amdgcn_ballot_w64(fabsf(mc) > kFarScore) != 0;
    }
  };
  // what is added to a score x log2(e) / sqrt(head_dim)
  auto offset = [&](floatx16 &s) __attribute__((always_inline)) {
    if (!far) return -mc;
    // the rounding of m x log2(e) would be most of the scores' difference: that first
    const float m = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] -= m;
    return 0.f;
  };
  auto exponentials = [&](floatx16 &s, float off) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c_log2, off));
  };
  auto add_up = [&](const floatx16 &s) __attribute__((always_inline)) {
    float sum[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
    for (int i = 4; i < 16; ++i) sum[i & 3] += s[i];
    const float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    l_run += all;                                     // this lane's tokens: the halves are added at the end
    return all;
  };
  auto softmax = [&](floatx16 &s) __attribute__((always_inline)) {
    raise(row_max(s));
    exponentials(s, offset(s));
    return add_up(s);
  };
  // eight probabilities of a page as an operand
  auto probs = [&](const floatx16 &p, int g) __attribute__((always_inline)) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = p[8 * g + i];
    Op8<T> pb;
    to_op(pb, e);
    return pb;
  };

  const_ids_t *ids = const_ids(a.page_table + (int64_t)it.table * a.pt_stride);
  const int page0 = it.t0 >> 4, page_end = (it.t1 - 1) >> 4;       // pages past the end: the last
  auto place = [&](int b) __attribute__((always_inline)) {
    return ((int64_t)min(max(b, 0), a.n_blocks - 1) * a.nkv + kvh) * PAGE;
  };
  const T *kp = static_cast<const T *>(a.k), *vp = static_cast<const T *>(a.v);
  const int k_lane = k_op_lane(lane), v_lane = v_op_lane(lane);
  const int n_tiles = (it.t1 - it.t0 + kTile - 1) / kTile;
  int x = part;                                        // the next tile of this wave

  if (wide) {
    // The tiles that every row of the item sees: pages go straight into LDS, STAGES - 1 tiles ahead, and lie
    // there in operand order (as they do in memory, a third of the LDS cycles were conflicts).
    constexpr int PIECE = (int)sizeof(T) / 2, LOADS = G_::PAGE_BYTES / 1024;   // 16-byte pieces of an operand; a wave's loads for a tile
    const int n = max(0, min(it.t1, it.ctx + by_g.of(it.tile0 * kTile) + 1) - it.t0) / kTile;
    // Block ids of 32 tiles sit in the lanes, those of the next 32 are on their way.  (Scalar loads share their counter with
    // LDS and return out of order: every operand read from LDS would wait for them.)
    const int32_t *table = a.page_table + (int64_t)it.table * a.pt_stride;
    auto window = [&](int w) __attribute__((always_inline)) { return table[min(page0 + 64 * w + lane, page_end)]; };
    int blk = window(0), after = window(1), b0 = 0, b1 = 0;
    auto ids_of = [&](int t) __attribute__((always_inline)) {          // of each tile in turn
      if (t % 32 == 0 && t > 0) {
        blk = after;
        after = window(t / 32 + 1);
      }
      b0 = __builtin_amdgcn_readlane(blk, 2 * t & 63);
      b1 = __builtin_amdgcn_readlane(blk, (2 * t & 63) + 1);
    };
    // A tile's buffer holds K's pages, then V's, each KiB of them as a load of 16 bytes a lane brings it: K's units in the
    // order of the rows that read them, V's as an operand has them.  The address is uniform but for the lane's place.
    constexpr int KIB = G_::PAGE_BYTES / 1024, OP_BYTES = 8 * (int)sizeof(T);
    const uint32_t k_from = ((lane >> 3 & 1) * 32 + (lane >> 4) * 8 + (lane & 7)) * OP_BYTES, v_from = (uint32_t)v_lane * (uint32_t)sizeof(T);
    auto bring = [&](int t) __attribute__((always_inline)) {
      // a wave: one page of K or of V
      const char *from = reinterpret_cast<const char *>((wave & 1 ? vp : kp) + place(wave & 2 ? b1 : b0));
      const uint32_t to = lds_address(smem) + (t % STAGES) * G_::STAGE_BYTES + (2 * (wave & 1) + (wave >> 1)) * G_::PAGE_BYTES;
#pragma unroll
      for (int u = 0; u < KIB / PIECE; ++u)
#pragma unroll
        for (int y = 0; y < PIECE; ++y)
          lds_dma16_at(from + u * 1024 * PIECE + 16 * y, wave & 1 ? v_from : k_from, to + (u * PIECE + y) * 1024);
    };
    const char *k_at = smem + (lane >> 4 & 1) * G_::PAGE_BYTES + ((lane >> 5) * 16 + (lane & 15)) * 16, *v_at = smem + 2 * G_::PAGE_BYTES + lane * 16;
    auto k_operand = [&](int buf, int kb) __attribute__((always_inline)) {
      Op8<T> r;
#pragma unroll
      for (int y = 0; y < PIECE; ++y) r.v[y] = ld16(k_at + buf * G_::STAGE_BYTES + ((kb >> 1) * PIECE + y) * 1024 + (kb & 1) * 512);
      return r;
    };
    auto v_operand = [&](int buf, int g, int mb) __attribute__((always_inline)) {
      Op8<T> r;
#pragma unroll
      for (int y = 0; y < PIECE; ++y) r.v[y] = ld16(v_at + buf * G_::STAGE_BYTES + g * G_::PAGE_BYTES + (mb * PIECE + y) * 1024);
      return r;
    };
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t) {
      ids_of(t);
      if (n > 0) bring(t);                             // past the end: pages of the item, not used
    }
    ids_of(STAGES - 1);
    loads_done();                                      // the queries
    auto products = [&](const Op8<T> (&k)[KB]) __attribute__((always_inline)) {
      floatx16 r;
#pragma unroll
      for (int i = 0; i < 16; ++i) r[i] = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) r = mma(r, k[kb], qf[kb]);
      return r;
    };
    // This wave's loads of a tile have landed (those of `behind` tiles after it may be on their way), and every wave's
    auto landed = [&](auto behind) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(behind)::value * LOADS) : "memory");
    };
    Op8<T> op[KB], ov[KB];
    if constexpr (STAGES > 2) {
      // A turn computes the scores of the next tile beside this one's exponentials, then this one's products with V
      // beside the next one's maximum: a wave's matrix and vector instructions run at the same time.
      floatx16 sc;
      if (n > 0) {
        landed(std::integral_constant<int, STAGES - 2>());
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) op[kb] = k_operand(0, kb);
        sc = products(op);
        raise(row_max(sc));
      }
      for (int t = 0; t < n; ++t) {
        landed(std::integral_constant<int, STAGES - 3>());
        bring(t + STAGES - 1);
        ids_of(t + STAGES);
        const float off = offset(sc);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) op[kb] = k_operand((t + 1) % STAGES, kb);
        const floatx16 next = products(op);              // past the end: not used
        exponentials(sc, off);
        add_up(sc);
        const Op8<T> p0 = probs(sc, 0), p1 = probs(sc, 1);
        d_run = op_sum(p0, p1, d_run);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) ov[kb] = v_operand(t % STAGES, kb / MB, kb % MB);
        if constexpr (sizeof(T) == 2) {
          __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);          // LDS reads
          __builtin_amdgcn_sched_group_barrier(0x2, 8, 0);             // vector instructions
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);           // a product
            __builtin_amdgcn_sched_group_barrier(0x2, 48 / KB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) o[mb] = mma(o[mb], ov[g * MB + mb], g ? p1 : p0);
        const float mx = row_max(next);
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < n) raise(mx);
        sc = next;
      }
    } else {
      for (int t = 0; t < n; ++t) {
        landed(std::integral_constant<int, 0>());
        bring(t + 1);
        ids_of(t + 2);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) op[kb] = k_operand(t % STAGES, kb);
        floatx16 sc = products(op);
        softmax(sc);
        const Op8<T> pb[2] = {probs(sc, 0), probs(sc, 1)};
        d_run = op_sum(pb[0], pb[1], d_run);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) o[mb] = mma(o[mb], v_operand(t % STAGES, g, mb), pb[g]);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // what was brought past the end has landed before LDS is used again
    x = n;
  }

  // A wave by itself, operands straight from memory, a tile ahead: the waves of a row tile take its token
  // tiles in turn; of a wide item each its rows' last tiles.
  {
    Op8<T> kf[KB], vf[2][MB];
    const T *vb[2];
    int b0 = 0, b1 = 0, later = INT_MAX;
    auto ids_of = [&](int t) __attribute__((always_inline)) {
      b0 = ids[min(page0 + 2 * t, page_end)];
      b1 = ids[min(page0 + 2 * t + 1, page_end)];
    };
    auto load_k = [&]() __attribute__((always_inline)) {
      const T *kt = kp + ((lane >> 4) & 1 ? place(b1) : place(b0)) + k_lane;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) kf[kb] = load_op(kt + k_op_step(kb));
    };
    auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) vf[g][mb] = load_op(vb[g] + v_lane + v_op_block(mb));
    };
    if (x < n_tiles) {
      ids_of(x);
      if constexpr (G_::AHEAD) load_k();
      vb[0] = vp + place(b0);
      vb[1] = vp + place(b1);
      if constexpr (G_::AHEAD) load_v();
    }
    for (; x < n_tiles; x += parts) {
      const int tp = it.t0 + x * kTile;
      if constexpr (!G_::AHEAD) {
        ids_of(x);
        load_k();
        vb[0] = vp + place(b0);
        vb[1] = vp + place(b1);
      } else {
        ids_of(x + parts);
      }
      floatx16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) sc = mma(sc, kf[kb], qf[kb]);
      // operands are asked for where those before them have been used: sooner, they would take registers of their own
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (G_::AHEAD) load_k();               // past the end: the last pages once more
      __builtin_amdgcn_sched_barrier(0);
      const bool masked = tp + kTile > open;
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = tp + reg_token(lane, i) < lim ? sc[i] : -INFINITY;
      }
      const float all = softmax(sc);
      if constexpr (!G_::AHEAD) load_v();
      if (masked) {
        // Slots past the last token may hold anything.  And a token that is there, but not seen by every row, may be
        // infinite or NaN, which a product with a probability of 0 would hand on: from such a tile on V is left for later
        bool special = false;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const Keep<T> keep(it.t1 - (tp + 16 * g + 8 * hf));
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            keep.apply(vf[g][mb]);
            special |= any_special(vf[g][mb]);
          }
        }
        if (__builtin_amdgcn_ballot_w64(special)) later = min(later, x);
      }
      if (later > x) {
        const Op8<T> pb[2] = {probs(sc, 0), probs(sc, 1)};
        d_run = op_sum(pb[0], pb[1], d_run);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) o[mb] = mma(o[mb], vf[g][mb], pb[g]);
      } else {
        d_run += all;                                  // they multiply V as they are
      }
      __builtin_amdgcn_sched_barrier(0);
      vb[0] = vp + place(b0);
      vb[1] = vp + place(b1);
      if constexpr (G_::AHEAD) load_v();
      __builtin_amdgcn_sched_barrier(0);
    }
    // V of the tiles that hold what some rows must not touch, token by token
#pragma unroll 1
    for (x = later; x < n_tiles; x += parts) {
      const int tp = it.t0 + x * kTile;
      ids_of(x);
      load_k();
      floatx16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) sc = mma(sc, kf[kb], qf[kb]);
      exponentials(sc, offset(sc));
#pragma unroll 1
      for (int t = 0; t < kTile && tp + t < it.t1; ++t) {
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) w = (t >> 4) * 8 + (t & 7) == i ? sc[i] : w;
        w = __shfl(w, lc + 32 * ((t >> 3) & 1));
        const T *from = vp + place(t < kPage ? b0 : b1) + v_page_off(t & 15, 4 * hf);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float v = as_float(from[512 * mb + (i >> 3) * 256 + ((i >> 2) & 1) * 64 + (i & 3) * 8]);
            asm volatile("" : "+v"(v));                // loaded by every lane: no branch around each load
            o[mb][i] = tp + t < lim ? __builtin_fmaf(w, v, o[mb][i]) : o[mb][i];
          }
      }
    }
  }

  // block ids out of range are reported (they were clamped above)
  for (int x = page0 + threadIdx.x; x <= page_end; x += 256) {
    const int b = a.page_table[(int64_t)it.table * a.pt_stride + x];
    if (b < 0 || b >= a.n_blocks) flag_error(a.err, kErrBlock);
  }
  // A row tile of one wave goes out as it lies in the registers, partial results in that order: 16 bytes a lane
  const float l = xor32_sum(l_run), d = sizeof(T) == 2 ? xor32_sum(d_run) : l;
  auto put_part = [&](int tile, int row_lane, int at, floatx4 v) __attribute__((always_inline)) {
    *reinterpret_cast<floatx4 *>(a.part_o + ((int64_t)it.part + (int64_t)kvh * it.step + tile) * (kTile * HD) + (at * 64 + row_lane) * 4) = v;
  };
  auto put_ml = [&](int tile, int row, float m, float l, float d) __attribute__((always_inline)) {
    a.part_ml[((int64_t)it.part + (int64_t)kvh * it.step + tile) * kTile + row] = make_float4(m, l, d, 0.f);
  };
  if (wide && it.part >= 0) {
    if (wave < it.tiles) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int y = 0; y < 4; ++y) put_part(wave, lane, 4 * mb + y, floatx4{o[mb][4 * y], o[mb][4 * y + 1], o[mb][4 * y + 2], o[mb][4 * y + 3]});
      if (hf == 0) put_ml(wave, lc, m_run, l, d);
    }
    return;
  }
  // through LDS: 8 dims of a row a thread, the waves of a row tile added in order
  __syncthreads();
  float(*jo)[kTile][LDJ] = reinterpret_cast<float(*)[kTile][LDJ]>(smem);
  if (hf == 0) sh_ml[wave][lc] = make_float4(m_run, l, d, 0.f);
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<floatx4 *>(&jo[wave][lc][32 * mb + 8 * x + 4 * hf]) =
          floatx4{o[mb][4 * x], o[mb][4 * x + 1], o[mb][4 * x + 2], o[mb][4 * x + 3]};
  __syncthreads();
  constexpr int CH = HD / 8;
  for (int u = threadIdx.x; u < it.tiles * kTile * CH; u += 256) {
    const int c0 = u % CH * 8, r = u / CH % kTile, t = u / CH / kTile;
    const int f = (it.tile0 + t) * kTile + r;
    if (f >= rows) continue;
    float m = -INFINITY, sum = 0.f, den = 0.f;
    for (int x = 0; x < parts; ++x) m = fmaxf(m, sh_ml[t + x * it.tiles][r].x);
    floatx4 y = {0.f, 0.f, 0.f, 0.f}, z = y;
    for (int x = 0; x < parts; ++x) {
      const float4 ml = sh_ml[t + x * it.tiles][r];
      if (ml.x == -INFINITY) {
        sum += ml.y;                                  // 0, or NaN of a row's NaN scores
        den += ml.z;
        continue;
      }
      const float w = __builtin_amdgcn_exp2f((ml.x - m) * c_log2);
      sum += ml.y * w;
      den += ml.z * w;
      y += *reinterpret_cast<const floatx4 *>(&jo[t + x * it.tiles][r][c0]) * w;
      z += *reinterpret_cast<const floatx4 *>(&jo[t + x * it.tiles][r][c0 + 4]) * w;
    }
    if (it.part >= 0) {
      put_part(t, r, c0 / 8, y);
      put_part(t, r + 32, c0 / 8, z);
      if (c0 == 0) put_ml(t, r, m, sum, den);
      continue;
    }
    const int j = by_g.of(f);
    const int64_t row = (int64_t)(it.row0 + j) * a.nq + kvh * G + f - j * G;
    const float inv = 1.0f / den;
    y *= inv;
    z *= inv;
    T *to = static_cast<T *>(a.out) + row * HD + c0;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4 *>(to) = make_uint4(pack2bf_rne(y[0], y[1]), pack2bf_rne(y[2], y[3]), pack2bf_rne(z[0], z[1]), pack2bf_rne(z[2], z[3]));
    } else {
      *reinterpret_cast<floatx4 *>(to) = y;
      *reinterpret_cast<floatx4 *>(to + 4) = z;
    }
    if (a.lse && c0 == 0) a.lse[row] = m * a.scale + logf(sum);
  }
}

// The partial results of a row, joined in order: its own segment's, then its group's.  A thread for 8 dims of a
// head; the loads of kJoinParts results are in flight at once.
constexpr int kJoinParts = 8, kJoinThreads = 128;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void shared_join_kernel(const SharedRow *rows, const SharedBundle *bundles, const float *part_o,
                                                                   const float4 *part_ml, T *out, float *lse, int n_rows, int nq, int nkv, int hd,
                                                                   int together, int per_block, float scale) {
  // Neighbouring threads have the heads of a kv head and then those of the next of `together` rows, whose results are
  // neighbours: 256 bytes, two lines.  per_block kv heads a workgroup.
  const int G = nq / nkv, ch = hd / 8;
  const Divisor by_g(G), by_rows(G * together), by_head(G * together * ch);
  const int at = blockIdx.z * blockDim.x + threadIdx.x, local = by_head.of(at), u = at - local * G * together * ch, c = by_rows.of(u);
  const int in_row = u - c * G * together, sub = by_g.of(in_row), g = in_row - sub * G;
  const int kvh = blockIdx.y * per_block + local, c0 = 8 * c, head = kvh * G + g, r = blockIdx.x * together + sub;
  if (local >= per_block || kvh >= nkv || r >= n_rows) return;
  const float c_log2 = scale * kLog2e;
  SharedBundle b0 = rows[r].own, b1 = rows[r].pre;
  int f0 = b0.row + g, f1 = b1.row + g;
  if (f0 >= kBundle * kTile) {
    b0 = bundles[rows[r].own_next];
    f0 -= kBundle * kTile;
  }
  if (f1 >= kBundle * kTile && b1.parts) {
    b1 = bundles[rows[r].pre_next];
    f1 -= kBundle * kTile;
  }
  const int n = b0.parts + b1.parts;
  if (n < 2) return;                                  // written as it was computed
  const int64_t own = ((int64_t)b0.at + (int64_t)kvh * b0.tiles) * kTile + f0, own_step = (int64_t)nkv * b0.tiles * kTile;
  const int64_t pre = ((int64_t)b1.at + (int64_t)kvh * b1.tiles) * kTile + f1, pre_step = (int64_t)nkv * b1.tiles * kTile;
  float m = -INFINITY, sum = 0.f, den = 0.f;
  floatx4 y = {0.f, 0.f, 0.f, 0.f}, z = y;
  for (int p0 = 0; p0 < n; p0 += kJoinParts) {
    float4 ml[kJoinParts];
    floatx4 a[kJoinParts], b[kJoinParts];
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
      ml[i] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
      a[i] = b[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (p0 + i < n) {
        const int p = p0 + i;
        const int64_t s = p < b0.parts ? own + p * own_step : pre + (p - b0.parts) * pre_step;
        ml[i] = part_ml[s];
        const float *o = part_o + (s >> 5) * kTile * hd + (c0 / 8 * 64 + (s & 31)) * 4;
        a[i] = *reinterpret_cast<const floatx4 *>(o);
        b[i] = *reinterpret_cast<const floatx4 *>(o + 32 * 4);
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) top = fmaxf(top, ml[i].x);
    const float was = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c_log2);
    m = top;
    sum *= was;
    den *= was;
    y *= was;
    z *= was;
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
      // of a part that saw no token the sum is 0, or NaN where the row's scores were
      const float w = ml[i].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml[i].x - m) * c_log2);
      sum += ml[i].y * w;
      den += ml[i].z * w;
      y += a[i] * w;
      z += b[i] * w;
    }
  }
  const int64_t row = (int64_t)r * nq + head;
  const float inv = 1.0f / den;
  y *= inv;
  z *= inv;
  T *to = out + row * hd + c0;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4 *>(to) = make_uint4(pack2bf_rne(y[0], y[1]), pack2bf_rne(y[2], y[3]), pack2bf_rne(z[0], z[1]), pack2bf_rne(z[2], z[3]));
  } else {
    *reinterpret_cast<floatx4 *>(to) = y;
    *reinterpret_cast<floatx4 *>(to + 4) = z;
  }
  if (lse && c0 == 0) lse[row] = m * scale + logf(sum);
}

}  // namespace

int shared_wgs_per_cu(int dtype, int hd) { return dtype == WISP_BF16 || hd <= 64 ? 2 : 1; }

void shared_attention(const SharedPlan &p, const SharedCache &c, const void *q, void *out, float *lse, int *err, hipStream_t s) {
  SharedArgs a{};
  a.items = reinterpret_cast<const SharedItem *>(p.ws + p.w_items);
  a.page_table = p.page_table;
  a.k = c.k;
  a.v = c.v;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.part_o = reinterpret_cast<float *>(p.ws + p.w_po);
  a.part_ml = reinterpret_cast<float4 *>(p.ws + p.w_pml);
  a.err = err;
  a.pt_stride = p.pt_stride;
  a.n_blocks = c.n_blocks;
  a.nq = p.nq;
  a.nkv = p.nkv;
  a.scale = 1.0f / sqrtf((float)p.hd);
  auto go = [&](auto kernel) { launch(kernel, p.n_items * p.nkv, 256, 0, s, a); };
  if (p.dtype == WISP_BF16) {
    if (p.hd == 128) go(shared_attn_kernel<uint16_t, 128>);
    else go(shared_attn_kernel<uint16_t, 64>);
  } else {
    switch (p.hd) {
      case 32: go(shared_attn_kernel<float, 32>); break;
      case 64: go(shared_attn_kernel<float, 64>); break;
      case 96: go(shared_attn_kernel<float, 96>); break;
      case 128: go(shared_attn_kernel<float, 128>); break;
      case 160: go(shared_attn_kernel<float, 160>); break;
      case 192: go(shared_attn_kernel<float, 192>); break;
      case 224: go(shared_attn_kernel<float, 224>); break;
      default: go(shared_attn_kernel<float, 256>);
    }
  }
  if (!p.joined) return;
  const SharedRow *rows = reinterpret_cast<const SharedRow *>(p.ws + p.w_join);
  const SharedBundle *bundles = reinterpret_cast<const SharedBundle *>(p.ws + p.w_bundles);
  const int G = p.nq / p.nkv, together = std::max(1, 16 / G), of_head = together * G * p.hd / 8;
  const int per_block = std::max(1, std::min(p.nkv, kJoinThreads / of_head)), threads = std::min(kJoinThreads, (per_block * of_head + 63) / 64 * 64);
  const dim3 grid((p.rows + together - 1) / together, (p.nkv + per_block - 1) / per_block, (per_block * of_head + threads - 1) / threads);
  auto join = [&](auto kernel, auto *to) {
    launch(kernel, grid, threads, 0, s, rows, bundles, (const float *)a.part_o, (const float4 *)a.part_ml, to, lse,
           p.rows, p.nq, p.nkv, p.hd, together, per_block, a.scale);
  };
  if (p.dtype == WISP_BF16) join(shared_join_kernel<uint16_t>, static_cast<uint16_t *>(out));
  else join(shared_join_kernel<float>, static_cast<float *>(out));
}

}  // namespace wisp
