// The attention weight that every cached token gets from a batch's rows: for token t and kv head h the sum
// over rows r that see t, and query heads g of h, of exp(q . k_t / sqrt(head_dim) - lse).
//
// The scores are computed once more: they are one product and not two, and kept they would be the rows x tokens that the
// attention does without.  A wave keeps the keys of 32 tokens in registers, as an operand, and adds up over the rows, which
// stream through LDS for the four waves; sums of fp32 in registers, a row's place in them fixed, so results do not vary.
//
// For a prompt (4096 rows x 32 heads over 4096 tokens, half of them seen) matrix and vector instructions take turns: 0.40 and
// 0.71 of the cycles, 16 exponentials of 64 lanes to a row tile's 8 products.  Three workgroups a CU hide most of the waits:
// 96 to 98 us, 720 TFLOP/s.  Two token tiles a wave, half the LDS reads, were 118 us where one took 106; the next tile's products
// beside a tile's exponentials, no change.  32 sessions on a document of 4096 tokens: 21 us, blocks of one row tile whose
// instructions before and after it are the most of it.  A few rows over many tokens are bound by latency: 4000 tokens 8 us.
#include <algorithm>

#include "../../include/wisp.h"
#include "kernels.h"
#include "shared.h"
#include "shared_tile.h"
#include "wave_reduce.h"

namespace wisp {

namespace {

struct MassArgs {
  const MassItem *items;
  const int32_t *page_table, *row;      // row: (request, row in it) of every row
  const void *k, *q;
  const float *lse;
  const int32_t *count;
  const float *prev;
  float *mass, *part;
  int *err;
  int pt_stride, n_blocks, nq, nkv;
  float scale, decay;
};

// A token's new weight: what it had, less the decay, if it was cached before, and what it got
__device__ __forceinline__ void put_mass(const int32_t *page_table, int pt_stride, int n_blocks, int nkv, int kvh, int table, int t,
                                         bool old, float decay, const float *prev, float got, float *mass, int *err) {
  const int b = page_table[(int64_t)table * pt_stride + (t >> 4)];
  if (b < 0 || b >= n_blocks) {
    flag_error(err, kErrBlock);
    return;
  }
  const int64_t at = ((int64_t)b * nkv + kvh) * kPage + (t & 15);
  mass[at] = old && prev ? __builtin_fmaf(decay, prev[at], got) : got;
}

// A weight's exponent in base 2 where the row's scores are large: the difference first, so that what is rounded before it is lse and
// the score, each as the attention rounded it (the product by itself, not in one with the difference), and a token that had all of its row
// has 0.  Roundings may make it positive: a weight is 1 at most.
__device__ __forceinline__ float far_exponent(float score, float scale, float lse) {
#pragma clang fp contract(off)
  const float scaled = score * scale;
  const float e = (scaled - lse) * kLog2e;
  return e > 0.f ? 0.f : e;                            // NaN stays
}

template <typename T, int HD>
__global__ __launch_bounds__(256, (sizeof(T) == 2 || HD <= 64) ? 3 : 1) void mass_kernel(MassArgs a) {
  constexpr int KB = HD / 16, UNITS = HD * (int)sizeof(T) / 16, PIECES = UNITS / 2;   // 16-byte units of a row; 1 KiB pieces of a row tile
  constexpr int TILES = PIECES <= 8 ? 2 : 1, RING = 3;             // row tiles of a stage; stages in LDS
  constexpr int STAGE = TILES * kTile;                              // its rows
  constexpr int SWIZZLE = UNITS % 16 ? 7 : 15;
  __shared__ uint4 rows_of[RING][TILES][kTile * UNITS];
  __shared__ float lse_of[RING][64];
  __shared__ uint32_t counts[kMassTiles];                           // of a group: which rows count
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lc = lane & 31, hf = lane >> 5;
  const int kvh = blockIdx.x % a.nkv;
  const MassItem it = a.items[blockIdx.x / a.nkv];
  const int G = a.nq / a.nkv, rows = it.nrow * G;
  // rows past those that count give nothing
  int counted = it.nrow;
  if (a.count && it.req >= 0) counted = min(max(a.count[it.req], 0), it.nrow);
  const int r_end = min(it.r1, counted * G);
  Op8<T> kf[KB];
  auto load_k = [&](int t0) __attribute__((always_inline)) {         // this wave's tokens of a block; past the end the last page
    const int32_t *ids = a.page_table + (int64_t)it.table * a.pt_stride;
    const int b = ids[min((t0 >> 4) + 2 * wave + ((lane >> 4) & 1), (it.t1 - 1) >> 4)];
    const T *kt = static_cast<const T *>(a.k) + ((int64_t)min(max(b, 0), a.n_blocks - 1) * a.nkv + kvh) * (kPage * HD);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) kf[kb] = load_op(kt + k_op_lane(lane) + k_op_step(kb));
  };
  load_k(it.t0);
  const float c_log2 = a.scale * kLog2e;
  // Row tiles go straight into LDS, RING - 1 stages ahead, whole rows at a time: unit u of row r lies at u ^ (r % 16 or 8), so
  // that the rows' operands are read without bank conflicts (in operand order, each load took 32 bytes of 32 rows: 115 us
  // for a prompt of 4096 rows).  Their lse goes with them.
  constexpr int WAVES = 4 / TILES, MINE = PIECES / WAVES, LOADS = MINE + 1;   // waves of a row tile's pieces; each one's; and the lse
  static_assert(PIECES % WAVES == 0, "a tile's pieces are shared equally");
  const Divisor by_g(G);
  // Where the query heads of a kv head divide a stage's rows (and the stage is whole) its rows lie as those of the stage
  // before, so many tokens on: their places are kept, and only a uniform address moves.
  const int my_tile = wave / WAVES, p0 = wave % WAVES * MINE;
  const bool steady = STAGE % G == 0;
  const int step = STAGE / G;            // rows of the batch, of a steady stage
  // of flat row f's query from row r's, in heads; j0: the batch's row of r
  auto behind = [&](int r, int j0, int f) __attribute__((always_inline)) {
    const int c = min(f, rows - 1);
    return (uint32_t)((by_g.of(c) - j0) * (a.nq - G) + c - r);
  };
  auto head_of = [&](int r, int j0) __attribute__((always_inline)) { return (int64_t)(it.row0 + j0) * a.nq + kvh * G + r - j0 * G; };
  uint32_t q_off[MINE], lse_off;
  auto places = [&](int r, int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < MINE; ++x) {
      const int at = (p0 + x) * 64 + lane, row = at / UNITS;
      q_off[x] = behind(r, j0, r + my_tile * kTile + row) * (uint32_t)(HD * sizeof(T)) + 16 * (at % UNITS ^ (row & SWIZZLE));
    }
    lse_off = behind(r, j0, r + lane) * 4;
  };
  const int first_j = by_g.of(it.r0);
  const int64_t head0 = head_of(it.r0, first_j);
  places(it.r0, first_j);
  auto bring = [&](int n) __attribute__((always_inline)) {           // stage n of the item, each in turn
    const int b = n % RING, r = it.r0 + n * STAGE;
    int64_t head = head0 + (int64_t)n * step * a.nq;
    if (n > 0 && !(steady && r + 64 <= rows)) {
      const int j0 = by_g.of(min(r, rows - 1));
      head = head_of(r, j0);
      places(r, j0);
    }
    const T *base = static_cast<const T *>(a.q) + head * HD;
    const uint32_t to = lds_address(rows_of) + ((b * TILES + my_tile) * kTile * UNITS + p0 * 64) * 16;
#pragma unroll
    for (int x = 0; x < MINE; ++x) lds_dma16_at(base, q_off[x], to + x * 1024);
    lds_dma4_at(a.lse + head, lse_off, lds_address(lse_of) + b * 256);
  };
  const bool by_request = a.count && it.req < 0;
  const int stages = (r_end - it.r0 + STAGE - 1) / STAGE;
  if (it.r0 < r_end) {
    for (int n = 0; n < min(stages, RING - 1); ++n) bring(n);
    if (by_request) {
      for (int f = it.r0 + threadIdx.x; f - lane < r_end; f += 256) {
        const int2 of = *reinterpret_cast<const int2 *>(a.row + 2 * (int64_t)(it.row0 + by_g.of(min(f, rows - 1))));
        const unsigned long long on = __builtin_amdgcn_ballot_w64(of.y < a.count[of.x]);
        if (lane < 2 && (f - lane - it.r0) / kTile + lane < kMassTiles) counts[(f - lane - it.r0) / kTile + lane] = lane ? on >> 32 : on;
      }
    }
  }
  floatx16 zero;                       // in registers: made anew for each tile, it would take 16 instructions
#pragma unroll
  for (int i = 0; i < 16; ++i) zero[i] = 0.f;
  asm volatile("" : "+v"(zero));
  // An item of one stage may have several blocks of tokens; the next one's keys are on their way while the sums go out.
  for (int t0 = it.t0;; t0 += kMassBlock) {
    const int tp = t0 + wave * kTile;
    floatx16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    loads_done();                        // K
    for (int n = 0; n < stages; ++n) {
      const int r0 = it.r0 + n * STAGE, b = n % RING, after = min(RING - 2, stages - 1 - n);
      // this wave's loads of the stage have landed, and every wave's
      if (t0 > it.t0) ;                  // the only one: it is there
      else if (after == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (n + RING - 1 < stages) bring(n + RING - 1);
#pragma unroll
      for (int y = 0; y < TILES; ++y) {
        if (r0 + y * kTile >= r_end) break;
        // all operands asked for, then the products: a pair at a time, each pair waited for LDS
        Op8<T> q[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int z = 0; z < (int)sizeof(T) / 2; ++z)
            q[kb].v[z] = rows_of[b][y][lc * UNITS + (((2 * kb + hf) * ((int)sizeof(T) / 2) + z) ^ (lc & SWIZZLE))];
        const float lse = lse_of[b][y * kTile + lc];
        const uint32_t on = by_request ? counts[n * TILES + y] : ~0u;
        __builtin_amdgcn_sched_barrier(0);
        floatx16 s;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s = mma(kb ? s : zero, kf[kb], q[kb]);
        const int f = r0 + y * kTile + lc;
        // tokens that this lane's row sees: none where it does not count
        const int lim = f < r_end && (on >> lc & 1) ? it.ctx + by_g.of(f) + 1 : 0;
        const float l2 = lse * kLog2e;
        const int seen = lim - tp - 8 * hf;
        if (__builtin_amdgcn_ballot_w64(fabsf(l2) > kFarScore)) {
          // scores so large that the roundings of both products with log2(e) would be most of their difference
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float p = __builtin_amdgcn_exp2f(fabsf(l2) > kFarScore ? far_exponent(s[i], a.scale, lse) : __builtin_fmaf(s[i], c_log2, -l2));
            acc[i] += reg_token(0, i) < seen ? p : 0.f;
          }
        } else if (__builtin_amdgcn_ballot_w64(lim < tp + kTile)) {
          // rows that do not see a token, or do not count
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c_log2, -l2));
            acc[i] += reg_token(0, i) < seen ? p : 0.f;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c_log2, -l2));
        }
      }
    }
    const bool more = t0 + kMassBlock < it.t1;
    if (more) load_k(t0 + kMassBlock);
    // over the rows: the lanes of a half
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = acc[i];
      v += dpp<kXor1>(v);
      v += dpp<kXor2>(v);
      v += dpp<kHalfMirror>(v);
      v += dpp<kMirror>(v);
      v = xor16_sum(v);
      sum = lc == i ? v : sum;
    }
    const int t = tp + reg_token(lane, lc & 15);
    if (lc < 16 && t < it.t1) {
      if (it.part >= 0) a.part[(int64_t)it.part + (int64_t)kvh * it.step + t - it.t0] = sum;
      else put_mass(a.page_table, a.pt_stride, a.n_blocks, a.nkv, kvh, it.table, t, t < it.ctx, a.decay, a.prev, sum, a.mass, a.err);
    }
    if (!more) break;
  }
}

__global__ __launch_bounds__(kMassBlock) void mass_join_kernel(const MassJoin *joins, const float *part, const int32_t *page_table,
                                                               int pt_stride, int n_blocks, int nkv, float decay, const float *prev,
                                                               float *mass, int *err) {
  const int kvh = blockIdx.x % nkv;
  const MassJoin j = joins[blockIdx.x / nkv];
  const int t = j.t0 + threadIdx.x;
  if (t >= j.t1) return;
  float got = 0.f;
  for (int p = 0; p < j.parts; ++p) got += part[(int64_t)j.part + (int64_t)kvh * j.step + (int64_t)p * kMassBlock + threadIdx.x];
  put_mass(page_table, pt_stride, n_blocks, nkv, kvh, j.table, t, t < j.ctx, decay, prev, got, mass, err);
}

}  // namespace

int mass_stage_tiles(int dtype, int hd) { return dtype == WISP_BF16 || hd <= 64 ? 2 : 1; }
int mass_wgs_per_cu(int dtype, int hd) { return dtype == WISP_BF16 || hd <= 64 ? 3 : 1; }

void shared_mass(const SharedPlan &p, const SharedCache &c, const void *q, const float *lse, const int32_t *count, float decay,
                 const float *prev, float *mass, int *err, hipStream_t s) {
  MassArgs a{};
  a.items = reinterpret_cast<const MassItem *>(p.ws + p.w_mass);
  a.page_table = p.page_table;
  a.row = reinterpret_cast<const int32_t *>(p.ws + p.w_row);
  a.k = c.k;
  a.q = q;
  a.lse = lse;
  a.count = count;
  a.prev = prev;
  a.mass = mass;
  a.part = reinterpret_cast<float *>(p.ws + p.w_pm);
  a.err = err;
  a.pt_stride = p.pt_stride;
  a.n_blocks = c.n_blocks;
  a.nq = p.nq;
  a.nkv = p.nkv;
  a.scale = 1.0f / sqrtf((float)p.hd);
  a.decay = decay;
  auto go = [&](auto kernel) { launch(kernel, p.n_mass * p.nkv, 256, 0, s, a); };
  if (p.dtype == WISP_BF16) {
    if (p.hd == 128) go(mass_kernel<uint16_t, 128>);
    else go(mass_kernel<uint16_t, 64>);
  } else {
    switch (p.hd) {
      case 32: go(mass_kernel<float, 32>); break;
      case 64: go(mass_kernel<float, 64>); break;
      case 96: go(mass_kernel<float, 96>); break;
      case 128: go(mass_kernel<float, 128>); break;
      case 160: go(mass_kernel<float, 160>); break;
      case 192: go(mass_kernel<float, 192>); break;
      case 224: go(mass_kernel<float, 224>); break;
      default: go(mass_kernel<float, 256>);
    }
  }
  if (p.n_mass_join > 0)
    launch(mass_join_kernel, p.n_mass_join * p.nkv, kMassBlock, 0, s, reinterpret_cast<const MassJoin *>(p.ws + p.w_mass_join),
           (const float *)a.part, p.page_table, p.pt_stride, c.n_blocks, p.nkv, decay, prev, mass, err);
}

}  // namespace wisp
