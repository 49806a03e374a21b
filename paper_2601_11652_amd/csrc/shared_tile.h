// Matrix products of 32 tokens x 32 query rows straight from the cache's pages, shared by the attention
// over shared prefixes and the accumulation of its weights.
//
// S^T = K Q^T and O^T += V^T P^T with 32 x 32 products: for bf16 16 dims (or tokens) a product, for fp32 two,
// eight of them in the place of one.  A query row stays in a lane column (lane % 32).  The tokens of a
// tile (two pages) are ordered so that lane half h = lane / 32 holds, in register i of its 16, token
// 16 (i / 8) + 8 h + i % 8: the eight registers of a page are then the second product's operand as they
// are, and an operand of K (8 dims of a slot) or V (8 slots of a dim) is 8 consecutive elements of a page.
#pragma once
#include <type_traits>

#include "common.h"

namespace wisp {

constexpr float kLog2e = 1.4426950408889634f;
// Magnitude of a score in base 2 up to which the rounding of its product with log2(e) may be taken out of the
// exponential's argument: above, differences of scores are formed first
constexpr float kFarScore = 65536.f;

template <typename T>
struct Op8 {                           // eight elements of an operand
  uint4 v[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Op8<T> load_op(const T *p) {
  Op8<T> o;
#pragma unroll
  for (int x = 0; x < (int)sizeof(T) / 2; ++x) o.v[x] = ld16(reinterpret_cast<const char *>(p) + 16 * x);
  return o;
}
__device__ __forceinline__ floatx16 mma(floatx16 c, const Op8<uint16_t> &a, const Op8<uint16_t> &b) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a.v[0]), as_bf16x8(b.v[0]), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mma(floatx16 c, const Op8<float> &a, const Op8<float> &b) {
  const floatx4 x[2] = {__builtin_bit_cast(floatx4, a.v[0]), __builtin_bit_cast(floatx4, a.v[1])};
  const floatx4 y[2] = {__builtin_bit_cast(floatx4, b.v[0]), __builtin_bit_cast(floatx4, b.v[1])};
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e / 4][e % 4], y[e / 4][e % 4], c, 0, 0, 0);
  return c;
}
// eight probabilities as an operand
__device__ __forceinline__ void to_op(Op8<uint16_t> &o, const float *p) {
  o.v[0] = make_uint4(pack2bf_rne(p[0], p[1]), pack2bf_rne(p[2], p[3]), pack2bf_rne(p[4], p[5]), pack2bf_rne(p[6], p[7]));
}
__device__ __forceinline__ void to_op(Op8<float> &o, const float *p) {
#pragma unroll
  for (int x = 0; x < 2; ++x)
    o.v[x] = make_uint4(__float_as_uint(p[4 * x]), __float_as_uint(p[4 * x + 1]), __float_as_uint(p[4 * x + 2]), __float_as_uint(p[4 * x + 3]));
}
// c and the sixteen probabilities of two operands, as they multiply V (fp32: as they are, and added already)
__device__ __forceinline__ float op_sum(const Op8<uint16_t> &a, const Op8<uint16_t> &b, float c) {
  const bf16x2_t one = {(__bf16)1.f, (__bf16)1.f};
  const uint32_t w[8] = {a.v[0].x, a.v[0].y, a.v[0].z, a.v[0].w, b.v[0].x, b.v[0].y, b.v[0].z, b.v[0].w};
  float s = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[x]), one, s, false);
    c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[x + 4]), one, c, false);
  }
  return c + s;
}
__device__ __forceinline__ float op_sum(const Op8<float> &, const Op8<float> &, float c) { return c; }
// The first n of eight elements: what is not theirs becomes zero.  Slots past a request's last token may hold
// anything.
template <typename T>
struct Keep {
  uint32_t mask[2 * sizeof(T)];
  __device__ __forceinline__ explicit Keep(int n) {
#pragma unroll
    for (int x = 0; x < 2 * (int)sizeof(T); ++x) {
      const int bits = min(max((n * (int)sizeof(T) - 4 * x) * 8, 0), 32);
      mask[x] = (uint32_t)((1ull << bits) - 1);
    }
  }
  __device__ __forceinline__ void apply(Op8<T> &o) const {
#pragma unroll
    for (int x = 0; x < (int)sizeof(T) / 2; ++x)
      o.v[x] = make_uint4(o.v[x].x & mask[4 * x], o.v[x].y & mask[4 * x + 1], o.v[x].z & mask[4 * x + 2], o.v[x].w & mask[4 * x + 3]);
  }
};
// whether an element is infinite or NaN
__device__ __forceinline__ bool any_special(const Op8<uint16_t> &o) {
  const uint32_t w[4] = {o.v[0].x, o.v[0].y, o.v[0].z, o.v[0].w};
  bool s = false;
#pragma unroll
  for (int x = 0; x < 4; ++x) s |= (w[x] & 0x7F80u) == 0x7F80u || (w[x] & 0x7F800000u) == 0x7F800000u;
  return s;
}
__device__ __forceinline__ bool any_special(const Op8<float> &o) {
  bool s = false;
#pragma unroll
  for (int x = 0; x < 2; ++x)
    s |= (o.v[x].x & 0x7F800000u) == 0x7F800000u || (o.v[x].y & 0x7F800000u) == 0x7F800000u ||
         (o.v[x].z & 0x7F800000u) == 0x7F800000u || (o.v[x].w & 0x7F800000u) == 0x7F800000u;
  return s;
}
__device__ __forceinline__ float as_float(uint16_t b) { return bf2f(b); }
__device__ __forceinline__ float as_float(float f) { return f; }

// A lane's operands inside a page, in elements.  K, 16-dim step kb: row r = lane % 32 of the product is slot
// 8 ((r / 4) % 2) + 4 ((r / 8) % 2) + r % 4 of page r / 16
__device__ __forceinline__ int k_op_lane(int lane) { return ((lane >> 3) & 1) * 256 + (lane >> 5) * 64 + (lane & 7) * 8; }
__device__ __forceinline__ constexpr int k_op_step(int kb) { return (kb >> 1) * 512 + (kb & 1) * 128; }
// V, 32-dim block mb: dim 32 mb + lane % 32, slots 8 (lane / 32) ..
__device__ __forceinline__ int v_op_lane(int lane) { return ((lane >> 4) & 1) * 256 + (lane >> 5) * 128 + (lane & 15) * 8; }
__device__ __forceinline__ constexpr int v_op_block(int mb) { return mb * 512; }
// token of register i, from the tile's first
__device__ __forceinline__ int reg_token(int lane, int i) { return 16 * (i >> 3) + 8 * (lane >> 5) + (i & 7); }

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}
// lds_dma16 from base + offset, base wave-uniform (no address to make for each lane), to an LDS address
__device__ __forceinline__ void lds_dma16_at(const void *base, uint32_t offset, uint32_t to) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane(to);
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(m0) : "memory", "m0");
}
// four bytes a lane
__device__ __forceinline__ void lds_dma4_at(const void *base, uint32_t offset, uint32_t to) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane(to);
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dword %0, %1" : : "v"(offset), "s"(base), "s"(m0) : "memory", "m0");
}

// Every load so far has returned, and the compiler knows it: operands that are first used inside a loop would make it
// wait there, in every turn, for whatever has been asked for since.
__device__ __forceinline__ void loads_done() {
  __builtin_amdgcn_s_waitcnt(0 | 7 << 4 | 15 << 8);
  asm volatile("" ::: "memory");
}

// x / d for x d below 2^32: one product (the quotient of a variable takes twenty instructions)
struct Divisor {
  uint32_t d, m;
  __device__ __forceinline__ explicit Divisor(int by) : d(by), m(0xFFFFFFFFu / (uint32_t)by + 1) {}
  __device__ __forceinline__ int of(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }
};

// block ids, read through the scalar cache: nothing writes them while a kernel runs
typedef const int32_t __attribute__((address_space(4))) const_ids_t;
__device__ __forceinline__ const_ids_t *const_ids(const int32_t *p) {
  return reinterpret_cast<const_ids_t *>(reinterpret_cast<uintptr_t>(p));
}

}  // namespace wisp
