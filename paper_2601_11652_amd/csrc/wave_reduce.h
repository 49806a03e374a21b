// Reductions over a wave on the VALU: lanes l ^ 1, l ^ 2 by quad permutes, the other quad and
// the other half of a 16-lane row by mirrors (every lane of a quad, then of an octet, already
// holds the same value), rows by lane swaps.  The same pairs as a butterfly in steps 1, 2, 4,
// 8, 16, 32, every lane ending with the same bits.
#pragma once
#include "common.h"

namespace wisp {

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  const int i = __float_as_int(v);
  return __int_as_float(__builtin_amdgcn_update_dpp(i, i, CTRL, 0xF, 0xF, false));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<kXor1>(v);
  v += dpp<kXor2>(v);
  v += dpp<kHalfMirror>(v);
  v += dpp<kMirror>(v);
  return xor32_sum(xor16_sum(v));
}
// over each half of the wave
__device__ __forceinline__ float half_wave_max(float v) {
  v = fmaxf(v, dpp<kXor1>(v));
  v = fmaxf(v, dpp<kXor2>(v));
  v = fmaxf(v, dpp<kHalfMirror>(v));
  v = fmaxf(v, dpp<kMirror>(v));
  return xor16_max(v);
}
__device__ __forceinline__ float wave_max(float v) { return xor32_max(half_wave_max(v)); }

}  // namespace wisp
