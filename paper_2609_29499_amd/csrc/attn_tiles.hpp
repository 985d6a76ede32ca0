// Pieces of attention kernels whose tiles of 16 query rows by 32 cache rows run on v_mfma_f32_16x16x32_bf16: operands,
// reductions over lanes, and small divisions without the integer divider.
#pragma once
#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// v[sub] of lane `owner`
__device__ __forceinline__ int pick(const int (&v)[4], int owner, int sub) {
  return __builtin_amdgcn_readlane(sub == 0 ? v[0] : sub == 1 ? v[1] : sub == 2 ? v[2] : v[3], owner);
}
// a / d for rows and items (a < 2^21): a + 1/2 is 1 / (2 d) away from a multiple of d at least, the product off by a / d 2^-22.
// (An integer division is 40 instructions one after the other: dealing took 2.9 us with a dozen of them.)
__device__ __forceinline__ int quot(int a, int d) { return int((float(a) + 0.5f) * __builtin_amdgcn_rcpf(float(d))); }
// a / d for steps, with a / d < 2^20: the product is off by less than one
__device__ __forceinline__ int quot_steps(int a, int d, float inv) {
  const int q = int(float(a) * inv), rest = a - q * d;
  return rest < 0 ? q - 1 : rest >= d ? q + 1 : q;
}
// Sums over lanes 0 .. own (row_shr:1, 2, 4, 8 within rows of 16, row_bcast:15 and :31 between them)
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}
__device__ __forceinline__ float quad_max(float v) {   // over lanes r, r + 16, r + 32, r + 48
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

__device__ __forceinline__ f32x4 mfma(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
      __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3])),
      __builtin_bit_cast(bf16x8, make_uint4(b[0], b[1], b[2], b[3])), acc, 0, 0, 0);
}

// four codes of a word -> two words of BF16 pairs (exact)
template <int TYPE>
__device__ __forceinline__ void widen(uint32_t w, uint32_t* o) {
  if constexpr (TYPE == SEQ_INT8) {
    const float f0 = float(int8_t(w)), f1 = float(int8_t(w >> 8)), f2 = float(int8_t(w >> 16)), f3 = float(int8_t(w >> 24));
    o[0] = __builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u);
    o[1] = __builtin_amdgcn_perm(__float_as_uint(f3), __float_as_uint(f2), 0x07060302u);
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
}

// NT BF16 terms of pairs (v0, v1): v = sum of terms to 8 NT bits
template <int NT>
__device__ __forceinline__ void terms(float v0, float v1, uint32_t* o, int stride) {
#pragma unroll
  for (int k = 0; k < NT; ++k) {
    o[k * stride] = pack_bf16(v0, v1);
    v0 -= bf16_lo(o[k * stride]);
    v1 -= bf16_hi(o[k * stride]);
  }
}

// Non-finite halves of V words become zeros; returns a non-zero word if there are any.
__device__ __forceinline__ uint32_t drop_odd(uint32_t& v) {
  const uint32_t top = ((v & 0x7f807f80u) + 0x00800080u) & 0x80008000u;      // a half's exponent is full
  v &= ~((top >> 15) * 0xffffu);
  return top;
}
// What load_q brought is here. Said in front of a loop over steps: a load that may still be on its way at its first
// turn is waited for in every turn, and with it all of the next step's loads, which are younger.
template <int QT, int NKC>
__device__ __forceinline__ void arrived(uint32_t (&qf)[QT][NKC][4]) {
#pragma unroll
  for (int k = 0; k < QT; ++k)
#pragma unroll
    for (int j = 0; j < NKC; ++j) asm volatile("" : "+v"(qf[k][j][0]), "+v"(qf[k][j][1]), "+v"(qf[k][j][2]), "+v"(qf[k][j][3]));
}

}  // namespace
}  // namespace tasp
