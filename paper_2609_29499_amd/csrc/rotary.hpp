// Head vectors of eight elements per lane, and rotary positions: what the kernels that write cache rows share.
#pragma once
#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

constexpr int kE = 8;                  // elements of a head per lane

struct Vec8 {
  float v[kE];
};

template <int ACT>
__device__ __forceinline__ Vec8 load8(const void* p, long at) {
  Vec8 x;
  if constexpr (ACT == SEQ_BF16) {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.v[2 * i] = bf16_lo(u[i]);
      x.v[2 * i + 1] = bf16_hi(u[i]);
    }
  } else {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = f[0], b = f[1];
    x.v[0] = a.x; x.v[1] = a.y; x.v[2] = a.z; x.v[3] = a.w;
    x.v[4] = b.x; x.v[5] = b.y; x.v[6] = b.z; x.v[7] = b.w;
  }
  return x;
}

// the same of a sum of arrays (a projection's splits), in their order
template <int ACT, class Args>
__device__ __forceinline__ Vec8 load8(const void* p, long at, const Args& a) {
  Vec8 x = load8<ACT>(p, at);
  if constexpr (ACT == SEQ_F32)
    for (int z = 1; z < a.ks; ++z) {
      const Vec8 y = load8<ACT>(p, at + z * a.split);
#pragma unroll
      for (int i = 0; i < kE; ++i) x.v[i] += y.v[i];
    }
  return x;
}

template <int ACT>
__device__ __forceinline__ void store8(void* p, long at, const Vec8& x) {
  if constexpr (ACT == SEQ_BF16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) =
        make_uint4(pack_bf16(x.v[0], x.v[1]), pack_bf16(x.v[2], x.v[3]), pack_bf16(x.v[4], x.v[5]), pack_bf16(x.v[6], x.v[7]));
  } else {
    float4* f = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
    f[0] = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
    f[1] = make_float4(x.v[4], x.v[5], x.v[6], x.v[7]);
  }
}

// Sine and cosine of pos * freq: turns = pos freq / 2 pi is formed and cut to [-1/2, 1/2] in 64 bits;
// what a 32-bit angle loses of it (d) is put back to first order.
__device__ __forceinline__ float2 turn(double pos, double freq, float m) {
  double a = pos * (freq * 0.15915494309189533577);
  a -= rint(a);
  a *= 6.28318530717958647693;
  const float x = float(a), d = float(a - double(x));
  float s, c;
  sincosf(x, &s, &c);
  return make_float2(fmaf(-s, d, c) * m, fmaf(c, d, s) * m);
}

// frequency of pair i (the launch's arguments hold what it is formed of: SeqAppendArgs)
template <class Args>
__device__ __forceinline__ double pair_freq(const Args& a, int i) {
  double f = 1.0;
#pragma unroll
  for (int k = 0; k < 6; ++k) f *= (i >> k) & 1 ? a.power[k] : 1.0;
  const double g = fmin(fmax(fma(a.by_index ? double(i) : f, a.mul, a.add), 0.0), 1.0);
  return f * fma(1.0 - g, a.keep, g);
}

}  // namespace
}  // namespace tasp
