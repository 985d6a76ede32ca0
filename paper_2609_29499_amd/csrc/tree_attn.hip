// Attention of drafted tokens over a cache whose sequences have their own lengths: node t of a
// sequence with L cached rows sees rows 0 .. L - 1, its ancestors' rows L + j and its own.
//
// o = softmax(scale q K^T) V per query head; a sequence's nodes and the query heads of one cache head
// form the rows of one product, row = node * group + head, so each K and V row is read once for all
// of them. A wave holds 16 of these rows and walks cache rows in steps of 32, straight from memory in the
// matrix instructions' layout (v_mfma_f32_16x16x32_bf16):
//   * S^T = K Q^T: lane (r, c) holds cache row r of a tile of 16 and, of its dimensions, the pieces that 16
//     bytes at 16 c of each 64 give (any order serves that q shares); it gets the scores of query row r
//     against cache rows 4 c .. 4 c + 3: P stays in registers, and is the A operand of
//   * O += P V over the step's two tiles: lane (r, c) loads cache rows 4 c .. 4 c + 3 of both tiles, dh / 16
//     dimensions from dh / 16 * r on, as whole coalesced rows, and turns them in registers (two rows' halves per
//     v_perm) into the operand's columns of eight rows. The output's dimensions are then dh / 16 * r + i: again
//     neighbours, so rows are stored whole. No LDS is used before the waves' results meet.
// Rows in 8 bits become BF16 exactly; their scales multiply scores and probabilities in 32 bits. P is
// carried as two BF16 terms (16 bits; one alone would double the error of a BF16 output), float32 q and P
// as three (24 bits, as exact as the products' float32 sums).
//
// Softmax with a running maximum per query row, raised only when a score passes it by 8 powers of two (sums
// are float32, so the slack costs no accuracy): most steps exchange nothing between lanes.
//
// The cache rows of all sequences are cut into chunks of equal length (from the lengths on the device: no
// host knows them), a workgroup takes one chunk of one cache head, its four waves every fourth
// step. Sequences of one chunk are written at once; the others leave (maximum, sum, unnormalised output)
// per query row in the workspace, which a second launch joins in chunk order.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

constexpr int kStep = 32;              // cache rows per step
constexpr int kMinSteps = 4;           // steps of a chunk at least: one per wave
constexpr float kSlack = 8.0f;         // powers of two a score may pass the running maximum by

// ---- which rows a workgroup serves
// Sequence b has steps(b) = ceil((L + T) / 32) steps and is cut in chunks of `chunk` steps. A wave holds four
// sequences per lane.
// How a call is launched: query rows in rb blocks of 16 mt, `target` workgroups aimed at, at most `most`
// chunks per sequence (what the workspace has room for), grid workgroups.
struct TreeShape {
  int mt, rb, target, most, grid;
};
struct Deal {
  int chunk;                           // steps per chunk
  int total;                           // chunks of all sequences
  int mine[4], before[4];              // of the lane's sequences: chunks, and chunks before them
};
__device__ __forceinline__ int steps_of(const TreeAttnArgs& a, int b) {
  const int L = b < a.c.batch ? seq_len(a.c.len, b, a.c.S) : -2;
  if (L == -2) return 0;               // no such sequence
  return L < 0 ? 1 : (min(L + a.T, a.c.S) + kStep - 1) / kStep;
}
__device__ __forceinline__ Deal deal(const TreeAttnArgs& a, const TreeShape& y, int lane) {
  Deal d;
  int n[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    n[i] = steps_of(a, 4 * lane + i);
    sum += n[i];
  }
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) sum += __shfl_xor(sum, k, kWave);
  const int chunk = max(kMinSteps, int((long(sum) * a.c.n_kv * y.rb + y.target - 1) / y.target));
  d.chunk = (chunk + 3) / 4 * 4;
  int own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d.mine[i] = min((n[i] + d.chunk - 1) / d.chunk, y.most);
    d.before[i] = own;
    own += d.mine[i];
  }
  int inc = own;
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) {
    const int o = __shfl_up(inc, k, kWave);
    if (lane >= k) inc += o;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) d.before[i] += inc - own;
  d.total = __builtin_amdgcn_readlane(inc, kWave - 1);
  return d;
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

template <int DH, int TYPE>
struct Rows32 {                        // a step's K and V as loaded
  static constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  static constexpr int KW = DH * ES / 64;          // 16-byte pieces of K per lane and tile
  static constexpr int VW = DH * ES / 64;          // words of V per lane and row: dh / 16 elements
  uint32_t k[2][KW][4];
  uint32_t v[8][VW];                   // rows 4 c + i of the first tile, then of the second
  float ks[8], vs[8];
};

// Waves per SIMD that the registers of MT tiles leave room for
template <int DH, int TYPE, int ACT, int MT>
constexpr int kWavesPerSimd = MT == 4 || (MT == 2 && DH == 128 && (TYPE == SEQ_BF16 || ACT == SEQ_F32)) ? 1 : 2;

// MT: tiles of 16 query rows per wave
template <int DH, int TYPE, int ACT, int MT>
__global__ __launch_bounds__(kBlock, (kWavesPerSimd<DH, TYPE, ACT, MT>)) void tree_attn_kernel(TreeAttnArgs a, TreeShape y) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  constexpr int NKC = DH / 32;         // score products per tile
  constexpr int NDT = DH / 16;         // dimensions per lane of V and O
  constexpr int QT = ACT == SEQ_F32 ? 3 : 1, PT = ACT == SEQ_F32 ? 3 : 2;
  using Rows = Rows32<DH, TYPE>;
  __shared__ float s_o[4][16][DH + 4];
  __shared__ float s_m[4][16 * MT], s_l[4][16 * MT];
  __shared__ int s_odd;                // a tree's row holds something not finite

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 15, c = lane >> 4;
  const int units = a.c.n_kv * y.rb;
  const Deal d = deal(a, y, lane);
  // workgroup -> row block (slowest), chunk of a sequence, cache head
  const int w = blockIdx.x;
  if (w >= d.total * units) return;
  const int g = w % a.c.n_kv, ch_all = (w / a.c.n_kv) % d.total, rb = w / (a.c.n_kv * d.total);
  int hit = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (ch_all >= d.before[i] && ch_all < d.before[i] + d.mine[i]) hit = i;
  const int owner = __ffsll((long long)__ballot(hit >= 0)) - 1;
  const int sub = __builtin_amdgcn_readlane(hit, owner);
  const int b = 4 * owner + sub;
  const int before = __builtin_amdgcn_readlane(sub == 0 ? d.before[0] : sub == 1 ? d.before[1] : sub == 2 ? d.before[2] : d.before[3], owner);
  const int n_ch = __builtin_amdgcn_readlane(sub == 0 ? d.mine[0] : sub == 1 ? d.mine[1] : sub == 2 ? d.mine[2] : d.mine[3], owner);
  const int ch = ch_all - before;

  const int L = seq_len(a.c.len, b, a.c.S);
  const int Lr = max(L, 0);                            // cached rows (none of a sequence passed over)
  const int end = L < 0 ? 0 : min(L + a.T, a.c.S);     // rows that may be read
  const int steps = (end + kStep - 1) / kStep;
  // the last chunk of a sequence takes what is left (with `most` chunks that may be more than a chunk)
  const int per = n_ch * d.chunk >= steps ? d.chunk : ((steps + n_ch - 1) / n_ch + 3) / 4 * 4;
  const int s0 = ch * per, s1 = ch == n_ch - 1 ? steps : min(steps, s0 + per);
  // steps from s_edge on hold rows of the tree: at most three, so a wave has one at most
  const int s_edge = min(Lr / kStep, s1);

  const size_t unit = size_t(b) * a.c.n_kv + g;
  const uint32_t row_bytes = DH * ES;
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char*>(a.c.k) + unit * a.c.S * row_bytes, uint32_t(end) * row_bytes);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const char*>(a.c.v) + unit * a.c.S * row_bytes, uint32_t(end) * row_bytes);
  const __amdgpu_buffer_rsrc_t rks = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.ks + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);
  const __amdgpu_buffer_rsrc_t rvs = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.vs + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);

  // Steps are loaded one ahead. Rows past `end`, and steps past `stop`, read as zeros without touching memory.
  auto load = [&](int s, int stop, Rows& x) {
    const uint32_t t0 = uint32_t(s) * kStep;
    const bool in = s < stop;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int j = 0; j < Rows::KW; ++j) {
        const int4 p = buf_load16_stream(rk, in ? (t0 + 16 * tt + r) * row_bytes + 64u * j + 16u * c : kOOB);
        x.k[tt][j][0] = p.x; x.k[tt][j][1] = p.y; x.k[tt][j][2] = p.z; x.k[tt][j][3] = p.w;
      }
    if constexpr (TYPE != SEQ_BF16) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const uint32_t off = in ? (t0 + 16 * tt + 4 * c) * 4u : kOOB;
        const float4 p = __builtin_bit_cast(float4, buf_load16(rks, off));
        const float4 q = __builtin_bit_cast(float4, buf_load16(rvs, off));
        x.ks[4 * tt] = p.x; x.ks[4 * tt + 1] = p.y; x.ks[4 * tt + 2] = p.z; x.ks[4 * tt + 3] = p.w;
        x.vs[4 * tt] = q.x; x.vs[4 * tt + 1] = q.y; x.vs[4 * tt + 2] = q.z; x.vs[4 * tt + 3] = q.w;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t off = in ? (t0 + 16 * (i >> 2) + 4 * c + (i & 3)) * row_bytes + uint32_t(NDT * ES) * r : kOOB;
      if constexpr (Rows::VW == 4) {
        const int4 p = buf_load16_stream(rv, off);
        x.v[i][0] = p.x; x.v[i][1] = p.y; x.v[i][2] = p.z; x.v[i][3] = p.w;
      } else if constexpr (Rows::VW == 2) {
        const auto p = __builtin_amdgcn_raw_buffer_load_b64(rv, int(off), 0, kCpolStream);
        x.v[i][0] = p[0]; x.v[i][1] = p[1];
      } else {
        x.v[i][0] = __builtin_amdgcn_raw_buffer_load_b32(rv, int(off), 0, kCpolStream);
      }
    }
  };
  const int s_own = s0 + wave;                         // this wave's steps: s_own, s_own + 4, ..
  const int s_late = s_own + max(0, (s_edge - s_own + 3) / 4) * 4;   // its first step at or behind s_edge
  const bool has_edge = s_late < s1;
  Rows xa, xb;
  load(s_late, s1, xa);
  load(s_own, s_edge, xb);

  // this lane's query rows, as rows of Q (B operand): node t, head h
  const int R = a.T * a.group;
  const TreeNode nd = tree_node(a.parent ? a.parent + size_t(b) * a.T : nullptr, a.T, L < 0 ? 0 : a.c.S - L, lane);
  unsigned long long anc[MT];
  uint32_t qf[MT][QT][NKC][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = min((rb * MT + mt) * 16 + r, R - 1);   // (rows past the last one repeat it and are not stored)
    const int t = row / a.group, h = g * a.group + row % a.group;
    anc[mt] = __shfl(nd.anc, t, kWave);
    const long at = b * a.q.seq + t * a.q.token + h * a.q.head;
#pragma unroll
    for (int kk = 0; kk < NKC; ++kk) {
      const int dim = ES == 2 ? 32 * kk + 8 * c : 64 * (kk >> 1) + 16 * c + 8 * (kk & 1);
      if constexpr (ACT == SEQ_BF16) {
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q.p) + at + dim);
        qf[mt][0][kk][0] = x.x; qf[mt][0][kk][1] = x.y; qf[mt][0][kk][2] = x.z; qf[mt][0][kk][3] = x.w;
      } else {
        const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(a.q.p) + at + dim);
        const float4 x = f[0], z = f[1];
        uint32_t* o = &qf[mt][0][kk][0];
        terms<QT>(x.x, x.y, o, NKC * 4);
        terms<QT>(x.z, x.w, o + 1, NKC * 4);
        terms<QT>(z.x, z.y, o + 2, NKC * 4);
        terms<QT>(z.z, z.w, o + 3, NKC * 4);
      }
    }
  }

  float m_run[MT], l_run[MT];                          // of query row r; l of this lane's cache rows
  f32x4 o[MT][NDT];                                    // lane (r, c): query rows 4 c + i, dimension NDT r + d
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = -INFINITY;
    l_run[mt] = 0.0f;
#pragma unroll
    for (int i = 0; i < NDT; ++i) o[mt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  auto process = [&](Rows& x, int s, auto edge_) {
    constexpr bool EDGE = decltype(edge_)::value;
    f32x4 sc[MT][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sc[mt][tt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < NKC; ++kk) {
        uint32_t kf[4];
        if constexpr (TYPE == SEQ_BF16) {
#pragma unroll
          for (int e = 0; e < 4; ++e) kf[e] = x.k[tt][kk][e];
        } else {
          widen<TYPE>(x.k[tt][kk >> 1][2 * (kk & 1)], kf);
          widen<TYPE>(x.k[tt][kk >> 1][2 * (kk & 1) + 1], kf + 2);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int q = 0; q < QT; ++q) sc[mt][tt] = mfma(kf, qf[mt][q][kk], sc[mt][tt]);
      }
    }
    uint32_t pf[MT][PT][4];
    float ks[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) ks[i] = TYPE == SEQ_BF16 ? a.scale2 : x.ks[i] * a.scale2;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = sc[mt][i >> 2][i & 3] * ks[i];
      uint32_t seen = 0xffu;                           // of the lane's eight cache rows
      if constexpr (EDGE) {
        seen = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = s * kStep + 16 * (i >> 2) + 4 * c + (i & 3) - Lr;
          const bool in = j < 0 || (j < kTreeMax && ((anc[mt] >> (j & 63)) & 1));
          seen |= uint32_t(in) << i;
          p[i] = in ? p[i] : -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
      if (__ballot(top > m_run[mt] + kSlack)) {        // (also the first rows: m_run is -inf)
        const float mn = fmaxf(m_run[mt], quad_max(top));
        const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[mt] - mn);
        m_run[mt] = mn;
        l_run[mt] *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = __shfl(alpha, 4 * c + i, kWave);
#pragma unroll
          for (int e = 0; e < NDT; ++e) o[mt][e][i] *= f;
        }
      }
      const float base = m_run[mt] == -INFINITY ? 0.0f : m_run[mt];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(p[i] - base);
        l_run[mt] += p[i];
        if constexpr (TYPE != SEQ_BF16) p[i] *= EDGE && !((seen >> i) & 1) ? 0.0f : x.vs[i];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) terms<PT>(p[2 * e], p[2 * e + 1], &pf[mt][0][e], 4);
    }
    // V: eight rows of NDT dimensions as BF16 pairs
    uint32_t v[8][NDT / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (TYPE == SEQ_BF16) {
#pragma unroll
        for (int e = 0; e < NDT / 2; ++e) v[i][e] = x.v[i][e];
      } else {
#pragma unroll
        for (int e = 0; e < NDT / 4; ++e) widen<TYPE>(x.v[i][e], &v[i][2 * e]);
      }
    }
    // A row of the tree that some nodes do not see must not reach them through 0 * inf: non-finite values of
    // the tree's rows are left out of the product, and added at the end to the outputs that see them
    if constexpr (EDGE && TYPE != SEQ_INT8) {
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < NDT / 2; ++e) {
          const uint32_t top = ((v[i][e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // a half's exponent is full
          bad |= top;
          v[i][e] &= ~((top >> 15) * 0xffffu);
        }
      if (bad) s_odd = 1;
    }
#pragma unroll
    for (int e = 0; e < NDT; ++e) {
      const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
      uint32_t vb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) vb[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], sel);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int k = 0; k < PT; ++k) o[mt][e] = mfma(pf[mt][k], vb, o[mt][e]);
    }
  };
  if constexpr (TYPE != SEQ_INT8) {
    if (tid == 0) s_odd = 0;
    __syncthreads();
  }
  if (has_edge) process(xa, s_late, std::true_type{});
  for (int s = s_own; s < s_edge; s += 8) {
    load(s + 4, s_edge, xa);
    process(xb, s, std::false_type{});
    if (s + 4 >= s_edge) break;
    load(s + 8, s_edge, xb);
    process(xa, s + 4, std::false_type{});
  }

  // the four waves' results, 16 query rows at a time
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float l_all = quad_sum(l_run[mt]);
    if (c == 0) {
      s_m[wave][16 * mt + r] = m_run[mt];
      s_l[wave][16 * mt + r] = l_all;
    }
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    if (mt > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < NDT; e += 4)
        *reinterpret_cast<float4*>(&s_o[wave][4 * c + i][NDT * r + e]) = make_float4(o[mt][e][i], o[mt][e + 1][i], o[mt][e + 2][i], o[mt][e + 3][i]);
    __syncthreads();
    // thread: query row tid / 16 of the tile, dimensions NDT (tid % 16) ..
    const int qr = tid >> 4, d0 = NDT * (tid & 15);
    float m = -INFINITY, l = 0.0f, f[4], v[NDT];
#pragma unroll
    for (int k = 0; k < 4; ++k) m = fmaxf(m, s_m[k][16 * mt + qr]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // (a wave that saw only rows scored -inf or none holds zeros; NaN stays)
      f[k] = s_m[k][16 * mt + qr] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s_m[k][16 * mt + qr] - m);
      l += s_l[k][16 * mt + qr] * f[k];
    }
#pragma unroll
    for (int e = 0; e < NDT; ++e) {
      v[e] = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[e] += s_o[k][qr][d0 + e] * f[k];
    }
    const int row_o = (rb * MT + mt) * 16 + qr;
    const int t_o = min(row_o, R - 1) / a.group;
    const unsigned long long anc_o = __shfl(nd.anc, t_o, kWave);
    const bool there = anc_o != 0;     // (a row of an absent node is zeros)
    if (row_o >= R) continue;
    if constexpr (TYPE != SEQ_INT8) {
      if (s_odd) {
        for (int j = max(0, max(s_edge, s0) * kStep - Lr); j < a.T && Lr + j < s1 * kStep; ++j) {
          if (!((anc_o >> j) & 1)) continue;
          const char* row = static_cast<const char*>(a.c.v) + (unit * a.c.S + Lr + j) * row_bytes + d0 * ES;
#pragma unroll
          for (int e = 0; e < NDT; ++e) {
            const float x = TYPE == SEQ_BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[e])
                                             : (row[e] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
            if (!(fabsf(x) < INFINITY)) v[e] += x;
          }
        }
      }
    }
    if (n_ch == 1) {
      const float inv = there && l != 0.0f ? 1.0f / l : 0.0f;
      const long at = b * a.o.seq + t_o * a.o.token + (g * a.group + row_o % a.group) * a.o.head + d0;
#pragma unroll
      for (int e = 0; e < NDT; e += 4) {
        float z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = there && l != 0.0f ? v[e + i] * inv : 0.0f;
        if constexpr (ACT == SEQ_BF16)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.p) + at + e) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
        else
          *reinterpret_cast<float4*>(static_cast<float*>(a.o.p) + at + e) = make_float4(z[0], z[1], z[2], z[3]);
      }
    } else {
      const size_t rec = ((size_t(ch_all) * a.c.n_kv + g) * y.rb + rb) * MT + mt;
      float* po = a.ws + (rec * 16 + qr) * (DH + 4);
      if (d0 == 0) {
        po[DH] = m;
        po[DH + 1] = there ? l : 0.0f;
      }
#pragma unroll
      for (int e = 0; e < NDT; e += 4)
        *reinterpret_cast<float4*>(po + d0 + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
  }
}

// Joins the chunks' records of one query row: 32 lanes over the dimensions, eight groups over the
// chunks. Grid (query rows of a sequence, sequences).
template <int DH, int ACT>
__global__ __launch_bounds__(kBlock) void tree_join_kernel(TreeAttnArgs a, TreeShape y) {
  constexpr int E = DH / 32;           // dimensions per lane
  __shared__ float s_m[8], s_l[8], s_o[8][DH];
  const int tid = threadIdx.x, lane = tid & 63;
  const int b = blockIdx.y;
  const Deal d = deal(a, y, lane);
  const int sub = b & 3;
  const int n = __builtin_amdgcn_readlane(sub == 0 ? d.mine[0] : sub == 1 ? d.mine[1] : sub == 2 ? d.mine[2] : d.mine[3], b >> 2);
  const int before = __builtin_amdgcn_readlane(sub == 0 ? d.before[0] : sub == 1 ? d.before[1] : sub == 2 ? d.before[2] : d.before[3], b >> 2);
  if (n <= 1) return;                  // written already
  const int t = blockIdx.x / a.n_q, h = blockIdx.x % a.n_q;
  const int g = h / a.group, row = t * a.group + h % a.group;
  const int grp = tid >> 5, d0 = E * (tid & 31);
  float m = -INFINITY, l = 0.0f, v[E] = {};
  for (int k = grp; k < n; k += 8) {
    const size_t rec = (size_t(before + k) * a.c.n_kv + g) * y.rb * y.mt + row / 16;
    const float* po = a.ws + (rec * 16 + row % 16) * (DH + 4);
    const float mk = po[DH], lk = po[DH + 1];
    const float mn = fmaxf(m, mk);
    const float fa = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    const float fb = mk == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mk - mn);
    m = mn;
    l = l * fa + lk * fb;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = v[e] * fa + po[d0 + e] * fb;
  }
  if ((tid & 31) == 0) {
    s_m[grp] = m;
    s_l[grp] = l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[grp][d0 + e] = v[e];
  __syncthreads();
  if (tid >= DH / 2) return;
  float mm = -INFINITY, ll = 0.0f, y0 = 0.0f, y1 = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) mm = fmaxf(mm, s_m[k]);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float f = s_m[k] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s_m[k] - mm);
    ll += s_l[k] * f;
    y0 += s_o[k][2 * tid] * f;
    y1 += s_o[k][2 * tid + 1] * f;
  }
  const bool any = ll != 0.0f;
  y0 = any ? y0 / ll : 0.0f;
  y1 = any ? y1 / ll : 0.0f;
  const long at = b * a.o.seq + t * a.o.token + h * a.o.head + 2 * tid;
  if constexpr (ACT == SEQ_BF16)
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.o.p) + at) = pack_bf16(y0, y1);
  else
    *reinterpret_cast<float2*>(static_cast<float*>(a.o.p) + at) = make_float2(y0, y1);
}

TreeShape shape(const TreeAttnArgs& a) {
  TreeShape y;
  const int tiles = (a.T * a.group + 15) / 16;
  y.mt = a.act == SEQ_F32 ? std::min(tiles, 2) : tiles > 2 ? 4 : tiles;
  y.rb = (tiles + y.mt - 1) / y.mt;
  y.target = y.mt == 4 ? 256 : 512;    // workgroups of four tiles fill a CU's registers alone
  const int units = a.c.n_kv * y.rb;
  const long steps = (std::min<long>(std::max(a.max_len, 0) + long(a.T), a.c.S) + kStep - 1) / kStep;
  y.most = int(std::max<long>(1, std::min<long>((steps + kMinSteps - 1) / kMinSteps, (y.target + units - 1) / units)));
  // chunks of all sequences: their steps over the chunk's, rounded up per sequence
  const long chunks = std::min<long>(long(a.c.batch) * y.most, y.target / units + 1 + a.c.batch);
  y.grid = int(chunks * units);
  return y;
}

}  // namespace

size_t tree_attn_workspace_bytes(const TreeAttnArgs& a) {
  const TreeShape y = shape(a);
  return y.most == 1 ? 0 : size_t(y.grid) * y.mt * 16 * (a.c.dh + 4) * 4;
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t s) {
  const TreeShape y = shape(a);
#define ATTN(DH, TYPE, ACT, MT) hipLaunchKernelGGL((tree_attn_kernel<DH, TYPE, ACT, MT>), dim3(y.grid), dim3(kBlock), 0, s, a, y)
#define ATTN_MT(DH, TYPE, ACT)                                            \
  do {                                                                    \
    if (y.mt == 1) ATTN(DH, TYPE, ACT, 1);                                \
    else if (y.mt == 2) ATTN(DH, TYPE, ACT, 2);                           \
    else if constexpr (ACT == SEQ_BF16) ATTN(DH, TYPE, ACT, 4);           \
  } while (0)
#define ATTN_TYPE(DH, ACT)                                      \
  do {                                                          \
    if (a.c.type == SEQ_BF16) ATTN_MT(DH, SEQ_BF16, ACT);       \
    else if (a.c.type == SEQ_INT8) ATTN_MT(DH, SEQ_INT8, ACT);  \
    else ATTN_MT(DH, SEQ_E4M3, ACT);                            \
  } while (0)
  if (a.c.dh == 128) {
    if (a.act == SEQ_BF16) ATTN_TYPE(128, SEQ_BF16);
    else ATTN_TYPE(128, SEQ_F32);
  } else {
    if (a.act == SEQ_BF16) ATTN_TYPE(64, SEQ_BF16);
    else ATTN_TYPE(64, SEQ_F32);
  }
#undef ATTN_TYPE
#undef ATTN_MT
#undef ATTN
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || y.most == 1) return e;
#define JOIN(DH, ACT) hipLaunchKernelGGL((tree_join_kernel<DH, ACT>), dim3(a.T * a.n_q, a.c.batch), dim3(kBlock), 0, s, a, y)
  if (a.c.dh == 128) {
    if (a.act == SEQ_BF16) JOIN(128, SEQ_BF16);
    else JOIN(128, SEQ_F32);
  } else {
    if (a.act == SEQ_BF16) JOIN(64, SEQ_BF16);
    else JOIN(64, SEQ_F32);
  }
#undef JOIN
  return hipGetLastError();
}

}  // namespace tasp
