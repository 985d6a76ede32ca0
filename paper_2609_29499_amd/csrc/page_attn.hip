// Causal attention of packed new tokens over caches in pages: token i of a sequence that held L rows sees rows 0 .. L + i.
//
// o = softmax(scale q K^T) V per query head; a sequence's tokens and the query heads of one cache head form the rows of
// one product, row = token * group + head, so each K and V row is read once for a block of them. Tiles of 16 query rows by
// 32 cache rows (a step) run on v_mfma_f32_16x16x32_bf16:
//   * S^T = K Q^T: lane (r, c) gets the scores of query row r against cache rows 4 c .. 4 c + 3 of each tile of
//     16: P stays in registers, and is the A operand of
//   * O += P V over the step's two tiles: lane (r, c) holds cache rows 4 c .. 4 c + 3 of both tiles, dh / 16
//     dimensions from dh / 16 * r on.
// Pages hold 16 rows or a multiple, so a tile of 16 cache rows lies in one page: its address and its scale are the same
// for all lanes. Codes become BF16 exactly; the scales multiply scores and probabilities in 32 bits. P is carried as two BF16
// terms (16 bits; one alone would double the error of a BF16 output), float32 q and P as three (24 bits).
//
// Softmax with a running maximum per query row, raised only when a score passes it by 8 powers of two (sums are
// float32, so the slack costs no accuracy): most steps exchange nothing between lanes.
//
// The cache rows of all sequences are cut into chunks of equal length (from the lengths on the device: no host knows
// them); a workgroup takes one chunk of one cache head. A sequence of one chunk is written at once; the others leave
// (maximum, sum, unnormalised output) per query row in the workspace, which a second launch joins in chunk order.
#include <algorithm>
#include <type_traits>

#include "attn_tiles.hpp"
#include "device_common.hpp"
#include "page.hpp"

namespace tasp {
namespace {

constexpr int kStep = 32;              // cache rows per step
constexpr int kMinSteps = 4;           // steps of a chunk at least, and its granule: one per wave
constexpr float kSlack = 8.0f;         // powers of two a score may pass the running maximum by
constexpr int kTarget = 512;           // workgroups aimed at: two per CU

// How a call is launched: query rows in blocks of `rows`, at most rb of them in a sequence that is cut; chunks of all
// sequences, `room` at most; items: of the grid
struct PageShape {
  int mt, rows, rows_log, rb, room, items, cut;
};
struct Deal {
  int chunk, total;                    // steps per chunk; chunks of all sequences
  int mine[4], before[4];              // of the lane's sequences: chunks, and those of the sequences before them
  int first[4], n[4], len[4];
};
// A lane holds four sequences. The chunk is the shortest multiple of kMinSteps that leaves at most `room` chunks.
__device__ __forceinline__ Deal deal(const PageAttnArgs& a, const PageShape& y, int lane) {
  Deal d;
  int steps[4], sum = 0, most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const PageSeq q = page_seq(a.start, a.N, a.c, min(4 * lane + i, a.c.batch - 1));
    d.first[i] = q.first; d.len[i] = q.L;
    d.n[i] = 4 * lane + i < a.c.batch ? q.n : 0;
    const int end = q.L < 0 ? 0 : min(q.L + d.n[i], a.c.cap);
    steps[i] = d.n[i] == 0 ? 0 : max(1, (end + kStep - 1) / kStep);
    sum += steps[i];
    most = max(most, steps[i]);
  }
  sum = __builtin_amdgcn_readlane(wave_scan(sum), kWave - 1);
  most = int(wave_max(float(most)));   // (below 2^24)
  auto count = [&](int chunk, int i, float inv) {
    return d.n[i] * a.group > y.rb * y.rows || !y.cut ? min(steps[i], 1) : quot_steps(steps[i] + chunk - 1, chunk, inv);
  };
  auto total = [&](int chunk) {
    const float inv = __builtin_amdgcn_rcpf(float(chunk));
    int own = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) own += count(chunk, i, inv);
    return __builtin_amdgcn_readlane(wave_scan(own), kWave - 1);
  };
  // in units of kMinSteps: lo may do, hi does
  int lo = max(1, ((sum + y.room - 1) / y.room + kMinSteps - 1) / kMinSteps), hi = max(lo, (most + kMinSteps - 1) / kMinSteps);
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (total(mid * kMinSteps) <= y.room) hi = mid;
    else lo = mid + 1;
  }
  d.chunk = lo * kMinSteps;
  const float inv = __builtin_amdgcn_rcpf(float(d.chunk));
  int own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d.mine[i] = count(d.chunk, i, inv);
    d.before[i] = own;
    own += d.mine[i];
  }
  const int all = wave_scan(own);
#pragma unroll
  for (int i = 0; i < 4; ++i) d.before[i] += all - own;
  d.total = __builtin_amdgcn_readlane(all, kWave - 1);
  return d;
}

// The part of the work that a workgroup takes.
struct Place {
  int b, g, head;                      // sequence, slot, its cache head
  int h0, group, R;                    // the slot's first query head, its heads, its query rows
  int n_ch, ch, before;                // chunks of the sequence, this one, those of the sequences before
  int first, n, L, end;                // its tokens, rows it held (-1: passed over), rows that may be read
  int s0, s1;                          // steps
};
__device__ __forceinline__ bool place(const PageAttnArgs& a, const PageShape& y, int lane, Place& p) {
  const int item = blockIdx.z * 8 + blockIdx.x, all = quot(item, a.slots);
  p.g = item - all * a.slots;
  const int slot = a.slot[p.g];
  const Deal d = deal(a, y, lane);
  if (all >= d.total) return false;
  int hit = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (all >= d.before[i] && all < d.before[i] + d.mine[i]) hit = i;
  const int owner = __builtin_amdgcn_readfirstlane(__ffsll((long long)__ballot(hit >= 0)) - 1), sub = __builtin_amdgcn_readlane(hit, owner);
  p.b = 4 * owner + sub;
  p.head = slot & 0xff;
  p.h0 = slot >> 8 & 0xfff;
  p.group = slot >> 20;
  p.first = pick(d.first, owner, sub);
  p.n = pick(d.n, owner, sub);
  p.L = pick(d.len, owner, sub);
  p.R = p.n * p.group;
  p.n_ch = pick(d.mine, owner, sub);
  p.before = pick(d.before, owner, sub);
  p.ch = all - p.before;
  p.end = p.L < 0 ? 0 : min(p.L + p.n, a.c.cap);
  const int steps = (p.end + kStep - 1) / kStep;
  p.s0 = p.ch * d.chunk;
  p.s1 = p.n_ch == 1 ? steps : min(steps, p.s0 + d.chunk);
  return true;
}

// One query row's output values (unnormalised) with their sum l: token t (of all), head h from dimension d0 on. there: the
// token is present.
template <int DH, int ACT, int N>
__device__ __forceinline__ void put_output(const PageAttnArgs& a, int t, int h, int d0, float l, bool there, const float (&v)[N]) {
  const float inv = there && l != 0.0f ? 1.0f / l : 0.0f;
  const long at = t * a.o.token + h * a.o.head + d0;
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = there && l != 0.0f ? v[e + i] * inv : 0.0f;
    if constexpr (ACT == SEQ_BF16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.p) + at + e) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(a.o.p) + at + e) = make_float4(z[0], z[1], z[2], z[3]);
  }
}

// The workspace: of each sequence (chunks, chunks of the sequences before, its first token, its tokens), then records of
// [rows][DH] outputs and [rows] (maximum, sum), [chunk][slot][block].
constexpr size_t kHeadFloats = 4 * kSeqMaxBatch;
__device__ __forceinline__ float* record(const PageAttnArgs& a, const PageShape& y, int chunk, int g, int rb) {
  return a.ws + kHeadFloats + ((size_t(chunk) * a.slots + g) * y.rb + rb) * (size_t(y.rows) * (a.c.dh + 2));
}

template <int DH, int TYPE>
struct Rows32 {                        // a step's K and V as loaded
  static constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  static constexpr int KW = DH * ES / 64;          // 16-byte pieces of K per lane and tile
  static constexpr int VW = DH * ES / 64;          // words of V per lane and row: dh / 16 elements
  uint32_t k[2][KW][4];
  uint32_t v[8][VW];                   // rows 4 c + i of the first tile, then of the second
  float ks[2], vs[2], bias[2];         // of the tiles' pages
};

// A query row's operand: from `at` on (elements from q.p) 8 values for each of dh / 32 products, those of product kk
// 32 kk further on, or (PAIRED) 64 floor(kk / 2) + 8 (kk mod 2)
template <int DH, int ACT, int QT, bool PAIRED>
__device__ __forceinline__ void load_q(const void* q, long at0, uint32_t (&qf)[QT][DH / 32][4]) {
#pragma unroll
  for (int kk = 0; kk < DH / 32; ++kk) {
    const long at = at0 + (PAIRED ? 64 * (kk >> 1) + 8 * (kk & 1) : 32 * kk);
    if constexpr (ACT == SEQ_BF16) {
      const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(q) + at);
      qf[0][kk][0] = x.x; qf[0][kk][1] = x.y; qf[0][kk][2] = x.z; qf[0][kk][3] = x.w;
    } else {
      const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(q) + at);
      const float4 x = f[0], z = f[1];
      uint32_t* o = &qf[0][kk][0];
      terms<QT>(x.x, x.y, o, DH / 8);
      terms<QT>(x.z, x.w, o + 1, DH / 8);
      terms<QT>(z.x, z.y, o + 2, DH / 8);
      terms<QT>(z.z, z.w, o + 3, DH / 8);
    }
  }
}

// One query row's scores of a step (lane (r, c): cache rows 4 c + i of both tiles) to the terms of P. bias: 0, or -inf for
// a tile without a page. EDGE: rows of the step may be hidden from some query rows; this one sees its rows below `seen`.
template <int NDT, int PT, bool SCALED, bool EDGE>
__device__ __forceinline__ void soft_step(const f32x4 (&sc)[2], const float (&ks)[2], const float (&vs)[2], const float (&bias)[2], int seen,
                                          int c, float& m_run, float& l_run, f32x4 (&o)[NDT], uint32_t (&pf)[PT][4]) {
  float p[8];
  bool in[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = fmaf(sc[i >> 2][i & 3], ks[i >> 2], bias[i >> 2]);
    in[i] = !EDGE || 16 * (i >> 2) + 4 * c + (i & 3) < seen;
    if constexpr (EDGE) p[i] = in[i] ? p[i] : -INFINITY;
  }
  const float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
  if (__ballot(top > m_run + kSlack)) {                // (also the first rows: m_run is -inf)
    const float mn = fmaxf(m_run, quad_max(top));
    const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run - mn);
    m_run = mn;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = __shfl(alpha, 4 * c + i, kWave);
#pragma unroll
      for (int e = 0; e < NDT; ++e) o[e][i] *= f;
    }
  }
  const float base = m_run == -INFINITY ? 0.0f : m_run;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = __builtin_amdgcn_exp2f(p[i] - base);
    l_run += p[i];
    if constexpr (SCALED) p[i] *= in[i] ? vs[i >> 2] : 0.0f;      // (a hidden row's scale may be anything)
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) terms<PT>(p[2 * e], p[2 * e + 1], &pf[0][e], 4);
}

// Adds the non-finite values that drop_odd left out to one query row's outputs: of the cache rows from .. to - 1.
template <int DH, int TYPE, int N>
__device__ __forceinline__ void add_odd(const PageAttnArgs& a, int b, int head, int from, int to, int d0, float (&v)[N]) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  for (int j = from; j < to; ++j) {
    const int page = a.c.table[size_t(b) * a.c.width + (j >> a.c.P_log)];
    if (page < 0 || page >= a.c.n_pages) continue;
    const size_t row = ((size_t(page) * a.c.n_kv + head) << a.c.P_log) + (j & (a.c.P - 1));
    const char* at = static_cast<const char*>(a.c.v) + (row * DH + d0) * ES;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float x = TYPE == SEQ_BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(at)[e])
                                       : (at[e] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
      if (!(fabsf(x) < INFINITY)) v[e] += x;
    }
  }
}

// Page ids and scales of a chunk: lane i holds those of page base + i, and of page base + 64 + i ahead of their use.
template <int TYPE>
struct PageLane {
  int id;
  float ks, vs;
  __device__ __forceinline__ void fetch(const PageAttnArgs& a, int b, int head, int pg, int pages) {
    id = pg < pages ? a.c.table[size_t(b) * a.c.width + pg] : -1;
    if (id < 0 || id >= a.c.n_pages) id = -1;
    if constexpr (TYPE != SEQ_BF16) {
      const size_t at = size_t(max(id, 0)) * a.c.n_kv + head;
      ks = a.c.ks[at];
      vs = a.c.vs[at];
    }
  }
};

// Waves per SIMD that the registers of MT tiles leave room for
template <int DH, int TYPE, int ACT, int MT>
constexpr int kWavesPerSimd = MT == 2 && DH == 128 && (TYPE == SEQ_BF16 || ACT == SEQ_F32) ? 1 : 2;

// MT: tiles of 16 query rows per wave; every wave holds all of the block's query rows and takes every fourth step of the
// chunk, the next step's loads in flight. Grid (8, row blocks, items / 8).
template <int DH, int TYPE, int ACT, int MT>
__global__ __launch_bounds__(kBlock, (kWavesPerSimd<DH, TYPE, ACT, MT>)) void page_attn_kernel(PageAttnArgs a, PageShape y) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  constexpr int NKC = DH / 32;         // score products per tile
  constexpr int NDT = DH / 16;         // dimensions per lane of V and O
  constexpr int QT = ACT == SEQ_F32 ? 3 : 1, PT = ACT == SEQ_F32 ? 3 : 2;
  using Rows = Rows32<DH, TYPE>;
  constexpr int RB = 16 * MT;
  constexpr uint32_t row_bytes = DH * ES;
  __shared__ float s_o[4][16][DH + 4];
  __shared__ float s_m[4][RB], s_l[4][RB];
  __shared__ int s_odd;                // a row that some query rows do not see holds something not finite

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, c = lane >> 4;
  Place p;
  if (!place(a, y, lane, p)) return;
  if (y.cut && p.ch == 0 && p.g == 0 && blockIdx.y == 0 && tid == 0)
    reinterpret_cast<int4*>(a.ws)[p.b] = make_int4(p.n_ch, p.before, p.first, p.n);
  const int pages = (p.end + a.c.P - 1) >> a.c.P_log;
  const size_t page_bytes = size_t(row_bytes) << a.c.P_log;

  for (int rb = blockIdx.y; rb * RB < p.R; rb += gridDim.y) {
    // rows that all of the block's tokens see, and that any of them does
    const int t_first = quot(rb * RB, p.group), t_last = quot(min(p.R, rb * RB + RB) - 1, p.group);
    const int common = p.L < 0 ? 0 : min(p.L + t_first + 1, p.end), end = p.L < 0 ? 0 : min(p.L + t_last + 1, p.end);
    const int s1 = min(p.s1, (end + kStep - 1) / kStep);

    // steps from s_edge on hold rows that some tokens do not see: at most three, so a wave has one at most
    const int s_own = p.s0 + wave;     // this wave's steps: s_own, s_own + 4, ..
    const int s_edge = min(common / kStep, s1), s_late = s_own + max(0, (s_edge - s_own + 3) / 4) * 4;
    const bool has_edge = s_late < s1;
    int base = p.s0 * kStep >> a.c.P_log;
    // Rows of a step, of the pages that ids holds from page `from` on. Rows past `end`, and of steps past `stop`, read as
    // zeros without touching memory.
    auto load = [&](int s, int stop, const PageLane<TYPE>& ids, int from, Rows& x) __attribute__((always_inline)) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int row = s * kStep + 16 * tt, at = (row >> a.c.P_log) - from, in_page = row & (a.c.P - 1);
        const int id = __builtin_amdgcn_readlane(ids.id, at);
        x.bias[tt] = id >= 0 ? 0.0f : -INFINITY;
        x.ks[tt] = id >= 0 ? a.scale2 : 0.0f;
        x.vs[tt] = 0.0f;
        if constexpr (TYPE != SEQ_BF16) {
          const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ids.ks), at));
          const float vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ids.vs), at));
          x.ks[tt] = id >= 0 ? ks * a.scale2 : 0.0f;
          x.vs[tt] = id >= 0 ? vs : 0.0f;
        }
        const size_t place = (size_t(max(id, 0)) * a.c.n_kv + p.head) * page_bytes + size_t(in_page) * row_bytes;
        const uint32_t bytes = id >= 0 && s < stop ? uint32_t(min(max(end - row, 0), 16)) * row_bytes : 0u;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char*>(a.c.k) + place, bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const char*>(a.c.v) + place, bytes);
#pragma unroll
        for (int j = 0; j < Rows::KW; ++j) {
          const int4 w = buf_load16_stream(rk, r * row_bytes + 64u * j + 16u * c);
          x.k[tt][j][0] = w.x; x.k[tt][j][1] = w.y; x.k[tt][j][2] = w.z; x.k[tt][j][3] = w.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t off = (4 * c + i) * row_bytes + uint32_t(NDT * ES) * r;
          uint32_t* v = x.v[4 * tt + i];
          if constexpr (Rows::VW == 4) {
            const int4 w = buf_load16_stream(rv, off);
            v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
          } else if constexpr (Rows::VW == 2) {
            const auto w = __builtin_amdgcn_raw_buffer_load_b64(rv, int(off), 0, kCpolStream);
            v[0] = w[0]; v[1] = w[1];
          } else {
            v[0] = __builtin_amdgcn_raw_buffer_load_b32(rv, int(off), 0, kCpolStream);
          }
        }
      }
    };
    PageLane<TYPE> now, next;
    now.fetch(a, p.b, p.head, base + lane, pages);
    next.fetch(a, p.b, p.head, base + kWave + lane, pages);
    // Steps before s_edge are loaded one ahead, their page ids and scales 64 pages ahead
    auto load_ahead = [&](int s, Rows& x) __attribute__((always_inline)) {
      if ((s * kStep >> a.c.P_log) - base >= kWave) {  // (by 8 pages at most: 64 to 71 pages on)
        base += kWave;
        now = next;
        next.fetch(a, p.b, p.head, base + kWave + lane, pages);
      }
      load(s, s_edge, now, base, x);
    };
    Rows xa, xb;
    {
      const int from = s_late * kStep >> a.c.P_log;
      PageLane<TYPE> late;
      late.fetch(a, p.b, p.head, from + lane, has_edge ? min(pages, from + 2) : 0);
      load(s_late, s1, late, from, xa);
    }
    load_ahead(s_own, xb);

    // this lane's query rows, as rows of Q (B operand): token t, head h; the cache rows below `lim` are seen
    int lim[MT];
    uint32_t qf[MT][QT][NKC][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int row = min(rb * RB + mt * 16 + r, p.R - 1);     // (rows past the last one repeat it and are not stored)
      const int t = quot(row, p.group), h = p.h0 + row - t * p.group;
      lim[mt] = p.L >= 0 && p.L + t < a.c.cap ? p.L + t + 1 : 0;
      load_q<DH, ACT, QT, ES == 1>(a.q.p, (p.first + t) * a.q.token + h * a.q.head + (ES == 2 ? 8 : 16) * c, qf[mt]);
    }

    float m_run[MT], l_run[MT];        // of query row r; l of this lane's cache rows
    f32x4 o[MT][NDT];                  // lane (r, c): query rows 4 c + i, dimension NDT r + d
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m_run[mt] = -INFINITY;
      l_run[mt] = 0.0f;
#pragma unroll
      for (int i = 0; i < NDT; ++i) o[mt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto process = [&](Rows& x, int s, auto edge_) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge_)::value;
      // (accumulators take turns: a product waits for the one before it on the same accumulator)
      f32x4 sc[MT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sc[mt][tt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < NKC; ++kk) {
        uint32_t kf[2][4];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          if constexpr (TYPE == SEQ_BF16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) kf[tt][e] = x.k[tt][kk][e];
          } else {
            widen<TYPE>(x.k[tt][kk >> 1][2 * (kk & 1)], kf[tt]);
            widen<TYPE>(x.k[tt][kk >> 1][2 * (kk & 1) + 1], kf[tt] + 2);
          }
        }
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sc[mt][tt] = mfma(kf[tt], qf[mt][q][kk], sc[mt][tt]);
      }
      uint32_t pf[MT][PT][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        soft_step<NDT, PT, TYPE != SEQ_BF16, EDGE>(sc[mt], x.ks, x.vs, x.bias, lim[mt] - s * kStep, c, m_run[mt], l_run[mt], o[mt], pf[mt]);
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
      // A row that some query rows do not see must not reach them through 0 * inf: its non-finite values are left out of
      // the product, and added at the end to the outputs that see them
      if constexpr (EDGE && TYPE != SEQ_INT8) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (s * kStep + 16 * (i >> 2) + 4 * c + (i & 3) >= common)
#pragma unroll
            for (int e = 0; e < NDT / 2; ++e) bad |= drop_odd(v[i][e]);
        if (bad) s_odd = 1;
      }
#pragma unroll
      for (int e = 0; e < NDT; e += 2) {
        uint32_t vb[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vb[0][i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], 0x05040100u);
          vb[1][i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], 0x07060302u);
        }
#pragma unroll
        for (int k = 0; k < PT; ++k)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][e + i] = mfma(pf[mt][k], vb[i], o[mt][e + i]);
      }
    };
    __syncthreads();                   // (the block of query rows before has been read)
    if (tid == 0) s_odd = 0;
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) arrived(qf[mt]);
    if (has_edge) process(xa, s_late, std::true_type{});
    for (int s = s_own; s < s_edge; s += 8) {
      load_ahead(s + 4, xa);
      process(xb, s, std::false_type{});
      if (s + 4 >= s_edge) break;
      load_ahead(s + 8, xb);
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
    float* rec = p.n_ch > 1 ? record(a, y, p.before + p.ch, p.g, rb) : nullptr;
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
      const int in = mt * 16 + qr, row = rb * RB + in;
      if (row >= p.R) continue;
      const int t = quot(row, p.group);
      const int mine = p.L >= 0 && p.L + t < a.c.cap ? p.L + t + 1 : 0;
      const bool there = mine > 0;     // (a row of an absent token is zeros)
      if constexpr (TYPE != SEQ_INT8) {
        if (s_odd) add_odd<DH, TYPE>(a, p.b, p.head, max(common, p.s0 * kStep), min(mine, s1 * kStep), d0, v);
      }
      if (p.n_ch == 1) {
        put_output<DH, ACT>(a, p.first + t, p.h0 + row - t * p.group, d0, l, there, v);
      } else {
#pragma unroll
        for (int e = 0; e < NDT; e += 4)
          *reinterpret_cast<float4*>(rec + in * DH + d0 + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        if (d0 == 0) *reinterpret_cast<float2*>(rec + RB * DH + 2 * in) = make_float2(m, there ? l : 0.0f);
      }
    }
  }
}

// Joins the chunks' records: dh / 4 lanes over a query row's dimensions, PARTS such groups of lanes over its
// chunks, the rest of the workgroup over rows. Grid (query rows of a sequence / rows, sequences).
template <int DH, int ACT, int PARTS>
__global__ __launch_bounds__(kBlock) void page_join_kernel(PageAttnArgs a, PageShape y) {
  constexpr int LPR = DH / 4, ROWS = kBlock / (LPR * PARTS);
  __shared__ float s_m[ROWS][PARTS], s_l[ROWS][PARTS];
  __shared__ float4 s_o[ROWS][PARTS][LPR];
  const int tid = threadIdx.x, b = blockIdx.y;
  if (page_seq(a.start, a.N, a.c, b).n == 0) return;   // (its entry of the workspace is not written)
  const int4 head = reinterpret_cast<const int4*>(a.ws)[b];
  const int n = head.x, before = head.y;
  if (n <= 1) return;                  // written already
  const int mine = tid / (LPR * PARTS), q_row = blockIdx.x * ROWS + mine;
  const int last = head.w * a.slots * a.group - 1;
  if (blockIdx.x * ROWS > last) return;
  const int th = quot(min(q_row, last), a.group), t = quot(th, a.slots), g = th - t * a.slots;
  const int slot = a.slot[g], h0 = slot >> 8 & 0xfff, group = slot >> 20;
  const int own = q_row - th * a.group, hh = min(own, group - 1);
  const bool there = own < group;      // (others repeat a row, and store nothing)
  const int row = t * group + hh, rows = y.rows, rb = row >> y.rows_log, in = row & (rows - 1);
  const size_t stride = size_t(rows) * (DH + 2) * a.slots * y.rb;
  const float* first = record(a, y, before, g, rb);
  const int part = tid / LPR % PARTS, d0 = 4 * (tid % LPR);
  float m = -INFINITY, l = 0.0f;
  float v[4] = {};
  auto add = [&](float mk, float lk, const float4& x) {
    const float mn = fmaxf(m, mk);
    const float fa = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    const float fb = mk == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mk - mn);
    m = mn;
    l = l * fa + lk * fb;
    v[0] = v[0] * fa + x.x * fb; v[1] = v[1] * fa + x.y * fb; v[2] = v[2] * fa + x.z * fb; v[3] = v[3] * fa + x.w * fb;
  };
  // four records in flight
  for (int k0 = part; k0 < n; k0 += 4 * PARTS) {
    float2 q[4];
    float4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* po = first + min(k0 + i * PARTS, n - 1) * stride;
      q[i] = *reinterpret_cast<const float2*>(po + rows * DH + 2 * in);
      x[i] = *reinterpret_cast<const float4*>(po + in * DH + d0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k0 + i * PARTS < n) add(q[i].x, q[i].y, x[i]);
  }
  if constexpr (PARTS > 1) {
    if (d0 == 0) {
      s_m[mine][part] = m;
      s_l[mine][part] = l;
    }
    s_o[mine][part][tid % LPR] = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    if (part > 0) return;
    m = -INFINITY;
    l = v[0] = v[1] = v[2] = v[3] = 0.0f;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) add(s_m[mine][k], s_l[mine][k], s_o[mine][k][tid % LPR]);
  }
  if (there) put_output<DH, ACT>(a, head.z + t, h0 + hh, d0, l, true, v);
}

PageShape shape(const PageAttnArgs& a) {
  PageShape y;
  const int tiles = int(std::min<long>(long(std::max(a.max_new, 1)) * a.group + 15, 1 << 21) / 16);
  y.mt = std::min(tiles, 2);
  y.rows = 16 * y.mt;
  y.rows_log = 31 - __builtin_clz(y.rows);
  const int blocks = std::min((tiles + y.mt - 1) / y.mt, 65535);
  y.rb = std::min(blocks, kTarget);
  const int units = a.slots * y.rb, seqs = std::min(a.c.batch, a.N);
  const long steps = (std::min<long>(std::max(a.max_len, 0) + long(std::max(a.max_new, 1)), a.c.cap) + kStep - 1) / kStep;
  y.room = std::max(seqs, (kTarget + units - 1) / units);
  y.cut = steps > kMinSteps && y.room > seqs;
  y.items = (y.room * a.slots + 7) / 8 * 8;
  y.rb = std::min(blocks, kTarget);
  return y;
}

}  // namespace

size_t page_attn_workspace_bytes(const PageAttnArgs& a) {
  const PageShape y = shape(a);
  return y.cut ? (kHeadFloats + size_t(y.room) * a.slots * y.rb * y.rows * (a.c.dh + 2)) * 4 : 0;
}

hipError_t launch_page_attn(const PageAttnArgs& a, hipStream_t s) {
  const PageShape y = shape(a);
  const int blocks = int(std::min<long>((long(std::max(a.max_new, 1)) * a.group + y.rows - 1) / y.rows, 65535));
#define ATTN(DH, TYPE, ACT, MT) \
  hipLaunchKernelGGL((page_attn_kernel<DH, TYPE, ACT, MT>), dim3(8, blocks, y.items / 8), dim3(kBlock), 0, s, a, y)
#define ATTN_MT(DH, TYPE, ACT)                   \
  do {                                           \
    if (y.mt == 1) ATTN(DH, TYPE, ACT, 1);       \
    else ATTN(DH, TYPE, ACT, 2);                 \
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
  if (e != hipSuccess || !y.cut) return e;
  const int rows = y.rb * y.rows * a.slots;
  const int seqs = std::min(a.c.batch, a.N);
#define JOIN_PARTS(DH, ACT, PARTS)                                                                                        \
  hipLaunchKernelGGL((page_join_kernel<DH, ACT, PARTS>), dim3((rows * PARTS + 4 * kBlock / DH - 1) / (4 * kBlock / DH), a.c.batch), \
                     dim3(kBlock), 0, s, a, y)
#define JOIN(DH, ACT)                                                        \
  do {                                                                       \
    if (rows * seqs < 2048) JOIN_PARTS(DH, ACT, 4 * kBlock / DH);            \
    else if (rows * seqs < 8192) JOIN_PARTS(DH, ACT, 4);                     \
    else JOIN_PARTS(DH, ACT, 1);                                             \
  } while (0)
  if (a.c.dh == 128 && a.act == SEQ_BF16) JOIN(128, SEQ_BF16);
  else if (a.c.dh == 128) JOIN(128, SEQ_F32);
  else if (a.act == SEQ_BF16) JOIN(64, SEQ_BF16);
  else JOIN(64, SEQ_F32);
#undef JOIN
#undef JOIN_PARTS
  return hipGetLastError();
}

}  // namespace tasp
