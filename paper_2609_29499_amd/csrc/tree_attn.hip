// Attention of drafted tokens over a cache whose sequences have their own lengths: node t of a
// sequence with L cached rows sees rows 0 .. L - 1, its ancestors' rows L + j and its own.
//
// o = softmax(scale q K^T) V per query head; a sequence's nodes and the query heads of one cache head
// form the rows of one product, row = node * group + head, so each K and V row is read once for all
// of them. Tiles of 16 query rows by 32 cache rows (a step) run on v_mfma_f32_16x16x32_bf16:
//   * S^T = K Q^T: lane (r, c) gets the scores of query row r against cache rows 4 c .. 4 c + 3 of each tile of
//     16: P stays in registers, and is the A operand of
//   * O += P V over the step's two tiles: lane (r, c) holds cache rows 4 c .. 4 c + 3 of both tiles, dh / 16
//     dimensions from dh / 16 * r on: whole coalesced rows, turned in registers (two rows' halves per
//     v_perm) into the operand's columns of eight rows. The output's dimensions are then dh / 16 * r + i: again
//     neighbours, so rows are stored whole.
// Rows in 8 bits become BF16 exactly; their scales multiply scores and probabilities in 32 bits. P is
// carried as two BF16 terms (16 bits; one alone would double the error of a BF16 output), float32 q and P
// as three (24 bits, as exact as the products' float32 sums). (One FP16 term has 11 bits, and not the range of a
// probability times a scale; calls of the 64-node case below took 170 us with it, 192 with two BF16 terms, 225 with three.)
//
// Softmax with a running maximum per query row, raised only when a score passes it by 8 powers of two (sums
// are float32, so the slack costs no accuracy): most steps exchange nothing between lanes.
//
// Measured, first launch + join: 64 nodes x 64 heads over 8 INT8 sequences of 8192 .. 4608 rows (108 GFLOP) 199 + 10 us,
// bound by instructions: some 640 of a wave's per step of 64 rows, 96 of them matrix products, two waves per SIMD; a tree of 16
// over 4 BF16 sequences of 4096 .. 2560 rows 20 + 5 us: 4 us until rows arrive, then 55 MB of them read and 15 MB of records
// written at 4.4 TB/s; 8 tokens over 131072 E4M3 rows (277 MB) 57 + 5 us, bound by memory (4.9 TB/s); one token over 2047
// INT8 rows 7 + 4 us, latency.
//
// Two kernels. Up to 32 query rows (tree_attn_kernel) a wave keeps all of them and walks every fourth step
// straight from memory in the operands' layout, the next step's loads in flight; no LDS is used before
// the four waves' results meet. More rows (tree_attn_wide_kernel) are dealt to the four waves, which share
// steps of 64 cache rows through LDS: two waves load, widen and lay out V, two K, for the next step while all
// compute on the present one, so that widening and turning are done once per row and not per wave.
//
// The cache rows of all sequences are cut into chunks of equal length (from the lengths on the device: no
// host knows them); a workgroup takes one chunk of one cache head, or a slot of several sequences' (below). A sequence of
// one chunk is written at once; the others leave (maximum, sum, unnormalised output) per query row in the workspace, which a
// second launch joins in chunk order. (Joining by the last workgroup of a sequence to finish was slower: one
// workgroup's latencies in a row, 8 us for 16 chunks of 16 query rows, 29 us for 64 of 32, against 4 and 7 us.)
#include <algorithm>
#include <type_traits>

#include "attn_tiles.hpp"
#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

constexpr int kStep = 32;              // cache rows per step
constexpr int kMinSteps = 4;           // steps of a chunk at least, and its granule: one per wave
constexpr int kMinWide = 2;            // and in the wide kernel: 64 rows that all waves share
constexpr float kSlack = 8.0f;         // powers of two a score may pass the running maximum by

// ---- which rows a workgroup serves
// Sequence b has steps(b) = ceil((L + T) / 32) steps. Two ways to deal them to workgroups, per cache head and block of
// query rows:
//   * span (few slots per sequence; the wide kernel): the sequences' steps in a row, each preceded by kSetup
//     steps for what a piece costs before its first row, are cut into `quota` equal slots; a workgroup takes its slot's
//     pieces one after the other. (In equal chunks of each sequence's own, eight sequences of 4608 .. 8192 rows in 16
//     slots left the fullest workgroup with 132 steps where the mean was 101.)
//   * otherwise each is cut in chunks of `chunk` steps, a workgroup for each.
// A piece or chunk of a sequence that has several leaves a record. A wave holds four sequences per lane.
//
// How a call is launched: query rows in rb blocks of `rows` = 2^rows_log (16 mt, wide: 64 mt), at most `most` chunks per
// sequence (what the workspace has room for), quota: slots per unit, room: records, items: of the grid
constexpr int kSetup = 4;
constexpr int kTarget = 512;           // workgroups aimed at: two per CU
struct TreeShape {
  int wide, mt, rows, rows_log, rb, most, quota, span, room, items;
};
struct Deal {
  int chunk;                           // steps per chunk or slot
  int total;                           // chunks of all sequences, or slots
  int mine[4], before[4];              // of the lane's sequences: chunks or pieces, and those of the sequences before them
  int len[4];                          // and their lengths, -1: passed over
  int at[4], slot[4], steps[4];        // span: place of the first step in the row, and its slot; steps
};
template <bool SPAN>
__device__ __forceinline__ Deal deal(const TreeAttnArgs& a, const TreeShape& y, int lane) {
  Deal d;
  int n[4], cost[4], sum_own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) d.len[i] = a.c.len[min(4 * lane + i, a.c.batch - 1)];    // (in flight together)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int L = d.len[i] = d.len[i] < 0 || d.len[i] > a.c.S ? -1 : d.len[i];
    n[i] = 4 * lane + i >= a.c.batch ? 0 : L < 0 ? 1 : (min(L + a.T, a.c.S) + kStep - 1) / kStep;
    cost[i] = SPAN && y.span && n[i] > 0 ? (n[i] + 3) / 4 * 4 + kSetup : n[i];
    sum_own += cost[i];
  }
  const int inc = wave_scan(sum_own), sum = __builtin_amdgcn_readlane(inc, kWave - 1);
  // (said to be the same in all lanes wherever it is: a buffer descriptor or a branch that the compiler takes for
  // divergent becomes a loop over lanes, around every load)
  d.total = y.quota;
  if (SPAN && y.span) {
    d.chunk = max(kMinSteps, (quot_steps(sum + y.quota - 1, y.quota, __builtin_amdgcn_rcpf(float(y.quota))) + 3) / 4 * 4);
    const float inv = __builtin_amdgcn_rcpf(float(d.chunk));
    int at = inc - sum_own;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      d.at[i] = at + kSetup;
      d.steps[i] = n[i];
      d.slot[i] = quot_steps(d.at[i], d.chunk, inv);
      d.mine[i] = cost[i] == 0 ? 0 : quot_steps(at + cost[i] - 1, d.chunk, inv) - d.slot[i] + 1;
      at += cost[i];
    }
  } else {
    const int units = a.slots * y.rb;
    const int least = y.wide ? kMinWide : kMinSteps;
    d.chunk = max(least, (int((long(sum) * units + kTarget - 1) / kTarget) + least - 1) / least * least);
    if (a.c.batch > 1 && 2 * a.c.batch <= y.quota) {
      // Sequences are rounded up to whole chunks: the shortest chunk that keeps all workgroups within the target is
      // looked for, a candidate per lane (workgroups beyond it would make a second round)
      const int mine = d.chunk + lane * max(4, d.chunk / 256 * 4);
      const float inv = __builtin_amdgcn_rcpf(float(mine));
      int count = 0;
      for (int b = 0; b < a.c.batch; ++b) {
        const int nb = pick(n, b >> 2, b & 3);
        const int q = int(float(nb) * inv);            // within one of the quotient; rounded up
        count += q + (q * mine < nb ? 1 : 0);
      }
      const unsigned long long fits = __ballot(count <= y.quota);
      d.chunk = __builtin_amdgcn_readlane(mine, fits ? __ffsll((long long)fits) - 1 : kWave - 1);
    }
    const float inv = __builtin_amdgcn_rcpf(float(d.chunk));
#pragma unroll
    for (int i = 0; i < 4; ++i) d.mine[i] = min(quot_steps(n[i] + d.chunk - 1, d.chunk, inv), y.most);
  }
  int own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d.before[i] = own;
    own += d.mine[i];
  }
  const int all = wave_scan(own);
#pragma unroll
  for (int i = 0; i < 4; ++i) d.before[i] += all - own;
  if (!(SPAN && y.span)) d.total = __builtin_amdgcn_readlane(all, kWave - 1);
  return d;
}
// One query row's scores of a step (lane (r, c): cache rows 4 c + i of both tiles) to the terms of P.
// t0: the step's first row minus the cached rows, i.e. rows from 0 on are the tree's; EDGE: there are
// such rows (or rows behind them), of which the row sees those in anc.
template <int NDT, int PT, bool SCALED, bool EDGE>
__device__ __forceinline__ void soft_step(const f32x4 (&sc)[2], const float (&ks)[8], const float (&vs)[8], float scale2, int t0, int c,
                                          unsigned long long anc, float& m_run, float& l_run, f32x4 (&o)[NDT], uint32_t (&pf)[PT][4]) {
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = sc[i >> 2][i & 3] * (SCALED ? ks[i] : scale2);
  uint32_t seen = 0;
  if constexpr (EDGE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = t0 + 16 * (i >> 2) + 4 * c + (i & 3);
      const bool in = j < 0 || (j < kTreeMax && ((anc >> (j & 63)) & 1));
      seen |= uint32_t(in) << i;
      p[i] = in ? p[i] : -INFINITY;
    }
  }
  const float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
  float w[8];                          // the scales of rows that the query row sees (others' may be anything)
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = !SCALED ? 1.0f : !EDGE || ((seen >> i) & 1) ? vs[i] : 0.0f;
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
    if constexpr (SCALED) p[i] *= w[i];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) terms<PT>(p[2 * e], p[2 * e + 1], &pf[0][e], 4);
}

// Adds the non-finite values that drop_odd left out to one query row's outputs: of the tree's rows
// from .. to - 1 (cache rows) that the row sees.
template <int DH, int TYPE, int N>
__device__ __forceinline__ void add_odd(const TreeAttnArgs& a, size_t unit, int Lr, int from, int to, unsigned long long anc, int d0, float (&v)[N]) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  for (int j = max(0, from - Lr); j < a.T && Lr + j < to; ++j) {
    if (!((anc >> j) & 1)) continue;
    const char* row = static_cast<const char*>(a.c.v) + ((unit * a.c.S + Lr + j) * DH + d0) * ES;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float x = TYPE == SEQ_BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[e])
                                       : (row[e] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f;
      if (!(fabsf(x) < INFINITY)) v[e] += x;
    }
  }
}

// The part of the work that a workgroup takes.
struct Place {
  int b, g, rb;                        // sequence, slot, block of query rows
  int h0, group, R;                    // the slot's first query head, its heads, its query rows
  size_t unit;                         // its cache head among those of all sequences
  int n_ch, ch, before, rec;           // chunks or pieces of the sequence, this one, those of the sequences before, its record
  int L, Lr, end;                      // length (-1: passed over), rows cached, rows that may be read
  int s0, s1;                          // steps
  bool more;                           // another piece follows
};
// piece: 0, 1, .. of the workgroup's
template <bool SPAN>
__device__ __forceinline__ bool place(const TreeAttnArgs& a, const TreeShape& y, int lane, int piece, Place& p) {
  // Grid (8, row blocks, items / 8): row blocks of one chunk and head read the same rows, and are eight workgroups
  // apart (one XCD, one L2) and next to each other in time. Item: chunk of a sequence x slot.
  p.rb = blockIdx.y;
  const int item = blockIdx.z * 8 + blockIdx.x, all = quot(item, a.slots);     // chunk, or slot of the row
  p.g = item - all * a.slots;
  const int slot = a.slot[p.g];                        // (on its way with the lengths)
  const Deal d = deal<SPAN>(a, y, lane);
  if (item >= d.total * a.slots) return false;
  p.h0 = slot >> 8 & 0xfff;
  p.group = slot >> 20;
  p.R = a.T * p.group;
  if (p.rb * y.rows >= p.R) return false;              // (a slot with fewer heads than the largest)
  p.more = false;
  if (SPAN && y.span) {
    // sequences that end before the slot come first; the slot's own follow one another
    int ended = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      ended += __popcll(__ballot(d.mine[i] > 0 && d.at[i] + (d.steps[i] + 3) / 4 * 4 <= all * d.chunk));
    p.b = ended + piece;
    auto starts = [&](int b) { return b < a.c.batch && pick(d.slot, b >> 2, b & 3) <= all; };
    if (!starts(p.b)) return false;
    p.more = starts(p.b + 1);
    p.ch = all - pick(d.slot, p.b >> 2, p.b & 3);
  } else {
    int hit = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (all >= d.before[i] && all < d.before[i] + d.mine[i]) hit = i;
    const int owner = __ffsll((long long)__ballot(hit >= 0)) - 1;
    p.b = 4 * owner + __builtin_amdgcn_readlane(hit, owner);
    p.ch = all - pick(d.before, owner, p.b & 3);
  }
  const int owner = p.b >> 2, sub = p.b & 3;
  p.n_ch = pick(d.mine, owner, sub);
  p.before = pick(d.before, owner, sub);
  p.rec = ((p.before + p.ch) * a.slots + p.g) * y.rb + p.rb;
  p.unit = size_t(p.b) * a.c.n_kv + (slot & 0xff);
  p.L = pick(d.len, owner, sub);
  p.Lr = max(p.L, 0);
  p.end = p.L < 0 ? 0 : min(p.L + a.T, a.c.S);
  const int steps = (p.end + kStep - 1) / kStep;
  if (SPAN && y.span) {
    const int at = all * d.chunk - pick(d.at, owner, sub);
    p.s0 = max(at, 0);
    p.s1 = min(at + d.chunk, steps);
  } else {
    // the last chunk of a sequence takes what is left (with `most` chunks that may be more than a chunk)
    const int per = p.n_ch * d.chunk >= steps ? d.chunk : ((steps + p.n_ch - 1) / p.n_ch + 3) / 4 * 4;
    p.s0 = p.ch * per;
    p.s1 = p.ch == p.n_ch - 1 ? steps : min(steps, p.s0 + per);
  }
  return true;
}

// One query row's output values (unnormalised) with their sum l: node t, head h from dimension d0 on. there: the
// node is present. put_record: the same with the maximum m to row `row` of the chunk's record of RB rows.
template <int DH, int ACT, int N>
__device__ __forceinline__ void put_output(const TreeAttnArgs& a, int b, int t, int h, int d0, float l, bool there, const float (&v)[N]) {
  const float inv = there && l != 0.0f ? 1.0f / l : 0.0f;
  const long at = b * a.o.seq + t * a.o.token + h * a.o.head + d0;
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

// A record: [RB][DH] outputs, then [RB] (maximum, sum).
template <int DH, int RB>
constexpr size_t kRecFloats = size_t(RB) * (DH + 2);
// The workspace starts with (chunks, chunks of the sequences before) of each sequence, for the join, which then has no
// lengths to read and nothing to deal (0.7 us).
constexpr size_t kHeadFloats = 2 * 256;
__device__ __forceinline__ void put_head(const TreeAttnArgs& a, const Place& p) {
  if (p.ch == 0 && p.g == 0 && p.rb == 0 && threadIdx.x == 0) reinterpret_cast<int2*>(a.ws)[p.b] = make_int2(p.n_ch, p.before);
}
template <int DH, int RB, int N>
__device__ __forceinline__ void put_record(const TreeAttnArgs& a, int rec, int row, int d0, float m, float l, const float (&v)[N]) {
  float* po = a.ws + kHeadFloats + size_t(rec) * kRecFloats<DH, RB>;
#pragma unroll
  for (int e = 0; e < N; e += 4)
    *reinterpret_cast<float4*>(po + row * DH + d0 + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
  if (d0 == 0) *reinterpret_cast<float2*>(po + RB * DH + 2 * row) = make_float2(m, l);
}

// A query row's operand: from `at` on (elements from q.p) 8 values for each of dh / 32 products, those of product
// kk 32 kk further on, or (PAIRED) 64 floor(kk / 2) + 8 (kk mod 2)
template <int DH, int ACT, int QT, bool PAIRED>
__device__ __forceinline__ void load_q(const TreeAttnArgs& a, long at0, uint32_t (&qf)[QT][DH / 32][4]) {
#pragma unroll
  for (int kk = 0; kk < DH / 32; ++kk) {
    const long at = at0 + (PAIRED ? 64 * (kk >> 1) + 8 * (kk & 1) : 32 * kk);
    if constexpr (ACT == SEQ_BF16) {
      const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q.p) + at);
      qf[0][kk][0] = x.x; qf[0][kk][1] = x.y; qf[0][kk][2] = x.z; qf[0][kk][3] = x.w;
    } else {
      const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(a.q.p) + at);
      const float4 x = f[0], z = f[1];
      uint32_t* o = &qf[0][kk][0];
      terms<QT>(x.x, x.y, o, DH / 8);
      terms<QT>(x.z, x.w, o + 1, DH / 8);
      terms<QT>(z.x, z.y, o + 2, DH / 8);
      terms<QT>(z.z, z.w, o + 3, DH / 8);
    }
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
constexpr int kWavesPerSimd = MT == 2 && DH == 128 && (TYPE == SEQ_BF16 || ACT == SEQ_F32) ? 1 : 2;

// MT: tiles of 16 query rows per wave. (Lambdas here are inlined by order: called, they would keep what they
// capture in memory, descriptors among it.)
template <int DH, int TYPE, int ACT, int MT>
__global__ __launch_bounds__(kBlock, (kWavesPerSimd<DH, TYPE, ACT, MT>)) void tree_attn_kernel(TreeAttnArgs a, TreeShape y) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  constexpr int NKC = DH / 32;         // score products per tile
  constexpr int NDT = DH / 16;         // dimensions per lane of V and O
  constexpr int QT = ACT == SEQ_F32 ? 3 : 1, PT = ACT == SEQ_F32 ? 3 : 2;
  using Rows = Rows32<DH, TYPE>;
  constexpr int RB = 16 * MT;
  __shared__ float s_o[4][16][DH + 4];
  __shared__ float s_m[4][RB], s_l[4][RB];
  __shared__ int s_odd;                // a tree's row holds something not finite

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, c = lane >> 4;
  Place p;
  if (!place<false>(a, y, lane, 0, p)) return;
  const int b = p.b, rb = p.rb, L = p.L, Lr = p.Lr, end = p.end, s0 = p.s0, s1 = p.s1;
  if (y.most > 1) put_head(a, p);
  // steps from s_edge on hold rows of the tree: at most three, so a wave has one at most
  const int s_edge = min(Lr / kStep, s1);

  const size_t unit = p.unit;
  const uint32_t row_bytes = DH * ES;
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char*>(a.c.k) + unit * a.c.S * row_bytes, uint32_t(end) * row_bytes);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const char*>(a.c.v) + unit * a.c.S * row_bytes, uint32_t(end) * row_bytes);
  const __amdgpu_buffer_rsrc_t rks = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.ks + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);
  const __amdgpu_buffer_rsrc_t rvs = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.vs + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);

  // Steps are loaded one ahead. Rows past `end`, and steps past `stop`, read as zeros without touching memory.
  auto load = [&](int s, int stop, Rows& x) __attribute__((always_inline)) {
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
  const int R = p.R;
  const TreeNode nd = tree_node(a.parent ? a.parent + size_t(b) * a.T : nullptr, a.T, L < 0 ? 0 : a.c.S - L, lane);
  unsigned long long anc[MT];
  uint32_t qf[MT][QT][NKC][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = min((rb * MT + mt) * 16 + r, R - 1);   // (rows past the last one repeat it and are not stored)
    const int t = quot(row, p.group), h = p.h0 + row - t * p.group;
    anc[mt] = __shfl(nd.anc, t, kWave);
    load_q<DH, ACT, QT, ES == 1>(a, b * a.q.seq + t * a.q.token + h * a.q.head + (ES == 2 ? 8 : 16) * c, qf[mt]);
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
    float ks[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) ks[i] = TYPE == SEQ_BF16 ? 0.0f : x.ks[i] * a.scale2;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      soft_step<NDT, PT, TYPE != SEQ_BF16, EDGE>(sc[mt], ks, x.vs, a.scale2, s * kStep - Lr, c, anc[mt], m_run[mt], l_run[mt], o[mt], pf[mt]);
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
        if (s * kStep + 16 * (i >> 2) + 4 * c + (i & 3) >= Lr)
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
  if constexpr (TYPE != SEQ_INT8) {
    if (tid == 0) s_odd = 0;
    __syncthreads();
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) arrived(qf[mt]);
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
    const int t_o = quot(min(row_o, R - 1), p.group);
    const unsigned long long anc_o = __shfl(nd.anc, t_o, kWave);
    const bool there = anc_o != 0;     // (a row of an absent node is zeros)
    if (row_o >= R) continue;
    if constexpr (TYPE != SEQ_INT8) {
      if (s_odd) add_odd<DH, TYPE>(a, unit, Lr, max(s_edge, s0) * kStep, s1 * kStep, anc_o, d0, v);
    }
    if (p.n_ch == 1) put_output<DH, ACT>(a, b, t_o, p.h0 + row_o - t_o * p.group, d0, l, there, v);
    else put_record<DH, RB>(a, p.rec, 16 * mt + qr, d0, m, there ? l : 0.0f, v);
  }
}

// MT: tiles of 16 query rows per wave; a workgroup holds 64 MT rows.
template <int DH, int TYPE, int ACT, int MT>
__global__ __launch_bounds__(kBlock, 2) void tree_attn_wide_kernel(TreeAttnArgs a, TreeShape y) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  constexpr int NKC = DH / 32, NDT = DH / 16, RB = 64 * MT;
  constexpr int QT = ACT == SEQ_F32 ? 3 : 1, PT = ACT == SEQ_F32 ? 3 : 2;
  constexpr int PPR = DH * ES / 16;    // 16-byte pieces of a K row as loaded
  constexpr int KL = 32 * PPR / kWave; // K loads per thread: 32 rows per wave
  constexpr int VW = NDT * ES / 4;     // words of V per lane and row
  constexpr int NW = 8 * VW;           // words per lane of 32 rows, of either
  static_assert(NW == 4 * KL, "K and V rows are equally wide");
  // Operands of a step of 64 rows, each 16 bytes per lane: K [tile of 16 rows][32 dimensions], V [32 rows][dimension i]
  struct Step {
    uint4 k[4][NKC][kWave];
    uint4 v[2][NDT][kWave];
  };
  __shared__ Step s_step[2];
  __shared__ float s_scale[2][2][64];  // [step][K / V][row]
  __shared__ int s_odd;

  for (int piece = 0;; ++piece) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));      // (new to the compiler in each piece: kept over pieces, what follows from it spills)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, c = lane >> 4;
    Place p;
    if (!place<true>(a, y, lane, piece, p)) return;
    if (piece > 0) __syncthreads();      // (LDS is read no more)
    const int Lr = p.Lr, end = p.end;
    if (y.most > 1) put_head(a, p);
    const size_t unit = p.unit;
    const uint32_t row_bytes = DH * ES;
    const bool for_v = wave < 2;         // this wave brings V (32 rows), or K
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const char*>(for_v ? a.c.v : a.c.k) + unit * a.c.S * row_bytes, uint32_t(end) * row_bytes);
    const __amdgpu_buffer_rsrc_t rks = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.ks + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);
    const __amdgpu_buffer_rsrc_t rvs = make_rsrc(TYPE == SEQ_BF16 ? nullptr : a.c.vs + unit * a.c.S, TYPE == SEQ_BF16 ? 0u : uint32_t(end) * 4u);
    const int half = 32 * (wave & 1);    // its rows of the step

    // what a wave has on its way: 32 rows of K or of V of the next step
    struct Raw {
      uint32_t w[NW];
      float scale;
    };
    auto load = [&](Raw& x, int s) __attribute__((always_inline)) {     // (steps past the last read as zeros)
      const uint32_t t0 = uint32_t(s) * kStep + half;
      const bool in = s < p.s1;
      if constexpr (TYPE != SEQ_BF16)
        x.scale = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(for_v ? rvs : rks, int(in && lane < 32 ? (t0 + lane) * 4u : kOOB), 0, 0));
      if (for_v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t off = in ? (t0 + 16 * (i >> 2) + 4 * c + (i & 3)) * row_bytes + uint32_t(NDT * ES) * r : kOOB;
          if constexpr (VW == 4) {
            const int4 q = buf_load16_stream(rx, off);
            x.w[4 * i] = q.x; x.w[4 * i + 1] = q.y; x.w[4 * i + 2] = q.z; x.w[4 * i + 3] = q.w;
          } else if constexpr (VW == 2) {
            const auto q = __builtin_amdgcn_raw_buffer_load_b64(rx, int(off), 0, kCpolStream);
            x.w[2 * i] = q[0]; x.w[2 * i + 1] = q[1];
          } else {
            x.w[i] = __builtin_amdgcn_raw_buffer_load_b32(rx, int(off), 0, kCpolStream);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const uint32_t row = t0 + i * (kWave / PPR) + lane / PPR;
          const int4 q = buf_load16_stream(rx, in ? row * row_bytes + 16u * (lane % PPR) : kOOB);
          x.w[4 * i] = q.x; x.w[4 * i + 1] = q.y; x.w[4 * i + 2] = q.z; x.w[4 * i + 3] = q.w;
        }
      }
    };
    auto commit = [&](const Raw& x, int buf, int s) __attribute__((always_inline)) {
      Step& z = s_step[buf];
      if constexpr (TYPE != SEQ_BF16)
        if (lane < 32) s_scale[buf][for_v][half + lane] = for_v ? x.scale : x.scale * a.scale2;
      if (for_v) {
        if constexpr (TYPE == SEQ_INT8) {
          // byte d of eight rows' words -> one operand: widened, and packed two rows at a time
#pragma unroll
          for (int e = 0; e < NDT; ++e) {
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float f0 = float(int8_t(x.w[2 * i * VW + e / 4] >> (8 * (e & 3)))), f1 = float(int8_t(x.w[(2 * i + 1) * VW + e / 4] >> (8 * (e & 3))));
              q[i] = __builtin_amdgcn_perm(__float_as_uint(f1), __float_as_uint(f0), 0x07060302u);
            }
            z.v[wave][e][lane] = make_uint4(q[0], q[1], q[2], q[3]);
          }
        } else {
          uint32_t v[8][NDT / 2];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (TYPE == SEQ_BF16) {
#pragma unroll
              for (int e = 0; e < NDT / 2; ++e) v[i][e] = x.w[i * VW + e];
            } else {
#pragma unroll
              for (int e = 0; e < NDT / 4; ++e) widen<TYPE>(x.w[i * VW + e], &v[i][2 * e]);
            }
          }
          const int new_row = Lr - s * kStep - half;     // the first of the wave's rows that is the tree's
          if (new_row < 32) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (16 * (i >> 2) + 4 * c + (i & 3) >= new_row)
#pragma unroll
                for (int e = 0; e < NDT / 2; ++e) bad |= drop_odd(v[i][e]);
            if (bad) s_odd = 1;
          }
#pragma unroll
          for (int e = 0; e < NDT; ++e) {
            const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
            z.v[wave][e][lane] = make_uint4(__builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], sel), __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], sel),
                                            __builtin_amdgcn_perm(v[5][e / 2], v[4][e / 2], sel), __builtin_amdgcn_perm(v[7][e / 2], v[6][e / 2], sel));
          }
        }
        // The two branches' last stores are kept apart by order: merged into one store behind both (three of its four
        // words, for BF16 rows and float32 q at dh 64), the compiler took one of V's words from the wrong register.
        asm volatile("; V is stored" ::: "memory");
      } else {
        // lane (r', c') of operand kk reads slot 16 c' + (r' ^ (4 kk + c')): the pieces of one row, written
        // together, go to different banks
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const int row = half + i * (kWave / PPR) + lane / PPR, j = lane % PPR;
          auto put = [&](int piece, uint4 q) __attribute__((always_inline)) {
            const int kk = piece >> 2, cc = piece & 3;
            z.k[row >> 4][kk][16 * cc + ((row & 15) ^ (4 * kk + cc))] = q;
          };
          if constexpr (TYPE == SEQ_BF16) {
            put(j, make_uint4(x.w[4 * i], x.w[4 * i + 1], x.w[4 * i + 2], x.w[4 * i + 3]));
          } else {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) widen<TYPE>(x.w[4 * i + e], &w[2 * e]);
            put(2 * j, make_uint4(w[0], w[1], w[2], w[3]));
            put(2 * j + 1, make_uint4(w[4], w[5], w[6], w[7]));
          }
        }
        asm volatile("; K is stored" ::: "memory");
      }
    };

    Raw x;
    load(x, p.s0);
    if (tid == 0) s_odd = 0;
    // this lane's query rows, as rows of Q (B operand): node t, head h
    const int R = p.R;
    const TreeNode nd = tree_node(a.parent ? a.parent + size_t(p.b) * a.T : nullptr, a.T, p.L < 0 ? 0 : a.c.S - p.L, lane);
    unsigned long long anc[MT];
    uint32_t qf[MT][QT][NKC][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int row = min(p.rb * RB + (wave * MT + mt) * 16 + r, R - 1);     // (rows past the last one repeat it and are not stored)
      const int t = quot(row, p.group), h = p.h0 + row - t * p.group;
      anc[mt] = __shfl(nd.anc, t, kWave);
      load_q<DH, ACT, QT, false>(a, p.b * a.q.seq + t * a.q.token + h * a.q.head + 8 * c, qf[mt]);
    }
    float m_run[MT], l_run[MT];          // of query row r; l of this lane's cache rows
    f32x4 o[MT][NDT];                    // lane (r, c): query rows 4 c + i, dimension NDT r + d
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m_run[mt] = -INFINITY;
      l_run[mt] = 0.0f;
#pragma unroll
      for (int i = 0; i < NDT; ++i) o[mt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) arrived(qf[mt]);
    __syncthreads();                     // s_odd

    // one barrier per step: whoever writes a buffer has passed the barrier that followed its last use
    auto step = [&](int s, int buf, auto edge_) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge_)::value;
      commit(x, buf, s);
      load(x, s + 2);
      __syncthreads();
      const Step& z = s_step[buf];
      const int t0 = s * kStep - Lr;
#pragma unroll 1
      for (int half_ = 0; half_ < 2; ++half_) {          // (unrolled, it does not fit the registers)
        // (accumulators take turns: a product waits for the one before it on the same accumulator)
        f32x4 sc[MT][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) sc[mt][tt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < NKC; ++kk) {
          uint4 kf[2];
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) kf[tt] = z.k[2 * half_ + tt][kk][16 * c + (r ^ (4 * kk + c))];
#pragma unroll
          for (int k = 0; k < QT; ++k)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) sc[mt][tt] = mfma({kf[tt].x, kf[tt].y, kf[tt].z, kf[tt].w}, qf[mt][k][kk], sc[mt][tt]);
        }
        float ks[8] = {}, vs[8] = {};
        if constexpr (TYPE != SEQ_BF16) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            const float4 x = *reinterpret_cast<const float4*>(&s_scale[buf][0][32 * half_ + 16 * tt + 4 * c]);
            const float4 w = *reinterpret_cast<const float4*>(&s_scale[buf][1][32 * half_ + 16 * tt + 4 * c]);
            ks[4 * tt] = x.x; ks[4 * tt + 1] = x.y; ks[4 * tt + 2] = x.z; ks[4 * tt + 3] = x.w;
            vs[4 * tt] = w.x; vs[4 * tt + 1] = w.y; vs[4 * tt + 2] = w.z; vs[4 * tt + 3] = w.w;
          }
        }
        uint32_t pf[MT][PT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          soft_step<NDT, PT, TYPE != SEQ_BF16, EDGE>(sc[mt], ks, vs, a.scale2, t0 + 32 * half_, c, anc[mt], m_run[mt], l_run[mt], o[mt], pf[mt]);
#pragma unroll
        for (int e = 0; e < NDT; e += 2) {
          uint4 vb[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) vb[i] = z.v[half_][e + i][lane];
#pragma unroll
          for (int k = 0; k < PT; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
                o[mt][e + i] = mfma(pf[mt][k], {vb[i].x, vb[i].y, vb[i].z, vb[i].w}, o[mt][e + i]);
        }
      }
    };
    int s = p.s0, buf = 0;
    for (; s < p.s1 && (s + 2) * kStep <= Lr; s += 2, buf ^= 1) step(s, buf, std::false_type{});
    for (; s < p.s1; s += 2, buf ^= 1) step(s, buf, std::true_type{});

    // every wave holds its rows' results: lane (r, c) rows 4 c + i of a tile, their maxima and sums in lanes 4 c + i
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float l_all = quad_sum(l_run[mt]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int in = (wave * MT + mt) * 16 + 4 * c + i, row = p.rb * RB + in;
        const float m = __shfl(m_run[mt], 4 * c + i, kWave), l = __shfl(l_all, 4 * c + i, kWave);
        const int t = quot(min(row, R - 1), p.group);
        const unsigned long long anc_o = __shfl(nd.anc, t, kWave);
        float v[NDT];
#pragma unroll
        for (int e = 0; e < NDT; ++e) v[e] = o[mt][e][i];
        if constexpr (TYPE != SEQ_INT8)
          if (s_odd) add_odd<DH, TYPE>(a, unit, Lr, p.s0 * kStep, p.s1 * kStep, anc_o, NDT * r, v);
        if (row < R) {
          if (p.n_ch == 1) put_output<DH, ACT>(a, p.b, t, p.h0 + row - t * p.group, NDT * r, l, anc_o != 0, v);
          else put_record<DH, RB>(a, p.rec, in, NDT * r, m, anc_o != 0 ? l : 0.0f, v);
        }
      }
    }
    if (!p.more) return;
  }
}

// Joins the chunks' records: dh / 4 lanes over a query row's dimensions, PARTS such groups of lanes over its
// chunks, the rest of the workgroup over rows. Grid (query rows of a sequence / rows, sequences).
template <int DH, int ACT, int PARTS>
__global__ __launch_bounds__(kBlock) void tree_join_kernel(TreeAttnArgs a, TreeShape y) {
  constexpr int LPR = DH / 4, ROWS = kBlock / (LPR * PARTS);
  __shared__ float s_m[ROWS][PARTS], s_l[ROWS][PARTS];
  __shared__ float4 s_o[ROWS][PARTS][LPR];
  const int tid = threadIdx.x, b = blockIdx.y;
  const int2 head = reinterpret_cast<const int2*>(a.ws)[b];
  const int n = head.x, before = head.y;
  if (n <= 1) return;                  // written already
  const int mine = tid / (LPR * PARTS), q_row = blockIdx.x * ROWS + mine;
  const int th = quot(min(q_row, a.T * a.slots * a.group - 1), a.group), t = quot(th, a.slots), g = th - t * a.slots;
  const int slot = a.slot[g], h0 = slot >> 8 & 0xfff, group = slot >> 20;
  const int own = q_row - th * a.group, hh = min(own, group - 1);
  const bool there = own < group;      // (others repeat a row, and store nothing)
  const int row = t * group + hh, rows = y.rows, rb = row >> y.rows_log, in = row & (rows - 1);
  const size_t rec = size_t(rows) * (DH + 2), stride = rec * a.slots * y.rb;
  const float* first = a.ws + kHeadFloats + before * stride + (size_t(g) * y.rb + rb) * rec;
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
  if (there) put_output<DH, ACT>(a, b, t, h0 + hh, d0, l, true, v);
}

TreeShape shape(const TreeAttnArgs& a) {
  TreeShape y;
  const int tiles = (a.T * a.group + 15) / 16;
  // One or two tiles stay in every wave (8 tokens over 131072 E4M3 rows 57 us, 93 through LDS; one token 7.2, 8.5); more go
  // through LDS (a tree of 16 with four tiles 20 us, 27 with four in every wave), two tiles per wave where there are
  // eight and registers for them (64 nodes x 64 heads 232 us when it was tried, 262 with one)
  y.wide = tiles > 2;
  y.mt = y.wide ? (tiles > 4 && a.act == SEQ_BF16 ? 2 : 1) : tiles;
  const int block = (y.wide ? 4 : 1) * y.mt;           // tiles of a workgroup
  y.rows = 16 * block;
  y.rows_log = 31 - __builtin_clz(y.rows);
  y.rb = (tiles + block - 1) / block;
  const int units = a.slots * y.rb, least = y.wide ? kMinWide : kMinSteps;
  const long steps = (std::min<long>(std::max(a.max_len, 0) + long(a.T), a.c.S) + kStep - 1) / kStep;
  y.most = int(std::max<long>(1, std::min<long>((steps + least - 1) / least, (kTarget + units - 1) / units)));
  // chunks of all sequences: their steps over the chunk's, rounded up per sequence
  const long chunks = std::min<long>(long(a.c.batch) * y.most, kTarget / units + 1 + a.c.batch);
  y.room = int(chunks) * a.slots * y.rb;
  // Spanned: two to eight slots per sequence (with more, chunks differ little, and a tree of 16 at 4 x 4096 rows took
  // 21.5 us instead of 19.7: two pieces in a row), and a record for every piece: a slot each and one more per further sequence
  y.quota = kTarget / units;
  y.span = y.wide && 2 * a.c.batch <= y.quota && y.quota < 8 * a.c.batch && y.quota + a.c.batch - 1 <= chunks;
  y.items = ((y.span ? y.quota : int(chunks)) * a.slots + 7) / 8 * 8;
  return y;
}

}  // namespace

size_t tree_attn_workspace_bytes(const TreeAttnArgs& a) {
  const TreeShape y = shape(a);
  return y.most == 1 ? 0 : (kHeadFloats + size_t(y.room) * y.rows * (a.c.dh + 2)) * 4;
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t s) {
  const TreeShape y = shape(a);
#define ATTN(KERNEL, DH, TYPE, ACT, MT) hipLaunchKernelGGL((KERNEL<DH, TYPE, ACT, MT>), dim3(8, y.rb, y.items / 8), dim3(kBlock), 0, s, a, y)
#define ATTN_MT(DH, TYPE, ACT)                                                                   \
  do {                                                                                           \
    if (!y.wide && y.mt == 1) ATTN(tree_attn_kernel, DH, TYPE, ACT, 1);                          \
    else if (!y.wide) ATTN(tree_attn_kernel, DH, TYPE, ACT, 2);                                  \
    else if (y.mt == 1) ATTN(tree_attn_wide_kernel, DH, TYPE, ACT, 1);                           \
    else if constexpr (ACT == SEQ_BF16) ATTN(tree_attn_wide_kernel, DH, TYPE, ACT, 2);           \
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
  const int rows = a.T * a.slots * a.group;
  // Few rows: a workgroup for each (latency); many: a group of lanes walks all of a row's records, which are few then
  // (the 64-node case took 72 us with a workgroup per row); between, four groups (a tree of 16 at 4 x 4096 rows, 16
  // records: 7.5 us with one).
#define JOIN_PARTS(DH, ACT, PARTS)                                                                                        \
  hipLaunchKernelGGL((tree_join_kernel<DH, ACT, PARTS>), dim3((rows * PARTS + 4 * kBlock / DH - 1) / (4 * kBlock / DH), a.c.batch), \
                     dim3(kBlock), 0, s, a, y)
#define JOIN(DH, ACT)                                                            \
  do {                                                                           \
    if (rows * a.c.batch < 2048) JOIN_PARTS(DH, ACT, 4 * kBlock / DH);           \
    else if (rows * a.c.batch < 8192) JOIN_PARTS(DH, ACT, 4);                    \
    else JOIN_PARTS(DH, ACT, 1);                                                 \
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
