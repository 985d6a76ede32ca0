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
// Two kernels. Up to 32 query rows of a sequence and cache head (page_attn_kernel): a wave keeps all of them and walks every
// fourth step straight from memory in the operands' layout, the next step's loads in flight. More
// (page_attn_wide_kernel): blocks of 64 to 256 rows are dealt to four or eight waves, which share steps of 64 cache rows
// through LDS (below).
//
// A workgroup takes one chunk of the cache rows of one block of query rows and cache head. Chunks have equal lengths, found
// from the lengths on the device (no host knows them) such that there are about two workgroups per CU. With more blocks than that
// the second kernel takes each whole, the first cuts those that are far longer than the others. A block of one chunk is written at
// once; the others leave (maximum, sum, unnormalised output) per query row in the workspace, which another launch joins in chunk order.
//
// What bounds them: the first, memory (4 tokens x 64 heads over 65,530 E4M3 rows 76 us and a join of 5: 5.8 TB/s; 32 tokens over 8190
// INT8 rows, a common prefix of 1024 read by each, 80: 5.1 TB/s); one token is latency (8.4 us and a join of 4.3 for
// 2047 rows). The second, matrix products and vector instructions, of which each waits for the other:
// a prompt of 8192 tokens x 64 heads in BF16 1236 us, 890 TFLOP/s of visible pairs, 72 % of what a library product of 8192^3
// reaches (1243): 386 M vector instructions for 68 M products, the matrix cores busy for 36 % of the cycles; 512 tokens behind 8191
// INT8 rows 111 us, 640 TFLOP/s, 33 M for 4.4 M, busy for 26 %.
#include <algorithm>
#include <type_traits>

#include "attn_tiles.hpp"
#include "device_common.hpp"
#include "page.hpp"

namespace tasp {
namespace {

constexpr int kStep = 32;              // cache rows per step
constexpr int kWideStep = 64;          // and in the wide kernel
constexpr int kMinSteps = 4;           // steps of a chunk at least, and its granule: one per wave
constexpr float kSlack = 8.0f;         // powers of two a score may pass the running maximum by
// workgroups aimed at: two per CU. (512 / 1024 / 2048, first version: 4 tokens x 64 heads over 65,530 rows 82 / 90 / 106 us, 32 tokens over
// 8190 rows 88 / 89 / 103, 512 tokens behind 8191 rows 153 / 163 / 177: more of them leave more records to join)
constexpr int kTarget = 512;
// query rows of a sequence and cache head that the first kernel serves: what a wave's registers hold. (Serving all, it took 262 us for 512
// tokens behind 8191 rows and 3904 for a prompt of 8192 tokens x 64 heads, where the wide one takes 133 and 1236)
constexpr int kFew = 32;

// Eight waves, one workgroup per CU in place of two, may share a step in LDS: bringing it (BF16 V to FP16 above all) takes each of them
// half the instructions, but a block's last steps and its empty waves take a whole CU. BF16 pages, from kEight query rows and
// kEightRows rows seen on, four / eight waves, 32 heads: 512 tokens behind 0 rows 30 / 33 us, 1000 45 / 45, 2000 54 / 53, 4000 72 / 67,
// 8191 113 / 103; 128 tokens behind 1000 29 / 33, 2000 35.4 / 34.5, 8191 51 / 48; a prompt of 1024 47.0 / 46.5, 2048 79 / 83, 4096
// 190 / 178, 8192 698 / 645. 8 bits: 512 tokens behind 0 30 / 35, 2000 54 / 58, 8191 112 / 113, a prompt of 8192 694 / 700; they have four. Nor where
// the other sequences, on average, fill less than a block and are not the first kernel's: a chunk of 512 beside 15 of 20 tokens behind 8191 207 / 316.
constexpr int kEight = 512, kEightRows = 2048;

// Steps of 64 cache rows, in all slots, of short sequences that the wide kernel takes beside its own, in place of a second launch:
// for float32, whose bits are the same in both kernels. Both / one, 32 heads of 128 over INT8 rows: 64 tokens and 11 single ones behind
// 1000 rows (1496 steps) 37 / 28 us, 2000 (2904) 49 / 38, 4000 (5632) 65 / 60, 8191 (11352) 99 / 105; 16 and 11 behind 1000 (1408) 34 / 26, 2000
// (2816) 41 / 38, 4000 (5544) 51 / 58. But not where the short sequences' workgroups take a chunk from the large one's blocks or run behind them: 512
// tokens and one behind 1000 rows 66 / 68, 2000 90 / 109, 8191 234 / 355; 1024 tokens and one behind 500 rows 82 / 69, 1000 106 / 98, 2000 151 / 172;
// 256 tokens, whose blocks have four chunks each and lose one of them, behind 8191 rows 142 / 132. (BF16 runs both kernels, for the bits of short
// sequences: beside 512 tokens behind 8191 rows all in the wide one took 137.6 us, both 131.7.)
constexpr int kAside = 2048, kAsideRows = 1024;

// How a kernel is launched. Sequences with least .. most query rows per cache head, in blocks of `rows` = 2^rows_log; steps of
// `step` rows; items: chunks of all blocks, at most; cut: there may be several chunks of a block, none shorter than all steps / share
struct PageShape {
  int least, most, mt, rows, rows_log, step, items, cut, share;
  size_t ws;                           // floats of the workspace in front of its records
};
struct Deal {
  int chunk, total;                    // steps per chunk; items of all sequences
  int nch[4], mine[4], before[4];      // of the lane's sequences: chunks of a block, items, items of the sequences before them
  int first[4], n[4], len[4];
};
// A lane holds four sequences. The chunk is the shortest multiple of kMinSteps, a share of all steps at least, that leaves at most `items` items.
__device__ __forceinline__ Deal deal(const PageAttnArgs& a, const PageShape& y, int lane) {
  Deal d;
  int steps[4], blocks[4], most = 0;
  uint32_t sum = 0;                    // (of 2^13 + 256 blocks of 2^18 steps at most)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const PageSeq q = page_seq(a.start, a.N, a.c, min(4 * lane + i, a.c.batch - 1));
    d.first[i] = q.first; d.len[i] = q.L;
    const int rows = q.n * a.group;
    d.n[i] = 4 * lane + i < a.c.batch && rows >= y.least && rows <= y.most ? q.n : 0;
    const int end = q.L < 0 ? 0 : min(q.L + d.n[i], a.c.cap);
    steps[i] = d.n[i] == 0 ? 0 : max(1, (end + y.step - 1) / y.step);
    blocks[i] = (d.n[i] * a.group + y.rows - 1) >> y.rows_log;
    sum += uint32_t(steps[i]) * uint32_t(min(blocks[i], kTarget));
    most = max(most, steps[i]);
  }
  d.chunk = 1 << 24;
  if (y.cut) {
    auto total = [&](int chunk) {
      const float inv = __builtin_amdgcn_rcpf(float(chunk));
      int own = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) own += blocks[i] * quot_steps(steps[i] + chunk - 1, chunk, inv);
      return __builtin_amdgcn_readlane(wave_scan(own), kWave - 1);
    };
    sum = uint32_t(__builtin_amdgcn_readlane(wave_scan(int(sum)), kWave - 1));
    most = int(wave_max(float(most)));                 // (below 2^24)
    // in units of kMinSteps: lo may do, hi does
    int lo = max(1, int((sum + y.share - 1) / y.share + kMinSteps - 1) / kMinSteps), hi = max(lo, (most + kMinSteps - 1) / kMinSteps);
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (total(mid * kMinSteps) <= y.items) hi = mid;
      else lo = mid + 1;
    }
    d.chunk = lo * kMinSteps;
  }
  const float inv = __builtin_amdgcn_rcpf(float(d.chunk));
  int own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    d.nch[i] = y.cut ? quot_steps(steps[i] + d.chunk - 1, d.chunk, inv) : min(steps[i], 1);
    d.mine[i] = blocks[i] * d.nch[i];
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
  int item, nch, ch, block;            // among all items; chunks of the block, this one; block of query rows
  int first, n, L;                     // the sequence's tokens, rows it held (-1: passed over)
  int common, end;                     // rows that all of the block's tokens see, and that any does
  int s0, s1;                          // steps
};
// false: nothing to do. Grid (slots, kItems, items / kItems): slots take turns, so that with eight of them a cache head's
// workgroups run on one XCD and share its L2.
constexpr int kItems = 1024;
__device__ __forceinline__ void note_tokens(const PageAttnArgs& a, const PageShape& y, const Place& p);
__device__ __forceinline__ bool place(const PageAttnArgs& a, const PageShape& y, int lane, Place& p) {
  p.item = blockIdx.z * kItems + blockIdx.y;
  p.g = blockIdx.x;
  const int slot = a.slot[p.g];
  const Deal d = deal(a, y, lane);
  if (p.item >= d.total) return false;
  int hit = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (p.item >= d.before[i] && p.item < d.before[i] + d.mine[i]) hit = i;
  const int owner = __builtin_amdgcn_readfirstlane(__ffsll((long long)__ballot(hit >= 0)) - 1), sub = __builtin_amdgcn_readlane(hit, owner);
  p.b = 4 * owner + sub;
  p.head = slot & 0xff;
  p.h0 = slot >> 8 & 0xfff;
  p.group = slot >> 20;
  p.first = pick(d.first, owner, sub);
  p.n = pick(d.n, owner, sub);
  p.L = pick(d.len, owner, sub);
  p.R = p.n * p.group;
  p.nch = pick(d.nch, owner, sub);
  const int local = p.item - pick(d.before, owner, sub), k = quot(local, p.nch), blocks = quot(pick(d.mine, owner, sub), p.nch);
  p.ch = local - k * p.nch;
  p.block = blocks - 1 - k;            // the last rows, which see the most, first
  const int r0 = p.block << y.rows_log;
  if (y.cut && p.ch == 0 && p.g == 0) note_tokens(a, y, p);
  if (r0 >= p.R) return false;         // (a slot with fewer heads than the largest)
  const int t_first = quot(r0, p.group), t_last = quot(min(p.R, r0 + y.rows) - 1, p.group);
  const int most = p.L < 0 ? 0 : min(p.L + p.n, a.c.cap);
  p.common = p.L < 0 ? 0 : min(p.L + t_first + 1, most);
  p.end = p.L < 0 ? 0 : min(p.L + t_last + 1, most);
  const int steps = (p.end + y.step - 1) / y.step;
  p.s0 = p.ch * min(d.chunk, 1 << 20);
  p.s1 = p.nch == 1 ? steps : min(steps, p.s0 + d.chunk);
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

// The workspace: of each token (its sequence, the sequence's first item, chunks of a block), then of each item and slot a
// record: [rows] (maximum, sum), [rows][DH] outputs. Both kernels' records lie behind each other.
__device__ __forceinline__ int4* token_notes(const PageAttnArgs& a) { return reinterpret_cast<int4*>(a.ws); }
__device__ __forceinline__ float* record(const PageAttnArgs& a, const PageShape& y, int item, int g) {
  return a.ws + y.ws + (size_t(item) * a.slots + g) * (size_t(y.rows) * (a.c.dh + 2));
}
// of the tokens whose first row (of the largest slot) lies in the block
__device__ __forceinline__ void note_tokens(const PageAttnArgs& a, const PageShape& y, const Place& p) {
  const int r0 = p.block << y.rows_log, blocks = (p.n * a.group + y.rows - 1) >> y.rows_log;
  const int t0 = quot(r0 + a.group - 1, a.group), t1 = min(p.n, quot(r0 + y.rows + a.group - 1, a.group));
  const int4 note = make_int4(p.b, p.item - (blocks - 1 - p.block) * p.nch, p.nch, 0);
  for (int t = t0 + int(threadIdx.x); t < t1; t += int(blockDim.x)) token_notes(a)[p.first + t] = note;
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

// Whether any of the cache rows from .. to - 1 has a page. (Asked only of query rows whose sum is NaN: scores against missing rows
// are NaN where the query is not finite, and a query row that sees none is zeros whatever it holds.)
__device__ __forceinline__ bool any_page(const PageAttnArgs& a, int b, int from, int to) {
  for (int j = from >> a.c.P_log; j << a.c.P_log < to; ++j) {
    const int page = a.c.table[size_t(b) * a.c.width + j];
    if (page >= 0 && page < a.c.n_pages) return true;
  }
  return false;
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
// chunk, the next step's loads in flight.
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
  const size_t page_bytes = size_t(row_bytes) << a.c.P_log;
  const int common = p.common, end = p.end, s1 = p.s1, r0 = p.block * RB;
  const int pages = (end + a.c.P - 1) >> a.c.P_log;
  {
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
        const size_t place = (size_t(max(id, 0)) * a.c.n_kv + p.head) * page_bytes + size_t(in_page) * row_bytes;
        // (said to be the same in all lanes: a descriptor that the compiler takes for divergent becomes a loop around every load)
        const uint32_t bytes = __builtin_amdgcn_readfirstlane(id >= 0 && s < stop ? min(max(end - row, 0), 16) * int(row_bytes) : 0);
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
      // (behind the rows' loads: the scales' own, which follow the page ids', are waited for here)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int at = ((s * kStep + 16 * tt) >> a.c.P_log) - from, id = __builtin_amdgcn_readlane(ids.id, at);
        x.bias[tt] = id >= 0 ? 0.0f : -INFINITY;
        x.ks[tt] = id >= 0 ? a.scale2 : 0.0f;
        x.vs[tt] = 0.0f;
        if constexpr (TYPE != SEQ_BF16) {
          const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ids.ks), at));
          const float vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ids.vs), at));
          x.ks[tt] = id >= 0 ? ks * a.scale2 : 0.0f;
          x.vs[tt] = id >= 0 ? vs : 0.0f;
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
      const int row = min(r0 + mt * 16 + r, p.R - 1);     // (rows past the last one repeat it and are not stored)
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
    float* rec = p.nch > 1 ? record(a, y, p.item, p.g) : nullptr;
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
      const int in = mt * 16 + qr, row = r0 + in;
      if (row >= p.R) continue;
      const int t = quot(row, p.group);
      const int mine = p.L >= 0 && p.L + t < a.c.cap ? p.L + t + 1 : 0;
      // (a row of an absent token is zeros, as is one that sees nothing)
      const bool there = mine > 0 && (l == l || any_page(a, p.b, p.s0 * kStep, min(mine, s1 * kStep)));
      if constexpr (TYPE != SEQ_INT8) {
        if (s_odd) add_odd<DH, TYPE>(a, p.b, p.head, max(common, p.s0 * kStep), min(mine, s1 * kStep), d0, v);
      }
      if (p.nch == 1) {
        put_output<DH, ACT>(a, p.first + t, p.h0 + row - t * p.group, d0, l, there, v);
      } else {
#pragma unroll
        for (int e = 0; e < NDT; e += 4)
          *reinterpret_cast<float4*>(rec + 2 * RB + in * DH + d0 + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        if (d0 == 0) *reinterpret_cast<float2*>(rec + 2 * in) = there ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
      }
    }
  }
}

// ---- more query rows
//
// A workgroup's four or eight waves (NW) hold MT tiles of 16 query rows each. Steps of 64 cache rows go through LDS, two of them in turn: all
// threads bring K and V of the next one (16 bytes a thread and row piece; loads in flight while the present step is computed),
// widen 8 bits and write rows of 16-bit values; chunks of 16 bytes change places by the row, so that no reader meets a
// bank twice. K rows are read as they lie (operand A of S^T = K Q^T); V is turned on its way from LDS
// (ds_read_b64_tr_b16: four rows of 16 dimensions, one per lane), cache rows 4 c .. 4 c + 3 of two tiles being the eight of
// operand B that meet the lane's P. So P stays in registers.
//   Float32 queries: three BF16 terms of q and of P, as above. BF16 queries, steps that all of the block's tokens see: P is one FP16
// term: 11 bits, an eighth of the output's rounding, and half the matrix products of two BF16 terms (with four waves, 8192 tokens x 64
// heads 1302 us, 1573 with two terms). V is FP16 too: codes are exact, and the page's scale over a reference (the power of two at or below
// the largest scale seen) goes into P, from 2^-kSpread to 2; BF16 values are multiplied by a power of two that brings the largest seen
// below 2^15 (lowered when a step has a larger one). P is at most 2^kWideSlack, and lifted by 2^kLift to just below FP16's end, so that
// half a step of its least numbers is 2^-35 of the row with the running maximum. (Slack of 2: 1320 us, of 8: 1303.) Lost at most, for
// each row: of BF16 values 2^-35 of the largest |v|, and 2^-36 for V's own least numbers; of 8 bits 2^-31 of the row's own |v|.
//   The units of V are the block's, so nothing that some of its tokens do not see may go into them: BF16 queries' last steps,
// which hold such rows, and all steps from one on whose pages' scales are further apart than 2^kSpread (a page's scale need not be
// reached by the rows that are left in it), have P in two BF16 terms and V as it is, as in the other kernel. Lift and units are
// taken out of the sums in front of them.
constexpr float kWideSlack = 4.0f;     // in place of kSlack
constexpr float kLift = 10.0f, kUnlift = 0x1p-10f;
constexpr uint32_t kSpread = 4;        // 8 bits: powers of two between a scale and the largest one
constexpr uint32_t kRise = 16;         // and between the first largest one and a later one: what was added up before stays far above 2^-126
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {         // round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, f16x2_t));
}
__device__ __forceinline__ f32x4 mfma_f16(const uint32_t (&a)[4], const uint32_t (&b)[4], f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, make_uint4(a[0], a[1], a[2], a[3])),
                                                __builtin_bit_cast(f16x8, make_uint4(b[0], b[1], b[2], b[3])), acc, 0, 0, 0);
}
// four codes -> two words of FP16 pairs (exact)
template <int TYPE>
__device__ __forceinline__ void widen_f16(uint32_t w, uint32_t* o) {
  if constexpr (TYPE == SEQ_INT8) {
    // 1024 + (code + 128) as an FP16 number is the byte under 0x64
    const uint32_t u = w ^ 0x80808080u;
    const f16x2_t bias = {_Float16(1152.0f), _Float16(1152.0f)};
    o[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias);
    o[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias);
  } else {
    o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
}
// E4M3 codes that are NaN become zeros; non-zero if there are any
__device__ __forceinline__ uint32_t drop_nan_codes(uint32_t& w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  w &= ~((top >> 7) * 0xffu);
  return top;
}
// the power of two that brings a largest magnitude to 2^11 .. 2^12
__device__ __forceinline__ float scale_for(float top) {
  const int e = int(__float_as_uint(top) >> 23);       // (0 for zero and what is next to it)
  return __uint_as_float(uint32_t(min(127 + 11 + 127 - e, 253)) << 23);
}

template <int DH, int TYPE, int ACT, int MT, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void page_attn_wide_kernel(PageAttnArgs a, PageShape y) {
  constexpr int ES = TYPE == SEQ_BF16 ? 2 : 1;
  constexpr int NKC = DH / 32, NDT = DH / 16, RB = 16 * NW * MT;
  constexpr int QT = ACT == SEQ_F32 ? 3 : 1;
  constexpr bool HALF = ACT == SEQ_BF16;               // P and V in FP16 in most steps
  constexpr int CPR = DH / 8;          // chunks (eight 16-bit values) of a row in LDS
  constexpr int PPR = DH * ES / 16;    // 16-byte pieces of a row as loaded
  constexpr int RPI = NW * kWave / PPR;    // rows per load of the workgroup
  constexpr int NL = kWideStep / RPI;  // loads of K, and of V, per thread and step
  constexpr uint32_t row_bytes = DH * ES;
  constexpr int LDO = DH + 4;
  union Lds {
    struct {
      uint4 k[kWideStep][CPR], v[kWideStep][CPR];
    } step[2];
    float o[NW][16][LDO];
  };
  __shared__ Lds z;
  __shared__ float s_top[NW];
  __shared__ uint32_t s_raise[3];      // a step's largest finite V where one does not fit (as its bits)
  __shared__ int s_odd;                // a row that some query rows do not see holds something not finite

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, c = lane >> 4;
  Place p;
  if (!place(a, y, lane, p)) return;
  const int common = p.common, end = p.end, s1 = p.s1, r0 = p.block * RB;
  float* rec = p.nch > 1 ? record(a, y, p.item, p.g) : nullptr;
  if (p.s0 >= s1 && p.nch > 1) {       // (a block that ends before this chunk)
    if (tid < RB) *reinterpret_cast<float2*>(rec + 2 * tid) = make_float2(-INFINITY, 0.0f);
    return;
  }
  const size_t page_bytes = size_t(row_bytes) << a.c.P_log;
  const int pages = (end + a.c.P - 1) >> a.c.P_log;

  int base = p.s0 * kWideStep >> a.c.P_log;
  PageLane<TYPE> now, next;
  now.fetch(a, p.b, p.head, base + lane, pages);
  next.fetch(a, p.b, p.head, base + kWave + lane, pages);
  struct Raw {
    uint32_t k[NL][4], v[NL][4];
    float ks[4], vs[4], bias[4];       // of the step's tiles of 16 rows
  };
  Raw x;
  const int piece = tid % PPR, row_in = tid / PPR;     // of its first load; the others are RPI rows on
  auto load = [&](int s) __attribute__((always_inline)) {
    if ((s * kWideStep >> a.c.P_log) - base >= kWave) {
      base += kWave;
      now = next;
      next.fetch(a, p.b, p.head, base + kWave + lane, pages);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int at = ((s * kWideStep + 16 * t) >> a.c.P_log) - base, id = __builtin_amdgcn_readlane(now.id, at);
      x.bias[t] = id >= 0 ? 0.0f : -INFINITY;
      x.ks[t] = id >= 0 ? a.scale2 : 0.0f;
      x.vs[t] = 0.0f;
      if constexpr (TYPE != SEQ_BF16) {
        x.ks[t] = id >= 0 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(now.ks), at)) * a.scale2 : 0.0f;
        x.vs[t] = id >= 0 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(now.vs), at)) : 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = s * kWideStep + 16 * (i * (RPI / 16) + wave * 4 / PPR);      // of the wave's tile
      const int id = __builtin_amdgcn_readlane(now.id, (row >> a.c.P_log) - base);
      const size_t at = (size_t(max(id, 0)) * a.c.n_kv + p.head) * page_bytes + size_t(row & (a.c.P - 1)) * row_bytes;
      // (said to be the same in all lanes: a descriptor that the compiler takes for divergent becomes a loop around every load)
      const uint32_t bytes = __builtin_amdgcn_readfirstlane(id >= 0 && s < s1 ? min(max(end - row, 0), 16) * int(row_bytes) : 0);
      const uint32_t off = uint32_t(row_in & 15) * row_bytes + 16u * piece;
      const int4 k = buf_load16(make_rsrc(static_cast<const char*>(a.c.k) + at, bytes), off);
      const int4 v = buf_load16(make_rsrc(static_cast<const char*>(a.c.v) + at, bytes), off);
      x.k[i][0] = k.x; x.k[i][1] = k.y; x.k[i][2] = k.z; x.k[i][3] = k.w;
      x.v[i][0] = v.x; x.v[i][1] = v.y; x.v[i][2] = v.z; x.v[i][3] = v.w;
    }
  };
  auto k_place = [](int row, int j) { return j ^ (DH == 128 ? row & 15 : row >> 1 & 7); };
  auto v_place = [](int row, int j) { return j ^ (DH == 128 ? 2 * (row & 7) : 2 * (row >> 1 & 3)); };
  float mul = 1.0f;                    // BF16: V's power of two
  // V into buffer buf, as FP16 or BF16; returns the largest magnitude (BF16 as FP16)
  auto commit_v = [&](int buf, auto f16_) __attribute__((always_inline)) {
    constexpr bool F16 = decltype(f16_)::value;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = row_in + i * RPI;
      if constexpr (TYPE == SEQ_BF16) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (!F16) {
            w[e] = x.v[i][e];
            continue;
          }
          const float f0 = bf16_lo(x.v[i][e]) * mul, f1 = bf16_hi(x.v[i][e]) * mul;
          top = fmaxf(fmaxf(fabsf(f0), fabsf(f1)), top);
          w[e] = pack_f16(f0, f1);
        }
        z.step[buf].v[row][v_place(row, piece)] = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) F16 ? widen_f16<TYPE>(x.v[i][e], &w[2 * e]) : widen<TYPE>(x.v[i][e], &w[2 * e]);
        z.step[buf].v[row][v_place(row, 2 * piece)] = make_uint4(w[0], w[1], w[2], w[3]);
        z.step[buf].v[row][v_place(row, 2 * piece + 1)] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
    return top;
  };
  auto commit_k = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = row_in + i * RPI;
      if constexpr (TYPE == SEQ_BF16) {
        z.step[buf].k[row][k_place(row, piece)] = make_uint4(x.k[i][0], x.k[i][1], x.k[i][2], x.k[i][3]);
      } else {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) widen<TYPE>(x.k[i][e], &w[2 * e]);
        z.step[buf].k[row][k_place(row, 2 * piece)] = make_uint4(w[0], w[1], w[2], w[3]);
        z.step[buf].k[row][k_place(row, 2 * piece + 1)] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
  };
  // the largest finite magnitude of the step's V in this wave
  auto top_v = [&]() __attribute__((always_inline)) {
    float top = 0.0f;
    if constexpr (TYPE == SEQ_BF16) {
#pragma unroll
      for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float f0 = fabsf(bf16_lo(x.v[i][e])), f1 = fabsf(bf16_hi(x.v[i][e]));
          top = fmaxf(top, f0 < INFINITY ? f0 : 0.0f);
          top = fmaxf(top, f1 < INFINITY ? f1 : 0.0f);
        }
    }
    return wave_max(top);
  };

  load(p.s0);
  // this lane's query rows, as rows of Q (B operand): token t, head h; the cache rows below `lim` are seen
  int lim[MT];
  uint32_t qf[MT][QT][NKC][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = min(r0 + (wave * MT + mt) * 16 + r, p.R - 1);      // (rows past the last one repeat it and are not stored)
    const int t = quot(row, p.group), h = p.h0 + row - t * p.group;
    lim[mt] = p.L >= 0 && p.L + t < a.c.cap ? p.L + t + 1 : 0;
    load_q<DH, ACT, QT, false>(a.q.p, (p.first + t) * a.q.token + h * a.q.head + 8 * c, qf[mt]);
  }
  float m_run[MT], l_run[MT];          // of query row r; l of this lane's cache rows
  f32x4 o[MT][NDT];                    // lane (r, c): query rows 4 c + i, dimension 16 d + r
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = -INFINITY;
    l_run[mt] = 0.0f;
#pragma unroll
    for (int i = 0; i < NDT; ++i) o[mt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int s_edge = min(s1, common / kWideStep);      // steps from it on hold rows that some tokens do not see
  uint32_t ref = 0, ref0 = 0;          // 8 bits: the exponent of the power of two that V's scales are divided by (0: none yet), the first one
  float inv_ref = 0.0f;
  if (tid == 0) s_odd = 0;
  if (tid < 3) s_raise[tid] = 0;
  if (TYPE == SEQ_BF16 && HALF && p.s0 < s_edge) {
    const float top = top_v();
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) most = fmaxf(most, s_top[k]);
    mul = scale_for(most);
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) arrived(qf[mt]);
  __syncthreads();                     // s_odd, s_raise
  // everything that has been added up is multiplied by f
  auto rescale = [&](float f) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < NDT; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[mt][e][i] *= f;
  };
  // 8 bits: whether the scales of the step that has been loaded are near enough to those before and to each other; ref then
  // covers them
  auto near = [&]() __attribute__((always_inline)) {
    uint32_t hi = 0, lo = 0xffffffffu; // (integers of the same order; a scale of 0 has no say)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t u = __builtin_amdgcn_readfirstlane(__float_as_uint(x.vs[t]));
      hi = max(hi, u);
      lo = min(lo, u - 1);
    }
    if (hi == 0) return true;
    const uint32_t e = max(ref, hi >> 23), least = max(e, kSpread + 1) - kSpread;
    if (hi >= 0x7f000000u || (lo + 1) >> 23 < least || (ref0 > 0 && e > ref0 + kRise)) return false;
    if (e > ref) {
      if (ref > 0) rescale(__uint_as_float((127 + ref - e) << 23));
      else ref0 = e;
      ref = e;
      inv_ref = __uint_as_float((254 - e) << 23);
    }
    return true;
  };
  // lane constants of the reads from LDS
  uint32_t k_at[NKC], v_at;
#pragma unroll
  for (int kk = 0; kk < NKC; ++kk) k_at[kk] = uint32_t(r * CPR + k_place(r, 4 * kk + c));
  const int v_row = 4 * c + (r >> 2);
  v_at = uint32_t(v_row * CPR + v_place(v_row, r >> 1 & 1)) * 16 + 8 * (r & 1);

  // Bringing a step goes first (priority 2: all waves wait for it), then scores (1: the matrix cores, while another wave's
  // softmax has the vector unit): 512 tokens behind 8191 rows 129.6 us, 140.8 without.
  // One barrier per step: whoever writes a buffer has passed the barrier that followed its last use
  auto step = [&](int s, int buf, int turn, auto edge_) __attribute__((always_inline)) {
    constexpr bool EDGE = decltype(edge_)::value, F16 = HALF && !EDGE;
    constexpr int PT = ACT == SEQ_F32 ? 3 : F16 ? 1 : 2;
    // A row that some query rows do not see must not reach them through 0 * inf: its non-finite values are left out
    // of the product, and added at the end to the outputs that see them
    if constexpr (EDGE && TYPE != SEQ_INT8) {
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (s * kWideStep + row_in + i * RPI >= common)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad |= TYPE == SEQ_BF16 ? drop_odd(x.v[i][e]) : drop_nan_codes(x.v[i][e]);
      if (bad) s_odd = 1;
    }
    __builtin_amdgcn_s_setprio(2);
    commit_k(buf);
    const float top = commit_v(buf, std::bool_constant<F16>{});
    __builtin_amdgcn_s_setprio(0);
    if constexpr (TYPE == SEQ_BF16 && F16) {
      if (__ballot(top >= 0x1p15f)) {                  // (an infinity too, each time)
        const float t = top_v();
        if (lane == 0) atomicMax(&s_raise[turn], __float_as_uint(t));
      }
    }
    __syncthreads();
    if constexpr (TYPE == SEQ_BF16 && F16) {
      if (tid == 0) s_raise[turn == 0 ? 2 : turn - 1] = 0;             // (the step after the next one's)
      const float most = __uint_as_float(__builtin_amdgcn_readfirstlane(s_raise[turn]));
      if (most * mul >= 0x1p15f) {
        const float to = scale_for(most);
        rescale(to / mul);
        mul = to;
        commit_v(buf, std::true_type{});
        __syncthreads();
      }
    }
    float ks[4], f[4], bias[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      ks[t] = x.ks[t]; bias[t] = x.bias[t];
      f[t] = TYPE == SEQ_BF16 ? 1.0f : F16 ? x.vs[t] * inv_ref : x.vs[t];
    }
    // K's operands are read two tiles ahead of their products: at most eight reads are on their way
    const char* kz = reinterpret_cast<const char*>(&z.step[buf].k[0][0]);
    uint4 kf[2][NKC];
    auto read_k = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int kk = 0; kk < NKC; ++kk) kf[t & 1][kk] = *reinterpret_cast<const uint4*>(kz + 16 * k_at[kk] + t * 16 * CPR * 16);
    };
    __builtin_amdgcn_s_setprio(1);
    read_k(0);
    read_k(1);
    __builtin_amdgcn_sched_barrier(0);
    load(s + 1);
    f32x4 sc[MT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) sc[mt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int kk = 0; kk < NKC; ++kk) {
        const uint32_t kw[4] = {kf[t & 1][kk].x, kf[t & 1][kk].y, kf[t & 1][kk].z, kf[t & 1][kk].w};
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) sc[mt][t] = mfma(kw, qf[mt][q][kk], sc[mt][t]);
      }
      if (t < 2) read_k(t + 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    uint32_t pf[MT][PT][2][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int seen = lim[mt] - s * kWideStep - 4 * c;                // rows 16 t + i below it are
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (EDGE) {
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, 16 * t + i < seen ? fmaf(sc[mt][t][i], ks[t], bias[t]) : -INFINITY);
        } else {
          const float q = fmaxf(fmaxf(sc[mt][t][0], sc[mt][t][1]), fmaxf(sc[mt][t][2], sc[mt][t][3]));
          top = fmaxf(top, fmaf(q, ks[t], bias[t]));
        }
      }
      if (__ballot(top > m_run[mt] + kWideSlack)) {        // (also the first rows: m_run is -inf)
        const float mn = fmaxf(m_run[mt], quad_max(top));
        const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_run[mt] - mn);
        m_run[mt] = mn;
        l_run[mt] *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float g = __shfl(alpha, 4 * c + i, kWave);
#pragma unroll
          for (int e = 0; e < NDT; ++e) o[mt][e][i] *= g;
        }
      }
      const float low = (F16 ? kLift : 0.0f) - (m_run[mt] == -INFINITY ? 0.0f : m_run[mt]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = __builtin_amdgcn_exp2f(fmaf(sc[mt][t][i], ks[t], bias[t] + low));
          if constexpr (EDGE) v[i] = 16 * t + i < seen ? v[i] : 0.0f;
          l_run[mt] += v[i];
          if constexpr (TYPE != SEQ_BF16) {
            v[i] *= f[t];
            if constexpr (EDGE) v[i] = 16 * t + i < seen ? v[i] : 0.0f;            // (a hidden row's scale may be anything)
          }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if constexpr (F16) pf[mt][0][t >> 1][2 * (t & 1) + e] = pack_f16(v[2 * e], v[2 * e + 1]);
          else terms<PT>(v[2 * e], v[2 * e + 1], &pf[mt][0][t >> 1][2 * (t & 1) + e], 8);
        }
      }
    }
    typedef __attribute__((address_space(3))) s16x4* lds_p;
    __attribute__((address_space(3))) char* vz = (__attribute__((address_space(3))) char*)(&z.step[buf].v[0][0]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < NDT; ++e) {
        __attribute__((address_space(3))) char* at = vz + (v_at ^ (32u * e)) + h * 32 * CPR * 16;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_p(at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_p(at + 16 * CPR * 16));
        const uint2 w0 = __builtin_bit_cast(uint2, lo), w1 = __builtin_bit_cast(uint2, hi);
        const uint32_t vf[4] = {w0.x, w0.y, w1.x, w1.y};
#pragma unroll
        for (int k = 0; k < PT; ++k)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) o[mt][e] = F16 ? mfma_f16(pf[mt][k][h], vf, o[mt][e]) : mfma(pf[mt][k][h], vf, o[mt][e]);
      }
  };
  int s = p.s0, buf = 0, turn = 0;
  for (; s < s_edge; ++s, buf ^= 1, turn = turn == 2 ? 0 : turn + 1) {
    if (TYPE != SEQ_BF16 && HALF && !near()) break;
    step(s, buf, turn, std::false_type{});
  }
  if constexpr (HALF) {
    rescale((TYPE == SEQ_BF16 ? 1.0f / mul : __uint_as_float(ref << 23)) * kUnlift);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) l_run[mt] *= kUnlift;
  }
  for (; s < s1; ++s, buf ^= 1, turn = turn == 2 ? 0 : turn + 1) step(s, buf, turn, std::true_type{});

  // every wave holds its rows' results; through LDS, 16 rows at a time, they become whole rows
  __syncthreads();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float l_all = quad_sum(l_run[mt]);
    if (l_all != l_all && !any_page(a, p.b, p.s0 * kWideStep, min(lim[mt], s1 * kWideStep))) {
      l_all = 0.0f;
      m_run[mt] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < NDT; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) z.o[wave][4 * c + i][16 * e + r] = o[mt][e][i];
#pragma unroll
    for (int k = 0; k < DH / 16; ++k) {
      const int in = (k * kWave + lane) / (DH / 4), d0 = 4 * (lane % (DH / 4));
      const float4 q = *reinterpret_cast<const float4*>(&z.o[wave][in][d0]);
      float v[4] = {q.x, q.y, q.z, q.w};
      const float m = __shfl(m_run[mt], in, kWave), l = __shfl(l_all, in, kWave);
      const int place = (wave * MT + mt) * 16 + in, row = r0 + place;
      if (row >= p.R) continue;
      const int t = quot(row, p.group);
      const int mine = p.L >= 0 && p.L + t < a.c.cap ? p.L + t + 1 : 0;
      if constexpr (TYPE != SEQ_INT8) {
        if (s_odd) add_odd<DH, TYPE>(a, p.b, p.head, max(common, p.s0 * kWideStep), min(mine, s1 * kWideStep), d0, v);
      }
      if (p.nch == 1) {
        put_output<DH, ACT>(a, p.first + t, p.h0 + row - t * p.group, d0, l, mine > 0, v);
      } else {
        *reinterpret_cast<float4*>(rec + 2 * RB + place * DH + d0) = make_float4(v[0], v[1], v[2], v[3]);
        if (d0 == 0) *reinterpret_cast<float2*>(rec + 2 * place) = mine > 0 ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
      }
    }
  }
}

// Joins the chunks' records: dh / 4 lanes over a query row's dimensions, PARTS such groups of lanes over its chunks, the
// rest of the workgroup over rows. Query rows of all tokens in a row; few, wide: the kernels' shapes.
template <int DH, int ACT, int PARTS>
__global__ __launch_bounds__(kBlock) void page_join_kernel(PageAttnArgs a, PageShape few, PageShape wide) {
  constexpr int LPR = DH / 4, ROWS = kBlock / (LPR * PARTS);
  __shared__ float s_m[ROWS][PARTS], s_l[ROWS][PARTS];
  __shared__ float4 s_o[ROWS][PARTS][LPR];
  const int tid = threadIdx.x;
  const int mine = tid / (LPR * PARTS), q_row = blockIdx.x * ROWS + mine;
  const int total = a.N * a.slots * a.group;           // (at most 2^17)
  const int th = quot(min(q_row, total - 1), a.group), token = quot(th, a.slots), g = th - token * a.slots;
  const int slot = a.slot[g], h0 = slot >> 8 & 0xfff, group = slot >> 20, own = q_row - th * a.group, hh = min(own, group - 1);
  // whose token it is: a note that names a sequence with this token, of a kernel that cuts blocks, was left by this call
  // (others may hold anything)
  const int4 note = token_notes(a)[token];
  const PageSeq seq = page_seq(a.start, a.N, a.c, min(max(note.x, 0), a.c.batch - 1));
  const int rows_all = seq.n * a.group;
  const PageShape& y = rows_all >= wide.least && rows_all <= wide.most ? wide : few;
  // (rows past a slot's last one repeat it, and store nothing; one chunk: written already)
  const bool there = own < group && q_row < total && token >= seq.first && token < seq.first + seq.n && y.cut && note.z > 1 &&
                     note.y >= 0 && note.z <= y.items && note.y <= y.items - ((rows_all + y.rows - 1) >> y.rows_log) * note.z;
  if (!__syncthreads_or(there)) return;
  const int n = there ? note.z : 1, row = there ? (token - seq.first) * group + hh : 0;
  const int blocks = (rows_all + y.rows - 1) >> y.rows_log, in = row & (y.rows - 1);
  const size_t stride = size_t(y.rows) * (DH + 2) * a.slots;
  const float* first = there ? record(a, y, note.y + (blocks - 1 - (row >> y.rows_log)) * n, g) : a.ws;
  const int part = tid / LPR % PARTS, d0 = 4 * (tid % LPR);
  float m = -INFINITY, l = 0.0f;
  float v[4] = {};
  auto add = [&](float mk, float lk, const float4& x) {
    if (mk == -INFINITY && lk == 0.0f) return;         // (rows that were not seen, or a chunk behind the block's end: x is not written)
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
      q[i] = *reinterpret_cast<const float2*>(po + 2 * in);
      x[i] = *reinterpret_cast<const float4*>(po + 2 * y.rows + in * DH + d0);
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
  if (there) put_output<DH, ACT>(a, token, h0 + hh, d0, l, true, v);
}

struct Shapes {
  PageShape few, wide;
  size_t floats;                       // of the workspace
};
Shapes shapes(const PageAttnArgs& a) {
  Shapes z{};
  const int seqs = std::min(a.c.batch, a.N), expected = std::min(a.max_new, a.N);
  const long rows = long(expected) * a.group;
  const long most = std::min<long>(std::max(a.max_len, 0) + long(expected), a.c.cap);
  // One kernel for all where it is what the expected number of tokens asks for, where there is one sequence, or where the
  // others' steps take the wide kernel less time than a second launch
  const long aside = (seqs - 1) * ((most + kWideStep - 1) / kWideStep) * a.slots;
  const long big = (rows + 16 * 4 - 1) / (16 * 4), room = (kTarget + a.slots - 1) / a.slots, share = room / big;      // (float32's blocks and chunks)
  const bool fits = a.max_len <= kAsideRows || share >= 3 || share * big + seqs - 1 <= room;
  const bool use_wide = rows > kFew, use_few = !use_wide || aside > (a.act == SEQ_F32 && fits ? kAside : 0);
  constexpr int kAll = 1 << 30;
  auto fill = [&](PageShape& y, bool use, int least, int limit, int step, int mt, int block) {
    y.least = use ? least : 1;
    y.most = use ? limit : 0;
    y.mt = mt; y.step = step; y.rows = block; y.rows_log = 31 - __builtin_clz(block);
    if (!use) return;
    const long blocks = std::min<long>(long(a.N) * a.group, limit == kFew ? long(seqs) * kFew : kAll) / block + seqs;    // of all sequences, at most
    const int quota = ((block == 256 ? kTarget / 2 : kTarget) + a.slots - 1) / a.slots;      // (of eight waves: half)
    // Blocks enough for all workgroups are cut too where the first kernel has them: lengths differ, and one workgroup per head would walk a
    // sequence far longer than the others by itself (131072 rows beside 63 of 1024, 32 heads: 1033 us uncut, 86 cut; three single tokens
    // behind 65530 rows beside a prompt of 4096 tokens 705, 280). Chunks of one and a half shares of all steps and more leave sequences of
    // like lengths whole (256 of 500 rows 64.6 us uncut, 67.2 so, 64 of 500 18.8, 20.7: the join). The join looks at every token's rows: a bound
    // on them, higher where the first kernel has the short sequences of a step.
    y.cut = (blocks < quota || block <= kFew) && most > kMinSteps * step && long(a.N) * a.slots * a.group <= (limit == kFew ? 1 << 20 : 1 << 17);
    y.share = blocks < quota ? quota : (2 * quota + 2) / 3;
    y.items = int(y.cut ? blocks < quota ? quota : blocks + y.share : blocks);
  };
  const int mt = rows > 16 && !use_wide ? 2 : 1;       // (beside the other kernel it has single tokens, mostly)
  fill(z.few, use_few, 1, use_wide ? kFew : kAll, kStep, mt, 16 * mt);
  const int wt = a.act == SEQ_BF16 ? 2 : 1;
  const long rest = seqs > 1 ? long(a.N - expected) * a.group / (seqs - 1) : 0;          // query rows of another sequence on average
  const bool eight = a.act == SEQ_BF16 && a.c.type == SEQ_BF16 && a.c.dh == 128 && rows >= kEight && most >= kEightRows && (rest <= kFew || rest >= 256);
  const int waves = eight ? 8 : 4;
  fill(z.wide, use_wide, use_few ? kFew + 1 : 1, kAll, kWideStep, wt, 16 * waves * wt);
  z.floats = z.few.cut || z.wide.cut ? (size_t(a.N) * 4 + 63) / 64 * 64 : 0;
  for (PageShape* y : {&z.few, &z.wide}) {
    y->ws = z.floats;
    if (y->cut) z.floats += size_t(y->items) * a.slots * y->rows * (a.c.dh + 2);
  }
  return z;
}

}  // namespace

size_t page_attn_workspace_bytes(const PageAttnArgs& a) { return shapes(a).floats * 4; }

hipError_t launch_page_attn(const PageAttnArgs& a, hipStream_t s) {
  const Shapes z = shapes(a);
#define ATTN(KERNEL, Y, THREADS, ...) hipLaunchKernelGGL((KERNEL<__VA_ARGS__>), dim3(a.slots, std::min(Y.items, kItems), (Y.items + kItems - 1) / kItems), dim3(THREADS), 0, s, a, Y)
#define ATTN_MT(DH, TYPE, ACT)                                                                      \
  do {                                                                                              \
    constexpr bool EIGHT = DH == 128 && TYPE == SEQ_BF16 && ACT == SEQ_BF16;                        \
    if (EIGHT && z.wide.items && z.wide.rows == 256) ATTN(page_attn_wide_kernel, z.wide, 8 * kWave, DH, TYPE, ACT, (ACT == SEQ_BF16 ? 2 : 1), (EIGHT ? 8 : 4)); \
    else if (z.wide.items) ATTN(page_attn_wide_kernel, z.wide, 4 * kWave, DH, TYPE, ACT, (ACT == SEQ_BF16 ? 2 : 1), 4); \
    if (z.few.items && z.few.mt == 1) ATTN(page_attn_kernel, z.few, kBlock, DH, TYPE, ACT, 1);      \
    else if (z.few.items) ATTN(page_attn_kernel, z.few, kBlock, DH, TYPE, ACT, 2);                  \
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
  if (e != hipSuccess || z.floats == 0) return e;
  const int rows = a.N * a.slots * a.group;
#define JOIN_PARTS(DH, ACT, PARTS)                                                                                      \
  hipLaunchKernelGGL((page_join_kernel<DH, ACT, PARTS>), dim3(int((long(rows) * PARTS + 4 * kBlock / DH - 1) / (4 * kBlock / DH))), \
                     dim3(kBlock), 0, s, a, z.few, z.wide)
#define JOIN(DH, ACT)                                                 \
  do {                                                                \
    if (rows < 2048) JOIN_PARTS(DH, ACT, 4 * kBlock / DH);            \
    else if (rows < 8192) JOIN_PARTS(DH, ACT, 4);                     \
    else JOIN_PARTS(DH, ACT, 1);                                      \
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
