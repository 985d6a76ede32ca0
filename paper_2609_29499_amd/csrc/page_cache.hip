// Caches in pages: packed tokens of several sequences written into their pages (rotary positions, quantised as they are
// written), and rows read back.
//
// Writing. y = rotation of x by position * frequency for k (and q), y = v for v. Pages in 8 bits hold codes and one scale
// s per page and KV head: s = max(|y|) / qmax (127 or 448) over all that was written there since row 0 was. A call whose rows
// raise it rounds the older rows' codes again, code' = round(code s_old / s); new rows are round(y / s). The rotated
// rows of a page and head must all be known before the first code is, so a workgroup holds them in registers: a lane eight
// elements of a head (both halves of four pairs) for each of NP rows, in float32. The page's sines and cosines go through LDS and serve all the heads
// that the workgroup walks.
//
// Bound by memory: 9750 tokens of 64 + 2 x 8 heads of 128, float32 into INT8 pages of 64, and back: 177 us, 4.5 TB/s in all (q's
// launch 125 us at 5.1 TB/s, rows back 18; k and v, in 160 pages x 4 slices of heads, 36 us at 2.8 TB/s: two and a half workgroups per CU,
// each of which waits twice per head for its largest value). A step of one token each is latency (7 us).
#include <algorithm>

#include "attn_tiles.hpp"
#include "device_common.hpp"
#include "page.hpp"
#include "rotary.hpp"

namespace tasp {
namespace {

struct KvMap {
  unsigned char h[64];
};

// How a call is launched: page items (upper bound), page items' slices of `per` of the 2 n_kv (k, v) heads, token groups of
// `tokens` and their slices of `rows` query head rows
struct AppendShape {
  int items, slices, per;
  int groups, tokens, q_slices, rows;
};

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = row_max_u32<16>(v);
  auto at = [&](int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); };
  return max(max(at(0), at(16)), max(at(32), at(48)));
}

// A lane's eight elements of a head: two pieces of four that hold both halves of four pairs, so that a row is read
// once. Rows of interleaved pairs, and what is not rotated: neighbours.
struct Pieces {
  int at[2];
  __device__ __forceinline__ Pieces(int lane, int rot, bool interleaved) {
    const int e0 = kE * lane;
    const bool apart = !interleaved && e0 < rot;
    at[0] = apart ? 4 * lane : e0;
    at[1] = apart ? rot / 2 + 4 * lane : e0 + 4;
  }
};
// the elements as they lie
template <int ACT>
struct Raw8 {
  uint32_t w[ACT == SEQ_BF16 ? 4 : 8];
};
template <int ACT>
__device__ __forceinline__ Raw8<ACT> load_raw(const void* p, long row, const Pieces& e) {
  Raw8<ACT> x;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (ACT == SEQ_BF16) {
      const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + row + e.at[k]);
      x.w[2 * k] = q.x; x.w[2 * k + 1] = q.y;
    } else {
      const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint32_t*>(p) + row + e.at[k]);
      x.w[4 * k] = q.x; x.w[4 * k + 1] = q.y; x.w[4 * k + 2] = q.z; x.w[4 * k + 3] = q.w;
    }
  }
  return x;
}
template <int ACT>
__device__ __forceinline__ Vec8 values_of(const Raw8<ACT>& x) {
  Vec8 v;
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    if constexpr (ACT == SEQ_BF16) v.v[i] = i & 1 ? bf16_hi(x.w[i / 2]) : bf16_lo(x.w[i / 2]);
    else v.v[i] = __uint_as_float(x.w[i]);
  }
  return v;
}
// the same of a sum of arrays (a projection's splits, a.split floats apart), in their order
template <int ACT>
__device__ __forceinline__ void add_splits(Vec8& x, const PageAppendArgs& a, const void* p, long row, const Pieces& e) {
  if constexpr (ACT == SEQ_F32)
    for (int z = 1; z < a.ks; ++z) {
      const Vec8 y = values_of<ACT>(load_raw<ACT>(p, row + z * a.split, e));
#pragma unroll
      for (int i = 0; i < kE; ++i) x.v[i] += y.v[i];
    }
}
template <int ACT>
__device__ __forceinline__ void store_pieces(void* p, long row, const Pieces& e, const Vec8& x) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float* v = x.v + 4 * k;
    if constexpr (ACT == SEQ_BF16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + row + e.at[k]) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(p) + row + e.at[k]) = make_float4(v[0], v[1], v[2], v[3]);
  }
}
// cs: the sines and cosines of the lane's four pairs
__device__ __forceinline__ void rotate_pieces(Vec8& x, const float2* cs, bool interleaved) {
  Vec8 y = x;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y.v[2 * i] = x.v[2 * i] * cs[i].x - x.v[2 * i + 1] * cs[i].y;
      y.v[2 * i + 1] = x.v[2 * i + 1] * cs[i].x + x.v[2 * i] * cs[i].y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y.v[i] = x.v[i] * cs[i].x - x.v[4 + i] * cs[i].y;
      y.v[4 + i] = x.v[i] * cs[i].y + x.v[4 + i] * cs[i].x;
    }
  }
  x = y;
}

// x / s for |x| up to qmax s about, by a refined reciprocal: s is brought near 1 by a power of two first
struct Quotient {
  float k, am, rc;
  __device__ __forceinline__ explicit Quotient(float s) {
    k = s < 0x1p-60f ? 0x1p80f : s > 0x1p60f ? 0x1p-40f : 1.0f;
    am = s * k;
    rc = __builtin_amdgcn_rcpf(am);
    rc = fmaf(fmaf(-am, rc, 1.0f), rc, rc);
  }
  __device__ __forceinline__ float operator()(float x) const {
    const float n = x * k, q = n * rc;
    return fmaf(fmaf(-q, am, n), rc, q);
  }
};

// eight values in units of the scale as codes
template <int TYPE>
__device__ __forceinline__ uint2 codes8(const float (&q)[kE]) {
  constexpr float QMAX = TYPE == SEQ_INT8 ? 127.0f : 448.0f;
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fminf(fmaxf(q[4 * j + i], -QMAX), QMAX);
    if constexpr (TYPE == SEQ_INT8) {
      w[j] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[j] |= (uint32_t(int(rintf(x[i]))) & 0xffu) << (8 * i);
    } else {
      const int o = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
      w[j] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], o, true));
    }
  }
  return make_uint2(w[0], w[1]);
}
template <int TYPE>
__device__ __forceinline__ void values8(uint2 w, float f, float (&x)[kE]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int wd = int(j ? w.y : w.x);
    if constexpr (TYPE == SEQ_INT8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * j + e] = f * float(int8_t(wd >> (8 * e)));
    } else {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(wd, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(wd, true);
      x[4 * j] = f * lo[0]; x[4 * j + 1] = f * lo[1]; x[4 * j + 2] = f * hi[0]; x[4 * j + 3] = f * hi[1];
    }
  }
}

// Grid (page items, then token groups; slices). NP: rows of a page per lane.
template <int DH, int ACT, int TYPE, int NP>
__global__ __launch_bounds__(kBlock) void page_append_kernel(PageAppendArgs a, KvMap map, AppendShape y) {
  constexpr int LPR = DH / kE;         // lanes per head row
  constexpr int RPP = kBlock / LPR;    // head rows per pass
  __shared__ float2 cs[NP * RPP][DH / 2];
  __shared__ uint32_t s_top[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = tid / LPR, half = a.rot / 2, pair0 = 4 * (tid % LPR);
  const Pieces e(tid % LPR, a.rot, a.interleaved);
  const bool turns = kE * (tid % LPR) < a.rot;

  if (int(blockIdx.x) >= y.items) {
    // ---- q of a token group
    if (int(blockIdx.y) >= y.q_slices) return;
    const int t0 = (blockIdx.x - y.items) * y.tokens;
    __shared__ int s_state[4];         // of a token: 0 no sequence's, 1 absent, 2 there
    // a pass's elements, asked for a pass ahead, the first ahead of the tokens' places
    struct Row {
      Raw8<ACT> x;
      int w, h;                        // token of the group, head
      bool in;
    };
    const int r0 = blockIdx.y * y.rows, r1 = min(min(y.tokens, a.N - t0) * a.n_q, r0 + y.rows);
    const float inv = 1.0f / float(a.n_q);
    auto fetch = [&](int r, Row& p) __attribute__((always_inline)) {
      p.in = r < r1;
      p.w = int((float(r) + 0.5f) * inv);              // (r < 4 * 512)
      p.h = r - p.w * a.n_q;
      if (p.in) p.x = load_raw<ACT>(a.q.p, (t0 + p.w) * a.q.token + p.h * a.q.head, e);
    };
    Row next;
    fetch(r0 + own, next);
    if (wave < y.tokens) {
      const int t = t0 + wave;
      int state = 0, pos = 0;
      if (t < a.N) {
        int b = t;
        if (a.start) {                 // the sequence that has the token
          b = a.c.batch;
#pragma unroll
          for (int i = 3; i >= 0; --i) {
            const int at = 64 * i + lane;
            bool mine = false;
            if (at < a.c.batch) {
              const int lo = a.start[at], hi = a.start[at + 1];
              mine = lo >= 0 && hi <= a.N && t >= lo && t < hi;
            }
            const unsigned long long who = __ballot(mine);
            if (who) b = 64 * i + __ffsll((long long)who) - 1;
          }
        }
        if (b < a.c.batch) {
          const PageSeq q = page_seq(a.start, a.N, a.c, b);
          if (t >= q.first && t < q.first + q.n) {
            pos = q.L + t - q.first;
            state = q.L >= 0 && pos < a.c.cap ? 2 : 1;
          }
        }
      }
      if (state == 2 && lane < half) cs[wave][lane] = turn(double(pos), pair_freq(a, lane), a.mscale);
      if (lane == 0) s_state[wave] = state;
    }
    __syncthreads();
    for (int r = r0 + own; r - own < r1; r += RPP) {
      const Row now = next;
      if (r - own + RPP < r1) fetch(r + RPP, next);
      if (!now.in) continue;
      const int state = s_state[now.w];
      const long to = (t0 + now.w) * a.q_out.token + now.h * a.q_out.head;
      if (state == 0) {
        if (a.rest.p) {
          store_pieces<ACT>(a.q_out.p, to, e, Vec8{});
          store_pieces<ACT>(a.rest.p, (t0 + now.w) * a.rest.token + now.h * a.rest.head, e, Vec8{});
        }
        continue;
      }
      Vec8 x{};
      if (state == 2) {
        x = values_of<ACT>(now.x);
        add_splits<ACT>(x, a, a.q.p, (t0 + now.w) * a.q.token + now.h * a.q.head, e);
        if (turns) rotate_pieces(x, &cs[now.w][pair0], a.interleaved);
      }
      store_pieces<ACT>(a.q_out.p, to, e, x);
    }
    return;
  }

  // ---- k and v of a page: which one, a sequence of 64 lanes' 4 each
  if (int(blockIdx.y) >= y.slices) return;
  int pages[4], before[4], L4[4], n4[4], f4[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const PageSeq q = page_seq(a.start, a.N, a.c, min(4 * lane + i, a.c.batch - 1));
    const int n = 4 * lane + i < a.c.batch && q.L >= 0 ? min(q.n, a.c.cap - q.L) : 0;
    L4[i] = q.L; n4[i] = n; f4[i] = q.first;
    pages[i] = n > 0 ? ((q.L + n - 1) >> a.c.P_log) - (q.L >> a.c.P_log) + 1 : 0;
    before[i] = sum;
    sum += pages[i];
  }
  const int all = wave_scan(sum) - sum, item = blockIdx.x;
  int hit = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    before[i] += all;
    if (item >= before[i] && item < before[i] + pages[i]) hit = i;
  }
  const unsigned long long owners = __ballot(hit >= 0);
  if (!owners) return;
  const int owner = __builtin_amdgcn_readfirstlane(__ffsll((long long)owners) - 1), sub = __builtin_amdgcn_readlane(hit, owner);
  const int b = 4 * owner + sub, L = pick(L4, owner, sub), n = pick(n4, owner, sub), first = pick(f4, owner, sub);
  const int pg = (L >> a.c.P_log) + item - pick(before, owner, sub), row0 = pg << a.c.P_log;
  const int page = a.c.table[size_t(b) * a.c.width + pg];
  if (page < 0 || page >= a.c.n_pages) return;          // rows without a page are not written
  const int lo = max(L - row0, 0), hi = min(L + n - row0, a.c.P);       // the page's new rows
  const int c0 = blockIdx.y * y.per, c1 = min(2 * a.n_kv, c0 + y.per);
  // A head's new rows, asked for a head ahead. (A branch around a load would wait for it: rows that are not new read the last one.)
  auto fetch = [&](int c, Raw8<ACT> (&raw)[NP]) __attribute__((always_inline)) {
    const SeqRows& src = c & 1 ? a.v : a.k;
#pragma unroll
    for (int p = 0; p < NP; ++p)
      raw[p] = load_raw<ACT>(src.p, long(first + row0 + min(max(p * RPP + own, lo), hi - 1) - L) * src.token + (c >> 1) * src.head, e);
  };
  Raw8<ACT> next[NP];
  fetch(c0, next);
  if (half > 0 && (c0 & 1 ? c0 + 1 : c0) < c1) {       // a head of k among them
    const double f = lane < half ? pair_freq(a, lane) : 0.0;
    for (int r = lo + wave; r < hi; r += 4)
      if (lane < half) cs[r][lane] = turn(double(row0 + r), f, a.mscale);
    __syncthreads();
  }
  for (int c = c0; c < c1; ++c) {                      // k and v of a head take turns
    const bool is_v = c & 1;
    const SeqRows& src = is_v ? a.v : a.k;
    const size_t unit = size_t(page) * a.c.n_kv + map.h[c >> 1];
    float* scale = TYPE == SEQ_BF16 ? nullptr : (is_v ? a.c.vs : a.c.ks) + unit;
    float was = TYPE != SEQ_BF16 && lo > 0 ? *scale : 0.0f;
    const size_t base = (unit << a.c.P_log) * DH;      // elements
    Vec8 x[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) x[p] = values_of<ACT>(next[p]);
    if (c + 1 < c1) fetch(c + 1, next);
    uint32_t top = 0;                  // magnitudes as integers: infinities and NaN on top
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int r = p * RPP + own;
      if (r >= lo && r < hi) {
        add_splits<ACT>(x[p], a, src.p, long(first + row0 + r - L) * src.token + (c >> 1) * src.head, e);
        if (!is_v && turns) rotate_pieces(x[p], &cs[r][pair0], a.interleaved);
        if constexpr (TYPE == SEQ_BF16) {
          store_pieces<SEQ_BF16>(is_v ? a.c.v : a.c.k, long(base + size_t(r) * DH), e, x[p]);
        } else {
#pragma unroll
          for (int i = 0; i < kE; ++i) top = max(top, __float_as_uint(x[p].v[i]) & 0x7fffffffu);
        }
      }
    }
    if constexpr (TYPE != SEQ_BF16) {
      constexpr float QMAX = TYPE == SEQ_INT8 ? 127.0f : 448.0f;
      top = wave_max_u32(top);
      asm volatile("" : "+v"(was));    // here in every wave before one stores the new scale: a barrier alone does not wait for loads
      __syncthreads();                 // (s_top of the head before is read no more)
      if (lane == 0) s_top[wave] = top;
      __syncthreads();
      top = max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3]));
      // an infinity or a NaN leaves the page and head without a scale: all of it reads as NaN
      const bool fine = top < 0x7f800000u && fabsf(was) < INFINITY;
      const float now = fine ? fmaxf(was, __uint_as_float(top) / QMAX) : __builtin_nanf("");
      const bool some = fine && now > 0.0f;
      const Quotient by(some ? now : 1.0f);
      const bool again = some && now > was;            // older rows' codes change
      const float f = again ? was / now : 0.0f;
      uint8_t* out = static_cast<uint8_t*>(is_v ? a.c.v : a.c.k) + base;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int r = p * RPP + own;
        uint32_t* w0 = reinterpret_cast<uint32_t*>(out + r * DH + e.at[0]);
        uint32_t* w1 = reinterpret_cast<uint32_t*>(out + r * DH + e.at[1]);
        float q[kE];
        if (r >= lo && r < hi) {
#pragma unroll
          for (int i = 0; i < kE; ++i) q[i] = some ? by(x[p].v[i]) : 0.0f;
        } else if (again && r < lo) {
          values8<TYPE>(make_uint2(*w0, *w1), f, q);
        } else {
          continue;
        }
        const uint2 w = codes8<TYPE>(q);
        *w0 = w.x;
        *w1 = w.y;
      }
      if (tid == 0) *scale = now;
    }
  }
}

// Rows first + i of every sequence and head as BF16 or float32; rows outside the table's pages or without a page read as
// zeros. A lane holds eight elements. Grid (rows, heads of all sequences, k / v).
template <int DH, int TYPE, int OUT>
__global__ __launch_bounds__(kBlock) void page_read_kernel(PageReadArgs a) {
  constexpr int LPR = DH / kE;
  const int i = blockIdx.x * (kBlock / LPR) + threadIdx.x / LPR, e0 = kE * (threadIdx.x % LPR);
  const int u = blockIdx.y, b = u / a.c.n_kv, h = u % a.c.n_kv;
  if (i >= a.n) return;
  const SeqRows& dst = blockIdx.z ? a.v : a.k;
  const void* src = blockIdx.z ? a.c.v : a.c.k;
  const long r = long(a.first ? a.first[b] : 0) + i;
  Vec8 x{};
  if (r >= 0 && r < a.c.cap) {
    const int page = a.c.table[size_t(b) * a.c.width + (r >> a.c.P_log)];
    if (page >= 0 && page < a.c.n_pages) {
      const size_t unit = size_t(page) * a.c.n_kv + h, at = ((unit << a.c.P_log) + (r & (a.c.P - 1))) * DH + e0;
      if constexpr (TYPE == SEQ_BF16)
        x = load8<SEQ_BF16>(src, long(at));
      else
        values8<TYPE>(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(src) + at), (blockIdx.z ? a.c.vs : a.c.ks)[unit], x.v);
    }
  }
  store8<OUT>(dst.p, b * dst.seq + i * dst.token + h * dst.head + e0, x);
}

// Lengths grow by the sequences' new tokens: a thread each.
__global__ __launch_bounds__(kBlock) void page_advance_kernel(PageAdvanceArgs a) {
  static_assert(kSeqMaxBatch <= kBlock, "one workgroup");
  const int b = threadIdx.x;
  if (b >= a.c.batch) return;
  const PageSeq q = page_seq(a.start, a.N, a.c, b);
  if (q.L >= 0 && q.n > 0) a.len[b] = min(q.L + min(q.n, a.c.cap), a.c.cap);
}

}  // namespace

hipError_t launch_page_advance(const PageAdvanceArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(page_advance_kernel, dim3(1), dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_append(const PageAppendArgs& a, hipStream_t s) {
  if (a.N < 1 || a.n_kv < 1 || a.n_kv > 64 || a.n_q < 0 || a.n_q > 512) return hipErrorInvalidValue;
  KvMap map{};
  for (int j = 0; j < a.n_kv; ++j) map.h[j] = (unsigned char)(a.kv_map ? a.kv_map[j] : j);
  const int rpp = kBlock / (a.c.dh / kE);
  AppendShape y{};
  // n tokens of a sequence touch at most n pages, and n / P + 2
  y.items = a.start ? int(std::min<long>(a.N, a.N / a.c.P + 2L * a.c.batch)) : a.c.batch;
  // two heads of k and of v per workgroup share a page's sines and cosines where that leaves enough of them (9750 tokens, pages of
  // 64: 177.7 us in all, 180.0 with one head, 180.4 with four, 181.7 with k or v of one; k or v of one against two heads of both, all
  // of a call: 128 single tokens of 64 / 8 heads into INT8 14.8 / 13.6 us, 1024 tokens of 4 prompts 25.0 / 30.1, 4096 63.9 / 66.3; 32 / 8 heads into BF16
  // pages of 16, 1024 tokens 15.1 / 15.1, 2048 20.3 / 18.6, 4096 29.1 / 24.0)
  y.per = long(y.items) * 2 * a.n_kv >= 2048 ? 4 : 1;
  y.slices = (2 * a.n_kv + y.per - 1) / y.per;
  y.tokens = a.N >= 1024 ? 4 : 1;
  y.groups = a.n_q ? (a.N + y.tokens - 1) / y.tokens : 0;
  y.rows = a.N >= 1024 ? y.tokens * a.n_q : rpp;
  y.q_slices = a.n_q ? (y.tokens * a.n_q + y.rows - 1) / y.rows : 0;
  // Many tokens: q in a launch of its own, which has the LDS of a small page, and so more workgroups per CU (one launch / two, 64 / 8 heads of
  // float32 into INT8 pages of 64: 512 tokens 18.3 / 22.3 us, 1000 24.5 / 23.9, 1500 31.8 / 28.5, 4096 77.5 / 64.4; 32 / 8 heads in BF16, pages of 16: 768
  // 11.7 / 14.0, 1024 13.7 / 15.2, 2048 17.2 / 18.5, 4096 26.2 / 24.0)
  AppendShape q = y;
  const bool apart = a.N >= 1024 && y.groups > 0;
  if (apart) {
    y.groups = y.q_slices = 0;
    q.items = q.slices = 0;
  }
#define APPEND(DH, ACT, TYPE, NP, Y) \
  hipLaunchKernelGGL((page_append_kernel<DH, ACT, TYPE, NP>), dim3(Y.items + Y.groups, std::max(Y.slices, Y.q_slices)), dim3(kBlock), 0, s, a, map, Y)
#define APPEND_NP(DH, ACT, TYPE)                                         \
  do {                                                                   \
    if (apart) APPEND(DH, ACT, TYPE, 1, q);                              \
    if (a.c.P <= kBlock * kE / DH) APPEND(DH, ACT, TYPE, 1, y);          \
    else if (a.c.P <= 2 * kBlock * kE / DH) APPEND(DH, ACT, TYPE, 2, y); \
    else if (a.c.P <= 4 * kBlock * kE / DH) APPEND(DH, ACT, TYPE, 4, y); \
    else if constexpr (DH == 128) APPEND(DH, ACT, TYPE, 8, y);           \
  } while (0)
#define APPEND_TYPE(DH, ACT)                                      \
  do {                                                            \
    if (a.c.type == SEQ_BF16) APPEND_NP(DH, ACT, SEQ_BF16);       \
    else if (a.c.type == SEQ_INT8) APPEND_NP(DH, ACT, SEQ_INT8);  \
    else APPEND_NP(DH, ACT, SEQ_E4M3);                            \
  } while (0)
  if (a.c.dh == 128) {
    if (a.act == SEQ_BF16) APPEND_TYPE(128, SEQ_BF16);
    else APPEND_TYPE(128, SEQ_F32);
  } else {
    if (a.act == SEQ_BF16) APPEND_TYPE(64, SEQ_BF16);
    else APPEND_TYPE(64, SEQ_F32);
  }
#undef APPEND_TYPE
#undef APPEND_NP
#undef APPEND
  return hipGetLastError();
}

hipError_t launch_page_read(const PageReadArgs& a, hipStream_t s) {
  const int rpp = kBlock / (a.c.dh / kE);
  const dim3 grid((a.n + rpp - 1) / rpp, a.c.batch * a.c.n_kv, 2);
#define READ(DH, TYPE, OUT) hipLaunchKernelGGL((page_read_kernel<DH, TYPE, OUT>), grid, dim3(kBlock), 0, s, a)
#define READ_TYPE(DH, OUT)                                   \
  do {                                                       \
    if (a.c.type == SEQ_BF16) READ(DH, SEQ_BF16, OUT);       \
    else if (a.c.type == SEQ_INT8) READ(DH, SEQ_INT8, OUT);  \
    else READ(DH, SEQ_E4M3, OUT);                            \
  } while (0)
  if (a.c.dh == 128) {
    if (a.out_type == SEQ_BF16) READ_TYPE(128, SEQ_BF16);
    else READ_TYPE(128, SEQ_F32);
  } else {
    if (a.out_type == SEQ_BF16) READ_TYPE(64, SEQ_BF16);
    else READ_TYPE(64, SEQ_F32);
  }
#undef READ_TYPE
#undef READ
  return hipGetLastError();
}

}  // namespace tasp
