// Caches whose sequences have their own lengths: rows written behind them (rotary positions,
// quantised as they are written), rows read back, and an accepted path's rows moved together.
//
// Writing. y = rotation of x by pos * inv_freq for q and k, y = v for v; a cache in 8 bits holds
// c = round(y qmax / max|y|) and the scale max|y| / qmax per row and head (qmax 127 or 448). The angle
// is a product of two 64-bit numbers, cut to one turn in 64 bits (positions of 10^5 and more leave
// nothing of a 32-bit angle's last digits), and its sine and cosine are taken in 32 bits of the rest. One workgroup serves
// head rows of one token: a lane holds eight elements of a head, so the row's maximum stays inside 8
// or 16 lanes and every access is 16 or 32 bytes wide; the token's sines and cosines go through LDS.
// Bound by memory: q, k and v are read once, q and the rows written once (2 x 8192 tokens of 32 + 2 x 8 heads of 128 in
// float32 into INT8, 705 MB: 141 us, 5.0 TB/s; 8 trees of 32, 10 MB: 6.7 us, latency: lengths and tree, then sines).
#include <algorithm>

#include "device_common.hpp"
#include "rotary.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

struct KvMap {
  unsigned char h[64];
};

// Grid (sequence tokens, slices of a token's head rows). rows: head rows per workgroup.
template <int DH, int ACT, int TYPE>
__global__ __launch_bounds__(kBlock) void seq_append_kernel(SeqAppendArgs a, KvMap map, int rows) {
  constexpr int LPR = DH / kE;         // lanes per head row
  constexpr int RPP = kBlock / LPR;    // head rows per pass
  __shared__ float2 cs[DH / 2];
  __shared__ int s_pos, s_row;
  const int tid = threadIdx.x;
  const int b = blockIdx.x / a.T, t = blockIdx.x % a.T;
  const int total = a.n_q + 2 * a.n_kv;
  const int r0 = blockIdx.y * rows, r1 = min(total, r0 + rows);
  const int e0 = kE * (tid % LPR);
  // A pass's elements, and their partners where pairs lie apart: asked for a pass ahead, the first ahead of the token's
  // place in its tree. (Rows of absent nodes are read like others; whole rows are in or out, reductions stay inside a row.)
  struct Pass {
    Vec8 x, y;
    int kind, h, head;                 // q, k, v; head; cache head
  };
  auto fetch = [&](int r, Pass& p) __attribute__((always_inline)) {
    const bool in = r < r1;
    p.kind = !in || r < a.n_q ? 0 : r < a.n_q + a.n_kv ? 1 : 2;
    const SeqRows& src = p.kind == 0 ? a.q : p.kind == 1 ? a.k : a.v;
    p.h = !in ? 0 : p.kind == 0 ? r : p.kind == 1 ? r - a.n_q : r - a.n_q - a.n_kv;
    if (!in) return;
    p.head = p.kind > 0 ? map.h[p.h] : 0;
    const long row = b * src.seq + t * src.token + p.h * src.head;
    p.x = load8<ACT>(src.p, row + e0, a);
    if (p.kind < 2 && e0 < a.rot && !a.interleaved)
      p.y = load8<ACT>(src.p, row + (e0 < a.rot / 2 ? e0 + a.rot / 2 : e0 - a.rot / 2), a);
  };
  Pass next;
  fetch(r0 + tid / LPR, next);
  if (tid < kWave) {
    const int L = seq_len(a.c.len, b, a.c.S);
    int depth = t, there = 1;
    if (a.parent) {                    // at most kTreeMax nodes
      const TreeNode nd = tree_node(a.parent + size_t(b) * a.T, a.T, a.T, tid);
      depth = __popcll(__shfl(nd.anc, t, kWave)) - 1;
      there = depth >= 0;
    }
    there = there && L >= 0 && L + t < a.c.S;
    for (int i = tid; i < a.rot / 2; i += kWave) cs[i] = turn(double(L + depth), pair_freq(a, i), a.mscale);
    if (tid == 0) {
      s_pos = there ? L + depth : -1;
      s_row = L + t;
    }
  }
  __syncthreads();
  const bool there = s_pos >= 0;
  for (int r = r0 + tid / LPR; r - tid / LPR < r1; r += RPP) {
    const bool in = r < r1;
    const Pass now = next;
    if (r - tid / LPR + RPP < r1) fetch(r + RPP, next);
    const int kind = now.kind, h = now.h;
    Vec8 x{};
    if (in && there) {
      x = now.x;
      if (kind < 2 && e0 < a.rot) {
        if (a.interleaved) {           // pairs (2 i, 2 i + 1)
#pragma unroll
          for (int i = 0; i < kE; i += 2) {
            const float2 w = cs[(e0 + i) / 2];
            const float p = x.v[i], q = x.v[i + 1];
            x.v[i] = p * w.x - q * w.y;
            x.v[i + 1] = q * w.x + p * w.y;
          }
        } else {                       // pairs (i, i + rot / 2): the partner's eight elements
          const int half = a.rot / 2;
          const bool first = e0 < half;
#pragma unroll
          for (int i = 0; i < kE; ++i) {
            const float2 w = cs[(first ? e0 : e0 - half) + i];
            x.v[i] = first ? x.v[i] * w.x - now.y.v[i] * w.y : x.v[i] * w.x + now.y.v[i] * w.y;
          }
        }
      }
    }
    if (in && kind == 0) {
      store8<ACT>(a.q_out.p, b * a.q_out.seq + t * a.q_out.token + h * a.q_out.head + e0, x);
    }
    if constexpr (TYPE == SEQ_BF16) {
      if (in && there && kind > 0) {
        const size_t at = (size_t(b) * a.c.n_kv + now.head) * a.c.S + s_row;
        store8<SEQ_BF16>(kind == 1 ? a.c.k : a.c.v, long(at * DH + e0), x);
      }
    } else {
      uint32_t top = 0;                // magnitudes as integers: infinities and NaN on top
#pragma unroll
      for (int i = 0; i < kE; ++i) top = max(top, __float_as_uint(x.v[i]) & 0x7fffffffu);
      top = row_max_u32<LPR>(top);
      if (in && there && kind > 0) {
        constexpr float QMAX = TYPE == SEQ_INT8 ? 127.0f : 448.0f;
        const float amax = __uint_as_float(top);
        const bool fine = top < 0x7f800000u && top > 0;
        // code = x qmax / amax by a refined reciprocal: exact where the quotient is (a code border is hit
        // by BF16 inputs), with rows far from 1 brought near it by a power of two first
        const float k = !fine ? 0.0f : amax < 0x1p-60f ? 0x1p80f : amax > 0x1p60f ? 0x1p-40f : 1.0f;
        const float am = fine ? amax * k : 1.0f;
        float rc = __builtin_amdgcn_rcpf(am);
        rc = fmaf(fmaf(-am, rc, 1.0f), rc, rc);
        float q[kE];
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          const float n = fine ? x.v[i] * k * QMAX : 0.0f;
          q[i] = n * rc;
          q[i] = fmaf(fmaf(-q[i], am, n), rc, q[i]);
        }
        uint32_t w[2];
        if constexpr (TYPE == SEQ_INT8) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            w[j] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[j] |= (uint32_t(int(rintf(q[4 * j + i]))) & 0xffu) << (8 * i);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            int o = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * j], q[4 * j + 1], 0, false);
            w[j] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * j + 2], q[4 * j + 3], o, true));
          }
        }
        const size_t at = (size_t(b) * a.c.n_kv + now.head) * a.c.S + s_row;
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(kind == 1 ? a.c.k : a.c.v) + at * DH + e0) = make_uint2(w[0], w[1]);
        // a row with an infinity or a NaN has no scale: it reads back as NaN
        if (e0 == 0) (kind == 1 ? a.c.ks : a.c.vs)[at] = top >= 0x7f800000u ? __builtin_nanf("") : amax / QMAX;
      }
    }
  }
}

// Rows first + i of every sequence and head as BF16 or float32; rows outside the cache read as zeros.
// A lane holds eight elements. Grid (rows, heads of all sequences, k / v).
template <int DH, int TYPE, int OUT>
__global__ __launch_bounds__(kBlock) void seq_read_kernel(SeqReadArgs a) {
  constexpr int LPR = DH / kE;
  const int i = blockIdx.x * (kBlock / LPR) + threadIdx.x / LPR, e0 = kE * (threadIdx.x % LPR);
  const int u = blockIdx.y, b = u / a.c.n_kv, h = u % a.c.n_kv;
  if (i >= a.n) return;
  const SeqRows& dst = blockIdx.z ? a.v : a.k;
  const void* src = blockIdx.z ? a.c.v : a.c.k;
  const long r = long(a.first ? a.first[b] : 0) + i;
  Vec8 x{};
  if (r >= 0 && r < a.c.S) {
    const size_t at = size_t(u) * a.c.S + size_t(r);
    if constexpr (TYPE == SEQ_BF16) {
      x = load8<SEQ_BF16>(src, long(at * DH + e0));
    } else {
      const float sc = (blockIdx.z ? a.c.vs : a.c.ks)[at];
      const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(src) + at * DH + e0);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int wd = int(j ? w.y : w.x);
        if constexpr (TYPE == SEQ_INT8) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[4 * j + e] = sc * float(int8_t(wd >> (8 * e)));
        } else {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(wd, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(wd, true);
          x.v[4 * j] = sc * lo[0]; x.v[4 * j + 1] = sc * lo[1]; x.v[4 * j + 2] = sc * hi[0]; x.v[4 * j + 3] = sc * hi[1];
        }
      }
    }
  }
  store8<OUT>(dst.p, b * dst.seq + i * dst.token + h * dst.head + e0, x);
}

__device__ __forceinline__ int next_len(const SeqCommitArgs& a, int b) {
  const int L = a.c.len[b], n = max(0, min(min(a.n[b], a.ld), kTreeMax));
  return L < 0 || L > a.c.S ? L : min(L + n, a.c.S);
}

// Rows len + path[i] -> len + i, i < n, of every layer, sequence and head: grid (HEADS heads of one layer and
// sequence, k / v). The workgroup reads every row that moves before it writes the first (path may
// name rows that earlier entries replace). Rows that stay are not touched. Bound by three latencies in a row
// (length and count, path, rows), which HEADS heads share: 80 layers of 8 x 8 heads, 9 of 64 nodes (42 MB moved):
// 16.7 us with one head per workgroup, 11 with four.
template <int RB, int HEADS>           // bytes of a row
__global__ __launch_bounds__(kBlock) void seq_commit_kernel(SeqCommitArgs a) {
  constexpr int LPR = RB / 16, RPP = kBlock / LPR, NP = kTreeMax / RPP;
  const int u = blockIdx.x * HEADS, lb = u / a.c.n_kv, b = lb % a.c.batch;
  const int L = seq_len(a.c.len, b, a.c.S);
  const int n = min(min(a.n[b], a.ld), kTreeMax);
  if (a.apart && lb < a.c.batch && u == lb * a.c.n_kv && blockIdx.y == 0 && threadIdx.x == 0)
    a.len_out[b] = next_len(a, b);
  if (L < 0) return;
  const size_t step = size_t(a.c.S) * RB;
  char* base = static_cast<char*>(blockIdx.y ? a.c.v : a.c.k) + size_t(u) * step;
  float* sc = a.c.ks ? (blockIdx.y ? a.c.vs : a.c.ks) + size_t(u) * a.c.S : nullptr;
  const int li = threadIdx.x / LPR, pc = threadIdx.x % LPR;
  int4 w[NP][HEADS] = {};
  float s[NP][HEADS] = {};
  bool go[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int i = p * RPP + li;
    const int from = i < n ? a.path[size_t(b) * a.ld + i] : -1;
    go[p] = from >= 0 && from < a.ld && from != i && long(L) + from < a.c.S && L + i < a.c.S;
    if (go[p]) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        w[p][h] = *reinterpret_cast<const int4*>(base + h * step + size_t(L + from) * RB + 16 * pc);
        if (sc && pc == 0) s[p][h] = sc[size_t(h) * a.c.S + L + from];
      }
    }
  }
  // the rows are here before any thread of the workgroup stores: a barrier alone does not wait for loads
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
      asm volatile("" : "+v"(w[p][h].x), "+v"(w[p][h].y), "+v"(w[p][h].z), "+v"(w[p][h].w), "+v"(s[p][h]));
  __syncthreads();
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int i = p * RPP + li;
    if (!go[p]) continue;
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      *reinterpret_cast<int4*>(base + h * step + size_t(L + i) * RB + 16 * pc) = w[p][h];
      if (sc && pc == 0) sc[size_t(h) * a.c.S + L + i] = s[p][h];
    }
  }
}

__global__ __launch_bounds__(kBlock) void seq_length_kernel(SeqCommitArgs a) {
  // (len_out may share memory with the lengths or counts, shifted too: all are read, and here, before any is written)
  const int b = threadIdx.x;
  static_assert(kSeqMaxBatch <= kBlock, "one workgroup");
  int L = b < a.c.batch ? next_len(a, b) : 0;
  asm volatile("" : "+v"(L));
  __syncthreads();
  if (b < a.c.batch) a.len_out[b] = L;
}

}  // namespace

hipError_t launch_seq_append(const SeqAppendArgs& a, hipStream_t s) {
  const int total = a.n_q + 2 * a.n_kv;
  if (total < 1 || a.T < 1 || a.n_kv > 64) return hipErrorInvalidValue;
  KvMap map{};
  for (int j = 0; j < a.n_kv; ++j) map.h[j] = (unsigned char)(a.kv_map ? a.kv_map[j] : j);
  const int rpp = kBlock / (a.c.dh / kE);
  // few tokens: one pass of head rows per workgroup (latency: 8 x 32 tokens 6.5 us, 9.4 the other way); many: a
  // workgroup walks its token's rows, so that its sines and cosines are formed once (2 x 8192 tokens 139 us, 151)
  const int rows = long(a.c.batch) * a.T < 1024 ? rpp : total;
  const dim3 grid(a.c.batch * a.T, (total + rows - 1) / rows);
#define APPEND(DH, ACT, TYPE) hipLaunchKernelGGL((seq_append_kernel<DH, ACT, TYPE>), grid, dim3(kBlock), 0, s, a, map, rows)
#define APPEND_TYPE(DH, ACT)                                   \
  do {                                                         \
    if (a.c.type == SEQ_BF16) APPEND(DH, ACT, SEQ_BF16);       \
    else if (a.c.type == SEQ_INT8) APPEND(DH, ACT, SEQ_INT8);  \
    else APPEND(DH, ACT, SEQ_E4M3);                            \
  } while (0)
  if (a.c.dh == 128) {
    if (a.act == SEQ_BF16) APPEND_TYPE(128, SEQ_BF16);
    else APPEND_TYPE(128, SEQ_F32);
  } else {
    if (a.act == SEQ_BF16) APPEND_TYPE(64, SEQ_BF16);
    else APPEND_TYPE(64, SEQ_F32);
  }
#undef APPEND_TYPE
#undef APPEND
  return hipGetLastError();
}

hipError_t launch_seq_read(const SeqReadArgs& a, hipStream_t s) {
  const int rpp = kBlock / (a.c.dh / kE);
  const dim3 grid((a.n + rpp - 1) / rpp, a.c.batch * a.c.n_kv, 2);
#define READ(DH, TYPE, OUT) hipLaunchKernelGGL((seq_read_kernel<DH, TYPE, OUT>), grid, dim3(kBlock), 0, s, a)
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

hipError_t launch_seq_commit(const SeqCommitArgs& a, hipStream_t s) {
  const int units = a.n_layers * a.c.batch * a.c.n_kv;
  // four heads per workgroup where that leaves four workgroups per CU (5120 heads 11 us, 16.7 the other way; 256 heads
  // one each 3.5 us, 3.8)
  const bool four = a.c.n_kv % 4 == 0 && units >= 2048;
  const dim3 grid(four ? units / 4 : units, 2);
  const int rb = a.c.dh * (a.c.type == SEQ_BF16 ? 2 : 1);
#define COMMIT(RB)                                                                                 \
  do {                                                                                             \
    if (four) hipLaunchKernelGGL((seq_commit_kernel<RB, 4>), grid, dim3(kBlock), 0, s, a);         \
    else hipLaunchKernelGGL((seq_commit_kernel<RB, 1>), grid, dim3(kBlock), 0, s, a);              \
  } while (0)
  if (rb == 256) COMMIT(256);
  else if (rb == 128) COMMIT(128);
  else COMMIT(64);
#undef COMMIT
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.apart) return hipSuccess;
  // a launch of its own, of one workgroup (a batch has as many sequences at most): all above read what this one replaces
  hipLaunchKernelGGL(seq_length_kernel, dim3(1), dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

}  // namespace tasp
