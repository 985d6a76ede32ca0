// Scores of given tokens: of every row x of logits the log probability of a token, the entropy, the token's rank, the
// `top` largest logits in order, and the mean log probability of every sequence of rows.
//
// In one pass over a row, in powers of two: t = (x - m) c with c = log2(e) / temperature and m the running maximum,
// s = sum 2^t, w = sum t 2^t. Then log p(x) = ln 2 ((x - m) c - log2 s) and the entropy is ln 2 (log2 s - w / s). Every
// thread has a maximum and sums of its own in float32 (some 500 terms); they meet in float64. (x c - m c, one instruction less,
// loses all digits at small temperatures.)
//
// The largest: elements above a bound go to a list in LDS as 64-bit keys (the logit as an integer that keeps its order,
// then the complement of the index: equal logits are in the order of their indices). The bound of the first 4096 elements is
// the smallest of 32 groups' maxima: at least 32 elements reach it, about 130 do. When the list has grown by 512 it is cut to
// its first `top`, and the last of them is the new bound: of 128256 logits in no particular order some 200 enter it.
//
// Bound by memory: a row is read once. Few rows are cut into pieces whose records a second launch joins.
#include <algorithm>
#include <cmath>

#include "device_common.hpp"
#include "logprob.hpp"

namespace tasp {
namespace {

constexpr int kPer = 16;               // elements of a thread and tile
constexpr int kTile = kBlock * kPer;
constexpr int kLimit = 512;            // keys that are ranked by comparing each with each
constexpr int kKeys = kLimit + kTile;  // the list has room for a whole tile more
constexpr int kTarget = 1024;          // workgroups aimed at
constexpr int kPieces = kKeys / kTopMax;          // of a row at most: the join's list holds all their keys

struct Sums {
  float m, s, w;                       // maximum; sums of 2^t and of t 2^t, t = (x - m) c
};
// the sums under a new maximum
__device__ __forceinline__ void move_to(Sums& a, float m, float c) {
  const float d = (a.m - m) * c, f = __builtin_amdgcn_exp2f(d);
  a.w = f == 0.0f ? 0.0f : (a.w + d * a.s) * f;        // (d s may be infinite then)
  a.s *= f;
  a.m = m;
}

// float -> integer of the same order (finite values), and back
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);        // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ unsigned long long key_of(float x, int i) {
  return (unsigned long long)(ordered(x)) << 32 | (0xffffffffu - uint32_t(i));
}

struct List {
  unsigned long long key[kKeys];
  unsigned long long best[kTopMax];
  int count, found;
  int part[4];
};
__device__ __forceinline__ int block_count(List& z, int v) {   // sum over the workgroup of a wave-uniform count
  __syncthreads();
  if ((threadIdx.x & 63) == 0) z.part[threadIdx.x >> 6] = v;
  __syncthreads();
  return z.part[0] + z.part[1] + z.part[2] + z.part[3];
}
// The list's `top` largest keys to its front, in order. All keys are different. Ends behind a barrier; returns their number.
__device__ __forceinline__ int rank_list(List& z, int top) {
  const int tid = threadIdx.x;
  __syncthreads();
  int n = z.count;
  const int out = min(n, top);
  if (n > kLimit) {
    // the top-th largest key, bit by bit: the largest value that `top` keys reach
    unsigned long long at = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long with = at | 1ull << bit;
      int own = 0;
      for (int i = tid; i - tid < n; i += kBlock) own += __popcll(__ballot(i < n && z.key[i] >= with));
      if (block_count(z, own) >= top) at = with;
    }
    __syncthreads();
    if (tid == 0) z.found = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kBlock)
      if (z.key[i] >= at) z.best[atomicAdd(&z.found, 1)] = z.key[i];
    __syncthreads();
    n = out;
    if (tid < n) z.key[tid] = z.best[tid];
    __syncthreads();
  }
  for (int i = tid; i < n; i += kBlock) {
    const unsigned long long mine = z.key[i];
    int before = 0;
    for (int j = 0; j < n; ++j) before += z.key[j] > mine;
    if (before < out) z.best[before] = mine;
  }
  __syncthreads();
  if (tid < out) z.key[tid] = z.best[tid];
  if (tid == 0) z.count = out;
  __syncthreads();
  return out;
}

// Of a row (or a piece of it): sums, elements that come before the token, and its largest keys
struct Record {
  double s, w;
  float m;
  int before;
};

// Results of a row from its joined record; keys: `n` of them in order. All threads of a wave at least.
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, const Record& z, const unsigned long long* key, int n) {
  const int tid = threadIdx.x;
  const bool empty = z.m <= -a.lim;              // no logit above -inf
  const double log_s = empty ? 0.0 : log2(z.s);
  constexpr double kLn2 = 0.693147180559945309417;
  auto lp = [&](float x) {
    // (an infinite logit leaves nothing to finite ones)
    return empty || x <= -a.lim || (z.m >= a.lim && x < z.m) ? -INFINITY : float(((double(x) - double(z.m)) * double(a.c) - log_s) * kLn2);
  };
  if (tid == 0) {
    const int t = a.tokens[row];
    const bool there = t >= 0 && t < a.V;
    float x = 0.0f;
    if (there) {
      const size_t at = size_t(row) * a.ld + t;
      x = a.f32 ? static_cast<const float*>(a.logits)[at] : bf16_to_f32(static_cast<const uint16_t*>(a.logits)[at]);
      x = fminf(fmaxf(x, -a.lim), a.lim);
    }
    a.logprob[row] = there ? lp(x) : 0.0f;
    if (a.rank) a.rank[row] = there ? z.before : -1;
    if (a.entropy) a.entropy[row] = empty ? 0.0f : float((log_s - z.w / z.s) * kLn2);
  }
  if (tid < a.top) {
    const bool in = tid < n;
    a.top_ids[size_t(row) * a.top + tid] = in ? int(0xffffffffu - uint32_t(key[tid])) : -1;
    a.top_logprobs[size_t(row) * a.top + tid] = in ? lp(unordered(uint32_t(key[tid] >> 32))) : -INFINITY;
  }
}

// The workspace: [rows][pieces] records, then [rows][pieces][top] keys (0: none).
__device__ __forceinline__ Record* records(const LogprobArgs& a) { return static_cast<Record*>(a.ws); }
__device__ __forceinline__ unsigned long long* keys(const LogprobArgs& a, int pieces) {
  return reinterpret_cast<unsigned long long*>(records(a) + size_t(a.rows) * pieces);
}

// A piece of a row: tiles blockIdx.x * per .. of row blockIdx.y.
template <bool F32, bool TOP>
__global__ __launch_bounds__(kBlock) void logprob_kernel(LogprobArgs a, int per) {
  __shared__ List z;
  __shared__ float s_group[32];
  __shared__ Sums s_sums[4];
  __shared__ int s_before[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const char* base = static_cast<const char*>(a.logits) + size_t(row) * a.ld * (F32 ? 4 : 2);
    const int first = blockIdx.x * per * kTile, end = min(long(a.V), long(first) + long(per) * kTile);
    // the token: the smallest key that comes before it in order is one more than its own
    const int token = a.tokens[row];
    const bool there = token >= 0 && token < a.V;
    float xt = INFINITY;
    if (there) {
      xt = F32 ? reinterpret_cast<const float*>(base)[token] : bf16_to_f32(reinterpret_cast<const uint16_t*>(base)[token]);
      xt = fminf(fmaxf(xt, -a.lim), a.lim);
    }
    // element j of this thread: index i0 + at(j)
    float x[kPer], nx[kPer];
    auto index = [&](int tile, int j, bool whole) {
      return !whole ? tile + j * kBlock + tid : F32 ? tile + (j >> 2) * 4 * kBlock + 4 * tid + (j & 3) : tile + (j >> 3) * 8 * kBlock + 8 * tid + (j & 7);
    };
    auto load = [&](int tile, float (&v)[kPer]) {
      if (tile + kTile <= end) {
        if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float4 q;
            __builtin_memcpy(&q, base + (size_t(tile) + j * 4 * kBlock + 4 * tid) * 4, 16);
            v[4 * j] = q.x; v[4 * j + 1] = q.y; v[4 * j + 2] = q.z; v[4 * j + 3] = q.w;
          }
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t q[4];
            __builtin_memcpy(q, base + (size_t(tile) + j * 8 * kBlock + 8 * tid) * 2, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              v[8 * j + 2 * i] = bf16_lo(q[i]);
              v[8 * j + 2 * i + 1] = bf16_hi(q[i]);
            }
          }
        }
      } else {                         // the row's last elements, one by one
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int i = tile + j * kBlock + tid;
          v[j] = i >= end ? -INFINITY : F32 ? reinterpret_cast<const float*>(base)[i] : bf16_to_f32(reinterpret_cast<const uint16_t*>(base)[i]);
        }
      }
    };
    Sums sum{-INFINITY, 0.0f, 0.0f};
    int before = 0;
    float bound = -a.lim;              // elements above it enter the list
    __syncthreads();                   // (the row before has been read)
    if (tid == 0) z.count = 0;
    load(first, nx);
    for (int tile = first; tile < end; tile += kTile) {
      const bool whole = tile + kTile <= end;
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] = fminf(fmaxf(nx[j], -a.lim), a.lim);      // (NaN is -lim)
      if (tile + kTile < end) load(tile + kTile, nx);
      float top = x[0];
#pragma unroll
      for (int j = 1; j < kPer; ++j) top = fmaxf(top, x[j]);
      if (top > sum.m) move_to(sum, top, a.c);
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const float t = (x[j] - sum.m) * a.c, e = __builtin_amdgcn_exp2f(t);
        const bool in = whole || index(tile, j, whole) < end;
        sum.s += in ? e : 0.0f;
        sum.w = fmaf(in ? e : 0.0f, t, sum.w);
      }
      if (token < tile || token >= tile + kTile) {     // (before the token equal ones come first too)
        const bool equal = token >= tile + kTile;
#pragma unroll
        for (int j = 0; j < kPer; ++j) before += __popcll(__ballot((x[j] > xt || (equal && x[j] == xt)) && (whole || index(tile, j, whole) < end)));
      } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int i = index(tile, j, whole);
          before += __popcll(__ballot((x[j] > xt || (i < token && x[j] == xt)) && i < end));
        }
      }
      if constexpr (TOP) {
        bool least = false;            // the bound itself is enough
        if (tile == first) {
          float g = top;
          g = fmaxf(g, dpp<kQuadXor1>(g));
          g = fmaxf(g, dpp<kQuadXor2>(g));
          g = fmaxf(g, dpp<kRowHalfMirror>(g));
          if ((lane & 7) == 0) s_group[tid >> 3] = g;
          __syncthreads();
          g = s_group[lane & 31];
          bound = -wave_max(-g);
          least = bound > -a.lim;
        }
        if (__ballot(top > bound || (least && top == bound))) {
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            const bool take = x[j] > bound || (least && x[j] == bound);
            const unsigned long long who = __ballot(take);
            if (who) {
              int at = 0;
              if (lane == 0) at = atomicAdd(&z.count, __popcll(who));
              at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0));
              if (take) z.key[at] = key_of(x[j], index(tile, j, whole));
            }
          }
        }
        __syncthreads();
        const int count = z.count;
        __syncthreads();               // (read by all before the next tile adds to it)
        if (count > kLimit) {
          rank_list(z, a.top);
          bound = fmaxf(bound, unordered(uint32_t(z.key[a.top - 1] >> 32)));
        }
      }
    }
    int n = 0;
    if constexpr (TOP) n = rank_list(z, a.top);
    // the workgroup's sums
    {
      const float m = wave_max(sum.m);
      if (sum.m > -INFINITY) move_to(sum, m, a.c);
      const float s = wave_sum(sum.s), w = wave_sum(sum.w);
      if (lane == 0) {
        s_sums[wave] = {m, s, w};
        s_before[wave] = before;
      }
      __syncthreads();
    }
    Record rec{0.0, 0.0, -INFINITY, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) rec.m = fmaxf(rec.m, s_sums[i].m);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Sums q = s_sums[i];
      rec.before += s_before[i];
      if (q.m == -INFINITY) continue;
      const double d = (double(q.m) - double(rec.m)) * double(a.c), f = exp2(d);
      rec.s += double(q.s) * f;
      rec.w += (double(q.w) + d * double(q.s)) * f;
    }
    if (gridDim.x == 1) {
      finish(a, row, rec, z.key, n);
    } else {
      const size_t at = size_t(row) * gridDim.x + blockIdx.x;
      if (tid == 0) records(a)[at] = rec;
      if (TOP && tid < a.top) keys(a, gridDim.x)[at * a.top + tid] = tid < n ? z.key[tid] : 0;
    }
  }
}

// Joins the pieces of a row: a workgroup each.
__global__ __launch_bounds__(kBlock) void logprob_join_kernel(LogprobArgs a, int pieces) {
  __shared__ List z;
  __shared__ Record s_rec[kBlock];
  const int row = blockIdx.x, tid = threadIdx.x;
  if (tid < pieces) s_rec[tid] = records(a)[size_t(row) * pieces + tid];
  if (tid == 0) z.count = 0;
  __syncthreads();
  const unsigned long long* from = keys(a, pieces) + size_t(row) * pieces * a.top;
  // a piece's last key has `top` keys at or above it: what lies below the largest of them is out
  unsigned long long least = 1;
  for (int i = 0; i < pieces && a.top > 0; ++i) least = max(least, from[i * a.top + a.top - 1]);
  for (int i = tid; i < pieces * a.top; i += kBlock) {
    const unsigned long long k = from[i];
    if (k >= least) z.key[atomicAdd(&z.count, 1)] = k;
  }
  int n = 0;
  if (a.top > 0) n = rank_list(z, a.top);
  Record rec{0.0, 0.0, -INFINITY, 0};
  for (int i = 0; i < pieces; ++i) rec.m = fmaxf(rec.m, s_rec[i].m);
  for (int i = 0; i < pieces; ++i) {
    const Record q = s_rec[i];
    rec.before += q.before;
    if (q.m == -INFINITY) continue;
    const double d = (double(q.m) - double(rec.m)) * double(a.c), f = exp2(d);
    rec.s += q.s * f;
    rec.w += (q.w + d * q.s) * f;
  }
  finish(a, row, rec, z.key, n);
}

// Mean log probability of the rows of a sequence that have a token (0 where none has): a workgroup each.
__global__ __launch_bounds__(kBlock) void logprob_mean_kernel(LogprobArgs a) {
  __shared__ double s_sum[kBlock];
  __shared__ int s_n[kBlock];
  const int tid = threadIdx.x, b = blockIdx.x;
  const int lo = max(a.start[b], 0), hi = min(a.start[b + 1], a.rows);
  double sum = 0.0;
  int n = 0;
  for (int i = lo + tid; i < hi; i += kBlock) {
    const int t = a.tokens[i];
    if (t < 0 || t >= a.V) continue;
    sum += double(a.logprob[i]);
    ++n;
  }
  s_sum[tid] = sum;
  s_n[tid] = n;
  for (int k = kBlock / 2; k > 0; k /= 2) {
    __syncthreads();
    if (tid < k) {
      s_sum[tid] += s_sum[tid + k];
      s_n[tid] += s_n[tid + k];
    }
  }
  if (tid == 0) a.mean[b] = s_n[0] ? float(s_sum[0] / s_n[0]) : 0.0f;
}

// pieces of a row: tiles of each, such that there are about kTarget workgroups
int tiles_per_piece(int rows, int V) {
  const int tiles = (V + kTile - 1) / kTile;
  const int pieces = std::min({std::max(1, kTarget / rows), tiles, kPieces});
  return (tiles + pieces - 1) / pieces;
}
int pieces_of(int rows, int V) {
  const int tiles = (V + kTile - 1) / kTile, per = tiles_per_piece(rows, V);
  return (tiles + per - 1) / per;
}

}  // namespace

size_t logprob_workspace_bytes(int rows, int V, int top) {
  const int pieces = pieces_of(rows, V);
  return pieces == 1 ? 0 : size_t(rows) * pieces * (sizeof(Record) + 8 * size_t(top));
}

hipError_t launch_logprob(const LogprobArgs& a, hipStream_t s) {
  const int per = tiles_per_piece(a.rows, a.V), pieces = pieces_of(a.rows, a.V);
  const dim3 grid(pieces, std::min(a.rows, 65535));
  if (a.f32) {
    if (a.top) hipLaunchKernelGGL((logprob_kernel<true, true>), grid, dim3(kBlock), 0, s, a, per);
    else hipLaunchKernelGGL((logprob_kernel<true, false>), grid, dim3(kBlock), 0, s, a, per);
  } else {
    if (a.top) hipLaunchKernelGGL((logprob_kernel<false, true>), grid, dim3(kBlock), 0, s, a, per);
    else hipLaunchKernelGGL((logprob_kernel<false, false>), grid, dim3(kBlock), 0, s, a, per);
  }
  if (pieces > 1) hipLaunchKernelGGL(logprob_join_kernel, dim3(a.rows), dim3(kBlock), 0, s, a, pieces);
  if (a.start) hipLaunchKernelGGL(logprob_mean_kernel, dim3(a.seqs), dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

}  // namespace tasp
