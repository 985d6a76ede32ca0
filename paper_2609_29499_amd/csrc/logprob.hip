// Scores of given tokens: of every row x of logits the log probability of a token, the entropy, the token's rank, the
// `top` largest logits in order, and the mean log probability of every sequence of rows.
//
// In one pass over a row, in powers of two: t = (x - m) c with c = log2(e) / temperature and m the running maximum,
// s = sum 2^t, w = sum t 2^t. Then log p(x) = ln 2 ((x - m) c - log2 s) and the entropy is ln 2 (log2 s - w / s). Every
// thread has a maximum and sums of its own in float32, of up to 512 terms; they meet in float64, behind every 32 tiles
// of a piece that has more, and at its end. (x c - m c, one instruction less, loses all digits at small temperatures.)
//
// The largest: every wave keeps a list in LDS of the elements that reach a bound, without a barrier: the `top`-th largest of its
// 64 lanes' maxima, which at least `top` elements reach (some 44 for 32), looked at again behind 1, 2, 4, .. tiles and where the list
// is full. At the end what reaches the largest of the four bounds becomes 64-bit keys (the logit as an integer that keeps
// its order, then the complement of the index: equal logits are in the order of their indices), and each is ranked against all. (One
// list of the workgroup, cut to its first as it grew, has two barriers per tile: 2048 rows of 128256 BF16, top 1 / 5 / 32,
// 154 / 157 / 182 us; this way 121 / 133 / 161; without alternatives 110. Folding into float64 took 513 x 32003 BF16, top 32,
// from 33.4 to 33.8.)
//
// Bound by memory: a row is read once (float32: 2048 rows of 128256 with 20 alternatives 190 us, 5.5 TB/s), BF16 with many alternatives by
// the instructions that enter elements into lists. Few rows are cut into pieces whose records a second launch joins: such that
// there are 512 workgroups (513 x 32003 BF16 in one piece each 30.6 us, cut in two for 1024 workgroups 41).
#include <algorithm>
#include <cmath>

#include "device_common.hpp"
#include "logprob.hpp"

namespace tasp {
namespace {

constexpr int kPer = 16;               // elements of a thread and tile
constexpr int kTile = kBlock * kPer;
constexpr int kFold = 32;              // tiles whose terms a thread adds up in float32
constexpr int kGrown = 96;             // elements that a wave's list may hold beyond `top` before it is cut
constexpr int kLimit = 256;            // keys that are ranked by comparing each with each: one per thread
constexpr int kKeys = 4192;            // of the join's list
constexpr int kWaveKeys = kTopMax + kGrown + kWave * kPer + 8; // a wave's list has room for its next elements, all of them
constexpr int kTarget = 512;           // workgroups aimed at
constexpr int kPieces = kKeys / kTopMax;               // of a row at most: the join's list holds all their keys

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
  __align__(16) unsigned long long key[kKeys + 2];
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
// The list's `top` largest keys to its front, in order. All keys are different. Begins and ends with a barrier; returns
// their number.
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
  if (tid == 0) z.key[n] = 0;          // (pairs are compared)
  __syncthreads();
  const unsigned long long mine = tid < n ? z.key[tid] : 0;
  int before = 0;
  if ((tid & ~63) < n) {
#pragma unroll 4
    for (int j = 0; j < n; j += 2) {
      const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(&z.key[j]);
      before += (k.x > mine) + (k.y > mine);
    }
  }
  if (tid < n && before < out) z.best[before] = mine;
  __syncthreads();
  if (tid < out) z.key[tid] = z.best[tid];
  if (tid == 0) z.count = out;
  __syncthreads();
  return out;
}

// The least number above x (finite, or the largest)
__device__ __forceinline__ float above(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return __uint_as_float(u & 0x80000000u ? u - 1 : u + 1);
}
// what lanes have written to LDS is what other lanes of the wave read
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ int lanes_before(unsigned long long who) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0));
}
// The top-th largest of a wave's 64 values g: that many lanes' reach it. z: 64 values of LDS.
__device__ __forceinline__ float nth_of_lanes(float g, int top, float* z, int lane) {
  if (top == 1) return wave_max(g);
  z[lane] = g;
  wave_sync();
  int larger = 0;
#pragma unroll
  for (int j = 0; j < kWave; j += 4) {
    const float4 q = *reinterpret_cast<const float4*>(&z[j]);
    larger += (q.x > g) + (q.y > g) + (q.z > g) + (q.w > g);
  }
  wave_sync();
  return -wave_max(larger < top ? -g : -INFINITY);
}
// A wave's candidates, as they come: logits and indexes
struct Found {
  float x[kWaveKeys];
  int i[kWaveKeys];
};
// Those that `stays` says true of to the front. Returns their number.
template <class Pred>
__device__ __forceinline__ int keep(Found& z, int n, int lane, Pred stays) {
  int kept = 0;
  wave_sync();
  for (int k = 0; k < n; k += kWave) {
    const bool in = k + lane < n;
    const float x = in ? z.x[k + lane] : 0.0f;
    const int i = in ? z.i[k + lane] : 0;
    const unsigned long long who = __ballot(in && stays(x, i));
    wave_sync();
    if ((who >> lane) & 1) {
      z.x[kept + lanes_before(who)] = x;
      z.i[kept + lanes_before(who)] = i;
    }
    kept += __popcll(who);
    wave_sync();
  }
  return kept;
}
// The top-th largest of a wave's n keys (n >= top), bit by bit: the largest value that `top` keys reach
__device__ __forceinline__ unsigned long long nth_key(const Found& z, int n, int top, int lane) {
  unsigned long long at = 0;
  wave_sync();
  for (int bit = 63; bit >= 0; --bit) {
    const unsigned long long with = at | 1ull << bit;
    int reach = 0;
    for (int k = lane; k - lane < n; k += kWave) reach += __popcll(__ballot(k < n && key_of(z.x[min(k, n - 1)], z.i[min(k, n - 1)]) >= with));
    if (reach >= top) at = with;
  }
  return at;
}

// Of a row (or a piece of it): sums under the maximum m, and elements that come before the token
struct Record {
  double s, w;
  float m;
  int before;
};
// q's sums under the maximum m (a float32 factor: its 2^-22 is what the terms have)
__device__ __forceinline__ void add_to(Record& rec, const Record& q, float c) {
  const double d = (double(q.m) - double(rec.m)) * double(c);
  const double f = double(__builtin_amdgcn_exp2f(float(d)));
  rec.before += q.before;
  if (f == 0.0) return;
  rec.s += q.s * f;
  rec.w += (q.w + d * q.s) * f;
}

// The same where q's maximum may be above, by less than the range of 64 bits
__device__ __forceinline__ void add_far(Record& rec, const Record& q, float c) {
  const double d = (double(q.m) - double(rec.m)) * double(c), k = rint(d);
  if (d < -1000.0) return;
  const double f = ldexp(double(__builtin_amdgcn_exp2f(float(d - k))), int(k));
  rec.s += q.s * f;
  rec.w += (q.w + d * q.s) * f;
}
// A wave's sums into what it has of the tiles before. rec.m stays (and with it what has been added, to the bit) until a maximum is
// 2^900 above it, which leaves nothing of the rest.
__device__ __forceinline__ void fold(Record& rec, const Record& q, float c) {
  if ((double(q.m) - double(rec.m)) * double(c) > 900.0) rec = Record{0.0, 0.0, q.m, 0};
  add_far(rec, q, c);
}

// A token's log probability under a row's record
struct Scale {
  double log_s;
  float m, c, lim;
  __device__ __forceinline__ Scale(const LogprobArgs& a, const Record& z) : log_s(z.m <= -a.lim ? 0.0 : log2(z.s)), m(z.m), c(a.c), lim(a.lim) {}
  // (an infinite logit leaves nothing to finite ones; a row without a logit above -inf nothing at all)
  __device__ __forceinline__ float operator()(float x) const {
    return m <= -lim || x <= -lim || (m >= lim && x < m) ? -INFINITY
                                                         : float(((double(x) - double(m)) * double(c) - log_s) * 0.693147180559945309417);
  }
};
// a row's token's logit; false: the token is padding
__device__ __forceinline__ bool token_logit(const LogprobArgs& a, int row, int t, float& x) {
  if (t < 0 || t >= a.V) return false;
  const size_t at = size_t(row) * a.ld + t;
  x = a.f32 ? static_cast<const float*>(a.logits)[at] : bf16_to_f32(static_cast<const uint16_t*>(a.logits)[at]);
  x = fminf(fmaxf(x, -a.lim), a.lim);
  return true;
}
// Results of a row from its joined record; xt: the token's logit (there: it has one); keys: `n` of them in order. Of one wave.
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, const Record& z, bool there, float xt, const unsigned long long* key, int n) {
  const int tid = threadIdx.x;
  const Scale lp(a, z);
  if (tid == 0) {
    a.logprob[row] = there ? lp(xt) : 0.0f;
    if (a.rank) a.rank[row] = there ? z.before : -1;
    if (a.entropy) a.entropy[row] = z.m <= -a.lim ? 0.0f : float((lp.log_s - z.w / z.s) * 0.693147180559945309417);
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
__global__ __launch_bounds__(kBlock, 4) void logprob_kernel(LogprobArgs a, int per) {
  constexpr int RAW = F32 ? 16 : 8;    // words of a tile's elements per thread
  constexpr int AHEAD = F32 ? 1 : 2;   // tiles on their way: 16 words either way
  __shared__ __align__(16) Found s_found[TOP ? 4 : 1];
  __shared__ unsigned long long s_best[kTopMax];
  __shared__ __align__(16) float s_group[TOP ? 4 : 1][kWave];
  __shared__ float s_bound[4];
  __shared__ int s_n;
  __shared__ Sums s_sums[4];
  __shared__ Record s_fold[4];         // of pieces of more than kFold tiles: a wave's sums of whole kFold tiles
  __shared__ int s_before[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const char* base = static_cast<const char*>(a.logits) + size_t(row) * a.ld * (F32 ? 4 : 2);
    const int first = blockIdx.x * per * kTile, end = int(min(long(a.V), long(first) + long(per) * kTile));
    // element j of this thread in a tile
    auto index = [&](int tile, int j) {
      const bool whole = tile + kTile <= end;
      constexpr int W = F32 ? 4 : 8;
      return tile + (whole ? W * tid : tid) + (whole ? j / W * W * kBlock + j % W : j * kBlock);
    };
    auto load = [&](int tile, uint32_t (&v)[RAW]) __attribute__((always_inline)) {
      if (tile + kTile <= end) {
#pragma unroll
        for (int j = 0; j < RAW / 4; ++j) __builtin_memcpy(&v[4 * j], base + size_t(tile) * (F32 ? 4 : 2) + j * 16 * kBlock + 16 * tid, 16);
      } else if (tile < end) {         // the row's last elements, one by one
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int i = tile + j * kBlock + tid;
          if constexpr (F32) {
            v[j] = i < end ? reinterpret_cast<const uint32_t*>(base)[i] : 0xff800000u;
          } else {
            const uint32_t u = i < end ? reinterpret_cast<const uint16_t*>(base)[i] : 0xff80u;
            v[j / 2] = j & 1 ? v[j / 2] | u << 16 : u;
          }
        }
      }
    };
    uint32_t raw[AHEAD][RAW];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) load(first + k * kTile, raw[k]);
    const int token = a.tokens[row];
    float xt = INFINITY;               // (padding: nothing comes before it)
    const bool there = token_logit(a, row, token, xt);
    Sums sum{-INFINITY, 0.0f, 0.0f};
    int before = 0, n = 0;
    Found& found = s_found[TOP ? wave : 0];
    float bound = above(-a.lim);       // elements from it on enter the wave's list
    float g = -a.lim;                  // the `top`-th largest of its lanes' maxima when last looked at
    const int tiles = (end - first + kTile - 1) / kTile;
    __syncthreads();                   // (the row before has been read)
    if (lane == 0) s_fold[wave] = Record{0.0, 0.0, -INFINITY, 0};
    for (int tile = first;;) {
      for (const int to = min(end, tile + kFold * kTile); tile < to; tile += kTile) {
        float x[kPer];
        if constexpr (F32) {
#pragma unroll
          for (int j = 0; j < kPer; ++j) x[j] = __uint_as_float(raw[0][j]);
        } else {
#pragma unroll
          for (int j = 0; j < RAW; ++j) {
            x[2 * j] = bf16_lo(raw[0][j]);
            x[2 * j + 1] = bf16_hi(raw[0][j]);
          }
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) x[j] = fmaxf(x[j], -a.lim);                         // (NaN is -lim)
        float top = fmaxf(x[0], x[1]);
#pragma unroll
        for (int j = 2; j < kPer; ++j) top = fmaxf(top, x[j]);
        if (__ballot(top > a.lim)) {
          top = fminf(top, a.lim);
#pragma unroll
          for (int j = 0; j < kPer; ++j) x[j] = fminf(x[j], a.lim);
        }
#pragma unroll
        for (int k = 0; k + 1 < AHEAD; ++k)
#pragma unroll
          for (int j = 0; j < RAW; ++j) raw[k][j] = raw[k + 1][j];
        load(tile + AHEAD * kTile, raw[AHEAD - 1]);
        // (places behind the row's end hold -lim: their terms are 0, or the row is empty)
        if (top > sum.m) move_to(sum, top, a.c);
        float s2 = 0.0f, w2 = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const float t = (x[j] - sum.m) * a.c, e = __builtin_amdgcn_exp2f(t);
          float& s = j & 1 ? s2 : sum.s;
          float& w = j & 1 ? w2 : sum.w;
          s += e;
          w = fmaf(e, t, w);
        }
        sum.s += s2;
        sum.w += w2;
        // before the token equal logits come first too
        if (token < tile || token >= tile + kTile) {
          if (token >= tile + kTile) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) before += __popcll(__ballot(x[j] >= xt));
          } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) before += __popcll(__ballot(x[j] > xt));
          }
        } else {
#pragma unroll
          for (int j = 0; j < kPer; ++j) before += __popcll(__ballot(x[j] > xt || (x[j] == xt && index(tile, j) < token)));
        }
        if constexpr (TOP) {
          // The `top`-th largest of the lanes' maxima so far: that many elements reach it, and later ones lose to equal ones.
          // Raised behind 1, 2, 4, .. tiles
          float from = bound;
          const int k = (tile - first) / kTile;
          if ((k & (k + 1)) == 0) {
            g = nth_of_lanes(sum.m, a.top, s_group[wave], lane);
            from = fmaxf(from, g);
            if (g > -a.lim) bound = fmaxf(bound, above(g));
          }
          if (__ballot(top >= from)) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
              const unsigned long long who = __ballot(x[j] >= from);
              if (who) {
                if (x[j] >= from) {
                  found.x[n + lanes_before(who)] = x[j];
                  found.i[n + lanes_before(who)] = index(tile, j);
                }
                n += __popcll(who);
              }
            }
          }
          if (n > a.top + kGrown) {
            g = nth_of_lanes(sum.m, a.top, s_group[wave], lane);
            n = keep(found, n, lane, [&](float x, int) { return x >= g; });
            if (g > -a.lim) bound = fmaxf(bound, above(g));
          }
          if (n > a.top + kGrown) {      // (many equal ones, or in few lanes)
            const unsigned long long least = nth_key(found, n, a.top, lane);
            n = keep(found, n, lane, [&](float x, int i) { return key_of(x, i) >= least; });
            bound = fmaxf(bound, above(unordered(uint32_t(least >> 32))));
          }
        }
      }
      if (tile >= end) break;
      const float m = wave_max(sum.m), own = sum.m;
      move_to(sum, m, a.c);
      const float s = wave_sum(sum.s), w = wave_sum(sum.w);
      if (lane == 0) fold(s_fold[wave], Record{double(s), double(w), m, 0}, a.c);
      sum = {own, 0.0f, 0.0f};
    }
    if constexpr (TOP) {
      if (tiles & (tiles - 1)) g = nth_of_lanes(sum.m, a.top, s_group[wave], lane);
      if (lane == 0) s_bound[wave] = g;
      if (tid == 0) s_n = 0;
    }
    // the workgroup's sums
    {
      const float m = wave_max(sum.m);
      move_to(sum, m, a.c);
      const float s = wave_sum(sum.s), w = wave_sum(sum.w);
      if (lane == 0) {
        s_sums[wave] = {m, s, w};
        s_before[wave] = before;
      }
      __syncthreads();
    }
    if constexpr (TOP) {
      // what reaches the largest of the four waves' bounds, in one list (where the first wave's next elements had room)
      constexpr int kUsed = kTopMax + kGrown;
      static_assert((4 * kUsed + 1) * 8 <= (kWaveKeys - kUsed) * 4 && kUsed % 4 == 0);
      unsigned long long* const s_all = reinterpret_cast<unsigned long long*>(&s_found[0].x[kUsed]);
      const float g = fmaxf(fmaxf(s_bound[0], s_bound[1]), fmaxf(s_bound[2], s_bound[3]));
      n = keep(found, n, lane, [&](float x, int) { return x >= g; });
      int at = 0;
      if (lane == 0) at = atomicAdd(&s_n, n);
      at = __builtin_amdgcn_readfirstlane(at);
      for (int i = lane; i < n; i += kWave) s_all[at + i] = key_of(found.x[i], found.i[i]);
      __syncthreads();
      n = s_n;
      if (tid == 0) s_all[n] = 0;      // (pairs are compared)
      __syncthreads();
      for (int i = tid; (i & ~63) < n; i += kBlock) {
        const unsigned long long mine = i < n ? s_all[i] : 0;
        int larger = 0;
#pragma unroll 4
        for (int j = 0; j < n; j += 2) {
          const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&s_all[j]);
          larger += (q.x > mine) + (q.y > mine);
        }
        if (i < n && larger < a.top) s_best[larger] = mine;
      }
      n = min(n, a.top);
      __syncthreads();
    }
    if (wave > 0) continue;
    Record rec{0.0, 0.0, -INFINITY, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) rec.m = fmaxf(rec.m, s_sums[i].m);
#pragma unroll
    for (int i = 0; i < 4; ++i) add_to(rec, Record{double(s_sums[i].s), double(s_sums[i].w), s_sums[i].m, s_before[i]}, a.c);
    if (tiles > kFold) {
      for (int i = 0; i < 4; ++i) add_far(rec, s_fold[i], a.c);
    }
    if (gridDim.x == 1) {
      finish(a, row, rec, there, xt, s_best, n);
    } else {
      const size_t at = size_t(row) * gridDim.x + blockIdx.x;
      if (tid == 0) records(a)[at] = rec;
      if (TOP && tid < a.top) keys(a, gridDim.x)[at * a.top + tid] = tid < n ? s_best[tid] : 0;
    }
  }
}

// A row's record of its pieces', in their order
__device__ __forceinline__ Record join(const LogprobArgs& a, const Record* of, int pieces) {
  Record rec{0.0, 0.0, -INFINITY, 0};
  for (int i = 0; i < pieces; ++i) rec.m = fmaxf(rec.m, of[i].m);
  for (int i = 0; i < pieces; ++i) add_to(rec, of[i], a.c);
  return rec;
}
__device__ __forceinline__ void put_mean(const LogprobArgs& a, int b, double sum, int n) {
  __shared__ double s_sum[kBlock];
  __shared__ int s_n[kBlock];
  const int tid = threadIdx.x;
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

// Joins the pieces of a row: a workgroup each, and behind them one for each sequence's mean, which forms the log
// probabilities that it needs by itself (a third launch would cost 4 us).
__global__ __launch_bounds__(kBlock) void logprob_join_kernel(LogprobArgs a, int pieces) {
  constexpr int kRecords = 1024;       // of several rows at a time, for the means
  __shared__ union {
    List z;
    Record rec[kRecords];
  } u;
  __shared__ Record s_rec[kPieces];
  __shared__ unsigned long long s_least[4];
  __shared__ __align__(16) unsigned long long s_key[kWave];
  List& z = u.z;
  const int row = blockIdx.x, tid = threadIdx.x;
  if (row >= a.rows) {
    const int b = row - a.rows, lo = max(a.start[b], 0), hi = min(a.start[b + 1], a.rows), per = min(kBlock, kRecords / pieces);
    double sum = 0.0;
    int n = 0;
    for (int i0 = lo; i0 < hi; i0 += per) {
      const int here = min(per, hi - i0);
      float x = 0.0f;
      const bool mine = tid < here && token_logit(a, i0 + tid, a.tokens[i0 + tid], x);
      __syncthreads();
      for (int k = tid; k < here * pieces; k += kBlock) u.rec[k] = records(a)[size_t(i0) * pieces + k];
      __syncthreads();
      if (mine) {
        sum += double(Scale(a, join(a, &u.rec[tid * pieces], pieces))(x));
        ++n;
      }
    }
    put_mean(a, b, sum, n);
    return;
  }
  float xt = 0.0f;                     // (asked for before the keys are ranked)
  const bool there = token_logit(a, row, a.tokens[row], xt);
  const unsigned long long* from = keys(a, pieces) + size_t(row) * pieces * a.top;
  // What lies below a key that `top` keys reach is out: the largest of the pieces' last keys is one, and, the j-th keys of the
  // pieces being taken, that of them which ceil(top / j) reach: half of the pieces' (of 32 pieces of 32 keys some 54 stay; with
  // j = 1 it was the least of the pieces' largest, which 256 keys and more may reach)
  unsigned long long least = 1;
  const int j = max(1, min(a.top, (2 * a.top + pieces - 1) / pieces));
  if (tid < pieces) {
    s_rec[tid] = records(a)[size_t(row) * pieces + tid];
    if (a.top > 0) least = max(least, from[tid * a.top + a.top - 1]);
  }
  if (a.top > 0 && tid < kWave) s_key[tid] = tid < pieces ? from[tid * a.top + j - 1] : 0;
#pragma unroll
  for (int k = 1; k < kWave; k *= 2) {
    const unsigned long long o = __shfl_xor(least, k, kWave);
    least = max(least, o);
  }
  if (tid == 0) z.count = 0;
  if ((tid & 63) == 0) s_least[tid >> 6] = least;
  __syncthreads();
  least = max(max(s_least[0], s_least[1]), max(s_least[2], s_least[3]));
  if (a.top > 0) {
    const unsigned long long mine = s_key[tid & 63];
    int larger = 0;
#pragma unroll 8
    for (int k = 0; k < kWave; k += 2) {
      const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&s_key[k]);
      larger += (q.x > mine) + (q.y > mine);
    }
    const unsigned long long who = __ballot(mine > 0 && larger == (a.top + j - 1) / j - 1);      // (keys are different)
    if (who) least = max(least, s_key[__ffsll((long long)who) - 1]);
  }
  for (int i = tid; i < pieces * a.top; i += kBlock) {
    const unsigned long long k = from[i];
    if (k >= least) z.key[atomicAdd(&z.count, 1)] = k;
  }
  int n = 0;
  if (a.top > 0) n = rank_list(z, a.top);
  if (tid < kWave) finish(a, row, join(a, s_rec, pieces), there, xt, z.key, n);
}

// Mean log probability of the rows of a sequence that have a token (0 where none has): a workgroup each.
__global__ __launch_bounds__(kBlock) void logprob_mean_kernel(LogprobArgs a) {
  const int b = blockIdx.x, lo = max(a.start[b], 0), hi = min(a.start[b + 1], a.rows);
  double sum = 0.0;
  int n = 0;
  for (int i = lo + threadIdx.x; i < hi; i += kBlock) {
    const int t = a.tokens[i];
    if (t < 0 || t >= a.V) continue;
    sum += double(a.logprob[i]);
    ++n;
  }
  put_mean(a, b, sum, n);
}

// pieces of a row: tiles of each, such that there are about kTarget workgroups
int tiles_per_piece(int rows, int V) {
  const int tiles = (V + kTile - 1) / kTile;
  const int pieces = std::min({(kTarget + rows - 1) / rows, tiles, kPieces});
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
  if (pieces > 1) hipLaunchKernelGGL(logprob_join_kernel, dim3(a.rows + (a.start ? a.seqs : 0)), dim3(kBlock), 0, s, a, pieces);
  else if (a.start) hipLaunchKernelGGL(logprob_mean_kernel, dim3(a.seqs), dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

}  // namespace tasp
