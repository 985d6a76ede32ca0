// Verification of drafted tokens against the target's distributions at given random numbers.
//
// p = softmax(l / temperature) of each node's logits. From node 0 the children of the current node are
// tried in node order: without draft logits child c with token x_c is accepted when
// u_c (Z - sum of e(x) over the earlier children's distinct tokens) < e(x_c), e = exp((l - max) / temperature),
// Z its sum, a token tried before counting 0 (the target's distribution without what was refused); with
// draft logits (a chain) when u_c q(x_c) < p(x_c). Where nothing is accepted, the last token is the lowest
// x whose cumulative weight exceeds u_0 times the total, of e without the children's tokens, or of
// max(p - q, 0). Everything is held in 64 bits: a vocabulary has 10^5 borders between two tokens'
// shares, and sums with an error of 10^-7 would move one of them across u_0 every few hundred calls.
//
// Launches: verify_stats_kernel (one chunk of 4096 logits per workgroup, held in registers: maximum,
// its lowest index and sum of e) over all rows of the tree and the draft; then verify_walk_kernel,
// which walks the tree and takes the last token. Without draft logits the chunks' weights follow
// from the first launch, so one workgroup per sequence reads one chunk again; with them
// each workgroup of a grid over the chunks walks the (short) chain for itself, sums its chunk of
// max(p - q, 0), and the last to finish takes the token.
//
// Bound by the read of the logits, and nearly as much by the exponentials: 16 trees of 32 over 128256 tokens, 263 MB, take
// 63 .. 72 us in the first launch (4.2 .. 3.7 TB/s; 20 instructions per logit are 40 us of every SIMD) and 13 in the second,
// which is latency: records from other dies' caches, the tree, a chunk of logits. Chains of 9 x 8 with drafts, 70 MB: 20 + 14 us;
// one row: 4 + 7.
#include <algorithm>

#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {
namespace {

constexpr int kVChunk = 4096;          // logits per workgroup of the first launch
constexpr int kVU = kVChunk / kBlock;  // logits per thread

// threads of the second launch: with 256, chains of 9 x 8 take 17.1 us in it instead of 14.0 and 32 nodes x 16 14.8
// instead of 12.0; with 1024 both as long as with 512
constexpr int kWalk = 512;

struct ChunkStat {
  double z;                            // sum of exp((l - m) / temperature) over the chunk
  float m;                             // its maximum
  int at;                              // lowest index of it
};

// exp((l - m) / temperature) = 2^(t / 64), t = (l - m) (64 log2(e) / temperature): t is cut at the nearest integer n by
// adding 1.5 2^52, which leaves n in the sum's low word; 2^((n mod 64) / 64) comes from a table in LDS, 2^(f / 64),
// |f| <= 1/2, from the Taylor polynomial of degree 4 (remainder (ln 2 / 128)^5 / 120 = 4e-14), and n / 64 is added to
// the exponent. 17 instructions, three of them conversions or compares (with rint, a conversion and ldexp, in 64 bits
// and at a quarter of the rate, the stats of the 32-node case took 80 us).
__constant__ double kPow64[64] = {
    1.0, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284,
    1.0442737824274138, 1.0556451783605572, 1.0671404006768237, 1.0787607977571199,
    1.0905077326652577, 1.102382583307841, 1.1143867425958924, 1.1265216186082418,
    1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812,
    1.189207115002721, 1.202156731452703, 1.215247359980469, 1.22848053610687,
    1.241857812073484, 1.255380757024691, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.339667524053303,
    1.3542555469368927, 1.3690024229745905, 1.383909881963832, 1.3989796725383112,
    1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647,
    1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384,
    1.5422108254079407, 1.559004400237837, 1.5759808451078865, 1.593142151342267,
    1.6104903319492543, 1.6280274218573478, 1.645755478153965, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.718619298122478, 1.7373338352737062,
    1.7562521603732995, 1.7753764925265212, 1.7947090750031072, 1.8142521755003989,
    1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656,
    1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.978456026387951,
};
constexpr double kLn2_64 = 0.69314718055994530942 / 64.0;
struct Exp {
  const double* table;                 // kPow64 in LDS
  double scale;                        // 64 log2(e) / temperature; greedy calls ask for no weight
  double low;                          // l - m below which a weight is 0: 2^-1020, what 64 bits hold in full
};
// Fills the table (by the first 64 threads; a barrier follows before its use)
__device__ __forceinline__ Exp exp_table(double* lds, double inv_temp) {
  if (threadIdx.x < 64) lds[threadIdx.x] = kPow64[threadIdx.x];
  const double scale = inv_temp * 64.0 * 1.44269504088896340736;
  return {lds, scale, -64.0 * 1020.0 / scale};
}
// 2^(d scale / 64) for low <= d <= 0
__device__ __forceinline__ double exp_of(double d, const Exp& e) {
  constexpr double magic = 0x1.8p52;
  const double s = fma(d, e.scale, magic), f = fma(d, e.scale, magic - s);
  const int n = __double2loint(s);
  constexpr double c = kLn2_64;
  double p = c * c * c * c / 24.0;
  p = fma(p, f, c * c * c / 6.0);
  p = fma(p, f, c * c / 2.0);
  p = fma(p, f, c);
  const double t = e.table[n & 63], y = fma(t, p * f, t);
  return __hiloint2double(__double2hiint(y) + int(uint32_t(n & ~63) << 14), __double2loint(y));
}
// The weight of a logit whose row's maximum is m: NaN counts as -inf, a row without anything above -inf has
// no weight, +inf shares it evenly.
__device__ __forceinline__ double weight(float l, float m, const Exp& e) {
  const double d = double(l) - double(m);
  const double y = exp_of(fmax(d, e.low), e);
  const double one = l == m ? 1.0 : 0.0;
  return m == INFINITY ? one : d > e.low ? y : 0.0;
}

// v of the lane that CTRL names, 0 where it names none, for the rows in ROWS; by DPP: through the lane crossbar
// (ds_bpermute) a scan of 64 doubles took 0.4 us
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double dpp_d(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xF, false),
                          __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ double lane_d(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// Sums over lanes 0 .. own (row_shr:1, 2, 4, 8 within rows of 16, then row_bcast:15 and :31 between them)
__device__ __forceinline__ double wave_scan(double v) {
  v += dpp_d<0x111>(v);
  v += dpp_d<0x112>(v);
  v += dpp_d<0x114>(v);
  v += dpp_d<0x118>(v);
  v += dpp_d<0x142, 0xA>(v);
  v += dpp_d<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ double wave_sum_d(double v) { return lane_d(wave_scan(v), 63); }

// Grid (chunks, rows). rows 0 .. n_target - 1 are the target's, the others the draft's. Also clears
// the next launch's counters (cnt[B]).
__global__ __launch_bounds__(kBlock) void verify_stats_kernel(VerifyArgs a, ChunkStat* stat, int* cnt) {
  __shared__ float sm[4];
  __shared__ int si[4];
  __shared__ double sz[4], table[64];
  const Exp ex = exp_table(table, a.inv_temp);
  const int tid = threadIdx.x, wave = tid >> 6;
  const int c = blockIdx.x, r = blockIdx.y, nt = a.B * a.T;
  const float* row = r < nt ? a.logits + size_t(r) * a.V : a.draft + size_t(r - nt) * a.V;
  if (c == 0 && r < a.B && tid == 0) cnt[r] = 0;
  const int k0 = c * kVChunk + tid;
  float x[kVU];
#pragma unroll
  for (int i = 0; i < kVU; ++i) {
    const int k = k0 + i * kBlock;
    x[i] = k < a.V ? row[k] : -INFINITY;
  }
  float m = -INFINITY;
  int at = 0x7fffffff;
  if (a.inv_temp == 0.0) {             // greedy: the maximum and its place are all
#pragma unroll
    for (int i = 0; i < kVU; ++i)
      if (x[i] > m) {
        m = x[i];
        at = k0 + i * kBlock;
      }
#pragma unroll
    for (int k = 1; k < kWave; k <<= 1) {
      const float om = __shfl_xor(m, k, kWave);
      const int oa = __shfl_xor(at, k, kWave);
      if (om > m || (om == m && oa < at)) {
        m = om;
        at = oa;
      }
    }
    if ((tid & 63) == 0) {
      sm[wave] = m;
      si[wave] = at;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (sm[w] > m || (sm[w] == m && si[w] < at)) {
        m = sm[w];
        at = si[w];
      }
    if (tid == 0) stat[size_t(r) * gridDim.x + c] = {0.0, m, at};
    return;
  }
#pragma unroll
  for (int i = 0; i < kVU; ++i) m = fmaxf(m, x[i]);
#pragma unroll
  for (int k = 1; k < kWave; k <<= 1) m = fmaxf(m, __shfl_xor(m, k, kWave));
  if ((tid & 63) == 0) sm[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  double z = 0.0;
  if (m == INFINITY) {                 // (uniform)
#pragma unroll
    for (int i = 0; i < kVU; ++i) z += x[i] == m ? 1.0 : 0.0;
  } else if (m > -INFINITY) {
    // what lies below the range adds 2^-1020 to a sum of 1 and more
#pragma unroll
    for (int i = 0; i < kVU; ++i) z += exp_of(fmax(double(x[i]) - double(m), ex.low), ex);
  }
  z = wave_sum_d(z);
  if ((tid & 63) == 0) sz[wave] = z;
  __syncthreads();
  z = (sz[0] + sz[1]) + (sz[2] + sz[3]);
  if (tid == 0) stat[size_t(r) * gridDim.x + c] = {z, m, at};
}

struct RowStat {
  double z;
  float m;
  int at;
};

struct WalkSmem {
  double table[64];
  RowStat row[2 * kTreeMax];           // the target's rows, then the draft's
  double e[kTreeMax];                  // weight of a node's token at its parent
  int token[kTreeMax];
  unsigned long long kids[kTreeMax];   // a node's children
  unsigned long long children;         // of the last node
  int last, n;
  uint32_t gone[kVChunk / 32];         // tokens of a chunk that were refused
  double part[kWalk / kWave + 1];
  int cand[kWalk / kWave], tail[kWalk / kWave];
  int found, is_last;
  double base;
};

// Maxima and sums from the chunks of rows `first` .. + n - 1 and, behind them, `first2` .. + n2 - 1: four threads per
// row, eight chunks of each in flight together (they come from other dies' caches: one by one, 32 chunks took 6 us).
__device__ __forceinline__ void row_stats(const VerifyArgs& a, const Exp& ex, const ChunkStat* stat, size_t first, int n, size_t first2,
                                          int n2, int chunks, RowStat* out, RowStat* out2) {
  const int q = threadIdx.x & 3;
  for (int t = threadIdx.x >> 2; t < n + n2; t += kWalk / 4) {          // (whole groups of four lanes)
    const ChunkStat* s = stat + (t < n ? first + t : first2 + (t - n)) * chunks;
    double z = 0.0;
    float m = -INFINITY;
    int at = 0x7fffffff;
    for (int c0 = 0; c0 < chunks; c0 += 32) {
      ChunkStat x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[min(c0 + 4 * i + q, chunks - 1)];
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (x[i].m > top) {
          top = x[i].m;
          at = x[i].at;
        }
      auto other = [&](float om, int oa) {
        if (om > top || (om == top && oa < at)) {
          top = om;
          at = oa;
        }
      };
      other(dpp<kQuadXor1>(top), __builtin_amdgcn_mov_dpp(at, kQuadXor1, 0xF, 0xF, true));
      other(dpp<kQuadXor2>(top), __builtin_amdgcn_mov_dpp(at, kQuadXor2, 0xF, 0xF, true));
      if (a.inv_temp > 0.0) {
        if (c0 > 0) z *= weight(m, top, ex);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double w = x[i].z * weight(x[i].m, top, ex);
          z += c0 + 4 * i + q < chunks ? w : 0.0;
        }
      }
      m = top;
    }
    z += dpp_d<kQuadXor1>(z);
    z += dpp_d<kQuadXor2>(z);
    if (q == 0) (t < n ? out[t] : out2[t - n]) = {z, m, at};
  }
}

// Nothing moves across: what a wave's lanes wrote to LDS before is there for its other lanes behind (LDS serves a wave in order)
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// The tree's walk by the first wave, a node per lane; path and n are written when `out` is set.
__device__ __forceinline__ void walk(const VerifyArgs& a, const Exp& ex, const ChunkStat* stat, int b, int chunks, WalkSmem& sm, bool out) {
  const int tid = threadIdx.x, T = a.T, t = tid;
  const bool greedy = a.inv_temp == 0.0, draft = a.draft && !greedy;
  // the tree and its tokens' logits are asked for first, so that they come with the chunks' records
  TreeNode nd{0, -2};
  int up = -1, x = -1;
  bool node = false, word = false;
  double u = 0.0;
  float lx = 0.0f, dx = 0.0f;
  if (tid < kWave) {
    sm.kids[t] = 0;
    int t_end = T;
    if (a.len) {
      const int L = seq_len(a.len, b, a.S);
      t_end = L < 0 ? 0 : a.S - L;
    }
    nd = tree_node(a.parent ? a.parent + size_t(b) * T : nullptr, T, t_end, t);
    node = nd.anc != 0 && nd.parent >= 0;
    up = node ? nd.parent : -1;
    x = t < T ? a.tokens[size_t(b) * T + t] : -1;
    word = node && x >= 0 && x < a.V;
    u = t < T && !greedy ? double(a.u[size_t(b) * T + t]) : 0.0;
    if (word && !greedy) {
      lx = a.logits[(size_t(b) * T + up) * a.V + x];
      if (draft) dx = a.draft[(size_t(b) * (T - 1) + up) * a.V + x];
    }
    sm.token[t] = x;
    wave_order();
    if (node && !draft) atomicOr(&sm.kids[up], 1ull << t);
  }
  __syncthreads();                     // the table
  row_stats(a, ex, stat, size_t(b) * T, T, size_t(a.B) * T + size_t(b) * (T - 1), draft ? T - 1 : 0, chunks, sm.row,
                sm.row + kTreeMax);
  __syncthreads();
  if (tid < kWave) {
    const RowStat rs = sm.row[max(up, 0)];
    double e = 0.0, q = 0.0;
    if (word && greedy) e = rs.at == x ? 1.0 : 0.0;
    if (word && !greedy) e = weight(lx, rs.m, ex);
    if (word && draft) {
      const RowStat ds = sm.row[kTreeMax + up];
      q = weight(dx, ds.m, ex);
      q = ds.z > 0.0 ? q / ds.z : 0.0;
    }
    bool good;
    unsigned long long older = 0;      // earlier children of the same parent
    if (draft) {
      good = word && rs.z > 0.0 && u * q < e / rs.z;
    } else {
      // (lists of children in LDS: two loops over all nodes took 4 us for 32)
      if (node) older = sm.kids[up] & ((1ull << t) - 1);
      bool again = false;              // the token was tried before
      for (unsigned long long k = older; k; k &= k - 1) again |= sm.token[__ffsll((long long)k) - 1] == x;
      if (again) e = 0.0;
      sm.e[t] = e;
      wave_order();
      double before = 0.0;
      for (unsigned long long k = older; k; k &= k - 1) before += sm.e[__ffsll((long long)k) - 1];
      good = word && u * ((greedy ? 1.0 : rs.z) - before) < e;
    }
    const unsigned long long goods = __ballot(good);
    const bool chosen = good && !(older & goods);
    const unsigned long long taken = __ballot(chosen) | 1ull;
    const bool on = nd.anc != 0 && (nd.anc & 1) && !(nd.anc & ~taken);
    const unsigned long long path = __ballot(on);
    // node 0 absent (its parent is not -1, or it does not fit): nothing is on the path. Without lengths it is the last node
    // all the same, with them nothing is emitted.
    const int n = a.len ? __popcll(path) : max(1, __popcll(path)), last = path ? 63 - __clzll(path) : 0;
    const unsigned long long kids = draft ? __ballot(node && up == last) : sm.kids[last];
    if (t == 0) {
      sm.n = n;
      sm.last = last;
      sm.children = kids;
    }
    if (out && t < T) {
      const int before = __popcll(path & ((1ull << t) - 1));
      int* po = a.path + size_t(b) * T;
      int* io = a.ids + size_t(b) * T;
      if (on || (t == 0 && n > 0)) po[before] = t;
      if (on && t > 0) io[before - 1] = x;
      if (t >= n) {
        po[t] = -1;
        io[t] = -1;
      }
      if (t == 0) a.n[b] = n;
    }
  }
  __syncthreads();
}

// The token of a chunk whose cumulative weight first exceeds `target`, the weights before it being
// `base`; also the chunk's last token with a weight. w(k, read(k)): weight of token k; the reads of all of a thread's
// tokens are in flight together. A wave holds consecutive groups of 64 tokens, so sums run in token order (16
// consecutive tokens per thread: 15000 cycles for two rows of logits, for their strided loads). found: -1 none, else the
// token; tail: the last token with a weight, -1 none; returns base plus the chunk's weight.
template <class R, class W>
__device__ __forceinline__ double scan_chunk(const VerifyArgs& a, int c, double base, double target, WalkSmem& sm, R&& read, W&& w,
                                             int* found, int* tail) {
  constexpr int U = kVChunk / kWalk, NWV = kWalk / kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int k0 = c * kVChunk + wave * (kWave * U) + lane;
  decltype(read(0)) x[U];
#pragma unroll
  for (int i = 0; i < U; ++i) x[i] = read(min(k0 + kWave * i, a.V - 1));
  double v[U], inc[U], sum = 0.0;      // weights, their sums over the group up to the lane
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const double y = w(k0 + kWave * i, x[i]);
    v[i] = k0 + kWave * i < a.V ? y : 0.0;
    inc[i] = wave_scan(v[i]);
    sum += lane_d(inc[i], 63);
  }
  if (lane == 0) sm.part[wave] = sum;
  __syncthreads();
  double cum = base, total = base;
#pragma unroll
  for (int j = 0; j < NWV; ++j) {
    const double pj = sm.part[j];
    cum += j < wave ? pj : 0.0;
    total += pj;
  }
  int hit = -1, end = -1;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const unsigned long long some = __ballot(v[i] > 0.0), over = __ballot(v[i] > 0.0 && cum + inc[i] > target);
    const int g0 = c * kVChunk + wave * (kWave * U) + kWave * i;
    if (over && hit < 0) hit = g0 + __ffsll((long long)over) - 1;
    if (some) end = g0 + 63 - __clzll(some);
    cum += lane_d(inc[i], 63);
  }
  if (lane == 0) {
    sm.cand[wave] = hit;
    sm.tail[wave] = end;
  }
  __syncthreads();
  int f = -1, g = -1;
#pragma unroll
  for (int j = 0; j < NWV; ++j) {
    f = f < 0 ? sm.cand[j] : f;
    g = max(g, sm.tail[j]);
  }
  *found = f;
  *tail = g;
  return total;
}

// The chunk's refused tokens as a bit mask
__device__ __forceinline__ void mark_gone(const VerifyArgs& a, int c, WalkSmem& sm) {
  for (int i = threadIdx.x; i < kVChunk / 32; i += kWalk) sm.gone[i] = 0;
  __syncthreads();
  const int t = threadIdx.x;
  if (t < a.T && ((sm.children >> t) & 1)) {
    const int k = sm.token[t] - c * kVChunk;
    if (k >= 0 && k < kVChunk && sm.token[t] < a.V) atomicOr(&sm.gone[k >> 5], 1u << (k & 31));
  }
  __syncthreads();
}

// Takes the last token of sequence b by the whole workgroup: chunk_weight(c) is the weight of chunk c
// (any thread may ask), read and w as for scan_chunk after mark_gone (remove: w asks for its mask).
template <class CW, class R, class W>
__device__ __forceinline__ int take(const VerifyArgs& a, int b, int chunks, WalkSmem& sm, bool remove, CW&& chunk_weight, R&& read, W&& w) {
  const int tid = threadIdx.x;
  // the chunk in which the cumulative weight passes the target: by the first wave, chunk sums in order
  if (tid < kWave) {
    const double u = double(a.u[size_t(b) * a.T]);
    const double w0 = tid < chunks ? chunk_weight(tid) : 0.0;        // (asked for once where there are up to 64)
    const double inc0 = wave_scan(w0);
    double total = lane_d(inc0, 63);
    for (int c0 = kWave; c0 < chunks; c0 += kWave) total += wave_sum_d(c0 + tid < chunks ? chunk_weight(c0 + tid) : 0.0);
    const double target = u * total;
    double base = 0.0;
    int at = -1;
    double before = 0.0;
    for (int c0 = 0; c0 < chunks && at < 0; c0 += kWave) {
      const double mine = c0 == 0 ? w0 : c0 + tid < chunks ? chunk_weight(c0 + tid) : 0.0;
      const double inc = c0 == 0 ? inc0 : wave_scan(mine);
      const unsigned long long over = __ballot(base + inc > target && mine > 0.0);
      if (over) {
        const int l = __ffsll((long long)over) - 1;
        at = c0 + l;
        before = base + lane_d(inc - mine, l);
      }
      base += lane_d(inc, 63);
    }
    if (tid == 0) {
      sm.found = total > 0.0 ? max(at, 0) : -1;
      sm.base = before;
      sm.part[kWalk / kWave] = target;
    }
  }
  __syncthreads();
  const int c_at = sm.found;
  double base = sm.base;
  const double target = sm.part[kWalk / kWave];
  if (c_at < 0) return -1;             // nothing has a weight
  int best = -1;                       // the last token with a weight, should rounding leave the target unreached
  for (int c = c_at; c < chunks; ++c) {
    int found, tail;
    if (remove) mark_gone(a, c, sm);
    base = scan_chunk(a, c, base, target, sm, read, w, &found, &tail);
    if (found >= 0) return found;
    if (tail >= 0) best = tail;
  }
  for (int c = c_at - 1; c >= 0 && best < 0; --c) {
    int found, tail;
    if (remove) mark_gone(a, c, sm);
    scan_chunk(a, c, 0.0, INFINITY, sm, read, w, &found, &tail);
    best = tail;
  }
  return best;
}

// Grid (1, or chunks with draft logits, B): see the head of the file.
__global__ __launch_bounds__(kWalk) void verify_walk_kernel(VerifyArgs a, const ChunkStat* stat, double* sums, int* cnt, int chunks) {
  __shared__ WalkSmem sm;
  const int tid = threadIdx.x, b = blockIdx.y, T = a.T;
  const bool greedy = a.inv_temp == 0.0;
  const Exp ex = exp_table(sm.table, a.inv_temp);
  walk(a, ex, stat, b, chunks, sm, blockIdx.x == 0);
  if (sm.n == 0) return;
  const int last = sm.last, slot = sm.n - 1;
  int* out = a.ids + size_t(b) * T + slot;
  const RowStat rs = sm.row[last];
  if (greedy) {
    if (tid == 0) *out = rs.m > -INFINITY ? rs.at : -1;
    return;
  }
  const size_t r = size_t(b) * T + last;
  const float* row = a.logits + r * a.V;
  const ChunkStat* st = stat + r * chunks;
  const bool kids = sm.children != 0;
  auto plain_sum = [&](int c) { return st[c].z * weight(st[c].m, rs.m, ex); };
  auto read = [&](int k) { return row[k]; };
  auto plain = [&](int, float l) { return weight(l, rs.m, ex); };
  if (!a.draft) {
    // e without the children's tokens: what they weigh is taken off their chunks
    auto left_sum = [&](int c) {
      double z = plain_sum(c);
      for (unsigned long long k = sm.children; k; k &= k - 1) {
        const int t = __ffsll((long long)k) - 1;
        if (sm.token[t] >= 0 && sm.token[t] / kVChunk == c) z -= sm.e[t];
      }
      return fmax(z, 0.0);
    };
    auto left = [&](int k, float l) {
      const int i = k % kVChunk;
      const double y = plain(k, l);
      return kids && ((sm.gone[i >> 5] >> (i & 31)) & 1) ? 0.0 : y;
    };
    int x = take(a, b, chunks, sm, kids, left_sum, read, left);
    if (x < 0 && kids) {               // (uniform)
      __syncthreads();
      x = take(a, b, chunks, sm, false, plain_sum, read, plain);
    }
    if (tid == 0) *out = x;
    return;
  }
  // max(p - q, 0) at a chain's refused token, p behind its end
  const RowStat ds = kids ? sm.row[kTreeMax + last] : RowStat{0.0, 0.0f, 0};
  const float* drow = kids ? a.draft + (size_t(b) * (T - 1) + last) * a.V : row;
  const double pz = rs.z > 0.0 ? 1.0 / rs.z : 0.0, qz = ds.z > 0.0 ? 1.0 / ds.z : 0.0;
  struct Two {
    float l, d;
  };
  auto read2 = [&](int k) { return Two{row[k], drow[k]}; };
  auto rest = [&](int, Two x) {
    const double p = weight(x.l, rs.m, ex) * pz;
    return kids ? fmax(p - weight(x.d, ds.m, ex) * qz, 0.0) : p;
  };
  const int c = blockIdx.x;
  constexpr int U = kVChunk / kWalk;
  Two in[U];                           // (all in flight together)
#pragma unroll
  for (int i = 0; i < U; ++i) in[i] = read2(min(c * kVChunk + i * kWalk + tid, a.V - 1));
  double z = 0.0;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const double y = rest(0, in[i]);
    z += c * kVChunk + i * kWalk + tid < a.V ? y : 0.0;
  }
  z = wave_sum_d(z);
  if ((tid & 63) == 0) sm.part[tid >> 6] = z;
  __syncthreads();
  const __amdgpu_buffer_rsrc_t rp = make_rsrc(sums + size_t(b) * chunks, uint32_t(chunks) * 8u);
  if (tid == 0) {
    z = 0.0;
    for (int j = 0; j < kWalk / kWave; ++j) z += sm.part[j];
    buf_store8_device(__builtin_bit_cast(int2, z), rp, uint32_t(c) * 8u);
    __builtin_amdgcn_s_waitcnt(0);                      // the sum is at the coherence point
    sm.is_last = __hip_atomic_fetch_add(cnt + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == chunks - 1;
  }
  __syncthreads();
  if (!sm.is_last) return;
  auto rest_sum = [&](int j) { return __builtin_bit_cast(double, buf_load8_device(rp, uint32_t(j) * 8u)); };
  int x = take(a, b, chunks, sm, false, rest_sum, read2, rest);
  if (x < 0) {                         // (uniform)
    __syncthreads();
    x = take(a, b, chunks, sm, false, plain_sum, read, plain);
  }
  if (tid == 0) *out = x;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t verify_workspace_bytes(int B, int T, int V) {
  const size_t chunks = size_t(V + kVChunk - 1) / kVChunk;
  return up256(size_t(B) * (2 * T - 1) * chunks * sizeof(ChunkStat)) + up256(size_t(B) * chunks * 8) + up256(size_t(B) * 4);
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  const int chunks = (a.V + kVChunk - 1) / kVChunk;
  const bool draft = a.draft && a.T > 1 && a.inv_temp > 0.0;
  const int rows = a.B * a.T + (draft ? a.B * (a.T - 1) : 0);
  char* ws = static_cast<char*>(a.ws);
  ChunkStat* stat = reinterpret_cast<ChunkStat*>(ws);
  ws += up256(size_t(a.B) * (2 * a.T - 1) * chunks * sizeof(ChunkStat));
  double* sums = reinterpret_cast<double*>(ws);
  ws += up256(size_t(a.B) * chunks * 8);
  VerifyArgs v = a;
  if (!draft) v.draft = nullptr;
  hipLaunchKernelGGL(verify_stats_kernel, dim3(chunks, rows), dim3(kBlock), 0, s, v, stat, reinterpret_cast<int*>(ws));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int* cnt = reinterpret_cast<int*>(ws);
  hipLaunchKernelGGL(verify_walk_kernel, dim3(draft ? chunks : 1, a.B), dim3(kWalk), 0, s, v, stat, sums, cnt, chunks);
  return hipGetLastError();
}

}  // namespace tasp
