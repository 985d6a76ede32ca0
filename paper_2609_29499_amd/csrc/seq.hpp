// Caches whose sequences have their own lengths, and trees of drafted tokens over them: arguments of
// the kernels in seq_cache.hip, tree_attn.hip and verify.hip, and the device helpers they share.
#pragma once
#include "device_common.hpp"

namespace tasp {

constexpr int kTreeMax = 64;           // nodes of a tree at most: a node's ancestors are one 64-bit word
constexpr int kSeqMaxBatch = 256;      // sequences of a cache at most: four per lane of a wave

enum SeqType { SEQ_BF16 = 0, SEQ_F32 = 1, SEQ_INT8 = 2, SEQ_E4M3 = 3 };

// rows of head vectors: element strides between sequences, tokens and heads
struct SeqRows {
  void* p;
  long seq, token, head;
};

// one layer of a cache: [batch][n_kv][S][dh] and scales [batch][n_kv][S]
struct SeqLayer {
  void* k; void* v;
  float* ks; float* vs;                // null for BF16
  const int* len;                      // [batch]
  int type, batch, n_kv, S, dh;
};

struct SeqAppendArgs {
  SeqLayer c;
  const int* parent; int T;            // [batch][T] or null: a chain
  int act;                             // SEQ_BF16 or SEQ_F32: type of q, k, v and q_out
  SeqRows q, k, v, q_out;
  int ks; long split;                  // ks > 1 (SEQ_F32): q, k, v are sums of ks arrays `split` floats apart
  int n_q, n_kv;                       // head rows of q; of k and v
  const int* kv_map;                   // host: cache head of k / v head j (null: j), used by the launch
  int rot, interleaved;                // rotated dimensions of a head; pair layout
  // Pair i's frequency: f = theta^(-2 i / rot), the product of power[k] = theta^(-2 2^k / rot) over the bits of i, times
  // g + (1 - g) keep, g = (by_index ? i : f) mul + add cut to 0 .. 1. (64 frequencies as arguments cost a launch 0.6 us.)
  double power[6];
  double mul, add, keep;
  float mscale;
  int by_index;
};
hipError_t launch_seq_append(const SeqAppendArgs& a, hipStream_t s);

struct SeqReadArgs {
  SeqLayer c;
  const int* first;                    // [batch] or null: row 0
  int n, out_type;                     // SEQ_BF16 or SEQ_F32
  SeqRows k, v;                        // token stride: between rows
};
hipError_t launch_seq_read(const SeqReadArgs& a, hipStream_t s);

struct SeqCommitArgs {
  SeqLayer c; int n_layers;            // c: layer 0
  const int* path; int ld;             // [batch][ld]
  const int* n;                        // [batch]
  int* len_out;                        // [batch]; may be c.len
  bool apart;                          // len_out shares nothing with what the launch reads
};
hipError_t launch_seq_commit(const SeqCommitArgs& a, hipStream_t s);

struct TreeAttnArgs {
  SeqLayer c;
  const int* parent; int T;
  int act;
  SeqRows q, o;
  // slots: cache heads that are read, slot[j] (tree_slot) says which and for which query heads,
  // 1 .. group of them
  int slots, group;
  int slot[64];
  float scale2;                        // scale * log2(e)
  int max_len;                         // largest length expected (sizes the grid; any length is served)
  float* ws;                           // tree_attn_workspace_bytes
};
size_t tree_attn_workspace_bytes(const TreeAttnArgs& a);
hipError_t launch_tree_attn(const TreeAttnArgs& a, hipStream_t s);

// a cache head, its first query head and their number in one word (a scalar load; one byte of an array is a vector's,
// 1 us where nothing else is on its way)
inline int tree_slot(int head, int first, int count) { return head | first << 8 | count << 20; }

struct VerifyArgs {
  const float* logits; const float* draft;   // [B][T][V], [B][T - 1][V] or null
  const int* tokens; const float* u; const int* parent;
  // rows that the sequences hold, of at most S (null: every node fits): nodes whose row does not fit are absent, and a
  // sequence whose node 0 is absent emits nothing
  const int* len; int S;
  int B, T, V;
  double inv_temp;                     // 0: greedy
  int* ids; int* path; int* n;         // [B][T], [B][T], [B]
  void* ws;
};
size_t verify_workspace_bytes(int B, int T, int V);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

#ifdef __HIPCC__
// The tree of one sequence, one node per lane (lanes T .. 63: absent). anc: bit j set for node j = the
// lane's node or one of its ancestors; 0 for an absent node (parent neither -1 nor an earlier node
// that is present, or t >= t_end). Pointer doubling: after step k a lane knows 2^k generations.
struct TreeNode {
  unsigned long long anc;
  int parent;                          // -1: root; -2: absent
};
__device__ __forceinline__ TreeNode tree_node(const int* parent, int T, int t_end, int lane) {
  if (!parent) {                       // a chain
    const bool in = lane < T && lane < t_end;
    return {in ? ~0ull >> (63 - lane) : 0ull, in ? lane - 1 : -2};
  }
  int p = lane < T ? parent[lane] : -2;
  if (p < -1 || p >= lane || lane >= t_end) p = -2;
  unsigned long long m = 1ull << lane;
  int up = p, gone = p == -2;
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    if (!__ballot(up >= 0)) break;     // (a tree of depth d takes the logarithm of d)
    const int at = up < 0 ? lane : up;
    const unsigned long long am = __shfl(m, at, kWave);
    const int ag = __shfl(gone, at, kWave), au = __shfl(up, at, kWave);
    if (up >= 0) {
      m |= am;
      gone |= ag;
      up = au;
    }
  }
  return {gone ? 0ull : m, gone ? -2 : p};
}

// Rows that a sequence holds; -1 for a length outside 0 .. S (the sequence is passed over).
__device__ __forceinline__ int seq_len(const int* len, int b, int S) {
  const int L = len[b];
  return L < 0 || L > S ? -1 : L;
}

typedef __bf16 bf16x2_seq __attribute__((ext_vector_type(2)));
typedef float f32x2_seq __attribute__((ext_vector_type(2)));
// two floats -> packed BF16 (hardware round to nearest even, NaN kept)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_seq{a, b}, bf16x2_seq));
}
// largest of each aligned group of 16 (LANES 16) or 8 lanes, unsigned
template <int LANES>
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  auto step = [](uint32_t x, int y) { return x > uint32_t(y) ? x : uint32_t(y); };
  v = step(v, __builtin_amdgcn_mov_dpp(int(v), kQuadXor1, 0xF, 0xF, true));
  v = step(v, __builtin_amdgcn_mov_dpp(int(v), kQuadXor2, 0xF, 0xF, true));
  v = step(v, __builtin_amdgcn_mov_dpp(int(v), kRowHalfMirror, 0xF, 0xF, true));
  if constexpr (LANES == 16) v = step(v, __builtin_amdgcn_mov_dpp(int(v), kRowMirror, 0xF, 0xF, true));
  return v;
}
#endif

}  // namespace tasp
