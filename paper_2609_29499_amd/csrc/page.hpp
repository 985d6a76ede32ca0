// Caches whose rows lie in pages of a pool, and packed tokens of several sequences: arguments of the kernels in
// page_cache.hip and page_attn.hip, and the device helpers they share.
#pragma once
#include "device_common.hpp"
#include "seq.hpp"

namespace tasp {

// one layer of a pool: [n_pages][n_kv][P][dh] and scales [n_pages][n_kv]; row r of sequence b lies in page
// table[b * width + r / P]
struct PageLayer {
  void* k; void* v;
  float* ks; float* vs;                // null for BF16
  const int* table; const int* len;    // [batch][width], [batch]
  int type, batch, n_kv, n_pages, width, P, P_log, dh;
  int cap;                             // rows of a sequence at most: width P
};

struct PageAppendArgs {
  PageLayer c;
  const int* start; int N;             // [batch + 1] or null: token b is sequence b's
  int act;                             // SEQ_BF16 or SEQ_F32: type of q, k, v and q_out
  SeqRows q, k, v, q_out;              // (seq is not used)
  SeqRows rest;                        // p not null: rows like q_out's; tokens of no sequence get zeros here and in q_out
  int ks; long split;                  // as SeqAppendArgs, and so on to the end
  int n_q, n_kv;
  const int* kv_map;
  int rot, interleaved;
  double power[6];
  double mul, add, keep;
  float mscale;
  int by_index;
};
hipError_t launch_page_append(const PageAppendArgs& a, hipStream_t s);

struct PageAdvanceArgs {
  PageLayer c;                         // any layer
  const int* start; int N;
  int* len;                            // c.len
};
hipError_t launch_page_advance(const PageAdvanceArgs& a, hipStream_t s);

struct PageReadArgs {
  PageLayer c;
  const int* first;                    // [batch] or null: row 0
  int n, out_type;                     // SEQ_BF16 or SEQ_F32
  SeqRows k, v;                        // token stride: between rows
};
hipError_t launch_page_read(const PageReadArgs& a, hipStream_t s);

struct PageAttnArgs {
  PageLayer c;
  const int* start; int N;
  int act;
  SeqRows q, o;                        // (seq is not used)
  int slots, group;                    // as TreeAttnArgs
  int slot[64];
  float scale2;                        // scale * log2(e)
  int max_len, max_new;                // largest length and number of new tokens expected (they size launches; any are served)
  float* ws;                           // page_attn_workspace_bytes
};
size_t page_attn_workspace_bytes(const PageAttnArgs& a);
hipError_t launch_page_attn(const PageAttnArgs& a, hipStream_t s);

#ifdef __HIPCC__
// A sequence's share of a step. n: its tokens, first .. first + n - 1 of the packed ones (0 where start is out of order or
// range); L: rows it holds, -1 for a length outside 0 .. cap (it is passed over).
struct PageSeq {
  int first, n, L;
};
__device__ __forceinline__ PageSeq page_seq(const int* start, int N, const PageLayer& c, int b) {
  PageSeq q{b, 1, c.len[b]};
  if (start) {
    q.first = start[b];
    const int end = start[b + 1];
    q.n = q.first >= 0 && end <= N && end > q.first ? end - q.first : 0;
  }
  if (q.L < 0 || q.L > c.cap) q.L = -1;
  return q;
}
#endif

}  // namespace tasp
