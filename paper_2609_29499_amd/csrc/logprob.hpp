// Log probabilities of given tokens: arguments of the kernels in logprob.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tasp {

constexpr int kTopMax = 32;            // alternatives at most

struct LogprobArgs {
  const void* logits; int f32;         // rows of V values (BF16, or float32), `ld` apart
  long ld;
  const int* tokens; int rows, V;
  float c, lim;                        // log2(e) / temperature; magnitude that logits are cut to
  int top;                             // alternatives, 0 .. kTopMax
  float* logprob; float* entropy; int* rank; int* top_ids; float* top_logprobs;    // entropy, rank may be null
  const int* start; int seqs; float* mean;                                        // start, mean null: no means
  void* ws;                            // logprob_workspace_bytes
};
size_t logprob_workspace_bytes(int rows, int V, int top);
hipError_t launch_logprob(const LogprobArgs& a, hipStream_t s);

}  // namespace tasp
