// Internal launch interface and device helpers of the language model operators
// (vocabulary rows, block norms, the gated linear recurrence).  Launchers
// assume validated arguments and only enqueue work.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sru_internal.h"

namespace sru {

// ------------------------------------------------------------ vocabulary rows
constexpr int kMaxTop = 64;       // alternatives: one lane of a wave each
constexpr int kMaxTeacher = 1024; // teacher's logits of a row
// Blocks a launch has at most; each then takes several (row, part) items.
constexpr long long kMaxGrid = 1 << 20;

// N rows of V logits of pitch ld (elements), fp32 or bf16.
struct VocabRows {
  const void* z;
  long long ld;
  int bf16;
  int N, V;
  float temperature;
};

struct LogprobArgs {
  VocabRows r;
  const int64_t* tokens;
  int top;
  float* logprob;
  float* entropy;
  float* stats;  // [N, 2]: max z, sum exp((z - max) / T)
  int64_t* top_ids;
  float* top_logprobs;
  void* workspace;
};
size_t logprob_workspace_bytes(int N, int V, int bf16, int top);
hipError_t logprob_launch(const LogprobArgs& a, hipStream_t stream);

struct LogprobGradArgs {
  VocabRows r;
  const int64_t* tokens;
  const float* stats;
  const float* entropy;
  const float* dlogprob;
  const float* dentropy;
  const int64_t* top_ids;
  const float* dtop;
  int top;
  void* dz;
  long long ldd;
};
hipError_t logprob_grad_launch(const LogprobGradArgs& a, hipStream_t stream);

struct DistillArgs {
  VocabRows r;
  const int64_t* ids;    // [N, K]
  const void* teacher;   // [N, K]
  int teacher_bf16;
  int K;
  const float* dloss;    // with dz: weight of each row's loss
  float* loss;           // nullptr: gradient only, from stats
  float* stats;          // out, or in where loss is nullptr
  void* dz;              // nullptr: loss only
  long long ldd;
  void* workspace;
};
size_t distill_workspace_bytes(int N, int V, int bf16);
hipError_t distill_launch(const DistillArgs& a, hipStream_t stream);

}  // namespace sru
