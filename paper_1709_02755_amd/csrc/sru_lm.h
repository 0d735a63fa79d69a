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

// ------------------------------------------------------------- residual norm
constexpr int kMaxNormWidth = 16384;  // a row is held in one workgroup's registers

// A matrix of M rows (data may be nullptr: absent), row pitch ld elements.
struct Rows {
  const void* p;
  long long ld;
};
struct NormArgs {
  int M, d;
  int act_bf16, res_bf16;
  int silu;  // gate z sigma(z), else sigma(z)
  float eps;
  Rows x, y, z;
  const float* w_post;
  const float* scale;
  const float* w_pre;
  float* rstd;  // [M, 2]: of y and of x_out; out in the forward, in for the gradient
  // forward
  Rows x_out, o;
  // gradient
  Rows dx_out, go;   // in: gradients of x_out and o
  Rows dx, dy, dz;   // out
  float* dw_post;
  float* dscale;
  float* dw_pre;
  float* partial;    // norm_grad_workspace_bytes
};
hipError_t norm_launch(const NormArgs& a, hipStream_t stream);
size_t norm_grad_workspace_bytes(int M, int d);
hipError_t norm_grad_launch(const NormArgs& a, hipStream_t stream);

// ------------------------------------------------- gated linear recurrence
constexpr int kLruSteps = 8;  // the steps that a wave holds, and that a state is kept for

// [L, B, d] with contiguous features; distances of steps and of sequences in
// elements.
struct Seq {
  const void* p;
  long long st, sb;
};
struct LruArgs {
  int L, B, d, bf16;
  Seq x, r, i;
  const float* lam;
  float c;
  const uint8_t* mask;   // [L, B] or nullptr
  const uint8_t* reset;  // [L, B] or nullptr
  // forward
  const float* h0;
  Seq h;
  float* h_last;
  float* states;  // [ceil(L / kLruSteps), B, d]; out, or in for the gradient
  // gradient
  Seq dh;
  const float* dh_last;
  Seq dx, dr, di;
  float* dlam;
  float* dh0;
  void* workspace;
};
size_t lru_workspace_bytes(int L, int B, int d);
size_t lru_grad_workspace_bytes(int L, int B, int d);
// Workgroups of a call, at most (they must fit a launch).
long long lru_blocks(int L, int B, int d);
hipError_t lru_launch(const LruArgs& a, hipStream_t stream);
hipError_t lru_grad_launch(const LruArgs& a, hipStream_t stream);

}  // namespace sru
