// C ABI of the language model operators: argument validation, workspace sizes
// and dispatch.  Every check runs before anything is enqueued; nothing here
// allocates, frees or synchronises.
#include <limits.h>

#include <cmath>

#include <initializer_list>

#include "../../include/sru.h"
#include "sru_lm.h"

namespace {

using sru::hip_status;

constexpr long long kMaxElems = 1LL << 40;  // per tensor, far beyond any HBM size

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool valid_dtype(int t) { return t == SRU_DTYPE_FP32 || t == SRU_DTYPE_BF16; }
size_t elem_size(int t) { return t == SRU_DTYPE_BF16 ? 2 : 4; }
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

bool any_null(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!p) return true;
  return false;
}
bool all_aligned(std::initializer_list<const void*> ptrs, size_t n) {
  for (const void* p : ptrs)
    if (!aligned(p, n)) return false;
  return true;
}

int check_workspace(size_t need, const void* workspace, size_t bytes) {
  if (need == 0) return SRU_OK;
  if (!workspace || bytes < need) return SRU_E_WORKSPACE;
  return aligned(workspace, 256) ? SRU_OK : SRU_E_ALIGN;
}

// Vocabulary rows: shared checks of the logits' sizes, type and temperature.
int check_rows(const void* z, long long ld, int dtype, int N, int V, float temperature,
               sru::VocabRows& r) {
  if (!valid_dtype(dtype)) return SRU_E_FLAG;
  // a column past a row's end is told by its sign
  if (N <= 0 || V <= 0 || V > INT_MAX / 2 || ld < V || ld > kMaxElems / N) return SRU_E_SHAPE;
  // log2(e) / T, in which the kernels count, is finite as well
  if (!std::isfinite(temperature) || !(temperature > 0.f) ||
      !std::isfinite(1.44269504088896341f / temperature))
    return SRU_E_SHAPE;
  if (!z) return SRU_E_NULLPTR;
  if (!aligned(z, elem_size(dtype))) return SRU_E_ALIGN;
  r = sru::VocabRows{z, ld, dtype == SRU_DTYPE_BF16, N, V, temperature};
  return SRU_OK;
}

int check_grad(const void* dz, long long ldd, int dtype, int N, int V) {
  if (ldd < V || ldd > kMaxElems / N) return SRU_E_SHAPE;
  if (!dz) return SRU_E_NULLPTR;
  return aligned(dz, elem_size(dtype)) ? SRU_OK : SRU_E_ALIGN;
}

int check_teacher(const int64_t* ids, const void* logits, int dtype, int N, int K) {
  if (!valid_dtype(dtype)) return SRU_E_FLAG;
  if (K <= 0 || K > SRU_MAX_TEACHER) return SRU_E_SHAPE;
  if (!ids || !logits) return SRU_E_NULLPTR;
  return aligned(ids, 8) && aligned(logits, elem_size(dtype)) ? SRU_OK : SRU_E_ALIGN;
}

// One matrix of the residual norm; a missing one is OK unless required.
struct RowsCheck {
  int M, d;
  int operator()(const void* p, long long ld, int dtype, bool required, sru::Rows& r) const {
    if (!p) {
      r = sru::Rows{nullptr, 0};
      return required ? SRU_E_NULLPTR : SRU_OK;
    }
    if (ld < d || ld > kMaxElems / M) return SRU_E_SHAPE;
    if (!aligned(p, elem_size(dtype))) return SRU_E_ALIGN;
    r = sru::Rows{p, ld};
    return SRU_OK;
  }
};

int check_norm(int M, int d, int dtype, int res_dtype, int gate, sru::NormArgs& a) {
  if (!valid_dtype(dtype) || (res_dtype != dtype && res_dtype != SRU_DTYPE_FP32))
    return SRU_E_FLAG;
  if (gate != SRU_GATE_SILU && gate != SRU_GATE_SIGMOID) return SRU_E_FLAG;
  if (M <= 0 || d <= 0 || d > SRU_MAX_NORM_WIDTH) return SRU_E_SHAPE;
  a.M = M;
  a.d = d;
  a.act_bf16 = dtype == SRU_DTYPE_BF16;
  a.res_bf16 = res_dtype == SRU_DTYPE_BF16;
  a.silu = gate == SRU_GATE_SILU;
  return SRU_OK;
}

// One [L, B, d] tensor of the recurrence.
struct SeqCheck {
  int L, B, d, dtype;
  int operator()(const void* p, long long st, long long sb, bool out, sru::Seq& s) const {
    if (!p) return SRU_E_NULLPTR;
    if (st < 0 || sb < 0 || st > kMaxElems / L || sb > kMaxElems / B) return SRU_E_SHAPE;
    // an output's steps and sequences lie apart
    if (out && L > 1 && st < d) return SRU_E_SHAPE;
    if (out && B > 1 && sb < d) return SRU_E_SHAPE;
    if (out && L > 1 && B > 1 && st < sb * (B - 1) + d && sb < st * (L - 1) + d)
      return SRU_E_SHAPE;
    if (!aligned(p, elem_size(dtype))) return SRU_E_ALIGN;
    // the distance over a dimension of one does not count
    s = sru::Seq{p, L > 1 ? st : 0, B > 1 ? sb : 0};
    return SRU_OK;
  }
};

int check_lru(int L, int B, int d, int dtype, float c) {
  if (!valid_dtype(dtype)) return SRU_E_FLAG;
  if (L <= 0 || B <= 0 || d <= 0) return SRU_E_SHAPE;
  if ((long long)B * d > INT_MAX || (long long)L * B > INT_MAX - 1024) return SRU_E_SHAPE;
  if ((long long)B * d > kMaxElems / L) return SRU_E_SHAPE;
  // 1024 threads a workgroup, below 2^32 in a launch
  if (sru::lru_blocks(L, B, d) >= 1LL << 22) return SRU_E_SHAPE;
  if (!std::isfinite(c) || c < 0.f) return SRU_E_SHAPE;
  return SRU_OK;
}

}  // namespace

static_assert(SRU_LRU_STEPS == sru::kLruSteps, "steps");
static_assert(SRU_MAX_NORM_WIDTH == sru::kMaxNormWidth, "limits");
static_assert(SRU_MAX_TOP == sru::kMaxTop && SRU_MAX_TEACHER == sru::kMaxTeacher, "limits");

extern "C" {

size_t sru_token_logprobs_workspace_bytes(int N, int V, int dtype, int top) {
  if (N <= 0 || V <= 0 || !valid_dtype(dtype) || top < 0 || top > SRU_MAX_TOP) return 0;
  return align_up(sru::logprob_workspace_bytes(N, V, dtype == SRU_DTYPE_BF16, top));
}

int sru_token_logprobs(const void* logits, long long ld, int dtype, const int64_t* tokens, int N,
                       int V, int top, float temperature, float* logprob, float* entropy,
                       float* stats, int64_t* top_ids, float* top_logprobs, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  sru::LogprobArgs a{};
  if (int e = check_rows(logits, ld, dtype, N, V, temperature, a.r)) return e;
  if (top < 0 || top > SRU_MAX_TOP || top > V) return SRU_E_SHAPE;
  if (any_null({tokens, logprob, entropy, stats})) return SRU_E_NULLPTR;
  if (top > 0 && any_null({top_ids, top_logprobs})) return SRU_E_NULLPTR;
  if (!all_aligned({tokens, top_ids}, 8) ||
      !all_aligned({logprob, entropy, stats, top_logprobs}, 4))
    return SRU_E_ALIGN;
  const size_t need = sru_token_logprobs_workspace_bytes(N, V, dtype, top);
  if (int e = check_workspace(need, workspace, workspace_bytes)) return e;
  a.tokens = tokens;
  a.top = top;
  a.logprob = logprob;
  a.entropy = entropy;
  a.stats = stats;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  a.workspace = workspace;
  return hip_status(sru::logprob_launch(a, stream));
}

int sru_token_logprobs_backward(const void* logits, long long ld, int dtype,
                                const int64_t* tokens, const float* stats, const float* entropy,
                                const float* dlogprob, const float* dentropy,
                                const int64_t* top_ids, const float* dtop, int N, int V, int top,
                                float temperature, void* dlogits, long long ldd,
                                hipStream_t stream) {
  sru::LogprobGradArgs a{};
  if (int e = check_rows(logits, ld, dtype, N, V, temperature, a.r)) return e;
  if (top < 0 || top > SRU_MAX_TOP || top > V || (dtop && top == 0)) return SRU_E_SHAPE;
  if (int e = check_grad(dlogits, ldd, dtype, N, V)) return e;
  if (any_null({tokens, stats}) || (dentropy && !entropy) || (dtop && !top_ids))
    return SRU_E_NULLPTR;
  if (!all_aligned({tokens, top_ids}, 8) ||
      !all_aligned({stats, entropy, dlogprob, dentropy, dtop}, 4))
    return SRU_E_ALIGN;
  a.tokens = tokens;
  a.stats = stats;
  a.entropy = entropy;
  a.dlogprob = dlogprob;
  a.dentropy = dentropy;
  a.top_ids = top_ids;
  a.dtop = dtop;
  a.top = top;
  a.dz = dlogits;
  a.ldd = ldd;
  return hip_status(sru::logprob_grad_launch(a, stream));
}

size_t sru_distill_workspace_bytes(int N, int V, int dtype) {
  if (N <= 0 || V <= 0 || !valid_dtype(dtype)) return 0;
  return align_up(sru::distill_workspace_bytes(N, V, dtype == SRU_DTYPE_BF16));
}

int sru_distill_forward(const void* logits, long long ld, int dtype, const int64_t* teacher_ids,
                        const void* teacher_logits, int teacher_dtype, int N, int V, int K,
                        float temperature, float* loss, float* stats, void* workspace,
                        size_t workspace_bytes, hipStream_t stream) {
  sru::DistillArgs a{};
  if (int e = check_rows(logits, ld, dtype, N, V, temperature, a.r)) return e;
  if (int e = check_teacher(teacher_ids, teacher_logits, teacher_dtype, N, K)) return e;
  if (any_null({loss, stats})) return SRU_E_NULLPTR;
  if (!all_aligned({loss, stats}, 4)) return SRU_E_ALIGN;
  if (int e = check_workspace(sru_distill_workspace_bytes(N, V, dtype), workspace,
                              workspace_bytes))
    return e;
  a.ids = teacher_ids;
  a.teacher = teacher_logits;
  a.teacher_bf16 = teacher_dtype == SRU_DTYPE_BF16;
  a.K = K;
  a.loss = loss;
  a.stats = stats;
  a.workspace = workspace;
  return hip_status(sru::distill_launch(a, stream));
}

int sru_distill_backward(const void* logits, long long ld, int dtype, const int64_t* teacher_ids,
                         const void* teacher_logits, int teacher_dtype, const float* stats,
                         const float* dloss, int N, int V, int K, float temperature,
                         void* dlogits, long long ldd, hipStream_t stream) {
  sru::DistillArgs a{};
  if (int e = check_rows(logits, ld, dtype, N, V, temperature, a.r)) return e;
  if (int e = check_teacher(teacher_ids, teacher_logits, teacher_dtype, N, K)) return e;
  if (int e = check_grad(dlogits, ldd, dtype, N, V)) return e;
  if (any_null({stats, dloss})) return SRU_E_NULLPTR;
  if (!all_aligned({stats, dloss}, 4)) return SRU_E_ALIGN;
  a.ids = teacher_ids;
  a.teacher = teacher_logits;
  a.teacher_bf16 = teacher_dtype == SRU_DTYPE_BF16;
  a.K = K;
  a.dloss = dloss;
  a.stats = const_cast<float*>(stats);  // read only where loss is NULL
  a.dz = dlogits;
  a.ldd = ldd;
  return hip_status(sru::distill_launch(a, stream));
}

int sru_distill_forward_backward(const void* logits, long long ld, int dtype,
                                 const int64_t* teacher_ids, const void* teacher_logits,
                                 int teacher_dtype, const float* dloss, int N, int V, int K,
                                 float temperature, float* loss, float* stats, void* dlogits,
                                 long long ldd, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream) {
  sru::DistillArgs a{};
  if (int e = check_rows(logits, ld, dtype, N, V, temperature, a.r)) return e;
  if (int e = check_teacher(teacher_ids, teacher_logits, teacher_dtype, N, K)) return e;
  if (int e = check_grad(dlogits, ldd, dtype, N, V)) return e;
  if (any_null({dloss, loss, stats})) return SRU_E_NULLPTR;
  if (!all_aligned({dloss, loss, stats}, 4)) return SRU_E_ALIGN;
  if (int e = check_workspace(sru_distill_workspace_bytes(N, V, dtype), workspace,
                              workspace_bytes))
    return e;
  a.ids = teacher_ids;
  a.teacher = teacher_logits;
  a.teacher_bf16 = teacher_dtype == SRU_DTYPE_BF16;
  a.K = K;
  a.dloss = dloss;
  a.loss = loss;
  a.stats = stats;
  a.dz = dlogits;
  a.ldd = ldd;
  a.workspace = workspace;
  return hip_status(sru::distill_launch(a, stream));
}

int sru_residual_norm_forward(int M, int d, int dtype, int res_dtype, int gate, float eps,
                              const void* x, long long ldx, const void* y, long long ldy,
                              const void* z, long long ldz, const float* w_post,
                              const float* scale, const float* w_pre, void* x_out,
                              long long ldx_out, void* o, long long ldo, float* rstd,
                              hipStream_t stream) {
  sru::NormArgs a{};
  if (int e = check_norm(M, d, dtype, res_dtype, gate, a)) return e;
  if (!std::isfinite(eps) || !(eps > 0.f)) return SRU_E_SHAPE;
  // without a block's output there is nothing but the norm of x, without
  // w_pre nothing but the sum
  if (!y && (z || w_post || scale || x_out || !w_pre)) return SRU_E_NULLPTR;
  if (!w_pre && o) return SRU_E_NULLPTR;
  const RowsCheck rows{M, d};
  if (int e = rows(x, ldx, res_dtype, true, a.x)) return e;
  if (int e = rows(y, ldy, dtype, false, a.y)) return e;
  if (int e = rows(z, ldz, dtype, false, a.z)) return e;
  if (int e = rows(x_out, ldx_out, res_dtype, y != nullptr, a.x_out)) return e;
  if (int e = rows(o, ldo, dtype, w_pre != nullptr, a.o)) return e;
  if (!rstd) return SRU_E_NULLPTR;
  if (!all_aligned({w_post, scale, w_pre, rstd}, 4)) return SRU_E_ALIGN;
  a.eps = eps;
  a.w_post = w_post;
  a.scale = scale;
  a.w_pre = w_pre;
  a.rstd = rstd;
  return hip_status(sru::norm_launch(a, stream));
}

size_t sru_residual_norm_backward_workspace_bytes(int M, int d) {
  if (M <= 0 || d <= 0 || d > SRU_MAX_NORM_WIDTH) return 0;
  return align_up(sru::norm_grad_workspace_bytes(M, d));
}

int sru_residual_norm_backward(int M, int d, int dtype, int res_dtype, int gate, const void* x,
                               long long ldx, const void* y, long long ldy, const void* z,
                               long long ldz, const float* w_post, const float* scale,
                               const float* w_pre, const float* rstd, const void* dx_out,
                               long long lddx_out, const void* do_, long long lddo, void* dx,
                               long long lddx, void* dy, long long lddy, void* dz, long long lddz,
                               float* dw_post, float* dscale, float* dw_pre, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
  sru::NormArgs a{};
  if (int e = check_norm(M, d, dtype, res_dtype, gate, a)) return e;
  if (!y && (z || w_post || scale || !w_pre)) return SRU_E_NULLPTR;
  // a gradient for every input that is there, and for no other
  if (!dy != !y || !dz != !z || !dw_post != !w_post || !dscale != !scale || !dw_pre != !w_pre)
    return SRU_E_NULLPTR;
  const RowsCheck rows{M, d};
  if (int e = rows(x, ldx, res_dtype, true, a.x)) return e;
  if (int e = rows(y, ldy, dtype, false, a.y)) return e;
  if (int e = rows(z, ldz, dtype, false, a.z)) return e;
  if (int e = rows(dx_out, lddx_out, res_dtype, false, a.dx_out)) return e;
  if (int e = rows(do_, lddo, dtype, false, a.go)) return e;
  if (int e = rows(dx, lddx, res_dtype, true, a.dx)) return e;
  if (int e = rows(dy, lddy, dtype, false, a.dy)) return e;
  if (int e = rows(dz, lddz, dtype, false, a.dz)) return e;
  if (!rstd) return SRU_E_NULLPTR;
  if (!all_aligned({w_post, scale, w_pre, rstd, dw_post, dscale, dw_pre}, 4)) return SRU_E_ALIGN;
  if (int e = check_workspace(sru_residual_norm_backward_workspace_bytes(M, d), workspace,
                              workspace_bytes))
    return e;
  a.w_post = w_post;
  a.scale = scale;
  a.w_pre = w_pre;
  a.rstd = const_cast<float*>(rstd);  // read only by the gradient
  a.dw_post = dw_post;
  a.dscale = dscale;
  a.dw_pre = dw_pre;
  a.partial = static_cast<float*>(workspace);
  return hip_status(sru::norm_grad_launch(a, stream));
}

size_t sru_lru_forward_workspace_bytes(int L, int B, int d) {
  if (check_lru(L, B, d, SRU_DTYPE_FP32, 0.f) != SRU_OK) return 0;
  return align_up(sru::lru_workspace_bytes(L, B, d));
}

int sru_lru_forward(int L, int B, int d, int dtype, const void* x, long long x_t, long long x_b,
                    const void* r, long long r_t, long long r_b, const void* i, long long i_t,
                    long long i_b, const float* lam, float c, const float* h0,
                    const uint8_t* pad_mask, const uint8_t* reset, void* H, long long H_t,
                    long long H_b, float* h_last, float* states, void* workspace,
                    size_t workspace_bytes, hipStream_t stream) {
  if (int e = check_lru(L, B, d, dtype, c)) return e;
  sru::LruArgs a{};
  const SeqCheck seq{L, B, d, dtype};
  if (int e = seq(x, x_t, x_b, false, a.x)) return e;
  if (int e = seq(r, r_t, r_b, false, a.r)) return e;
  if (int e = seq(i, i_t, i_b, false, a.i)) return e;
  if (int e = seq(H, H_t, H_b, true, a.h)) return e;
  if (!lam) return SRU_E_NULLPTR;
  if (!all_aligned({lam, h0, h_last, states}, 4)) return SRU_E_ALIGN;
  if (int e = check_workspace(sru_lru_forward_workspace_bytes(L, B, d), workspace,
                              workspace_bytes))
    return e;
  a.L = L;
  a.B = B;
  a.d = d;
  a.bf16 = dtype == SRU_DTYPE_BF16;
  a.lam = lam;
  a.c = c;
  a.mask = pad_mask;
  a.reset = reset;
  a.h0 = h0;
  a.h_last = h_last;
  a.states = states;
  a.workspace = workspace;
  return hip_status(sru::lru_launch(a, stream));
}

size_t sru_lru_backward_workspace_bytes(int L, int B, int d) {
  if (check_lru(L, B, d, SRU_DTYPE_FP32, 0.f) != SRU_OK) return 0;
  return align_up(sru::lru_grad_workspace_bytes(L, B, d));
}

int sru_lru_backward(int L, int B, int d, int dtype, const void* x, long long x_t, long long x_b,
                     const void* r, long long r_t, long long r_b, const void* i, long long i_t,
                     long long i_b, const float* lam, float c, const float* states,
                     const void* dH, long long dH_t, long long dH_b, const float* dh_last,
                     const uint8_t* pad_mask, const uint8_t* reset, void* dx, long long dx_t,
                     long long dx_b, void* dr, long long dr_t, long long dr_b, void* di,
                     long long di_t, long long di_b, float* dlam, float* dh0, void* workspace,
                     size_t workspace_bytes, hipStream_t stream) {
  if (int e = check_lru(L, B, d, dtype, c)) return e;
  sru::LruArgs a{};
  const SeqCheck seq{L, B, d, dtype};
  if (int e = seq(x, x_t, x_b, false, a.x)) return e;
  if (int e = seq(r, r_t, r_b, false, a.r)) return e;
  if (int e = seq(i, i_t, i_b, false, a.i)) return e;
  if (int e = seq(dH, dH_t, dH_b, false, a.dh)) return e;
  if (int e = seq(dx, dx_t, dx_b, true, a.dx)) return e;
  if (int e = seq(dr, dr_t, dr_b, true, a.dr)) return e;
  if (int e = seq(di, di_t, di_b, true, a.di)) return e;
  if (any_null({lam, states, dlam})) return SRU_E_NULLPTR;
  if (!all_aligned({lam, states, dh_last, dlam, dh0}, 4)) return SRU_E_ALIGN;
  if (int e = check_workspace(sru_lru_backward_workspace_bytes(L, B, d), workspace,
                              workspace_bytes))
    return e;
  a.L = L;
  a.B = B;
  a.d = d;
  a.bf16 = dtype == SRU_DTYPE_BF16;
  a.lam = lam;
  a.c = c;
  a.mask = pad_mask;
  a.reset = reset;
  a.states = const_cast<float*>(states);  // read only by the gradient
  a.dh_last = dh_last;
  a.dlam = dlam;
  a.dh0 = dh0;
  a.workspace = workspace;
  return hip_status(sru::lru_grad_launch(a, stream));
}

}  // extern "C"
