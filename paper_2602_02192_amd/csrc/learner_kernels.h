// Launches of the learner's kernels (kernels_logits.hip, kernels_adamw.hip) for echo_learner.hip, which has checked the arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace echo {

struct LogitRows {
  const void *x;
  const int32_t *targets;   // nullable: every row takes part
  int64_t rows, stride;
  int32_t vocab, dtype;
  float temperature;
  const float *weights;     // nullable; a row of weight 0 takes no part
};

struct RowOutputs {
  float *logprobs, *entropy, *lse;   // nullable
  int32_t *top_ids;
  float *top_logprobs;
  int32_t top_k;
};

struct PolicyTerms {
  const float *advantages, *old_logprobs, *sampler, *ref;   // sampler, ref nullable
  float lo, hi, ratio_cap, sampler_cap, kl, entropy;                  // lo, hi: bounds of the clipped ratio
};

size_t logprobs_workspace(const LogitRows &x, int top_k);
size_t policy_workspace(const LogitRows &x);
void launch_token_logprobs(const LogitRows &x, const RowOutputs &out, void *workspace, hipStream_t st);
void launch_token_logprobs_grad(const LogitRows &x, const float *lse, const float *entropy, const float *g, const float *h, void *out, int64_t out_stride,
                                hipStream_t st);
void launch_policy_loss(const LogitRows &x, const PolicyTerms &p, float *loss, float *logprobs, float *entropy, void *grad, int64_t grad_stride,
                        void *workspace, hipStream_t st);

// The tensors of one launch, by value in its arguments (4 KiB hold them): what is queued refers to no host memory, so a call can
// be recorded into a graph and its arrays freed.
constexpr int TENSORS_PER_LAUNCH = 64;
struct NormTensors {
  const void *grad[TENSORS_PER_LAUNCH];
  int64_t numel[TENSORS_PER_LAUNCH];
  uint32_t chunk0[TENSORS_PER_LAUNCH + 1];   // first chunk of each tensor
  int32_t n;
  int64_t chunk;                             // elements of a workgroup
};
struct StepTensors {
  void *param[TENSORS_PER_LAUNCH];
  const void *grad[TENSORS_PER_LAUNCH];
  uint16_t *snapshot[TENSORS_PER_LAUNCH];
  int64_t numel[TENSORS_PER_LAUNCH];
  int64_t state0[TENSORS_PER_LAUNCH];        // first element in the states
  float decay[TENSORS_PER_LAUNCH];           // 1 - lr weight_decay
  uint32_t chunk0[TENSORS_PER_LAUNCH + 1];
  int32_t n;
};
struct StepConstants {
  void *m, *v;
  float *m_scale, *v_scale;
  const float *norm;
  float max_norm, beta1, fresh1, beta2, fresh2, root, eps, size;   // fresh: 1 - beta; root: (1 - beta2^t)^-1/2; size: lr / (1 - beta1^t)
  uint32_t step;
  uint64_t seed;
  bool moderate;   // eps and root keep the denominators of moderate averages within 2^-60 .. 2^90
};
constexpr int64_t STEP_CHUNK = 4096;          // elements of a workgroup
// Elements of a workgroup of the norm: enough of them to fill the GPU, and, of many elements, few enough partial sums for the one workgroup that adds them up.
inline int64_t norm_chunk(int64_t elements) { return elements < (int64_t)1 << 26 ? 8192 : 65536; }
void launch_grad_norm(const NormTensors &t, int dtype, double *partial, hipStream_t st);          // partial[chunk]
void launch_norm_finish(const double *partial, int64_t n, float *out, hipStream_t st);
void launch_adamw(const StepTensors &t, const StepConstants &c, int param_dtype, int grad_dtype, int state_dtype, hipStream_t st);

}  // namespace echo
