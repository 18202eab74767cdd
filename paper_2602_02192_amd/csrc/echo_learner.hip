// Entry points of include/echo_learner.h: argument checks, workspace sizes, launches.  No state and no device memory of their own.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>

#include "../../include/echo_learner.h"
#include "learner_kernels.h"

void echo_set_call_error(const char *msg);   // echo_engine.hip: the message echo_last_error(NULL) returns on this thread

using namespace echo;

namespace {

int refuse(int code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  echo_set_call_error(buf);
  return code;
}

// Nothing a call does may leave through the C boundary but its code.
template <typename F> int guarded(F f) {
  try {
    return f();
  } catch (const std::exception &) {
    return ECHO_ENOMEM;   // the library itself throws nothing; the runtime's own containers can run out of memory
  } catch (...) {
    return ECHO_EHIP;
  }
}

// Drops what the runtime holds as this thread's last error, queues, and reports what the launches said.
template <typename F> int queue(F launches) {
  (void)hipGetLastError();
  launches();
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ECHO_OK : refuse(ECHO_EHIP, "kernel launch: %s", hipGetErrorString(e));
}

size_t element_bytes(int dtype) { return dtype == ECHO_F32 ? 4 : dtype == ECHO_BF16 || dtype == ECHO_F16 ? 2 : 0; }
bool misaligned(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

const char *wrong_logits(const echo_logits *x) {
  if (!x) return "logits description is NULL";
  const size_t e = element_bytes(x->dtype);
  if (!e) return "logits must be ECHO_F32, ECHO_BF16 or ECHO_F16";
  if (x->rows < 0) return "rows must not be negative";
  if (x->vocab < 1 || x->vocab > 1 << 28) return "vocab must lie in 1 .. 2^28";
  // A launch has less than 2^32 threads: 256 for every 8192 entries of a row at most, and 512 or 1024 for a row of two or five times as many.
  if (x->rows > ((1 << 24) - 1) / ((x->vocab + 8191) / 8192)) return "rows * ceil(vocab / 8192) must be less than 2^24";
  if (x->row_stride < x->vocab) return "row_stride is less than vocab";
  if (x->rows > 0 && x->row_stride > INT64_MAX / 16 / x->rows) return "rows * row_stride is out of range";
  if (!(x->temperature > 0.f) || !std::isfinite(x->temperature) || !std::isfinite(2.0f / x->temperature)) return "temperature must be positive, finite, and its reciprocal too";
  return nullptr;
}
const char *wrong_pointers(const echo_logits *x) {
  if (x->rows == 0) return nullptr;
  if (!x->logits) return "logits are NULL";
  if (misaligned(x->logits, element_bytes(x->dtype))) return "logits are not aligned to their elements";
  if (misaligned(x->targets, 4)) return "targets are not aligned to their elements";
  return nullptr;
}
LogitRows rows_of(const echo_logits *x) { return {x->logits, x->targets, x->rows, x->row_stride, x->vocab, x->dtype, x->temperature, nullptr}; }

bool any_misaligned4(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (misaligned(p, 4)) return true;
  return false;
}

const char *wrong_workspace(const void *p, size_t have, size_t need) {
  if (need == 0) return nullptr;
  if (!p || have < need) return "the workspace is smaller than its size function says";
  if (misaligned(p, 256)) return "the workspace is not 256-byte aligned";
  return nullptr;
}

const char *wrong_grad(const echo_logits *x, const void *out, int64_t stride) {
  if (stride < x->vocab) return "the gradient's row stride is less than vocab";
  if (x->rows > 0 && stride > INT64_MAX / 16 / x->rows) return "rows * gradient stride is out of range";
  if (misaligned(out, element_bytes(x->dtype))) return "the gradient is not aligned to its elements";
  if (out == x->logits && stride != x->row_stride) return "a gradient in place of the logits needs their row stride";
  return nullptr;
}

// First chunk behind n tensors; -1 where a size is negative or the chunks pass a grid's limit.
int64_t chunks_of(const int64_t *numel, int32_t n, int64_t chunk) {
  if (n < 0 || (n > 0 && !numel)) return -1;
  int64_t c = 0;
  for (int i = 0; i < n; ++i) {
    if (numel[i] < 0 || numel[i] > ((int64_t)1 << 42)) return -1;
    c += (numel[i] + chunk - 1) / chunk;
    if (c > INT32_MAX) return -1;
  }
  return c;
}

// Chunks of a norm, and their size; -1 as above.
int64_t norm_chunks(const int64_t *numel, int32_t n, int64_t *chunk) {
  int64_t total = 0;
  if (chunks_of(numel, n, 65536) < 0) return -1;
  for (int i = 0; i < n; ++i) total += numel[i];
  *chunk = norm_chunk(total);
  return chunks_of(numel, n, *chunk);
}

}  // namespace

extern "C" {

size_t echo_token_logprobs_workspace(const echo_logits *x, int32_t top_k) {
  if (wrong_logits(x) || top_k < 0 || top_k > ECHO_TOP_MAX || top_k > x->vocab) return 0;
  return logprobs_workspace(rows_of(x), top_k);
}

int echo_token_logprobs(const echo_logits *x, int32_t top_k, float *out_logprobs, float *out_entropy, float *out_lse, int32_t *out_top_ids, float *out_top_logprobs,
                        void *workspace, size_t workspace_bytes, void *stream) {
  return guarded([&] {
    if (const char *why = wrong_logits(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (const char *why = wrong_pointers(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (top_k < 0 || top_k > ECHO_TOP_MAX || top_k > x->vocab) return refuse(ECHO_EINVAL, "top_k = %d outside 0 .. min(%d, vocab)", top_k, ECHO_TOP_MAX);
    if (x->rows == 0) return (int)ECHO_OK;
    if ((top_k > 0) != (out_top_ids != nullptr) || (top_k > 0) != (out_top_logprobs != nullptr))
      return refuse(ECHO_EINVAL, "top outputs and top_k = %d do not go together", top_k);
    if (!x->targets && out_logprobs) return refuse(ECHO_EINVAL, "log-probabilities need targets");
    if (any_misaligned4({out_logprobs, out_entropy, out_lse, out_top_ids, out_top_logprobs})) return refuse(ECHO_EINVAL, "an output is not aligned to its elements");
    const LogitRows r = rows_of(x);
    if (const char *why = wrong_workspace(workspace, workspace_bytes, logprobs_workspace(r, top_k))) return refuse(ECHO_ENOMEM, "%s", why);
    const RowOutputs out = {out_logprobs, out_entropy, out_lse, out_top_ids, out_top_logprobs, top_k};
    return queue([&] { launch_token_logprobs(r, out, workspace, (hipStream_t)stream); });
  });
}

int echo_token_logprobs_grad(const echo_logits *x, const float *lse, const float *entropy, const float *grad_logprobs, const float *grad_entropy, void *out,
                             int64_t out_stride, void *stream) {
  return guarded([&] {
    if (const char *why = wrong_logits(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (const char *why = wrong_pointers(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (const char *why = wrong_grad(x, out, out_stride)) return refuse(ECHO_EINVAL, "%s", why);
    if (x->rows == 0) return (int)ECHO_OK;
    if (!lse || !out) return refuse(ECHO_EINVAL, "lse and the gradient are needed");
    if (!grad_logprobs && !grad_entropy) return refuse(ECHO_EINVAL, "grad_logprobs or grad_entropy is needed");
    if (grad_logprobs && !x->targets) return refuse(ECHO_EINVAL, "grad_logprobs needs targets");
    if (grad_entropy && !entropy) return refuse(ECHO_EINVAL, "grad_entropy needs the entropy");
    if (any_misaligned4({lse, entropy, grad_logprobs, grad_entropy})) return refuse(ECHO_EINVAL, "an input is not aligned to its elements");
    return queue([&] { launch_token_logprobs_grad(rows_of(x), lse, entropy, grad_logprobs, grad_entropy, out, out_stride, (hipStream_t)stream); });
  });
}

size_t echo_policy_loss_workspace(const echo_logits *x) { return wrong_logits(x) ? 0 : policy_workspace(rows_of(x)); }

int echo_policy_loss(const echo_logits *x, const float *advantages, const float *old_logprobs, const float *weights, const float *sampler_logprobs,
                     const float *ref_logprobs, const echo_policy_loss_opts *o, float *out_loss, float *out_logprobs, float *out_entropy, void *out_grad,
                     int64_t grad_stride, void *workspace, size_t workspace_bytes, void *stream) {
  return guarded([&] {
    if (const char *why = wrong_logits(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (const char *why = wrong_pointers(x)) return refuse(ECHO_EINVAL, "%s", why);
    if (!o) return refuse(ECHO_EINVAL, "opts are NULL");
    if (!(o->clip_low >= 0.f) || !(o->clip_high >= 0.f)) return refuse(ECHO_EINVAL, "clip_low and clip_high must be >= 0");
    if (!(o->ratio_cap > 0.f) || !(o->sampler_cap > 0.f)) return refuse(ECHO_EINVAL, "ratio_cap and sampler_cap must be positive");
    if (!std::isfinite(o->kl_coef) || !std::isfinite(o->entropy_coef)) return refuse(ECHO_EINVAL, "kl_coef and entropy_coef must be finite");
    if (out_grad)
      if (const char *why = wrong_grad(x, out_grad, grad_stride)) return refuse(ECHO_EINVAL, "%s", why);
    if (x->rows == 0) return (int)ECHO_OK;
    if (!x->targets || !advantages || !old_logprobs) return refuse(ECHO_EINVAL, "targets, advantages and old_logprobs are needed");
    if (o->kl_coef != 0.f && !ref_logprobs) return refuse(ECHO_EINVAL, "kl_coef = %g needs ref_logprobs", (double)o->kl_coef);
    if (any_misaligned4({advantages, old_logprobs, weights, sampler_logprobs, ref_logprobs, out_loss, out_logprobs, out_entropy}))
      return refuse(ECHO_EINVAL, "an array is not aligned to its elements");
    LogitRows r = rows_of(x);
    r.weights = weights;
    if (const char *why = wrong_workspace(workspace, workspace_bytes, policy_workspace(r))) return refuse(ECHO_ENOMEM, "%s", why);
    const PolicyTerms p = {advantages, old_logprobs, sampler_logprobs, ref_logprobs, (float)(1.0 - (double)o->clip_low), (float)(1.0 + (double)o->clip_high),
                           o->ratio_cap, o->sampler_cap, o->kl_coef, o->entropy_coef};
    return queue([&] { launch_policy_loss(r, p, out_loss, out_logprobs, out_entropy, out_grad, grad_stride, workspace, (hipStream_t)stream); });
  });
}

size_t echo_grad_norm_workspace(const int64_t *numel, int32_t n_tensors) {
  int64_t chunk;
  const int64_t c = norm_chunks(numel, n_tensors, &chunk);
  return c < 0 ? 0 : (size_t)(c + 1) * sizeof(double);
}

int echo_grad_norm(const void *const *grads, const int64_t *numel, int32_t n_tensors, int32_t dtype, float *out_norm, void *workspace, size_t workspace_bytes,
                   void *stream) {
  return guarded([&] {
    const size_t e = element_bytes(dtype);
    if (!e) return refuse(ECHO_EINVAL, "gradients must be ECHO_F32, ECHO_BF16 or ECHO_F16");
    int64_t chunk;
    const int64_t chunks = norm_chunks(numel, n_tensors, &chunk);
    if (chunks < 0 || (n_tensors > 0 && !grads)) return refuse(ECHO_EINVAL, "bad sizes");
    if (!out_norm || misaligned(out_norm, 4)) return refuse(ECHO_EINVAL, "out_norm is NULL or not aligned");
    for (int i = 0; i < n_tensors; ++i)
      if (numel[i] > 0 && (!grads[i] || misaligned(grads[i], e))) return refuse(ECHO_EINVAL, "gradient %d is NULL or not aligned to its elements", i);
    if (const char *why = wrong_workspace(workspace, workspace_bytes, echo_grad_norm_workspace(numel, n_tensors))) return refuse(ECHO_ENOMEM, "%s", why);
    double *partial = (double *)workspace;
    hipStream_t st = (hipStream_t)stream;
    return queue([&] {
      NormTensors t;
      t.chunk = chunk;
      int64_t done = 0;
      for (int i = 0; i < n_tensors;) {
        t.n = 0;
        t.chunk0[0] = 0;
        for (; i < n_tensors && t.n < TENSORS_PER_LAUNCH; ++i) {
          if (numel[i] == 0) continue;
          t.grad[t.n] = grads[i];
          t.numel[t.n] = numel[i];
          t.chunk0[t.n + 1] = t.chunk0[t.n] + (uint32_t)((numel[i] + chunk - 1) / chunk);
          ++t.n;
        }
        if (t.n) launch_grad_norm(t, dtype, partial + done, st);
        done += t.chunk0[t.n];
      }
      launch_norm_finish(partial, done, out_norm, st);
    });
  });
}

int64_t echo_adamw_state_numel(const int64_t *numel, int32_t n_tensors) {
  if (chunks_of(numel, n_tensors, STEP_CHUNK) < 0) return -1;
  int64_t s = 0;
  for (int i = 0; i < n_tensors; ++i) s += (numel[i] + ECHO_ADAMW_BLOCK - 1) / ECHO_ADAMW_BLOCK * ECHO_ADAMW_BLOCK;
  return s;
}

int echo_adamw_step(const echo_adamw_args *a, void *stream) {
  return guarded([&] {
    if (!a) return refuse(ECHO_EINVAL, "args are NULL");
    if (a->param_dtype != ECHO_F32 && a->param_dtype != ECHO_BF16) return refuse(ECHO_EINVAL, "parameters must be ECHO_F32 or ECHO_BF16");
    if (a->grad_dtype != ECHO_F32 && a->grad_dtype != ECHO_BF16) return refuse(ECHO_EINVAL, "gradients must be ECHO_F32 or ECHO_BF16");
    if (a->state_dtype != ECHO_F32 && a->state_dtype != ECHO_E4M3) return refuse(ECHO_EINVAL, "states must be ECHO_F32 or ECHO_E4M3");
    if (chunks_of(a->numel, a->n_tensors, STEP_CHUNK) < 0) return refuse(ECHO_EINVAL, "bad sizes");
    const int64_t states = echo_adamw_state_numel(a->numel, a->n_tensors);
    if (!(a->lr >= 0) || !std::isfinite(a->lr) || !(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1) || !((float)a->eps > 0.f) || !std::isfinite(a->eps))
      return refuse(ECHO_EINVAL, "lr >= 0, 0 <= beta < 1 and eps > 0 are needed");
    if (a->step < 1 || a->step > INT32_MAX) return refuse(ECHO_EINVAL, "step = %lld outside 1 .. 2^31 - 1", (long long)a->step);
    if (a->norm && !(a->max_norm > 0.f)) return refuse(ECHO_EINVAL, "max_norm must be positive");
    if (states == 0) return (int)ECHO_OK;
    if (!a->params || !a->grads || !a->weight_decay || !a->m || !a->v) return refuse(ECHO_EINVAL, "params, grads, weight_decay, m and v are needed");
    const bool f8 = a->state_dtype == ECHO_E4M3;
    if (f8 != (a->m_scale != nullptr) || f8 != (a->v_scale != nullptr)) return refuse(ECHO_EINVAL, "scales go with ECHO_E4M3 states, and with no others");
    if (a->snapshot && a->param_dtype != ECHO_F32) return refuse(ECHO_EINVAL, "a snapshot goes with ECHO_F32 parameters");
    if (misaligned(a->m, 16) || misaligned(a->v, 16)) return refuse(ECHO_EINVAL, "m and v must be 16-byte aligned");
    if (any_misaligned4({a->m_scale, a->v_scale, a->norm})) return refuse(ECHO_EINVAL, "an array is not aligned to its elements");
    for (int i = 0; i < a->n_tensors; ++i) {
      if (a->numel[i] == 0) continue;
      if (!a->params[i] || misaligned(a->params[i], element_bytes(a->param_dtype))) return refuse(ECHO_EINVAL, "parameter %d is NULL or not aligned to its elements", i);
      if (!a->grads[i] || misaligned(a->grads[i], element_bytes(a->grad_dtype))) return refuse(ECHO_EINVAL, "gradient %d is NULL or not aligned to its elements", i);
      if (a->snapshot && (!a->snapshot[i] || misaligned(a->snapshot[i], 2))) return refuse(ECHO_EINVAL, "snapshot %d is NULL or not aligned to its elements", i);
      if (!std::isfinite(a->weight_decay[i])) return refuse(ECHO_EINVAL, "weight_decay[%d] is not finite", i);
    }
    StepConstants c;
    c.m = a->m; c.v = a->v; c.m_scale = a->m_scale; c.v_scale = a->v_scale; c.norm = a->norm; c.max_norm = a->max_norm;
    c.beta1 = (float)a->beta1; c.fresh1 = (float)(1.0 - a->beta1);
    c.beta2 = (float)a->beta2; c.fresh2 = (float)(1.0 - a->beta2);
    c.root = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, (double)a->step)));
    c.size = (float)(a->lr / (1.0 - std::pow(a->beta1, (double)a->step)));
    c.eps = (float)a->eps;
    c.step = (uint32_t)a->step;
    c.seed = a->seed;
    c.moderate = c.eps >= 0x1p-60f && c.eps <= 0x1p30f && c.root <= 0x1p40f;
    return queue([&] {
      StepTensors t;
      int64_t state0 = 0;
      for (int i = 0; i < a->n_tensors;) {
        t.n = 0;
        t.chunk0[0] = 0;
        for (; i < a->n_tensors && t.n < TENSORS_PER_LAUNCH; ++i) {
          const int64_t n = a->numel[i];
          if (n == 0) continue;
          t.param[t.n] = a->params[i];
          t.grad[t.n] = a->grads[i];
          t.snapshot[t.n] = a->snapshot ? (uint16_t *)a->snapshot[i] : nullptr;
          t.numel[t.n] = n;
          t.state0[t.n] = state0;
          t.decay[t.n] = (float)(1.0 - a->lr * a->weight_decay[i]);
          t.chunk0[t.n + 1] = t.chunk0[t.n] + (uint32_t)((n + STEP_CHUNK - 1) / STEP_CHUNK);
          state0 += (n + ECHO_ADAMW_BLOCK - 1) / ECHO_ADAMW_BLOCK * ECHO_ADAMW_BLOCK;
          ++t.n;
        }
        if (t.n) launch_adamw(t, c, a->param_dtype, a->grad_dtype, a->state_dtype, (hipStream_t)stream);
      }
    });
  });
}

}  // extern "C"
