// Operators on rows of logits (include/echo_learner.h): log-probability of the given token with entropy and top entries, its
// gradient, and the policy loss with its gradient.
#include "echo_device.h"
#include "learner_kernels.h"
#include "../../include/echo_learner.h"

namespace echo {
namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr int THREADS = 256;

template <int DT> struct Elem;
template <> struct Elem<ECHO_F32> { typedef float type; };
template <> struct Elem<ECHO_BF16> { typedef uint16_t type; };
template <> struct Elem<ECHO_F16> { typedef _Float16 type; };

template <int DT> __device__ __forceinline__ float get(const void *p, int64_t i) {
  if (DT == ECHO_BF16) return bf16_bits_to_f32(((const uint16_t *)p)[i]);
  return (float)((const typename Elem<DT>::type *)p)[i];
}
template <int DT> __device__ __forceinline__ void put(void *p, int64_t i, float f) {
  if (DT == ECHO_BF16) ((uint16_t *)p)[i] = f32_to_bf16_bits(f);
  else ((typename Elem<DT>::type *)p)[i] = (typename Elem<DT>::type)f;
}

__device__ __forceinline__ bool row_live(const LogitRows &r, int64_t t) {
  return !r.targets || (uint32_t)r.targets[t] < (uint32_t)r.vocab;
}

__device__ float block_max(float v, float *sh) {
  v = wave_max(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < THREADS / 64; ++i) v = fmaxf(v, sh[i]);
  return v;
}
__device__ float block_sum(float v, float *sh) {
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < THREADS / 64; ++i) v += sh[i];
  return v;
}

// Order of the entries of a row: by logit, then by falling index; 0 is below every entry.
__device__ __forceinline__ uint64_t order_key(float x, int32_t j) {
  const uint32_t b = __float_as_uint(x + 0.0f), k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)k << 32 | (uint32_t)~j;
}

// Statistics of entries of a row with d_j = (x_j - top) c, c = log2(e) / T: the largest entry, sum = sum 2^d_j, turn = sum 2^d_j d_j.  The difference first: it is
// exact near the top, nought for the largest entry itself, and does not overflow where entries are ruled out by the lowest value of a type.
struct RowStats { float top, sum, turn; };
template <int DT> __device__ RowStats row_stats(const void *x, int vocab, float c, float *sh) {
  float top = -INFINITY;
  for (int j = threadIdx.x; j < vocab; j += THREADS) top = fmaxf(top, get<DT>(x, j));
  top = block_max(top, sh);
  const float safe = top == -INFINITY ? 0.f : top;
  float sum = 0.f, turn = 0.f;
  for (int j = threadIdx.x; j < vocab; j += THREADS) {
    const float d = (get<DT>(x, j) - safe) * c, e = exp2f(d);
    sum += e;
    turn = fmaf(e, fmaxf(d, -200.f), turn);
  }
  sum = block_sum(sum, sh);
  return {top, sum, block_sum(turn, sh)};
}
// Log-sum, entropy and the log-probability of an entry; a row without weight has sum 0.
__device__ __forceinline__ float stats_lse(const RowStats &s, float inv_t) { return s.sum == 0.f ? -INFINITY : fmaf(s.top, inv_t, LN2 * log2f(s.sum)); }
__device__ __forceinline__ float stats_entropy(const RowStats &s) { return s.sum == 0.f ? 0.f : LN2 * (log2f(s.sum) - s.turn / s.sum); }
__device__ __forceinline__ float logprob(float x, const RowStats &s, float inv_t) {
  return x == -INFINITY && s.sum == s.sum ? -INFINITY : (x - s.top) * inv_t - LN2 * log2f(s.sum);
}

template <int DT> __global__ __launch_bounds__(THREADS) void logprobs_kernel(LogitRows r, RowOutputs out) {
  __shared__ float sh[THREADS / 64];
  __shared__ uint64_t shk[THREADS / 64];
  const int64_t t = blockIdx.x;
  if (!row_live(r, t)) {
    if (threadIdx.x == 0) {
      if (out.logprobs) out.logprobs[t] = 0.f;
      if (out.entropy) out.entropy[t] = 0.f;
      if (out.lse) out.lse[t] = 0.f;
    }
    for (int k = threadIdx.x; k < out.top_k; k += THREADS) { out.top_ids[t * out.top_k + k] = -1; out.top_logprobs[t * out.top_k + k] = 0.f; }
    return;
  }
  const auto *x = (const typename Elem<DT>::type *)r.x + t * r.stride;
  const float inv_t = 1.0f / r.temperature;
  const RowStats s = row_stats<DT>(x, r.vocab, LOG2E / r.temperature, sh);
  if (threadIdx.x == 0) {
    if (out.logprobs) out.logprobs[t] = logprob(get<DT>(x, r.targets[t]), s, inv_t);
    if (out.entropy) out.entropy[t] = stats_entropy(s);
    if (out.lse) out.lse[t] = stats_lse(s, inv_t);
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < out.top_k; ++k) {   // the largest key below the last one
    uint64_t best = 0;
    for (int j = threadIdx.x; j < r.vocab; j += THREADS) {
      const float v = get<DT>(x, j);
      const uint64_t key = v == -INFINITY ? 0 : order_key(v, j);
      if (key < last && key > best) best = key;
    }
    for (int o = 32; o > 0; o >>= 1) { const uint64_t b = __shfl_xor(best, o, 64); best = b > best ? b : best; }
    __syncthreads();
    if (threadIdx.x % 64 == 0) shk[threadIdx.x / 64] = best;
    __syncthreads();
    for (int i = 0; i < THREADS / 64; ++i) best = shk[i] > best ? shk[i] : best;
    last = best;
    if (threadIdx.x == 0) {
      const int32_t id = best ? (int32_t)~(uint32_t)best : -1;
      out.top_ids[t * out.top_k + k] = id;
      out.top_logprobs[t * out.top_k + k] = id < 0 ? -INFINITY : logprob(get<DT>(x, id), s, inv_t);
    }
  }
}

// Gradient of a row: with d_j = (x_j scale - from) unit and p_j a factor (in a and b) times 2^d_j, out_j = 2^d_j (a + b d_j), at_target more at the
// target.
struct RowGrad { float scale, from, unit, a, b, at_target; };
template <int DT> __device__ void write_grad(const void *x, void *out, int vocab, int target, const RowGrad &q) {
  for (int j = threadIdx.x; j < vocab; j += THREADS) {
    const float d = fmaf(get<DT>(x, j), q.scale, -q.from) * q.unit;
    float v = exp2f(d) * fmaf(q.b, fmaxf(d, -200.f), q.a);
    if (j == target) v += q.at_target;
    put<DT>(out, j, v);
  }
}
// Coefficients for d/dlogprob = g and d/dentropy = h, where p_j = k 2^d_j and ln p_j = ln 2 d_j - lo.
__device__ __forceinline__ RowGrad row_grad(float scale, float from, float unit, float k, float lo, float g, float h, float H, float inv_t) {
  return {scale, from, unit, -k * inv_t * (g + h * (H - lo)), -k * inv_t * h * LN2, g * inv_t};
}
template <int DT> __device__ void write_zeros(void *out, int vocab) {
  for (int j = threadIdx.x; j < vocab; j += THREADS) put<DT>(out, j, 0.f);
}

template <int DT> __global__ __launch_bounds__(THREADS) void logprobs_grad_kernel(LogitRows r, const float *lse, const float *entropy, const float *g, const float *h,
                                                                               void *out, int64_t out_stride) {
  const int64_t t = blockIdx.x;
  auto *o = (typename Elem<DT>::type *)out + t * out_stride;
  if (!row_live(r, t) || lse[t] == -INFINITY) return write_zeros<DT>(o, r.vocab);
  const float inv_t = 1.0f / r.temperature, gt = g ? g[t] : 0.f, ht = h ? h[t] : 0.f, H = h ? entropy[t] : 0.f;
  write_grad<DT>((const typename Elem<DT>::type *)r.x + t * r.stride, o, r.vocab, g ? r.targets[t] : -1,
                 row_grad(inv_t, lse[t], LOG2E, 1.f, 0.f, gt, ht, H, inv_t));
}

struct TokenLoss { float loss, logprob, g, h; };
__device__ TokenLoss token_loss(const PolicyTerms &p, int64_t t, float lp, float H) {
  const float w = p.weights ? p.weights[t] : 1.f, A = p.advantages[t], old = p.old_logprobs[t];
  const float ratio = expf(lp - old), trust = p.sampler ? fminf(expf(old - p.sampler[t]), p.sampler_cap) : 1.f;
  const float free = fminf(ratio, p.ratio_cap) * A, held = fminf(fmaxf(ratio, p.lo), p.hi) * A;
  float kl = 0.f, kl_slope = 0.f;
  if (p.kl != 0.f) {
    const float off = p.ref[t] - lp, e = expm1f(off);
    kl = p.kl * (e - off);
    kl_slope = -p.kl * e;
  }
  const float slope = free <= held && ratio < p.ratio_cap ? A * ratio : 0.f;
  return {w * (-trust * fminf(free, held) + kl - p.entropy * H), lp, w * (kl_slope - trust * slope), -p.entropy * w};
}

template <int DT> __global__ __launch_bounds__(THREADS) void policy_kernel(LogitRows r, PolicyTerms p, float *loss, float *logprobs, float *entropy, void *grad,
                                                                        int64_t grad_stride) {
  __shared__ float sh[THREADS / 64];
  const int64_t t = blockIdx.x;
  const bool live = row_live(r, t) && (!p.weights || p.weights[t] != 0.f);
  RowStats s = {0.f, 0.f, 0.f};
  TokenLoss l = {0.f, 0.f, 0.f, 0.f};
  float H = 0.f;
  const auto *x = (const typename Elem<DT>::type *)r.x + t * r.stride;
  const float inv_t = 1.0f / r.temperature, c = LOG2E / r.temperature;
  if (live) {
    s = row_stats<DT>(x, r.vocab, c, sh);
    H = stats_entropy(s);
    l = token_loss(p, t, logprob(get<DT>(x, r.targets[t]), s, inv_t), H);
  }
  if (threadIdx.x == 0) {
    if (loss) loss[t] = l.loss;
    if (logprobs) logprobs[t] = l.logprob;
    if (entropy) entropy[t] = H;
  }
  if (!grad) return;
  auto *o = (typename Elem<DT>::type *)grad + t * grad_stride;
  if (!live || s.sum == 0.f) return write_zeros<DT>(o, r.vocab);
  write_grad<DT>(x, o, r.vocab, r.targets[t], row_grad(1.f, s.top, c, 1.0f / s.sum, LN2 * log2f(s.sum), l.g, l.h, H, inv_t));
}

}  // namespace

size_t logprobs_workspace(const LogitRows &, int) { return 0; }
size_t policy_workspace(const LogitRows &) { return 0; }

#define FOR_DTYPE(dt, CALL)                                    \
  do {                                                         \
    if ((dt) == ECHO_F32) { constexpr int DT = ECHO_F32; CALL; } \
    else if ((dt) == ECHO_BF16) { constexpr int DT = ECHO_BF16; CALL; } \
    else { constexpr int DT = ECHO_F16; CALL; }                \
  } while (0)

void launch_token_logprobs(const LogitRows &x, const RowOutputs &out, void *, hipStream_t st) {
  FOR_DTYPE(x.dtype, (logprobs_kernel<DT><<<dim3((uint32_t)x.rows), THREADS, 0, st>>>(x, out)));
}
void launch_token_logprobs_grad(const LogitRows &x, const float *lse, const float *entropy, const float *g, const float *h, void *out, int64_t out_stride,
                                hipStream_t st) {
  FOR_DTYPE(x.dtype, (logprobs_grad_kernel<DT><<<dim3((uint32_t)x.rows), THREADS, 0, st>>>(x, lse, entropy, g, h, out, out_stride)));
}
void launch_policy_loss(const LogitRows &x, const PolicyTerms &p, float *loss, float *logprobs, float *entropy, void *grad, int64_t grad_stride, void *,
                        hipStream_t st) {
  FOR_DTYPE(x.dtype, (policy_kernel<DT><<<dim3((uint32_t)x.rows), THREADS, 0, st>>>(x, p, loss, logprobs, entropy, grad, grad_stride)));
}

}  // namespace echo
