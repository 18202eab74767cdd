// Operators on rows of logits (include/echo_learner.h): log-probability of the given token with entropy and top entries, its
// gradient, and the policy loss with its gradient.
#include "echo_device.h"
#include "learner_kernels.h"
#include "../../include/echo_learner.h"

namespace echo {
namespace {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr int THREADS = 256, BATCH = 8;   // vectors of 16 bytes that a thread holds at a time
constexpr int CANDIDATES = 1024;

typedef uint32_t vec16 __attribute__((ext_vector_type(4)));

template <int DT> struct Elem { typedef uint16_t type; static constexpr int VEC = 8; };
template <> struct Elem<ECHO_F32> { typedef float type; static constexpr int VEC = 4; };

template <int DT> __device__ __forceinline__ float widen(typename Elem<DT>::type b) {
  if constexpr (DT == ECHO_F32) return b;
  else if constexpr (DT == ECHO_BF16) return bf16_bits_to_f32(b);
  else return h16_bits_to_f32(b);
}
template <int DT> __device__ __forceinline__ typename Elem<DT>::type narrow(float f) {
  if constexpr (DT == ECHO_F32) return f;
  else if constexpr (DT == ECHO_BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  else return __builtin_bit_cast(uint16_t, (_Float16)f);
}
// Element e of a vector.
template <int DT> __device__ __forceinline__ float element(const vec16 &q, int e) {
  if constexpr (DT == ECHO_F32) return __uint_as_float(q[e]);
  else if constexpr (DT == ECHO_BF16) return __uint_as_float(e % 2 ? q[e / 2] & 0xffff0000u : q[e / 2] << 16);
  else return h16_bits_to_f32((uint16_t)(e % 2 ? q[e / 2] >> 16 : q[e / 2]));
}
template <int DT> __device__ __forceinline__ vec16 pack(const float *v) {
  vec16 q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == ECHO_F32) q[i] = __float_as_uint(v[i]);
    else q[i] = (uint32_t)narrow<DT>(v[2 * i]) | (uint32_t)narrow<DT>(v[2 * i + 1]) << 16;
  }
  return q;
}
// The compiler would keep the widened elements of a vector from one use to the next, in twice its registers; after this it widens them again.
__device__ __forceinline__ void as_loaded(vec16 &q) { asm volatile("" : "+v"(q)); }
template <int DT> __device__ __forceinline__ vec16 filled(float f) {
  float v[8] = {f, f, f, f, f, f, f, f};
  return pack<DT>(v);
}

// Vectors of a row: rows of any stride start at any element, so these are loads and stores of 16 bytes at the elements' alignment.  A vector that
// passes the end is filled up with -inf, and stored element by element.
template <int DT> __device__ __forceinline__ vec16 load_vector(const typename Elem<DT>::type *x, int j, int end) {
  constexpr int VEC = Elem<DT>::VEC;
  vec16 q;
  if (j + VEC <= end) { __builtin_memcpy(&q, x + j, 16); return q; }
  q = filled<DT>(-INFINITY);
  if (j < end) {
    typename Elem<DT>::type e[VEC];
    __builtin_memcpy(e, &q, 16);
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (j + i < end) e[i] = x[j + i];
    __builtin_memcpy(&q, e, 16);
  }
  return q;
}
template <int DT> __device__ __forceinline__ void store_vector(typename Elem<DT>::type *x, int j, int end, const vec16 &q) {
  constexpr int VEC = Elem<DT>::VEC;
  if (j + VEC <= end) { __builtin_memcpy(x + j, &q, 16); return; }
  if (j < end) {
    typename Elem<DT>::type e[VEC];
    __builtin_memcpy(e, &q, 16);
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (j + i < end) x[j + i] = e[i];
  }
}

__device__ __forceinline__ bool row_live(const LogitRows &r, int64_t t) {
  return !r.targets || (uint32_t)r.targets[t] < (uint32_t)r.vocab;
}

// Order of the entries of a row: by logit, then by falling index; 0 is below every entry.
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_order_bits(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint64_t order_key(float x, int32_t j) { return (uint64_t)order_bits(x) << 32 | (uint32_t)~j; }
__device__ __forceinline__ int32_t key_index(uint64_t key) { return (int32_t)~(uint32_t)key; }
__device__ __forceinline__ float key_value(uint64_t key) { return from_order_bits((uint32_t)(key >> 32)); }

// Statistics of entries of a row with d_j = (x_j - top) c, c = log2(e) / T: the largest entry, sum = sum 2^d_j, turn = sum 2^d_j d_j.  The difference first: it is
// exact near the top, nought for the largest entry itself, and does not overflow where entries are ruled out by the lowest value of a type.
struct RowStats { float top, sum, turn; };

// The same relative to another top (>= s.top): a difference beyond 2^-200 leaves nothing.
__device__ __forceinline__ RowStats moved(const RowStats &s, float top, float c) {
  const float d = fmaxf((s.top - top) * c, -200.f), k = __builtin_amdgcn_exp2f(d);
  return s.top == top ? s : RowStats{top, s.sum * k, fmaf(d, s.sum, s.turn) * k};
}
__device__ __forceinline__ RowStats wave_stats(RowStats s, float c) {
  s = moved(s, wave_max(s.top), c);
  return {s.top, wave_sum(s.sum), wave_sum(s.turn)};
}
// Of a whole workgroup, in every thread.
template <int WAVES> __device__ __forceinline__ RowStats block_stats(RowStats s, float c, RowStats *sh) {
  s = wave_stats(s, c);
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = s;
  __syncthreads();
  s = sh[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) s.top = fmaxf(s.top, sh[i].top);
  s = moved(sh[0], s.top, c);
#pragma unroll
  for (int i = 1; i < WAVES; ++i) {
    const RowStats o = moved(sh[i], s.top, c);
    s.sum += o.sum; s.turn += o.turn;
  }
  return s;
}
// Log-sum, entropy and the log-probability of an entry; a row without weight has sum 0.
__device__ __forceinline__ float stats_lse(const RowStats &s, float inv_t) { return s.sum == 0.f ? -INFINITY : fmaf(s.top, inv_t, LN2 * log2f(s.sum)); }
__device__ __forceinline__ float stats_entropy(const RowStats &s) { return s.sum == 0.f ? 0.f : LN2 * (log2f(s.sum) - s.turn / s.sum); }
__device__ __forceinline__ float logprob(float x, const RowStats &s, float inv_t) {
  return x == -INFINITY && s.sum == s.sum ? -INFINITY : (x - s.top) * inv_t - LN2 * log2f(s.sum);
}

// Adds the entries of N vectors to a thread's statistics.
template <int DT, int N> __device__ __forceinline__ float largest(const vec16 *q, float *of_vector = nullptr) {
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < Elem<DT>::VEC; ++e) m = fmaxf(m, element<DT>(q[u], e));
    if (of_vector) of_vector[u] = m;
    top = fmaxf(top, m);
  }
  return top;
}
template <int DT, int N> __device__ __forceinline__ void add_entries(RowStats &s, vec16 *q, float top, float c) {
  s = moved(s, top, c);
  const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    as_loaded(q[u]);
#pragma unroll
    for (int e = 0; e < Elem<DT>::VEC; ++e) {
      const float d = (element<DT>(q[u], e) - from) * c, p = __builtin_amdgcn_exp2f(d);
      s.sum += p;
      s.turn = fmaf(p, fmaxf(d, -200.f), s.turn);
    }
  }
}

// A part of a row: its statistics, and the given entry's logit where it holds it.
struct RowPart { RowStats s; float given; };
struct Parts { RowPart *part; uint64_t *top; };   // [rows, splits], [rows, splits, top_k]

// The k largest of n <= CANDIDATES keys (different ones but for 0), in order, by their rank among all; what is left of out is 0.
__device__ __forceinline__ void select_top(const uint64_t *keys, int n, int k, uint64_t *out) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const uint64_t mine = keys[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += keys[j] > mine || (keys[j] == mine && j < i);
    if (rank < k) out[rank] = mine;
  }
  for (int i = n + threadIdx.x; i < k; i += THREADS) out[i] = 0;
}

template <int DT, bool TOP> __global__ __launch_bounds__(THREADS) void stats_kernel(LogitRows r, Parts p, int splits, int span, int top_k) {
  constexpr int VEC = Elem<DT>::VEC;
  __shared__ RowStats sh[THREADS / 64];
  const int64_t t = blockIdx.x / (uint32_t)splits;
  const int part = blockIdx.x % (uint32_t)splits;
  if (!row_live(r, t)) return;
  const auto *x = (const typename Elem<DT>::type *)r.x + t * r.stride;
  const float c = LOG2E / r.temperature;
  const int begin = part * span, end = min(r.vocab, begin + span);
  RowStats s = {-INFINITY, 0.f, 0.f};
  vec16 q[BATCH];
  float of_vector[BATCH];
#pragma unroll
  for (int u = 0; u < BATCH; ++u) of_vector[u] = -INFINITY;
  for (int j = begin + threadIdx.x * VEC; j - (int)threadIdx.x * VEC < end; j += THREADS * VEC * BATCH) {
#pragma unroll
    for (int u = 0; u < BATCH; ++u) q[u] = load_vector<DT>(x, j + u * THREADS * VEC, end);
    add_entries<DT, BATCH>(s, q, fmaxf(s.top, largest<DT, BATCH>(q, of_vector)), c);
  }
  const float mine = s.top;
  s = block_stats<THREADS / 64>(s, c, sh);
  if (threadIdx.x == 0) {
    const int given = r.targets ? r.targets[t] : -1;
    p.part[blockIdx.x] = {s, given >= begin && given < end ? widen<DT>(x[given]) : -INFINITY};
  }
  if constexpr (TOP) {   // (the part is one batch: it is still in q)
    __shared__ uint64_t keys[CANDIDATES];
    __shared__ uint32_t bound[THREADS / 64], count;
    uint64_t *out = p.top + (int64_t)blockIdx.x * top_k;
    // A value that at least top_k entries of a wave reach: its lanes' largest entries, cut to 16 bits, by bisection.
    const uint32_t key = order_bits(mine) >> 16;
    uint32_t low = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
      const uint32_t tried = low | 1u << b;
      if (__popcll(__ballot(key >= tried)) >= top_k) low = tried;
    }
    if (threadIdx.x % 64 == 0) bound[threadIdx.x / 64] = low;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) low = max(low, bound[i]);
    const uint32_t least = max(low << 16, order_bits(-INFINITY) + 1);
    const float floor = from_order_bits(least);
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      if (!(of_vector[u] >= floor)) continue;
      as_loaded(q[u]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = element<DT>(q[u], e);
        if (v >= floor) {
          const uint32_t at = atomicAdd(&count, 1u);
          if (at < CANDIDATES) keys[at] = order_key(v, begin + (u * THREADS + (int)threadIdx.x) * VEC + e);
        }
      }
    }
    __syncthreads();
    if (count <= CANDIDATES) return select_top(keys, count, top_k, out);
    // Too many equal ones: one entry after the other, each the largest below the last.
    uint64_t last = ~0ull;
    for (int k = 0; k < top_k; ++k) {
      uint64_t best = 0;
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        as_loaded(q[u]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float v = element<DT>(q[u], e);
          const uint64_t key = order_key(v, begin + (u * THREADS + (int)threadIdx.x) * VEC + e);
          if (v >= floor && key < last && key > best) best = key;
        }
      }
      for (int o = 32; o > 0; o >>= 1) { const uint64_t b = __shfl_xor(best, o, 64); best = b > best ? b : best; }
      __syncthreads();
      if (threadIdx.x % 64 == 0) keys[threadIdx.x / 64] = best;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < THREADS / 64; ++i) best = max(best, keys[i]);
      if (threadIdx.x == 0) out[k] = best;
      last = best;
    }
  }
}

// The parts of a row put together, by the first wave of a workgroup.
__device__ __forceinline__ RowPart joined(const RowPart *part, int splits, float c) {
  RowPart m = {{-INFINITY, 0.f, 0.f}, -INFINITY};
  for (int i = threadIdx.x % 64; i < splits; i += 64) {
    const RowPart o = part[i];
    const float top = fmaxf(m.s.top, o.s.top);
    m.s = moved(m.s, top, c);
    const RowStats n = moved(o.s, top, c);
    m.s.sum += n.sum; m.s.turn += n.turn;
    m.given = fmaxf(m.given, o.given);
  }
  return {wave_stats(m.s, c), wave_max(m.given)};
}

template <bool TOP> __global__ __launch_bounds__(THREADS) void stats_finish_kernel(LogitRows r, Parts p, int splits, RowOutputs out) {
  const int64_t t = blockIdx.x;
  const float inv_t = 1.0f / r.temperature;
  const bool live = row_live(r, t);
  __shared__ RowStats all;
  if (threadIdx.x < 64) {
    RowPart m = {{0.f, 0.f, 0.f}, 0.f};
    if (live) m = joined(p.part + t * splits, splits, LOG2E / r.temperature);
    if (threadIdx.x == 0) {
      if (out.logprobs) out.logprobs[t] = live ? logprob(m.given, m.s, inv_t) : 0.f;
      if (out.entropy) out.entropy[t] = live ? stats_entropy(m.s) : 0.f;
      if (out.lse) out.lse[t] = live ? stats_lse(m.s, inv_t) : 0.f;
      all = m.s;
    }
  }
  if constexpr (TOP) {
    // The parts' lists, as many at a time as fit: of the best so far and of the new ones only those count that reach the last of a list, since that many
    // entries are as large as it is.
    __shared__ uint64_t keys[CANDIDATES], best[ECHO_TOP_MAX], bound;
    __shared__ uint32_t count;
    const int k = out.top_k, n = splits * k, at_once = (CANDIDATES / k - 1) * k;
    const uint64_t *lists = p.top + t * n;
    if (threadIdx.x == 0) { bound = 1; count = 0; }
    __syncthreads();
    for (int done = 0; live && done < n; done += at_once) {
      const int more = min(n - done, at_once);
      for (int i = threadIdx.x; i < more / k; i += THREADS) atomicMax((unsigned long long *)&bound, lists[done + i * k + k - 1]);
      __syncthreads();
      const uint64_t least = bound;
      for (int i = threadIdx.x; i < more; i += THREADS) {
        const uint64_t key = lists[done + i];
        if (key >= least) keys[atomicAdd(&count, 1u)] = key;
      }
      if (done && threadIdx.x < k && best[threadIdx.x] >= least) keys[atomicAdd(&count, 1u)] = best[threadIdx.x];
      __syncthreads();
      select_top(keys, count, k, best);
      __syncthreads();
      if (threadIdx.x == 0) { bound = max(best[k - 1], (uint64_t)1); count = 0; }
      __syncthreads();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < k; i += THREADS) {
      const uint64_t key = live ? best[i] : 0;
      out.top_ids[t * k + i] = key ? key_index(key) : -1;
      out.top_logprobs[t * k + i] = !live ? 0.f : key ? logprob(key_value(key), all, inv_t) : -INFINITY;
    }
  }
}

// Gradient of a row: with d_j = (x_j scale - from) unit and p_j a factor (in a and b) times 2^d_j, out_j = 2^d_j (a + b d_j), at_target more at the
// target.
struct RowGrad { float scale, from, unit, a, b, at_target; };
// Coefficients for d/dlogprob = g and d/dentropy = h, where p_j = k 2^d_j and ln p_j = ln 2 d_j - lo.
__device__ __forceinline__ RowGrad row_grad(float scale, float from, float unit, float k, float lo, float g, float h, float H, float inv_t) {
  return {scale, from, unit, -k * inv_t * (g + h * (H - lo)), -k * inv_t * h * LN2, g * inv_t};
}
template <int DT> __device__ __forceinline__ vec16 grad_vector(const vec16 &q, int from_target, const RowGrad &c) {
  constexpr int VEC = Elem<DT>::VEC;
  float v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const float d = fmaf(element<DT>(q, e), c.scale, -c.from) * c.unit;
    v[e] = __builtin_amdgcn_exp2f(d) * fmaf(c.b, fmaxf(d, -200.f), c.a);
  }
  if ((uint32_t)from_target < (uint32_t)VEC) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e == from_target) v[e] += c.at_target;
  }
  return pack<DT>(v);
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
__device__ __forceinline__ bool token_live(const LogitRows &r, const PolicyTerms &p, int64_t t) {
  return row_live(r, t) && (!p.weights || p.weights[t] != 0.f);
}

struct LossOutputs { float *loss, *logprobs, *entropy; void *grad; int64_t stride; };

// Loss of a row from its statistics; its outputs by the thread that `writes`.
__device__ __forceinline__ RowGrad finish_loss(const LogitRows &r, const PolicyTerms &p, const LossOutputs &out, int64_t t, const RowStats &s, float given, bool writes) {
  const float inv_t = 1.0f / r.temperature, H = stats_entropy(s);
  const TokenLoss l = token_loss(p, t, logprob(given, s, inv_t), H);
  if (writes) {
    if (out.loss) out.loss[t] = l.loss;
    if (out.logprobs) out.logprobs[t] = l.logprob;
    if (out.entropy) out.entropy[t] = H;
  }
  if (s.sum == 0.f) return {1.f, 0.f, 1.f, 0.f, 0.f, 0.f};   // without weight anywhere: entries of -inf
  return row_grad(1.f, s.top, LOG2E / r.temperature, 1.0f / s.sum, LN2 * log2f(s.sum), l.g, l.h, H, inv_t);
}
__device__ __forceinline__ void no_loss(const LossOutputs &out, int64_t t) {
  if (out.loss) out.loss[t] = 0.f;
  if (out.logprobs) out.logprobs[t] = 0.f;
  if (out.entropy) out.entropy[t] = 0.f;
}

struct GivenStats { const float *lse, *entropy, *g, *h; };   // g, h nullable

// One batch of a row's gradient: from given statistics (LOSS false), or from the parts of stats_kernel, which every workgroup of a row joins while its
// vectors are on their way.
template <int DT, bool LOSS> __global__ __launch_bounds__(THREADS) void grad_kernel(LogitRows r, GivenStats given, PolicyTerms terms, Parts p, int splits, LossOutputs out,
                                                                                 int batches) {
  constexpr int VEC = Elem<DT>::VEC;
  const int64_t t = blockIdx.x / (uint32_t)batches;
  const int j = (int)(blockIdx.x % (uint32_t)batches) * THREADS * VEC * BATCH + threadIdx.x * VEC;
  const bool first = blockIdx.x % (uint32_t)batches == 0;
  const auto *x = (const typename Elem<DT>::type *)r.x + t * r.stride;
  auto *o = (typename Elem<DT>::type *)out.grad + t * out.stride;
  bool live;
  if constexpr (LOSS) live = token_live(r, terms, t); else live = row_live(r, t) && given.lse[t] != -INFINITY;
  if (!live) {
    if (LOSS && first && threadIdx.x == 0) no_loss(out, t);
#pragma unroll
    for (int u = 0; u < BATCH; ++u) store_vector<DT>(o, j + u * THREADS * VEC, r.vocab, vec16{0, 0, 0, 0});
    return;
  }
  vec16 q[BATCH];
#pragma unroll
  for (int u = 0; u < BATCH; ++u) q[u] = load_vector<DT>(x, j + u * THREADS * VEC, r.vocab);
  RowGrad c;
  int target = -1;
  if constexpr (LOSS) {
    __shared__ RowGrad sh;
    if (threadIdx.x < 64) {
      const RowPart m = joined(p.part + t * splits, splits, LOG2E / r.temperature);
      const RowGrad mine = finish_loss(r, terms, out, t, m.s, m.given, first && threadIdx.x == 0);
      if (threadIdx.x == 0) sh = mine;
    }
    __syncthreads();
    c = sh;
    target = r.targets[t];
  } else {
    const float inv_t = 1.0f / r.temperature, h = given.h ? given.h[t] : 0.f;
    c = row_grad(inv_t, given.lse[t], LOG2E, 1.f, 0.f, given.g ? given.g[t] : 0.f, h, given.h ? given.entropy[t] : 0.f, inv_t);
    if (given.g) target = r.targets[t];
  }
#pragma unroll
  for (int u = 0; u < BATCH; ++u) {
    const int at = j + u * THREADS * VEC;
    store_vector<DT>(o, at, r.vocab, grad_vector<DT>(q[u], target - at, c));
  }
}

// A whole row by one workgroup: its first N vectors a thread stay in registers between the statistics and the gradient, what is beyond them is read
// again.
template <int DT, int W, int N> __global__ __launch_bounds__(W) void loss_row_kernel(LogitRows r, PolicyTerms terms, LossOutputs out) {
  constexpr int VEC = Elem<DT>::VEC, AGAIN = 4;
  __shared__ RowStats sh[W / 64];
  const int64_t t = blockIdx.x;
  const auto *x = (const typename Elem<DT>::type *)r.x + t * r.stride;
  auto *o = (typename Elem<DT>::type *)out.grad + t * out.stride;
  const int mine = threadIdx.x * VEC;
  if (!token_live(r, terms, t)) {
    if (threadIdx.x == 0) no_loss(out, t);
    for (int j = mine; j < r.vocab; j += W * VEC) store_vector<DT>(o, j, r.vocab, vec16{0, 0, 0, 0});
    return;
  }
  const float c = LOG2E / r.temperature;
  const int target = r.targets[t];
  const float given = widen<DT>(x[target]);
  vec16 q[N];
#pragma unroll
  for (int u = 0; u < N; ++u) q[u] = load_vector<DT>(x, mine + u * W * VEC, r.vocab);
  RowStats s = {-INFINITY, 0.f, 0.f};
  for (int j = N * W * VEC; j < r.vocab; j += AGAIN * W * VEC) {
    vec16 a[AGAIN];
#pragma unroll
    for (int u = 0; u < AGAIN; ++u) a[u] = load_vector<DT>(x, j + mine + u * W * VEC, r.vocab);
    add_entries<DT, AGAIN>(s, a, fmaxf(s.top, largest<DT, AGAIN>(a)), c);
  }
  add_entries<DT, N>(s, q, fmaxf(s.top, largest<DT, N>(q)), c);
  s = block_stats<W / 64>(s, c, sh);   // (its barrier: the target's logit has been read before any gradient is written)
  const RowGrad g = finish_loss(r, terms, out, t, s, given, threadIdx.x == 0);
  for (int j = N * W * VEC; j < r.vocab; j += AGAIN * W * VEC) {
    vec16 a[AGAIN];
#pragma unroll
    for (int u = 0; u < AGAIN; ++u) a[u] = load_vector<DT>(x, j + mine + u * W * VEC, r.vocab);
#pragma unroll
    for (int u = 0; u < AGAIN; ++u) {
      const int at = j + mine + u * W * VEC;
      store_vector<DT>(o, at, r.vocab, grad_vector<DT>(a[u], target - at, g));
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int at = mine + u * W * VEC;
    as_loaded(q[u]);
    store_vector<DT>(o, at, r.vocab, grad_vector<DT>(q[u], target - at, g));
  }
}

// The loss alone.
__global__ __launch_bounds__(64) void loss_finish_kernel(LogitRows r, PolicyTerms terms, Parts p, int splits, LossOutputs out) {
  const int64_t t = blockIdx.x;
  if (!token_live(r, terms, t)) {
    if (threadIdx.x == 0) no_loss(out, t);
    return;
  }
  const RowPart m = joined(p.part + t * splits, splits, LOG2E / r.temperature);
  finish_loss(r, terms, out, t, m.s, m.given, threadIdx.x == 0);
}

// Parts of a row: one batch each where the top entries are wanted, a few batches otherwise.
struct Split { int splits, span; };
Split split_of(const LogitRows &x, bool top) {
  const int vec = x.dtype == ECHO_F32 ? 4 : 8, batch = THREADS * vec * BATCH;
  const int whole = batch * (top ? 1 : 4);
  const int splits = (x.vocab + whole - 1) / whole;
  const int span = ((x.vocab + splits - 1) / splits + vec - 1) / vec * vec;   // (at most `whole`)
  return {splits, span};
}
size_t parts_bytes(const LogitRows &x, const Split &s) { return ((size_t)x.rows * s.splits * sizeof(RowPart) + 255) / 256 * 256; }

}  // namespace

size_t logprobs_workspace(const LogitRows &x, int top_k) {
  const Split s = split_of(x, top_k > 0);
  return parts_bytes(x, s) + (size_t)x.rows * s.splits * top_k * sizeof(uint64_t);
}
size_t policy_workspace(const LogitRows &x) { return parts_bytes(x, split_of(x, false)); }

#define FOR_DTYPE(dt, CALL)                                    \
  do {                                                         \
    if ((dt) == ECHO_F32) { constexpr int DT = ECHO_F32; CALL; } \
    else if ((dt) == ECHO_BF16) { constexpr int DT = ECHO_BF16; CALL; } \
    else { constexpr int DT = ECHO_F16; CALL; }                \
  } while (0)

void launch_token_logprobs(const LogitRows &x, const RowOutputs &out, void *workspace, hipStream_t st) {
  const Split s = split_of(x, out.top_k > 0);
  const Parts p = {(RowPart *)workspace, (uint64_t *)((char *)workspace + parts_bytes(x, s))};
  const dim3 grid((uint32_t)(x.rows * s.splits));
  if (out.top_k > 0) {
    FOR_DTYPE(x.dtype, (stats_kernel<DT, true><<<grid, THREADS, 0, st>>>(x, p, s.splits, s.span, out.top_k)));
    stats_finish_kernel<true><<<dim3((uint32_t)x.rows), THREADS, 0, st>>>(x, p, s.splits, out);
  } else {
    FOR_DTYPE(x.dtype, (stats_kernel<DT, false><<<grid, THREADS, 0, st>>>(x, p, s.splits, s.span, 0)));
    stats_finish_kernel<false><<<dim3((uint32_t)x.rows), 64, 0, st>>>(x, p, s.splits, out);
  }
}
static int grad_batches(const LogitRows &x) {
  const int batch = THREADS * (x.dtype == ECHO_F32 ? 4 : 8) * BATCH;
  return (x.vocab + batch - 1) / batch;
}
void launch_token_logprobs_grad(const LogitRows &x, const float *lse, const float *entropy, const float *g, const float *h, void *out, int64_t out_stride,
                                hipStream_t st) {
  const int batches = grad_batches(x);
  const LossOutputs o = {nullptr, nullptr, nullptr, out, out_stride};
  FOR_DTYPE(x.dtype, (grad_kernel<DT, false><<<dim3((uint32_t)(x.rows * batches)), THREADS, 0, st>>>(x, GivenStats{lse, entropy, g, h}, PolicyTerms{}, Parts{}, 0, o, batches)));
}
void launch_policy_loss(const LogitRows &x, const PolicyTerms &terms, float *loss, float *logprobs, float *entropy, void *grad, int64_t grad_stride, void *workspace,
                        hipStream_t st) {
  const Split s = split_of(x, false);
  const Parts p = {(RowPart *)workspace, nullptr};
  const LossOutputs o = {loss, logprobs, entropy, grad, grad_stride};
  if (grad && x.rows >= 200) {
    FOR_DTYPE(x.dtype, (loss_row_kernel<DT, 1024, DT == ECHO_F32 ? 17 : 19><<<dim3((uint32_t)x.rows), 1024, 0, st>>>(x, terms, o)));
    return;
  }
  FOR_DTYPE(x.dtype, (stats_kernel<DT, false><<<dim3((uint32_t)(x.rows * s.splits)), THREADS, 0, st>>>(x, p, s.splits, s.span, 0)));
  if (!grad) {
    loss_finish_kernel<<<dim3((uint32_t)x.rows), 64, 0, st>>>(x, terms, p, s.splits, o);
    return;
  }
  const int batches = grad_batches(x);
  FOR_DTYPE(x.dtype, (grad_kernel<DT, true><<<dim3((uint32_t)(x.rows * batches)), THREADS, 0, st>>>(x, GivenStats{}, terms, p, s.splits, o, batches)));
}

}  // namespace echo
