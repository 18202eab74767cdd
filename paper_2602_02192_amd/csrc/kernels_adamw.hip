// The update (include/echo_learner.h): norm of many gradients, one AdamW step over many tensors.
#include "echo_device.h"
#include "learner_kernels.h"
#include "../../include/echo_learner.h"

namespace echo {
namespace {

constexpr int THREADS = 256;

// The tensor that holds a workgroup's chunk.
__device__ __forceinline__ int tensor_of(const uint32_t *chunk0, int n, uint32_t chunk) {
  int lo = 0, hi = n;                    // chunk0[lo] <= chunk < chunk0[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (chunk0[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

template <int DT> __device__ __forceinline__ float get(const void *p, int64_t i) {
  if (DT == ECHO_BF16) return bf16_bits_to_f32(((const uint16_t *)p)[i]);
  if (DT == ECHO_F16) return (float)((const _Float16 *)p)[i];
  return ((const float *)p)[i];
}

__device__ double block_sum(double v, double *sh) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < THREADS / 64; ++i) v += sh[i];
  return v;
}

template <int DT> __global__ __launch_bounds__(THREADS) void norm_kernel(NormTensors t, double *partial) {
  __shared__ double sh[THREADS / 64];
  const int i = tensor_of(t.chunk0, t.n, blockIdx.x);
  const int64_t a = (int64_t)(blockIdx.x - t.chunk0[i]) * NORM_CHUNK, left = t.numel[i] - a, n = left < NORM_CHUNK ? left : NORM_CHUNK;
  double s = 0;
  for (int64_t j = threadIdx.x; j < n; j += THREADS) {
    const double g = get<DT>(t.grad[i], a + j);
    s = fma(g, g, s);
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(THREADS) void norm_finish_kernel(const double *partial, int64_t n, float *out) {
  __shared__ double sh[THREADS / 64];
  double s = 0;
  for (int64_t j = threadIdx.x; j < n; j += THREADS) s += partial[j];
  s = block_sum(s, sh);
  if (threadIdx.x == 0) *out = (float)sqrt(s);
}

// Magnitude and sign bits of an E4M3 code as f32 (codes 0x7f and 0xff are NaN).
__device__ __forceinline__ float e4m3_value(uint32_t code) {
  const uint32_t m = code & 0x7f;
  const float f = m == 0x7f ? NAN : m >= 8 ? __uint_as_float((m + (120u << 3)) << 20) : (float)m * 0x1p-9f;
  return code & 0x80 ? -f : f;
}

// z in [0, 448] (a rounding above at most, or NaN) to the code below or above it, by 16 random bits: in f32 the three significand bits that stay end at
// bit 20, so adding the random bits below them and cutting carries with the right probability; below 2^-6 codes are multiples of 2^-9.
__device__ __forceinline__ uint32_t e4m3_code(float z, uint32_t bits) {
  if (z != z) return 0x7f;
  z = fminf(z, 448.0f);
  uint32_t code;
  if (z < 0x1p-6f) code = (uint32_t)floorf(z * 512.0f + (float)bits * 0x1p-16f);
  else code = ((__float_as_uint(z) + (bits << 4)) >> 20) - (120u << 3);
  return code < 0x7eu ? code : 0x7eu;
}

// A bf16 next to f, by 16 random bits; infinities and NaN stay what they are.
__device__ __forceinline__ uint16_t bf16_by_chance(float f, uint32_t bits) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7f800000u) == 0x7f800000u) return f32_to_bf16_bits(f);
  return (uint16_t)((u + bits) >> 16);
}

// Scale of a block whose largest magnitude is `top`, and its reciprocal (0 for a block without weight).
__device__ __forceinline__ float block_scale(float top, float &inv) {
#pragma clang fp contract(off)
  const float scale = top < 0x1p-100f ? 0.f : top * (1.0f / 448.0f);
  inv = scale > 0.f ? 1.0f / scale : scale;
  return scale;
}

// A wave takes 256 consecutive elements, a lane four of them: one call of the generator, one block of the 8-bit states.
template <int PT, int GT, int ST> __global__ __launch_bounds__(THREADS) void adamw_kernel(StepTensors t, StepConstants c) {
#pragma clang fp contract(off)
  float factor = 1.0f;
  if (c.norm) {
    const float norm = *c.norm;
    if (!(fabsf(norm) < INFINITY)) return;
    if (norm > c.max_norm) factor = c.max_norm / norm;
  }
  const int i = tensor_of(t.chunk0, t.n, blockIdx.x);
  const int64_t n = t.numel[i], a = (int64_t)(blockIdx.x - t.chunk0[i]) * STEP_CHUNK, s0 = t.state0[i];
  const float decay = t.decay[i];
  for (int64_t b = a + threadIdx.x * 4; b < a + STEP_CHUNK; b += THREADS * 4) {
    if (b - threadIdx.x % 64 * 4 >= n) break;   // (whole waves)
    const int64_t s = s0 + b;
    float m[4], v[4];
    if (ST == ECHO_F32) {
      const f32x4 m4 = *(const f32x4 *)((const float *)c.m + s), v4 = *(const f32x4 *)((const float *)c.v + s);
      for (int k = 0; k < 4; ++k) { m[k] = m4[k]; v[k] = v4[k]; }
    } else {
      const uint32_t m4 = *(const uint32_t *)((const uint8_t *)c.m + s), v4 = *(const uint32_t *)((const uint8_t *)c.v + s);
      const float ms = c.m_scale[s / ECHO_ADAMW_BLOCK], vs = c.v_scale[s / ECHO_ADAMW_BLOCK];
      for (int k = 0; k < 4; ++k) { m[k] = e4m3_value(m4 >> 8 * k & 0xff) * ms; v[k] = e4m3_value(v4 >> 8 * k & 0xff) * vs; }
    }
    u32x4 by_chance = {0, 0, 0, 0};
    if (PT == ECHO_BF16) by_chance = philox4x32_10((uint32_t)(s >> 2), (uint32_t)(s >> 34), c.step, 1, (uint32_t)c.seed, (uint32_t)(c.seed >> 32));
    const uint32_t rp[4] = {by_chance.x, by_chance.y, by_chance.z, by_chance.w};
    for (int k = 0; k < 4; ++k) {
      const bool in = b + k < n;
      if (!in) { m[k] = 0.f; v[k] = 0.f; continue; }
      const float g = get<GT>(t.grad[i], b + k) * factor;
      m[k] = m[k] * c.beta1 + g * c.fresh1;
      v[k] = v[k] * c.beta2 + g * c.fresh2 * g;
      const float p = get<PT>(t.param[i], b + k) * decay - m[k] / (sqrtf(v[k]) * c.root + c.eps) * c.size;
      if (PT == ECHO_F32) ((float *)t.param[i])[b + k] = p;
      else ((uint16_t *)t.param[i])[b + k] = bf16_by_chance(p, rp[k] & 0xffff);
      if (PT == ECHO_F32 && t.snapshot[i]) t.snapshot[i][b + k] = f32_to_bf16_bits(p);
    }
    if (ST == ECHO_F32) {
      *(f32x4 *)((float *)c.m + s) = f32x4{m[0], m[1], m[2], m[3]};
      *(f32x4 *)((float *)c.v + s) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      const u32x4 r = philox4x32_10((uint32_t)(s >> 2), (uint32_t)(s >> 34), c.step, 0, (uint32_t)c.seed, (uint32_t)(c.seed >> 32));
      const uint32_t rs[4] = {r.x, r.y, r.z, r.w};
      float mi, vi;
      const float ms = block_scale(wave_max(fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])))), mi);
      const float vs = block_scale(wave_max(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]))), vi);
      uint32_t m4 = 0, v4 = 0;
      for (int k = 0; k < 4; ++k) {
        uint32_t mc = e4m3_code(fabsf(m[k]) * mi, rs[k] & 0xffff), vc = e4m3_code(v[k] * vi, rs[k] >> 16);
        if (m[k] < 0.f && mc) mc |= 0x80;
        if (v[k] > 0.f && vs > 0.f && !vc) vc = 1;
        m4 |= mc << 8 * k; v4 |= vc << 8 * k;
      }
      *(uint32_t *)((uint8_t *)c.m + s) = m4;
      *(uint32_t *)((uint8_t *)c.v + s) = v4;
      if (threadIdx.x % 64 == 0) { c.m_scale[s / ECHO_ADAMW_BLOCK] = ms; c.v_scale[s / ECHO_ADAMW_BLOCK] = vs; }
    }
  }
}

template <int PT, int GT> void launch_states(const StepTensors &t, const StepConstants &c, int state_dtype, hipStream_t st) {
  const dim3 grid(t.chunk0[t.n]);
  if (state_dtype == ECHO_F32) adamw_kernel<PT, GT, ECHO_F32><<<grid, THREADS, 0, st>>>(t, c);
  else adamw_kernel<PT, GT, ECHO_E4M3><<<grid, THREADS, 0, st>>>(t, c);
}

}  // namespace

void launch_grad_norm(const NormTensors &t, int dtype, double *partial, hipStream_t st) {
  const dim3 grid(t.chunk0[t.n]);
  if (dtype == ECHO_F32) norm_kernel<ECHO_F32><<<grid, THREADS, 0, st>>>(t, partial);
  else if (dtype == ECHO_BF16) norm_kernel<ECHO_BF16><<<grid, THREADS, 0, st>>>(t, partial);
  else norm_kernel<ECHO_F16><<<grid, THREADS, 0, st>>>(t, partial);
}
void launch_norm_finish(const double *partial, int64_t n, float *out, hipStream_t st) { norm_finish_kernel<<<1, THREADS, 0, st>>>(partial, n, out); }

void launch_adamw(const StepTensors &t, const StepConstants &c, int param_dtype, int grad_dtype, int state_dtype, hipStream_t st) {
  if (param_dtype == ECHO_F32) {
    if (grad_dtype == ECHO_F32) launch_states<ECHO_F32, ECHO_F32>(t, c, state_dtype, st);
    else launch_states<ECHO_F32, ECHO_BF16>(t, c, state_dtype, st);
  } else {
    if (grad_dtype == ECHO_F32) launch_states<ECHO_BF16, ECHO_F32>(t, c, state_dtype, st);
    else launch_states<ECHO_BF16, ECHO_BF16>(t, c, state_dtype, st);
  }
}

}  // namespace echo
