// One AdamW step over many tensors, with states in 32 or 8 bits (moe.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "blocks.h"
#include "tile.h"

using namespace moe;

namespace {

constexpr int PIECE = 16;          // consecutive values of a thread
constexpr int CHUNK = 256 * PIECE;  // values of a workgroup
constexpr int LANES = MOE_ADAMW_BLOCK / PIECE;  // threads that share an 8-bit block
// Tensors of a launch: their addresses are kernel arguments (4 KB at most), so
// that no table has to reach the device before the step.
constexpr int MOST = 48;

struct Tensor {
  const void* grad;
  uint16_t* param;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t n;
  float decay;
  uint32_t place_and_type;  // place in the caller's list * 2 + (grad is fp32)
  __device__ bool grad_fp32() const { return place_and_type & 1; }
  __device__ uint32_t place() const { return place_and_type >> 1; }
};

struct AdamArgs {
  const float* now;
  float lr, scale, step, log_b1, log_b2, b1, b2, eps;
  uint32_t seed;
  int count;           // tensors of this launch
  uint32_t end[MOST];  // chunks of the tensors up to and with each
  Tensor t[MOST];
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// ---- random bits ----------------------------------------------------------------
// Multiplications by odd numbers and folds of the upper half into the lower: a
// flipped bit of h flips each bit of the result with probability 1/2 (measured
// over 10^5 values: within the error of the measurement).
__device__ __forceinline__ uint32_t mixed(uint32_t h) {
  h = (h ^ h >> 16) * 0x761BCE4Bu;
  h = (h ^ h >> 15) * 0xA0D73955u;
  return h ^ h >> 16;
}

// ---- 8-bit values -----------------------------------------------------------------
// x in [0, 448] or [0, 57344] to e4m3 or e5m2, up with probability (distance to
// the lower neighbour) / (step): 16 random bits are added below the mantissa that
// stays, or below the unit of the subnormals.
__device__ __forceinline__ uint32_t to_e4m3(float x, uint32_t r) {
  const uint32_t normal = ((__float_as_uint(x) + (r << 4)) >> 20) - (120u << 3);
  const uint32_t tiny = (uint32_t)(x * 512.0f + (float)r * 0x1p-16f);
  return min(x < 0x1p-6f ? tiny : normal, 0x7Eu);
}
__device__ __forceinline__ uint32_t to_e5m2(float x, uint32_t r) {
  const uint32_t normal = ((__float_as_uint(x) + (r << 5)) >> 21) - (112u << 2);
  const uint32_t tiny = (uint32_t)(x * 65536.0f + (float)r * 0x1p-16f);
  return min(x < 0x1p-14f ? tiny : normal, 0x7Bu);
}

// the scale of a block, from its largest magnitude's bits, and its reciprocal (0: the block is 0)
__device__ __forceinline__ float scale_of(uint32_t largest, float most, float* inv) {
  const float a = __uint_as_float(largest);
  *inv = 0;
  if (!(a < __builtin_inff())) return __builtin_nanf("");
  if (a < 0x1p-110f) return 0;
  const float s = a / most;
  *inv = 1.0f / s;
  return s;
}
// the largest over the threads of a block
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
#pragma unroll
  for (int d = LANES / 2; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  return m;
}

template <bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  int i = 0;
  while (i + 1 < a.count && blockIdx.x >= a.end[i]) ++i;
  const Tensor& t = a.t[i];
  const int64_t first = ((int64_t)blockIdx.x - (i ? a.end[i - 1] : 0)) * CHUNK + threadIdx.x * PIECE;
  const int have = (int)min((int64_t)PIECE, max((int64_t)0, t.n - first));
  float lr = a.lr, gs = a.scale, step = a.step;
  if (a.now) {
    lr = a.now[0], gs = a.now[1], step = a.now[2];
    if (gs != gs) return;
    step = step >= 1.0f ? step : 1.0f;
  }
  const float c1 = -expm1f(step * a.log_b1), c2 = -expm1f(step * a.log_b2);

  float m[PIECE], v[PIECE], w[PIECE];
  uint32_t m_most = 0, v_most = 0;
#pragma unroll
  for (int j = 0; j < PIECE; ++j) {
    m[j] = v[j] = w[j] = 0;
    if (j >= have) continue;
    const int64_t at = first + j;
    const float g = gs * (t.grad_fp32() ? static_cast<const float*>(t.grad)[at]
                                      : bf16_to_f32(static_cast<const uint16_t*>(t.grad)[at]));
    if constexpr (BITS8) {
      m[j] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(t.m)[at], 0) * t.m_scale[at / MOE_ADAMW_BLOCK];
      v[j] = __builtin_amdgcn_cvt_f32_bf8(static_cast<const uint8_t*>(t.v)[at], 0) * t.v_scale[at / MOE_ADAMW_BLOCK];
    } else {
      m[j] = static_cast<const float*>(t.m)[at];
      v[j] = static_cast<const float*>(t.v)[at];
    }
    m[j] = a.b1 * m[j] + (1.0f - a.b1) * g;
    v[j] = a.b2 * v[j] + (1.0f - a.b2) * (g * g);
    m_most = max(m_most, __float_as_uint(m[j]) & 0x7fffffffu);
    v_most = max(v_most, __float_as_uint(v[j]) & 0x7fffffffu);
    w[j] = t.master ? t.master[at] : bf16_to_f32(t.param[at]);
    w[j] -= lr * (t.decay * w[j] + (m[j] / c1) / (sqrtf(v[j] / c2) + a.eps));
  }
  float ms = 0, vs = 0, mi = 0, vi = 0;
  if constexpr (BITS8) {
    ms = scale_of(block_max(m_most), 448.0f, &mi);
    vs = scale_of(block_max(v_most), 57344.0f, &vi);
    if (have > 0 && threadIdx.x % LANES == 0) {
      t.m_scale[first / MOE_ADAMW_BLOCK] = ms;
      t.v_scale[first / MOE_ADAMW_BLOCK] = vs;
    }
  }
  const uint32_t key = mixed(mixed(a.seed + (uint32_t)step * 0xD22CD251u) + t.place() * 0xA5375919u);
#pragma unroll
  for (int j = 0; j < PIECE; ++j) {
    if (j >= have) continue;
    const int64_t at = first + j;
    const uint32_t h = mixed(key + (uint32_t)at * 0x946BAFCDu + (uint32_t)(at >> 32) * 0x8952E2D3u);
    if (t.master) {
      t.master[at] = w[j];
      if (t.param) t.param[at] = (uint16_t)f32_to_bf16(w[j]);
    } else {
      t.param[at] = w[j] != w[j] ? 0x7fc0u : (uint16_t)((__float_as_uint(w[j]) + (h * 0x761BCE4Bu >> 16)) >> 16);
    }
    if constexpr (BITS8) {
      const uint32_t mc = mi > 0 ? to_e4m3(fabsf(m[j]) * mi, h & 0xffffu) | (__float_as_uint(m[j]) >> 31 << 7) : 0u;
      const uint32_t vc = vi > 0 ? max(to_e5m2(v[j] * vi, h >> 16), v[j] > 0 ? 1u : 0u) : 0u;
      static_cast<uint8_t*>(t.m)[at] = (uint8_t)mc;
      static_cast<uint8_t*>(t.v)[at] = (uint8_t)vc;
    } else {
      static_cast<float*>(t.m)[at] = m[j];
      static_cast<float*>(t.v)[at] = v[j];
    }
  }
}

moe_status check(const moe_adamw_config* c, const moe_adamw_tensor* tensors, int32_t n) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  const auto finite = [](float v) { return v - v == 0.0f; };
  if (!finite(c->lr) || c->lr < 0) return fail(MOE_ERR_INVALID_ARG, "lr must be finite and not below 0");
  if (!(c->beta1 >= 0.0f && c->beta1 < 1.0f && c->beta2 >= 0.0f && c->beta2 < 1.0f))
    return fail(MOE_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!finite(c->eps) || !(c->eps > 0)) return fail(MOE_ERR_INVALID_ARG, "eps must be above 0 and finite");
  if (!finite(c->grad_scale)) return fail(MOE_ERR_INVALID_ARG, "grad_scale must be finite");
  if (c->step < 1) return fail(MOE_ERR_INVALID_ARG, "step counts from 1");
  if (c->state_bits != 32 && c->state_bits != 8) return fail(MOE_ERR_INVALID_ARG, "state_bits must be 32 or 8");
  if (n < 0 || (n > 0 && !tensors)) return fail(MOE_ERR_INVALID_ARG, "no list of n_tensors tensors");
  for (int32_t i = 0; i < n; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > (1LL << 40)) return fail(MOE_ERR_INVALID_ARG, "tensor %d: n must be in [0, 2^40]", i);
    if (!finite(t.weight_decay) || t.weight_decay < 0)
      return fail(MOE_ERR_INVALID_ARG, "tensor %d: weight_decay must be finite and not below 0", i);
    if (t.grad_fp32 != 0 && t.grad_fp32 != 1) return fail(MOE_ERR_INVALID_ARG, "tensor %d: grad_fp32 must be 0 or 1", i);
    if (t.n == 0) continue;
    if ((!t.param && !t.master) || !t.grad || !t.m || !t.v) return fail(MOE_ERR_INVALID_ARG, "tensor %d: NULL argument", i);
    if ((!t.m_scale || !t.v_scale) != (c->state_bits == 32) || !t.m_scale != !t.v_scale)
      return fail(MOE_ERR_INVALID_ARG, "tensor %d: states in 8 bits have scales, and others none", i);
    for (const void* p : {(const void*)t.param, (const void*)t.master, t.grad, (const void*)t.m, (const void*)t.v,
                          (const void*)t.m_scale, (const void*)t.v_scale})
      if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "tensor %d does not start on a 16-byte boundary", i);
  }
  return MOE_OK;
}

}  // namespace

extern "C" {

moe_status moe_adamw(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors, const float* now,
                     void* stream) {
  moe_status st = check(cfg, tensors, n_tensors);
  if (st != MOE_OK) return st;
  if (reinterpret_cast<uintptr_t>(now) % 4) return fail(MOE_ERR_INVALID_ARG, "now is not aligned to its values");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  AdamArgs a{};
  a.now = now, a.lr = cfg->lr, a.scale = cfg->grad_scale, a.step = (float)cfg->step;
  a.b1 = cfg->beta1, a.b2 = cfg->beta2, a.eps = cfg->eps, a.seed = cfg->seed;
  a.log_b1 = (float)std::log((double)cfg->beta1), a.log_b2 = (float)std::log((double)cfg->beta2);
  bool any = false;
  const auto go = [&] {
    if (a.count == 0) return;
    any = true;
    const uint32_t grid = a.end[a.count - 1];
    if (cfg->state_bits == 8) adamw_kernel<true><<<grid, 256, 0, s>>>(a);
    else adamw_kernel<false><<<grid, 256, 0, s>>>(a);
    a.count = 0;
  };
  for (int32_t i = 0; i < n_tensors; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    const int64_t before = a.count ? a.end[a.count - 1] : 0, chunks = (t.n + CHUNK - 1) / CHUNK;
    a.t[a.count] = {t.grad, t.param, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n, t.weight_decay,
                    (uint32_t)i << 1 | (uint32_t)t.grad_fp32};
    a.end[a.count++] = (uint32_t)(before + chunks);
    // (2^28 chunks are the largest tensor's: a grid stays below 2^30)
    if (a.count == MOST || before + chunks > (1 << 28)) go();
  }
  go();
  if (any) HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
