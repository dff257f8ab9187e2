// One AdamW step over many tensors, with states in 32 or 8 bits (moe.h).
#include <hip/hip_runtime.h>

#include <cmath>

#include "blocks.h"
#include "tile.h"

using namespace moe;

namespace {

constexpr int VALUES = 16;           // of a thread
constexpr int CHUNK = 256 * VALUES;  // of a workgroup
// Chunks of a launch: a launch has fewer than 2^32 threads
constexpr int64_t MOST_CHUNKS = (1 << 24) - 1;
// Tensors of a launch: their addresses are kernel arguments (4 KB at most), so
// that no table has to reach the device before the step.  A tensor and its end take 48
// bytes (8 bits: 60), addresses as multiples of 16 (scales': of 4): 150 small tensors in
// two launches, 20 us, against 29 in four of 48 tensors.
template <bool BITS8>
struct Packed {
  static constexpr int N = BITS8 ? 7 : 5;  // grad, param, master, m, v, m_scale, v_scale
  uint32_t low[N];
  uint32_t high[N / 2 + 1];  // 16 bits each, n's behind them (words: scalar loads have no halves)
  uint32_t n_low;
  float decay;
  uint32_t place_and_type;  // place in the caller's list * 2 + (grad is fp32)

  __host__ __device__ __forceinline__ uint32_t half(int i) const { return i % 2 ? high[i / 2] >> 16 : high[i / 2] & 0xffffu; }
  static __host__ __device__ __forceinline__ constexpr int unit(int i) { return i < 5 ? 4 : 2; }  // bits that are 0 in address i
  __device__ __forceinline__ char* at(int i) const { return reinterpret_cast<char*>(((uint64_t)half(i) << 32 | low[i]) << unit(i)); }
  __device__ __forceinline__ int64_t n() const { return (int64_t)((uint64_t)half(N) << 32 | n_low); }
  __device__ __forceinline__ bool grad_fp32() const { return place_and_type & 1; }
  __device__ __forceinline__ uint32_t place() const { return place_and_type >> 1; }
};
template <bool BITS8>
constexpr int MOST = BITS8 ? 67 : 84;

template <bool BITS8>
struct AdamArgs {
  const float* now;
  float lr, scale, log_b1, log_b2, b1, b2, rest1, rest2, eps;  // rest: 1 - beta
  int32_t step;
  uint32_t seed;
  int count;                  // tensors of this launch
  uint32_t end[MOST<BITS8>];  // chunks of the tensors up to and with each
  Packed<BITS8> t[MOST<BITS8>];
};
static_assert(sizeof(Packed<true>) == 56 && sizeof(Packed<false>) == 44 && sizeof(AdamArgs<true>) <= 4096 &&
              sizeof(AdamArgs<false>) <= 4096, "kernel arguments");

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
// the lower neighbour) / (step): 16 random bits r are added below the mantissa
// that stays.  Below the smallest normal value the steps are those of its
// binade, so x is rounded as x + that value and 8 (4) steps are taken off.
__device__ __forceinline__ uint32_t to_e4m3(float x, uint32_t r) {
  const bool tiny = x < 0x1p-6f;
  const uint32_t bits = __float_as_uint(tiny ? x + 0x1p-6f : x) + (r << 4);
  return min((bits >> 20) - (tiny ? (121u << 3) : (120u << 3)), 0x7Eu);
}
__device__ __forceinline__ uint32_t to_e5m2(float x, uint32_t r) {
  const bool tiny = x < 0x1p-14f;
  const uint32_t bits = __float_as_uint(tiny ? x + 0x1p-14f : x) + (r << 5);
  return min((bits >> 21) - (tiny ? (113u << 2) : (112u << 2)), 0x7Bu);
}

// value i of four in e4m3 (M) or e5m2
template <bool M>
__device__ __forceinline__ float from_8bit(uint32_t four, int i) {
  if constexpr (M)
    return i < 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)four, false)[i] : __builtin_amdgcn_cvt_pk_f32_fp8((int)four, true)[i - 2];
  else
    return i < 2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)four, false)[i] : __builtin_amdgcn_cvt_pk_f32_bf8((int)four, true)[i - 2];
}

// b old + rest x, rounded operation by operation: which of an 8-bit state's two
// neighbours is taken then does not depend on what a compiler fuses.
__device__ __forceinline__ float average(float b, float old, float rest, float x) {
#pragma clang fp contract(off)
  return b * old + rest * x;
}

// the scale of a block, from its largest magnitude's bits, and its reciprocal (0: the block is 0)
__device__ __forceinline__ float scale_of(uint32_t largest, float one_over_most, float* inv) {
  const float a = __uint_as_float(largest);
  *inv = 0;
  if (!(a < __builtin_inff())) return __builtin_nanf("");
  if (a < 0x1p-110f) return 0;
  const float s = a * one_over_most;
  *inv = 1.0f / s;
  return s;
}

// GROUP consecutive values in registers as they lie in memory, and in fp32
template <int GROUP>
struct Raw {
  u32x4_t w[GROUP / 4];
};
template <int GROUP>
__device__ __forceinline__ void load_f32(Raw<GROUP>& r, const float* p) {
#pragma unroll
  for (int i = 0; i < GROUP / 4; ++i) r.w[i] = reinterpret_cast<const u32x4_t*>(p)[i];
}
template <int GROUP>
__device__ __forceinline__ void load_bf16(Raw<GROUP>& r, const uint16_t* p) {
  if constexpr (GROUP == 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    r.w[0] = u32x4_t{v.x, v.y, 0, 0};
  } else {
#pragma unroll
    for (int i = 0; i < GROUP / 8; ++i) r.w[i] = reinterpret_cast<const u32x4_t*>(p)[i];
  }
}
template <int GROUP>
__device__ __forceinline__ float f32_of(const Raw<GROUP>& r, int j) { return __uint_as_float(r.w[j / 4][j % 4]); }
template <int GROUP>
__device__ __forceinline__ float bf16_of(const Raw<GROUP>& r, int j) {
  const uint32_t w = r.w[j / 8][j / 2 % 4];
  return j % 2 ? bf16_hi(w) : bf16_lo(w);
}

// One workgroup steps CHUNK values of a tensor, in groups of GROUP consecutive
// ones a thread: 16 where states have 8 bits (one 16-byte load of each, a block's
// scale from 16 threads), 4 where they have 32.  Bound by memory: 604 million values,
// 8-bit states and bf16 weights and gradients, 1183 to 1262 us, 4.8 to 5.1 TB/s; 134 million
// with 32-bit states, master weights and fp32 gradients 744 to 770, 5.2 to 5.4.
// GRAD32: gradients in fp32; MASTER, PARAM: which weights there are.
template <bool BITS8, bool GRAD32, bool MASTER, bool PARAM>
__device__ __forceinline__ void step_chunk(const AdamArgs<BITS8>& a, const Packed<BITS8>& t, int64_t chunk) {
  constexpr int GROUP = BITS8 ? 16 : 4, GROUPS = VALUES / GROUP;
  const int lane = threadIdx.x & 63;
  const int inside = (int)min((int64_t)CHUNK, t.n() - chunk);  // values of this chunk
  float lr = a.lr, gs = a.scale, step = (float)a.step;
  uint32_t count = (uint32_t)a.step;  // of the random bits: fp32 would give neighbouring steps from 2^24 on the same
  if (a.now) {
    lr = a.now[0], gs = a.now[1], step = a.now[2];
    if (gs != gs) return;
    step = step >= 1.0f ? step : 1.0f;
    count = (uint32_t)fminf(step, 0x1.fffffep31f);
  }
  const float c1 = 1.0f / -expm1f(step * a.log_b1), c2 = 1.0f / -expm1f(step * a.log_b2);
  const uint32_t key = mixed(mixed(a.seed + count * 0xD22CD251u) + t.place() * 0xA5375919u);
  const float* grad_f = reinterpret_cast<const float*>(t.at(0)) + chunk;
  const uint16_t* grad_h = reinterpret_cast<const uint16_t*>(t.at(0)) + chunk;
  uint16_t* param = reinterpret_cast<uint16_t*>(t.at(1)) + chunk;
  float* master = reinterpret_cast<float*>(t.at(2)) + chunk;
  uint8_t *m8 = reinterpret_cast<uint8_t*>(t.at(3)) + chunk, *v8 = reinterpret_cast<uint8_t*>(t.at(4)) + chunk;
  float *m32 = reinterpret_cast<float*>(t.at(3)) + chunk, *v32 = reinterpret_cast<float*>(t.at(4)) + chunk;
  float *m_scale = nullptr, *v_scale = nullptr;
  if constexpr (BITS8) {
    m_scale = reinterpret_cast<float*>(t.at(5)) + chunk / MOE_ADAMW_BLOCK;
    v_scale = reinterpret_cast<float*>(t.at(6)) + chunk / MOE_ADAMW_BLOCK;
  }

  Raw<GROUP> g[GROUPS], w[GROUPS];
  u32x4_t m[GROUPS], v[GROUPS];  // 16 states of 8 bits or 4 of 32
  float ms = 0, vs = 0;
  const auto at_of = [&](int k) { return ((int)(threadIdx.x >> 6) * GROUPS * 64 + k * 64 + lane) * GROUP; };
  // A group that the tensor's end cuts is read value by value, zeros behind it
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    const int at = at_of(k), have = inside - at;
    g[k] = w[k] = {};
    m[k] = v[k] = u32x4_t{0, 0, 0, 0};
    if (have >= GROUP) {
      if constexpr (GRAD32) load_f32(g[k], grad_f + at);
      else load_bf16(g[k], grad_h + at);
      if constexpr (MASTER) load_f32(w[k], master + at);
      else load_bf16(w[k], param + at);
      m[k] = BITS8 ? *reinterpret_cast<const u32x4_t*>(m8 + at) : *reinterpret_cast<const u32x4_t*>(m32 + at);
      v[k] = BITS8 ? *reinterpret_cast<const u32x4_t*>(v8 + at) : *reinterpret_cast<const u32x4_t*>(v32 + at);
    } else if (have > 0) {
#pragma unroll
      for (int j = 0; j < GROUP; ++j) {
        if (j >= have) continue;
        if constexpr (GRAD32) g[k].w[j / 4][j % 4] = __float_as_uint(grad_f[at + j]);
        else g[k].w[j / 8][j / 2 % 4] |= (uint32_t)grad_h[at + j] << (j % 2 * 16);
        if constexpr (MASTER) w[k].w[j / 4][j % 4] = __float_as_uint(master[at + j]);
        else w[k].w[j / 8][j / 2 % 4] |= (uint32_t)param[at + j] << (j % 2 * 16);
        if constexpr (BITS8) {
          m[k][j / 4] |= (uint32_t)m8[at + j] << (j % 4 * 8);
          v[k][j / 4] |= (uint32_t)v8[at + j] << (j % 4 * 8);
        } else {
          m[k][j] = __float_as_uint(m32[at + j]);
          v[k][j] = __float_as_uint(v32[at + j]);
        }
      }
    }
    if (BITS8 && have > 0) {
      ms = m_scale[at / MOE_ADAMW_BLOCK];
      vs = v_scale[at / MOE_ADAMW_BLOCK];
    }
  }
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    const int at = at_of(k), have = inside - at;
    float fm[GROUP], fv[GROUP], fw[GROUP];
    uint32_t m_most = 0, v_most = 0;
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      const float gr = gs * (GRAD32 ? f32_of(g[k], j) : bf16_of(g[k], j));
      if constexpr (BITS8) {
        fm[j] = from_8bit<true>(m[k][j / 4], j % 4) * ms;
        fv[j] = from_8bit<false>(v[k][j / 4], j % 4) * vs;
      } else {
        fm[j] = __uint_as_float(m[k][j]);
        fv[j] = __uint_as_float(v[k][j]);
      }
      fm[j] = average(a.b1, fm[j], a.rest1, gr);
      fv[j] = average(a.b2, fv[j], a.rest2, gr * gr);
      if constexpr (BITS8) {
        m_most = max(m_most, __float_as_uint(fm[j]) & 0x7fffffffu);
        v_most = max(v_most, __float_as_uint(fv[j]) & 0x7fffffffu);
      }
      // the hardware's root and reciprocal, each within 2^-23 of the exact one
      const float old = MASTER ? f32_of(w[k], j) : bf16_of(w[k], j);
      const float den = __builtin_amdgcn_sqrtf(fv[j] * c2) + a.eps;
      fw[j] = old - lr * (t.decay * old + fm[j] * c1 * __builtin_amdgcn_rcpf(den));
    }
    float mi = 0, vi = 0;
    if constexpr (BITS8) {
#pragma unroll
      for (int d = MOE_ADAMW_BLOCK / GROUP / 2; d; d >>= 1) {
        m_most = max(m_most, (uint32_t)__shfl_xor((int)m_most, d));
        v_most = max(v_most, (uint32_t)__shfl_xor((int)v_most, d));
      }
      ms = scale_of(m_most, 1.0f / 448.0f, &mi);
      vs = scale_of(v_most, 1.0f / 57344.0f, &vi);
      if (have > 0 && threadIdx.x % (MOE_ADAMW_BLOCK / GROUP) == 0) {
        m_scale[at / MOE_ADAMW_BLOCK] = ms;
        v_scale[at / MOE_ADAMW_BLOCK] = vs;
      }
    }
    // random bits, where something is rounded at random
    uint32_t h[GROUP] = {};
    if constexpr (BITS8 || !MASTER) {
      const uint64_t first = (uint64_t)(chunk + at);
      uint32_t x = key + (uint32_t)first * 0x946BAFCDu + (uint32_t)(first >> 32) * 0x8952E2D3u;
#pragma unroll
      for (int j = 0; j < GROUP; ++j, x += 0x946BAFCDu) h[j] = mixed(x);
    }
    uint32_t pw[GROUP / 2];  // param's values
    u32x4_t ow[GROUP / 4];   // master's
#pragma unroll
    for (int j = 0; j < GROUP; ++j) ow[j / 4][j % 4] = __float_as_uint(fw[j]);
#pragma unroll
    for (int j = 0; j < GROUP; j += 2) {
      if constexpr (MASTER) {
        pw[j / 2] = pack_bf16x2(fw[j], fw[j + 1]);
      } else {
        uint32_t r[2];
#pragma unroll
        for (int n = 0; n < 2; ++n)
          r[n] = fw[j + n] != fw[j + n] ? 0x7fc00000u : __float_as_uint(fw[j + n]) + (h[j + n] * 0x761BCE4Bu >> 16);
        pw[j / 2] = r[0] >> 16 | (r[1] & 0xffff0000u);
      }
    }
    u32x4_t om{0, 0, 0, 0}, ov{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < GROUP; ++j) {
      if constexpr (BITS8) {
        const uint32_t mc = to_e4m3(fabsf(fm[j]) * mi, h[j] & 0xffffu) | (__float_as_uint(fm[j]) >> 24 & 0x80u);
        // (what is not 0 stays so: its root is divided by)
        const uint32_t vc = max(to_e5m2(fv[j] * vi, h[j] >> 16), min(__float_as_uint(fv[j]), 1u));
        om[j / 4] |= mc << (j % 4 * 8);
        ov[j / 4] |= vc << (j % 4 * 8);
      } else {
        om[j] = __float_as_uint(fm[j]);
        ov[j] = __float_as_uint(fv[j]);
      }
    }
    if constexpr (BITS8) {  // a block that is 0, or NaN
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        om[j] = mi > 0 ? om[j] : 0u;
        ov[j] = vi > 0 ? ov[j] : 0u;
      }
    }
    if (have >= GROUP) {
      if constexpr (MASTER) {
#pragma unroll
        for (int j = 0; j < GROUP / 4; ++j) reinterpret_cast<u32x4_t*>(master + at)[j] = ow[j];
      }
      if constexpr (PARAM) {
        if constexpr (GROUP == 4) {
          *reinterpret_cast<uint2*>(param + at) = uint2{pw[0], pw[1]};
        } else {
#pragma unroll
          for (int j = 0; j < GROUP / 8; ++j)
            reinterpret_cast<u32x4_t*>(param + at)[j] = u32x4_t{pw[4 * j], pw[4 * j + 1], pw[4 * j + 2], pw[4 * j + 3]};
        }
      }
      *(BITS8 ? reinterpret_cast<u32x4_t*>(m8 + at) : reinterpret_cast<u32x4_t*>(m32 + at)) = om;
      *(BITS8 ? reinterpret_cast<u32x4_t*>(v8 + at) : reinterpret_cast<u32x4_t*>(v32 + at)) = ov;
    } else if (have > 0) {
#pragma unroll
      for (int j = 0; j < GROUP; ++j) {
        if (j >= have) continue;
        if constexpr (MASTER) master[at + j] = fw[j];
        if constexpr (PARAM) param[at + j] = (uint16_t)(pw[j / 2] >> (j % 2 * 16));
        if constexpr (BITS8) {
          m8[at + j] = (uint8_t)(om[j / 4] >> (j % 4 * 8));
          v8[at + j] = (uint8_t)(ov[j / 4] >> (j % 4 * 8));
        } else {
          m32[at + j] = __uint_as_float(om[j]);
          v32[at + j] = __uint_as_float(ov[j]);
        }
      }
    }
  }
}

template <bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs<BITS8> a) {
  const int lane = threadIdx.x & 63;
  int i = 0;  // tensors that end before this chunk
#pragma unroll
  for (int first = 0; first < MOST<BITS8>; first += 64) {
    const int k = first + lane;
    i += __popcll(__ballot(k < a.count && blockIdx.x >= a.end[min(k, MOST<BITS8> - 1)]));
  }
  const Packed<BITS8>& t = a.t[i];
  const int64_t chunk = (int64_t)(blockIdx.x - (i ? a.end[i - 1] : 0)) * CHUNK;
  const bool param = t.at(1) != nullptr, master = t.at(2) != nullptr;
  if (t.grad_fp32()) {
    if (!master) step_chunk<BITS8, true, false, true>(a, t, chunk);
    else if (param) step_chunk<BITS8, true, true, true>(a, t, chunk);
    else step_chunk<BITS8, true, true, false>(a, t, chunk);
  } else {
    if (!master) step_chunk<BITS8, false, false, true>(a, t, chunk);
    else if (param) step_chunk<BITS8, false, true, true>(a, t, chunk);
    else step_chunk<BITS8, false, true, false>(a, t, chunk);
  }
}

moe_status check(const moe_adamw_config* c, const moe_adamw_tensor* tensors, int32_t n) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  const auto finite = [](double v) { return std::isfinite((float)v); };
  if (!finite(c->lr) || c->lr < 0) return fail(MOE_ERR_INVALID_ARG, "lr must be finite and not below 0");
  if (!(c->beta1 >= 0 && c->beta1 < 1 && c->beta2 >= 0 && c->beta2 < 1))
    return fail(MOE_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!finite(c->eps) || !(c->eps >= 1e-15)) return fail(MOE_ERR_INVALID_ARG, "eps must be finite and at least 1e-15");
  if (!finite(c->grad_scale)) return fail(MOE_ERR_INVALID_ARG, "grad_scale must be finite");
  if (c->step < 1) return fail(MOE_ERR_INVALID_ARG, "step counts from 1");
  if (c->state_bits != 32 && c->state_bits != 8) return fail(MOE_ERR_INVALID_ARG, "state_bits must be 32 or 8");
  if (n < 0 || (n > 0 && !tensors)) return fail(MOE_ERR_INVALID_ARG, "no list of n_tensors tensors");
  for (int32_t i = 0; i < n; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > MOST_CHUNKS * CHUNK) return fail(MOE_ERR_INVALID_ARG, "tensor %d: n must be in [0, 2^36 - 4096]", i);
    if (!finite(t.weight_decay) || t.weight_decay < 0)
      return fail(MOE_ERR_INVALID_ARG, "tensor %d: weight_decay must be finite and not below 0", i);
    if (t.grad_fp32 != 0 && t.grad_fp32 != 1) return fail(MOE_ERR_INVALID_ARG, "tensor %d: grad_fp32 must be 0 or 1", i);
    if (t.n == 0) continue;
    if ((!t.param && !t.master) || !t.grad || !t.m || !t.v) return fail(MOE_ERR_INVALID_ARG, "tensor %d: NULL argument", i);
    if ((!t.m_scale || !t.v_scale) != (c->state_bits == 32) || !t.m_scale != !t.v_scale)
      return fail(MOE_ERR_INVALID_ARG, "tensor %d: states in 8 bits have scales, and others none", i);
    for (const void* p : {(const void*)t.param, (const void*)t.master, t.grad, (const void*)t.m, (const void*)t.v})
      if (!aligned16(p) || reinterpret_cast<uint64_t>(p) >> 50)
        return fail(MOE_ERR_INVALID_ARG, "tensor %d does not start on a 16-byte boundary", i);
    for (const float* p : {t.m_scale, t.v_scale})
      if (reinterpret_cast<uint64_t>(p) % 4 || reinterpret_cast<uint64_t>(p) >> 50)
        return fail(MOE_ERR_INVALID_ARG, "tensor %d: scales are not aligned to their values", i);
  }
  return MOE_OK;
}

template <bool BITS8>
bool launch(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors, const float* now, hipStream_t s) {
  AdamArgs<BITS8> a{};
  a.now = now, a.lr = (float)cfg->lr, a.scale = (float)cfg->grad_scale, a.step = cfg->step;
  a.b1 = (float)cfg->beta1, a.b2 = (float)cfg->beta2, a.eps = (float)cfg->eps, a.seed = cfg->seed;
  a.rest1 = (float)(1 - cfg->beta1), a.rest2 = (float)(1 - cfg->beta2);
  a.log_b1 = (float)std::log(cfg->beta1), a.log_b2 = (float)std::log(cfg->beta2);
  bool any = false;
  const auto go = [&] {
    if (a.count == 0) return;
    any = true;
    adamw_kernel<BITS8><<<a.end[a.count - 1], 256, 0, s>>>(a);
    a.count = 0;
  };
  for (int32_t i = 0; i < n_tensors; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    const int64_t chunks = (t.n + CHUNK - 1) / CHUNK;
    if (a.count == MOST<BITS8> || (a.count && a.end[a.count - 1] + chunks > MOST_CHUNKS)) go();
    const int64_t before = a.count ? a.end[a.count - 1] : 0;
    Packed<BITS8>& p = a.t[a.count];
    p = {};
    const auto put_half = [&](int k, uint32_t v) { p.high[k / 2] |= v << (k % 2 * 16); };
    const void* const at[7] = {t.grad, t.param, t.master, t.m, t.v, t.m_scale, t.v_scale};
    for (int k = 0; k < Packed<BITS8>::N; ++k) {
      const uint64_t v = reinterpret_cast<uint64_t>(at[k]) >> Packed<BITS8>::unit(k);
      p.low[k] = (uint32_t)v;
      put_half(k, (uint32_t)(v >> 32));
    }
    p.n_low = (uint32_t)t.n;
    put_half(Packed<BITS8>::N, (uint32_t)(t.n >> 32));
    p.decay = t.weight_decay;
    p.place_and_type = (uint32_t)i << 1 | (uint32_t)t.grad_fp32;
    a.end[a.count++] = (uint32_t)(before + chunks);
  }
  go();
  return any;
}

}  // namespace

extern "C" {

moe_status moe_adamw(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors, const float* now,
                     void* stream) {
  moe_status st = check(cfg, tensors, n_tensors);
  if (st != MOE_OK) return st;
  if (reinterpret_cast<uintptr_t>(now) % 4) return fail(MOE_ERR_INVALID_ARG, "now is not aligned to its values");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool any = cfg->state_bits == 8 ? launch<true>(cfg, tensors, n_tensors, now, s) : launch<false>(cfg, tensors, n_tensors, now, s);
  if (any) HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
