// Root-mean-square norm with the residual's addition, in bf16 or in 8 bits, and
// its backward pass (moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "blocks.h"
#include "tile.h"

using namespace moe;

namespace {

struct NormArgs {
  int T, H;
  float eps;
  const uint16_t *x, *residual, *weight;
  uint16_t *sum, *y;
  float* rstd;
  int8_t* q;
  float* scale;
};

struct NormGradArgs {
  int T, H;
  const uint16_t *dy, *dsum, *sum, *weight;
  const float* rstd;
  uint16_t* dx;
  float *dweight, *part;  // part: [parts][H]
  int parts;
};

// Threads of a workgroup whose rows take THREADS threads each
template <int THREADS>
constexpr int group_of = THREADS > 256 ? THREADS : 256;

// Sum and largest of (a, m) over the THREADS threads of a row.  red: a slot for
// each wavefront; a caller in a loop takes two sets in turn.
template <int THREADS>
__device__ __forceinline__ void reduce(float& a, uint32_t& m, float* red_a, uint32_t* red_m) {
#pragma unroll
  for (int d = (THREADS < 64 ? THREADS : 64) / 2; d; d >>= 1) {
    a += __shfl_xor(a, d);
    m = max(m, (uint32_t)__shfl_xor((int)m, d));
  }
  if constexpr (THREADS > 64) {
    if (threadIdx.x % 64 == 0) {
      red_a[threadIdx.x / 64] = a;
      red_m[threadIdx.x / 64] = m;
    }
    __syncthreads();
    a = red_a[0], m = red_m[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) {
      a += red_a[i];
      m = max(m, red_m[i]);
    }
  }
}

template <int THREADS>
__device__ __forceinline__ float sum_of(float a, float* red) {
#pragma unroll
  for (int d = (THREADS < 64 ? THREADS : 64) / 2; d; d >>= 1) a += __shfl_xor(a, d);
  if constexpr (THREADS > 64) {
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = a;
    __syncthreads();
    a = red[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) a += red[i];
  }
  return a;
}

// One row by THREADS threads, held in registers: LOADS pieces of 8 values each.
// s w is exact in fp32 (two bf16 values), so y = (s w) r is rounded once, and the
// largest |y| is the largest |s w| times r: one reduction gives the norm and the
// 8-bit scale.  Bound by memory: 32768 x 4096 with a residual, sum and y 181 us, 5.9
// TB/s; 6007 x 2048 in 8 bits 16 us, 5.4; one row of 4096 3.3, a launch's latency.
template <int THREADS, int LOADS>
__global__ __launch_bounds__(group_of<THREADS>) void rms_norm_kernel(NormArgs a) {
  constexpr int PER = group_of<THREADS> / THREADS;  // rows of a workgroup
  __shared__ float red_a[16];
  __shared__ uint32_t red_m[16];
  const int t = threadIdx.x % THREADS, row = blockIdx.x * PER + threadIdx.x / THREADS;
  const bool some = row < a.T;
  const size_t at = (size_t)row * a.H;
  u32x4_t s[LOADS], r[LOADS], w[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int c = (t + i * THREADS) * 8;
    const bool in = some && c < a.H;
    s[i] = in ? *reinterpret_cast<const u32x4_t*>(a.x + at + c) : u32x4_t{0, 0, 0, 0};
    r[i] = in && a.residual ? *reinterpret_cast<const u32x4_t*>(a.residual + at + c) : u32x4_t{0, 0, 0, 0};
    w[i] = in ? *reinterpret_cast<const u32x4_t*>(a.weight + c) : u32x4_t{0, 0, 0, 0};
  }
  float squares = 0;
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    float v[8], g[8];
    tile::unpack8(s[i], v);
    if (a.residual) {
      tile::unpack8(r[i], g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += g[j];
      s[i] = tile::pack8(v);
      tile::unpack8(s[i], v);
    }
    tile::unpack8(w[i], g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      squares += v[j] * v[j];
      most = max(most, __float_as_uint(v[j] * g[j]) & 0x7fffffffu);
    }
  }
  reduce<THREADS>(squares, most, red_a, red_m);
  if (!some) return;
  const float rstd = 1.0f / sqrtf(squares / a.H + a.eps);
  float scale = 0;
  if (a.q) {
    scale = __uint_as_float(most) * rstd;
    scale = scale < __builtin_inff() ? scale / 127.0f : __builtin_nanf("");
  }
  if (t == 0) {
    if (a.rstd) a.rstd[row] = rstd;
    if (a.q) a.scale[row] = scale;
  }
  const bool zero = !(scale > 0.0f);
  const Quantizer quant(scale);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int c = (t + i * THREADS) * 8;
    if (c >= a.H) break;
    if (a.sum) *reinterpret_cast<u32x4_t*>(a.sum + at + c) = s[i];
    float v[8], g[8];
    tile::unpack8(s[i], v);
    tile::unpack8(w[i], g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * g[j] * rstd;
    if (a.y) *reinterpret_cast<u32x4_t*>(a.y + at + c) = tile::pack8(v);
    if (a.q) {
      uint32_t p[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        p[j] = zero ? 0u
                    : (uint32_t)(quant(v[4 * j]) & 255) | (uint32_t)(quant(v[4 * j + 1]) & 255) << 8 |
                          (uint32_t)(quant(v[4 * j + 2]) & 255) << 16 | (uint32_t)quant(v[4 * j + 3]) << 24;
      *reinterpret_cast<uint2*>(a.q + at + c) = uint2{p[0], p[1]};
    }
  }
}

// dx row by row, and each workgroup's part of dweight over its rows: bound by memory,
// so the next row's loads are under way while a row is worked on.  32768 x 4096 with
// dsum 179 to 212 us by a trace, 186 with the next kernel's 5 in a row of calls, 5.8 TB/s
// (without the next row's loads 200 to 215 by a trace); 333 x 1000 3.5 and 3.0.
template <int THREADS, int LOADS>
__global__ __launch_bounds__(group_of<THREADS>) void rms_norm_grad_kernel(NormGradArgs a) {
  constexpr int PER = group_of<THREADS> / THREADS, W = THREADS * LOADS * 8;
  constexpr bool AHEAD = THREADS < 1024;  // (1024 threads have no registers for two rows: 222 us against 202, 8192 x 16384)
  __shared__ float red[2][16];
  __shared__ __attribute__((aligned(16))) float sums[PER > 1 ? PER * W : 4];
  const int t = threadIdx.x % THREADS, group = threadIdx.x / THREADS;
  u32x4_t w[LOADS];
  float dw[LOADS][8] = {};
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int c = (t + i * THREADS) * 8;
    w[i] = c < a.H ? *reinterpret_cast<const u32x4_t*>(a.weight + c) : u32x4_t{0, 0, 0, 0};
  }
  struct Given {  // of a row: dy, s, dsum and rstd
    u32x4_t d[LOADS], s[LOADS], more[LOADS];
    float r;
  };
  const auto load = [&](Given& g, int row) {
    const bool some = row < a.T;
    const size_t at = (size_t)row * a.H;
    g.r = some ? a.rstd[row] : 0.0f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c = (t + i * THREADS) * 8;
      const bool in = some && c < a.H;
      g.d[i] = in ? *reinterpret_cast<const u32x4_t*>(a.dy + at + c) : u32x4_t{0, 0, 0, 0};
      g.s[i] = in ? *reinterpret_cast<const u32x4_t*>(a.sum + at + c) : u32x4_t{0, 0, 0, 0};
      g.more[i] = in && a.dsum ? *reinterpret_cast<const u32x4_t*>(a.dsum + at + c) : u32x4_t{0, 0, 0, 0};
    }
  };
  int turn = 0;  // two sets of slots in turn: one barrier a row
  Given next;
  if (AHEAD) load(next, blockIdx.x * PER + group);
  for (int row0 = blockIdx.x * PER; row0 < a.T; row0 += a.parts * PER, turn ^= 1) {
    const int row = row0 + group;
    if (!AHEAD) load(next, row);
    const Given g = next;
    if (AHEAD) load(next, row + a.parts * PER);
    float dot = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      float dv[8], sv[8], wv[8];
      tile::unpack8(g.d[i], dv);
      tile::unpack8(g.s[i], sv);
      tile::unpack8(w[i], wv);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = sv[j] * g.r;
        dw[i][j] += dv[j] * n;
        dot += dv[j] * wv[j] * n;
      }
    }
    if (!a.dx) continue;
    const float c0 = sum_of<THREADS>(dot, red[turn]) / a.H;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c = (t + i * THREADS) * 8;
      if (row >= a.T || c >= a.H) break;
      float dv[8], sv[8], wv[8];
      tile::unpack8(g.d[i], dv);
      tile::unpack8(g.s[i], sv);
      tile::unpack8(w[i], wv);
#pragma unroll
      for (int j = 0; j < 8; ++j) dv[j] = g.r * (dv[j] * wv[j] - sv[j] * g.r * c0);
      if (a.dsum) {
        tile::unpack8(g.more[i], sv);
#pragma unroll
        for (int j = 0; j < 8; ++j) dv[j] += sv[j];
      }
      *reinterpret_cast<u32x4_t*>(a.dx + (size_t)row * a.H + c) = tile::pack8(dv);
    }
  }
  if (!a.dweight) return;
  float* part = a.part + (size_t)blockIdx.x * a.H;
  if constexpr (PER > 1) {  // the groups' sums first
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<f32x4_t*>(sums + group * W + (t + i * THREADS) * 8 + j) =
            f32x4_t{dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]};
    __syncthreads();
    for (int c = threadIdx.x * 4; c < a.H; c += group_of<THREADS> * 4) {
      f32x4_t v = *reinterpret_cast<const f32x4_t*>(sums + c);
#pragma unroll
      for (int i = 1; i < PER; ++i) v += *reinterpret_cast<const f32x4_t*>(sums + i * W + c);
      *reinterpret_cast<f32x4_t*>(part + c) = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c = (t + i * THREADS) * 8;
      if (c >= a.H) break;
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<f32x4_t*>(part + c + j) = f32x4_t{dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]};
    }
  }
}

// The parts' sum in a fixed order: 32 columns a workgroup, 8 threads side by side
// and 128 groups of them that take the parts in turn.
__global__ __launch_bounds__(1024) void rms_norm_dweight_kernel(NormGradArgs a) {
  __shared__ f32x4_t red[128][8];
  const int c = blockIdx.x * 32 + threadIdx.x % 8 * 4, first = threadIdx.x / 8;
  f32x4_t v{0, 0, 0, 0};
  if (c < a.H) {
#pragma unroll 8
    for (int i = first; i < a.parts; i += 128) v += *reinterpret_cast<const f32x4_t*>(a.part + (size_t)i * a.H + c);
  }
  red[first][threadIdx.x % 8] = v;
#pragma unroll
  for (int n = 64; n; n >>= 1) {
    __syncthreads();
    if (first < n) red[first][threadIdx.x % 8] += red[first + n][threadIdx.x % 8];
  }
  if (first == 0 && c < a.H) *reinterpret_cast<f32x4_t*>(a.dweight + c) = red[0][threadIdx.x % 8];
}

// fn(constants THREADS and LOADS) for rows of H values
template <typename Fn>
void for_width(int H, Fn&& fn) {
  using std::integral_constant;
  if (H <= 128) fn(integral_constant<int, 16>(), integral_constant<int, 1>());
  else if (H <= 512) fn(integral_constant<int, 64>(), integral_constant<int, 1>());
  else if (H <= 1024) fn(integral_constant<int, 64>(), integral_constant<int, 2>());
  else if (H <= 2048) fn(integral_constant<int, 256>(), integral_constant<int, 1>());
  else if (H <= 4096) fn(integral_constant<int, 256>(), integral_constant<int, 2>());
  else if (H <= 8192) fn(integral_constant<int, 512>(), integral_constant<int, 2>());
  else fn(integral_constant<int, 1024>(), integral_constant<int, 2>());
}

// Workgroups of the backward pass, each with a part of dweight's sum: as many as
// load 6 MB of rows at once (dy, s and dsum), whole rounds of 256 CUs (32768 x 1000 in
// 262 workgroups 69 us, in 256 51).  More cost their parts'
// way out and back.  In 256, 512, 1024 and 2048 workgroups, us: 32768 x 4096 185, 197,
// 221 and 220; 32768 x 2048 129, 97, 106 and 114; 65536 x 512 67, 48, 52 and 55; 262144
// x 64 58, 39, 30 and 33.
int grad_parts(int T, int H) {
  int per = 1;
  for_width(H, [&](auto threads, auto) { per = group_of<threads()> / threads(); });
  return std::min(ceil_div(T, per), std::clamp((1 << 20) / (per * H) / 256, 1, 4) * 256);
}

moe_status check_cfg(const moe_rms_norm_config* c) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  if (c->rows < 0 || c->rows > (1 << 22)) return fail(MOE_ERR_INVALID_ARG, "rows must be in [0, 2^22]");
  if (c->hidden < 8 || c->hidden % 8 || c->hidden > 16384)
    return fail(MOE_ERR_INVALID_ARG, "hidden must be a multiple of 8 in [8, 16384]");
  if (c->rows == 1 << 22 && c->hidden > 8192)  // (1024 threads each: a launch has fewer than 2^32)
    return fail(MOE_ERR_INVALID_ARG, "rows must be below 2^22 where hidden is above 8192");
  if (!(c->eps > 0.0f) || !(c->eps < __builtin_inff())) return fail(MOE_ERR_INVALID_ARG, "eps must be above 0 and finite");
  return MOE_OK;
}

size_t ws_size(const moe_rms_norm_config* c) {
  return 256 + sizeof(float) * (size_t)grad_parts(c->rows, c->hidden) * c->hidden;
}

}  // namespace

extern "C" {

moe_status moe_rms_norm_forward(const moe_rms_norm_config* cfg, const uint16_t* x, const uint16_t* residual,
                                const uint16_t* weight, uint16_t* sum, float* rstd, uint16_t* y, int8_t* q,
                                float* scale, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!x || !weight) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!y && !q) return fail(MOE_ERR_INVALID_ARG, "y or q is wanted, or both");
  if (y && y == sum) return fail(MOE_ERR_INVALID_ARG, "y and sum are the same");
  if (!q != !scale) return fail(MOE_ERR_INVALID_ARG, "q and scale are wanted both or neither");
  for (const void* p : {(const void*)x, (const void*)residual, (const void*)weight, (const void*)sum, (const void*)rstd,
                        (const void*)y, (const void*)q, (const void*)scale})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  const NormArgs a{cfg->rows, cfg->hidden, cfg->eps, x, residual, weight, sum, y, rstd, q, scale};
  for_width(a.H, [&](auto threads, auto loads) {
    constexpr int group = group_of<threads()>;
    rms_norm_kernel<threads(), loads()>
        <<<ceil_div(a.T, group / threads()), group, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  });
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_rms_norm_workspace_size(const moe_rms_norm_config* cfg, size_t* bytes) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = ws_size(cfg);
  return MOE_OK;
}

moe_status moe_rms_norm_backward(const moe_rms_norm_config* cfg, const uint16_t* dy, const uint16_t* dsum,
                                 const uint16_t* sum, const uint16_t* weight, const float* rstd, uint16_t* dx,
                                 float* dweight, void* ws, size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows > 0 && (!dy || !sum || !weight || !rstd)) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  for (const void* p : {(const void*)dy, (const void*)dsum, (const void*)sum, (const void*)weight, (const void*)rstd,
                        (const void*)dx, (const void*)dweight})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if (!ws || ws_bytes < ws_size(cfg))
    return fail(MOE_ERR_INVALID_ARG, "the workspace holds %zu of %zu bytes", ws ? ws_bytes : 0, ws_size(cfg));
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MOE_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  NormGradArgs a{cfg->rows, cfg->hidden, dy, dsum, sum, weight, rstd, dx, dweight, static_cast<float*>(ws),
                 grad_parts(cfg->rows, cfg->hidden)};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (a.T > 0 && (dx || dweight))
    for_width(a.H, [&](auto threads, auto loads) {
      constexpr int group = group_of<threads()>;
      rms_norm_grad_kernel<threads(), loads()><<<a.parts, group, 0, s>>>(a);
    });
  if (dweight) rms_norm_dweight_kernel<<<ceil_div(a.H, 32), 1024, 0, s>>>(a);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
