// Products in 8-bit integers over row groups, and the quantisers that feed
// them (moe.h).
#include <hip/hip_runtime.h>

#include "blocks.h"

using namespace moe;

namespace {

// ---- quantisers -----------------------------------------------------------------
// scale = max|x| / 127 and q = rint(x / scale), both divisions IEEE fp32, so
// the same on every machine.  The maximum runs over the magnitudes' bit
// patterns, which order as the values do; infinity and NaN come out as 0x7f80
// and above.
constexpr uint32_t BF16_INF = 0x7f80;

__device__ __forceinline__ float scale_of(uint32_t amax) {
  return amax >= BF16_INF ? __builtin_nanf("") : bf16_to_f32((uint16_t)amax) / 127.0f;
}
// (a scale rounded down in the subnormal range can give a quotient above 127)
__device__ __forceinline__ int quantize(uint16_t v, float scale) {
  if (!(scale > 0.0f)) return 0;
  return (int)fminf(fmaxf(rintf(bf16_to_f32(v) / scale), -127.0f), 127.0f);
}

__global__ __launch_bounds__(256) void quantize_rows_kernel(int cols, const uint16_t* x, int8_t* q, float* scale) {
  __shared__ uint32_t red[4];
  const size_t row = blockIdx.x;
  uint32_t m = 0;
  for (int c = threadIdx.x; c < cols; c += 256) m = max(m, x[row * cols + c] & 0x7fffu);
  for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = m;
  __syncthreads();
  m = max(max(red[0], red[1]), max(red[2], red[3]));
  const float s = scale_of(m);
  if (threadIdx.x == 0) scale[row] = s;
  for (int c = threadIdx.x; c < cols; c += 256) q[row * cols + c] = (int8_t)quantize(x[row * cols + c], s);
}

// a workgroup takes 64 channels of a group: the largest magnitudes, then the
// values, transposed through LDS 64 rows of the depth at a time
__global__ __launch_bounds__(256) void quantize_weights_kernel(int K, int N, int Nq, int first, const uint16_t* w,
                                                               int8_t* wq, float* scale) {
  __shared__ uint32_t red[4][64];
  __shared__ int8_t tile[64][65];
  const int g = blockIdx.y, n0 = blockIdx.x * 64, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint16_t* wg = w + (size_t)g * K * N + n0;
  uint32_t m = 0;
  for (int k = wave; k < K; k += 4) m = max(m, wg[(size_t)k * N + lane] & 0x7fffu);
  red[wave][lane] = m;
  __syncthreads();
  m = max(max(red[0][lane], red[1][lane]), max(red[2][lane], red[3][lane]));
  const float s = scale_of(m);
  if (wave == 0) scale[(size_t)g * Nq + first + n0 + lane] = s;
  for (int k0 = 0; k0 < K; k0 += 64) {
    __syncthreads();
    for (int k = wave; k < 64; k += 4) tile[lane][k] = (int8_t)quantize(wg[(size_t)(k0 + k) * N + lane], s);
    __syncthreads();
    for (int n = wave; n < 64; n += 4) wq[((size_t)g * Nq + first + n0 + n) * K + k0 + lane] = tile[n][lane];
  }
}

// ---- the product ----------------------------------------------------------------
constexpr int TS = 64, KS = 64;

__device__ void product(int (&acc)[4][4], const int8_t* a, int rows, const int8_t* b, int cols, int K) {
  __shared__ int sa[TS][KS / 4 + 1], sb[TS][KS / 4 + 1];
  const int t = threadIdx.x, tx = t % 16, ty = t / 16;
  for (int k0 = 0; k0 < K; k0 += KS) {
    __syncthreads();
    for (int i = t; i < TS * (KS / 4); i += 256) {
      const int r = i / (KS / 4), c = i % (KS / 4);
      sa[r][c] = r < rows ? reinterpret_cast<const int*>(a + (size_t)r * K + k0)[c] : 0;
      sb[r][c] = r < cols ? reinterpret_cast<const int*>(b + (size_t)r * K + k0)[c] : 0;
    }
    __syncthreads();
    for (int k = 0; k < KS / 4; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
          for (int byte = 0; byte < 32; byte += 8)
            acc[i][j] += (int)(int8_t)(sa[ty + 16 * i][k] >> byte) * (int)(int8_t)(sb[tx + 16 * j][k] >> byte);
  }
}

struct I8Args {
  int T, K, N, G, act;
  const int32_t* off;
  const int8_t *x, *w;
  const float *sx, *sw;
  uint16_t* y;
};

__global__ __launch_bounds__(256) void gemm_i8_kernel(I8Args a) {
  RowTile rt;
  int total;
  if (!row_tile(a.off, a.G, a.T, TS, blockIdx.y, &rt, &total)) return;
  const bool gated = a.act != MOE_ACT_NONE;
  const int out = gated ? a.N / 2 : a.N, n0 = blockIdx.x * TS, rows = rt.end - rt.begin, cols = min(TS, out - n0);
  const int8_t* x = a.x + (size_t)rt.begin * a.K;
  const int8_t* w = a.w + ((size_t)rt.group * a.N + n0) * a.K;
  const float* sw = a.sw + (size_t)rt.group * a.N + n0;
  int v[4][4] = {}, u[4][4] = {};
  product(v, x, rows, w, cols, a.K);
  if (gated) product(u, x, rows, w + (size_t)out * a.K, cols, a.K);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = ty + 16 * i, n = tx + 16 * j;
      if (m >= rows || n >= cols) continue;
      const float s = a.sx[rt.begin + m];
      float r = (float)v[i][j] * (s * sw[n]);
      if (gated) r = act_of(r, a.act) * ((float)u[i][j] * (s * sw[out + n]));
      a.y[(size_t)(rt.begin + m) * out + n0 + n] = f32_to_bf16(r);
    }
}

moe_status check_cfg(const moe_gemm_i8_config* c) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  if (c->rows < 0 || c->rows > (1 << 22)) return fail(MOE_ERR_INVALID_ARG, "rows must be in [0, 2^22]");
  if (c->depth < 64 || c->depth % 64 || c->depth > 32768)
    return fail(MOE_ERR_INVALID_ARG, "depth must be a multiple of 64 in [64, 32768]");
  if (c->n_groups < 1 || c->n_groups > MOE_MAX_GROUPS)
    return fail(MOE_ERR_INVALID_ARG, "n_groups must be in [1, %d]", MOE_MAX_GROUPS);
  if (c->act != MOE_ACT_NONE && c->act != MOE_ACT_SILU && c->act != MOE_ACT_GELU)
    return fail(MOE_ERR_INVALID_ARG, "act must be a MOE_ACT_* value");
  const int step = c->act == MOE_ACT_NONE ? 8 : 16;
  if (c->channels < step || c->channels % step || c->channels > 65536)
    return fail(MOE_ERR_INVALID_ARG, "channels must be a multiple of %d in [%d, 65536]", step, step);
  return MOE_OK;
}

size_t ws_size(const moe_gemm_i8_config*) { return 256; }

}  // namespace

extern "C" {

moe_status moe_quantize_rows_i8(int32_t rows, int32_t cols, const uint16_t* x, int8_t* q, float* scale, void* stream) {
  if (rows < 0 || rows > (1 << 22)) return fail(MOE_ERR_INVALID_ARG, "rows must be in [0, 2^22]");
  if (cols < 64 || cols % 64 || cols > 32768)
    return fail(MOE_ERR_INVALID_ARG, "cols must be a multiple of 64 in [64, 32768]");
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!aligned16(x) || !aligned16(q) || !aligned16(scale))
    return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  quantize_rows_kernel<<<rows, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(cols, x, q, scale);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_quantize_weights_i8(int32_t n_groups, int32_t depth, int32_t channels, int32_t q_channels,
                                   int32_t first, const uint16_t* w, int8_t* wq, float* scale, void* stream) {
  if (n_groups < 1 || n_groups > MOE_MAX_GROUPS)
    return fail(MOE_ERR_INVALID_ARG, "n_groups must be in [1, %d]", MOE_MAX_GROUPS);
  if (depth < 64 || depth % 64 || depth > 32768)
    return fail(MOE_ERR_INVALID_ARG, "depth must be a multiple of 64 in [64, 32768]");
  if (q_channels < 64 || q_channels > 65536) return fail(MOE_ERR_INVALID_ARG, "q_channels must be in [64, 65536]");
  if (channels < 64 || channels % 64 || channels > q_channels || first < 0 || first > q_channels - channels)
    return fail(MOE_ERR_INVALID_ARG, "channels must be a multiple of 64, and [first, first + channels) in [0, q_channels)");
  if (!w || !wq || !scale) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!aligned16(w) || !aligned16(wq) || !aligned16(scale))
    return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  quantize_weights_kernel<<<dim3(channels / 64, n_groups), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(
      depth, channels, q_channels, first, w, wq, scale);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_gemm_i8_workspace_size(const moe_gemm_i8_config* cfg, size_t* bytes) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = ws_size(cfg);
  return MOE_OK;
}

moe_status moe_gemm_i8(const moe_gemm_i8_config* cfg, const int8_t* xq, const float* x_scale, const int32_t* group_off,
                       const int8_t* wq, const float* w_scale, uint16_t* y, void* ws, size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!xq || !x_scale || !wq || !w_scale || !y) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!group_off && cfg->n_groups > 1) return fail(MOE_ERR_INVALID_ARG, "group_off is NULL with more than one group");
  for (const void* p : {(const void*)xq, (const void*)x_scale, (const void*)wq, (const void*)w_scale, (const void*)y})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if (!ws || ws_bytes < ws_size(cfg))
    return fail(MOE_ERR_INVALID_ARG, "the workspace holds %zu of %zu bytes", ws ? ws_bytes : 0, ws_size(cfg));
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MOE_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  I8Args a{cfg->rows, cfg->depth, cfg->channels, cfg->n_groups, cfg->act, group_off, xq, wq, x_scale, w_scale, y};
  const int out = cfg->act == MOE_ACT_NONE ? cfg->channels : cfg->channels / 2;
  gemm_i8_kernel<<<dim3(ceil_div(out, TS), max_row_tiles(a.T, a.G, TS)), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
