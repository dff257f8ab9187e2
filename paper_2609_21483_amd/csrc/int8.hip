// Products in 8-bit integers over row groups, and the quantisers that feed
// them (moe.h).
#include <hip/hip_runtime.h>

#include "blocks.h"
#include "tile.h"

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
struct I8Args {
  int T, K, N, G, act;
  const int32_t* off;
  const int8_t *x, *w;
  const float *sx, *sw;
  uint16_t* y;
};

template <typename S>
using I8 = tile::Tile<S, true, false, false>;

template <typename Tl, bool GATED>
__global__ __launch_bounds__(Tl::THREADS) void gemm_i8_kernel(I8Args a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  constexpr int COLS = GATED ? Tl::BN / 2 : Tl::BN;
  const int out = GATED ? a.N / 2 : a.N;
  int m, n;
  if (!tile::pick(list.total, ceil_div(out, COLS), &m, &n)) return;
  const RowTile rt = list.at(m);
  const int n0 = n * COLS, rows = rt.end - rt.begin;
  const char* w = reinterpret_cast<const char*>(a.w) + ((size_t)rt.group * a.N + n0) * a.K;
  const tile::Operand A{reinterpret_cast<const char*>(a.x) + (size_t)rt.begin * a.K, nullptr, (uint32_t)a.K, rows, 0, 0};
  const tile::Operand B{w, GATED ? w + (size_t)out * a.K : nullptr, (uint32_t)a.K, out - n0, 0, 0};
  const float* sw = a.sw + (size_t)rt.group * a.N + n0;
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.K, A, B, 0);
  Tl::template epilogue<GATED>(acc, lds, rows, [&](int r, int c, const auto& v) {
    if (n0 + c >= out) return;
    const float sx = a.sx[rt.begin + r];
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = (float)(int)v[i] * (sx * sw[c + i]);
      if constexpr (GATED) y[i] = act_of(y[i], a.act) * ((float)(int)v[8 + i] * (sx * sw[out + c + i]));
    }
    *reinterpret_cast<u32x4_t*>(a.y + (size_t)(rt.begin + r) * out + n0 + c) = tile::pack8(y);
  });
}

template <typename S>
void launch_gemm(const I8Args& a, hipStream_t s) {
  using Tl = I8<S>;
  const bool gated = a.act != MOE_ACT_NONE;
  const int nt = gated ? ceil_div(a.N / 2, Tl::BN / 2) : ceil_div(a.N, Tl::BN);
  const int g = tile::grid_of(max_row_tiles(a.T, a.G, Tl::BM), nt);
  (gated ? gemm_i8_kernel<Tl, true> : gemm_i8_kernel<Tl, false>)<<<g, Tl::THREADS, 0, s>>>(a);
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
  launch_gemm<tile::Wide>(a, reinterpret_cast<hipStream_t>(stream));
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
