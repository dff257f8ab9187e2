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

// One row by THREADS threads, held in registers: each takes LOADS pieces of 8
// values.  Bound by memory: 16384 x 14336 in 124 us, 5.7 TB/s (2 bytes read and
// 1 written per value); one row of 4096 in 3.
template <int THREADS, int LOADS>
__global__ __launch_bounds__(256) void quantize_rows_kernel(int rows, int cols, const uint16_t* x, int8_t* q, float* scale) {
  constexpr int PER = 256 / THREADS;  // rows of a workgroup
  __shared__ uint32_t red[4];
  const int t = threadIdx.x % THREADS, row = blockIdx.x * PER + threadIdx.x / THREADS;
  const bool some = row < rows;
  const uint16_t* xr = x + (size_t)row * cols;
  u32x4_t v[LOADS];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int c = (t + i * THREADS) * 8;
    v[i] = some && c < cols ? *reinterpret_cast<const u32x4_t*>(xr + c) : u32x4_t{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, max(v[i][j] & 0x7fffu, (v[i][j] >> 16) & 0x7fffu));
#pragma unroll
  for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if constexpr (THREADS > 64) {
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = m;
    __syncthreads();
    m = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  if (!some) return;
  const float s = scale_of(m);
  if (t == 0) scale[row] = s;
  const bool zero = !(s > 0.0f);
  const Quantizer quant(s);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int c = (t + i * THREADS) * 8;
    if (c >= cols) break;
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t lo = v[i][2 * j], hi = v[i][2 * j + 1];
      w[j] = zero ? 0u
                  : (uint32_t)(quant(bf16_lo(lo)) & 255) | (uint32_t)(quant(bf16_hi(lo)) & 255) << 8 |
                        (uint32_t)(quant(bf16_lo(hi)) & 255) << 16 | (uint32_t)quant(bf16_hi(hi)) << 24;
    }
    *reinterpret_cast<uint2*>(q + (size_t)row * cols + c) = uint2{w[0], w[1]};
  }
}

// Weights: 64 channels x 256 rows of the depth a workgroup, in three passes, the
// largest magnitudes of the channels (their bits gathered where the scales go;
// a maximum does not depend on the order), the values, transposed through LDS,
// and the scales.  14336 x 4096 in 62 us, 71 where other weights pass between
// (1.8 and 2.1 times what one read of them takes at 5.1 TB/s): a channel's
// values lie a row apart, so its largest is known only after the whole depth,
// and a strip of 64 channels by the depth that a workgroup would keep for its
// second pass (1.8 MB here) does not fit its LDS.
constexpr int QW_N = 64, QW_K = 256;

// what = 0: clears, 1: turns magnitudes into scales
__global__ __launch_bounds__(256) void quantize_scales_kernel(int N, int Nq, int first, float* scale, int what) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  float* p = scale + (size_t)blockIdx.y * Nq + first + n;
  *p = what ? scale_of(__float_as_uint(*p)) : 0.0f;
}

__global__ __launch_bounds__(256) void quantize_max_kernel(int K, int N, int Nq, int first, const uint16_t* w, float* scale) {
  __shared__ uint32_t red[4][QW_N];
  const int k0 = blockIdx.x * QW_K, n0 = blockIdx.y * QW_N, g = blockIdx.z;
  const int c = threadIdx.x % 8 * 8, r = threadIdx.x / 8;
  const uint16_t* p = w + ((size_t)g * K + k0) * N + n0 + c;
  u32x4_t v[QW_K / 32];
#pragma unroll
  for (int i = 0; i < QW_K / 32; ++i)
    v[i] = k0 + r + i * 32 < K ? *reinterpret_cast<const u32x4_t*>(p + (size_t)(r + i * 32) * N) : u32x4_t{0, 0, 0, 0};
  uint32_t m[8] = {};
#pragma unroll
  for (int i = 0; i < QW_K / 32; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[2 * j] = max(m[2 * j], v[i][j] & 0x7fffu);
      m[2 * j + 1] = max(m[2 * j + 1], (v[i][j] >> 16) & 0x7fffu);
    }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int d = 8; d < 64; d <<= 1) m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], d));
    if (threadIdx.x % 64 < 8) red[threadIdx.x / 64][c + j] = m[j];
  }
  __syncthreads();
  if (threadIdx.x < QW_N) {
    const int t = threadIdx.x;
    atomicMax(reinterpret_cast<uint32_t*>(scale + (size_t)g * Nq + first + n0 + t),
              max(max(red[0][t], red[1][t]), max(red[2][t], red[3][t])));
  }
}

__global__ __launch_bounds__(256) void quantize_weights_kernel(int K, int N, int Nq, int first, const uint16_t* w,
                                                               int8_t* wq, const float* scale) {
  // rows of 65 words: a wavefront's 8 channel groups x 8 words fall on 64 banks
  __shared__ uint32_t tile[QW_N][QW_K / 4 + 1];
  const int k0 = blockIdx.x * QW_K, n0 = blockIdx.y * QW_N, g = blockIdx.z;
  const int c = threadIdx.x % 8 * 8, r = threadIdx.x / 8;
  const uint16_t* p = w + ((size_t)g * K + k0) * N + n0 + c;
  const float* sc = scale + (size_t)g * Nq + first + n0 + c;
  u32x4_t v[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = i * 128 + r * 4 + j;
      v[i][j] = k0 + k < K ? *reinterpret_cast<const u32x4_t*>(p + (size_t)k * N) : u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float s = scale_of(__float_as_uint(sc[n]));
    const bool zero = !(s > 0.0f);
    const Quantizer quant(s);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t q = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q |= (uint32_t)(quant(n % 2 ? bf16_hi(v[i][j][n / 2]) : bf16_lo(v[i][j][n / 2])) & 255) << (8 * j);
      tile[c + n][i * 32 + r] = zero ? 0u : q;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QW_N * QW_K / 16 / 256; ++i) {
    const int piece = threadIdx.x + i * 256, n = piece / (QW_K / 16), k = piece % (QW_K / 16);
    if (k0 + k * 16 < K) {
      const uint32_t* t = &tile[n][k * 4];
      *reinterpret_cast<u32x4_t*>(wq + ((size_t)g * Nq + first + n0 + n) * K + k0 + k * 16) = u32x4_t{t[0], t[1], t[2], t[3]};
    }
  }
}

// ---- the product ----------------------------------------------------------------
struct I8Args {
  int T, K, N, G, act;
  const int32_t* off;
  const int8_t *x, *w;
  const float *sx, *sw;
  uint16_t* y;
  int32_t* part;  // partial sums [split][T][N] of a split product
  int split;
};

// A row's scale, times which a sum and its channel's scale are multiplied:
// mantissas (0.5 to 1) first and the powers of two in one step at the end, since
// the product of the scales, or of a sum and one of them, may leave fp32 where
// the result does not (1e25 * 1e14 * 0 is 0).  The same bits as v * (x * w)
// where nothing of that is subnormal or infinite.
struct RowScale {
  float mant;
  int exp;
  __device__ __forceinline__ explicit RowScale(float x)
      : mant(__builtin_amdgcn_frexp_mantf(x)), exp(__builtin_amdgcn_frexp_expf(x)) {}
  __device__ __forceinline__ float times(uint32_t v, float w) const {
    return __builtin_amdgcn_ldexpf((float)(int)v * (mant * __builtin_amdgcn_frexp_mantf(w)),
                                   exp + __builtin_amdgcn_frexp_expf(w));
  }
};

// 8 columns of y from their sums (gated: v[8..15] the ups'): n the column of y
template <bool GATED>
__device__ __forceinline__ void finish(const I8Args& a, size_t row, int group, int n, const uint32_t* v) {
  const int out = GATED ? a.N / 2 : a.N;
  const RowScale sx(a.sx[row]);
  const float* sw = a.sw + (size_t)group * a.N + n;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = sx.times(v[i], sw[i]);
    if constexpr (GATED) y[i] = act_of(y[i], a.act) * sx.times(v[8 + i], sw[out + i]);
  }
  *reinterpret_cast<u32x4_t*>(a.y + row * out + n) = tile::pack8(y);
}

// The same, or the partial sums where the product is split.
template <bool GATED>
__device__ __forceinline__ void put(const I8Args& a, int part, size_t row, int group, int n, const uint32_t* v) {
  if (a.split == 1) {
    finish<GATED>(a, row, group, n, v);
    return;
  }
  int32_t* p = a.part + ((size_t)part * a.T + row) * a.N + n;
#pragma unroll
  for (int i = 0; i < (GATED ? 4 : 2); ++i)
    *reinterpret_cast<u32x4_t*>(p + i / 2 * (a.N / 2) + i % 2 * 4) = u32x4_t{v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]};
}

// Operands of a tile from depth k and column n0 on
template <bool GATED>
__device__ __forceinline__ tile::Operand rows_op(const I8Args& a, const RowTile& rt, int k) {
  return {reinterpret_cast<const char*>(a.x) + (size_t)rt.begin * a.K + k, nullptr, (uint32_t)a.K, rt.end - rt.begin, 0, 0};
}
template <bool GATED>
__device__ __forceinline__ tile::Operand weights_op(const I8Args& a, const RowTile& rt, int k, int n0) {
  const int out = GATED ? a.N / 2 : a.N;
  const char* w = reinterpret_cast<const char*>(a.w) + ((size_t)rt.group * a.N + n0) * a.K + k;
  return {w, GATED ? w + (size_t)out * a.K : nullptr, (uint32_t)a.K, out - n0, 0, 0};
}

// 16384 x 14336 x 4096 in 805 us, 2.4 POP/s (Wide; calls in a row, 850 to 880 one
// by one under the profiler); 6007 rows in 16 groups, 2048 x 2816 gated, in 57 to
// 67 us by what the caches hold, 1.03 to 1.2 (Small).
template <typename S, bool GATED>
__global__ __launch_bounds__(S::THREADS) void gemm_i8_kernel(I8Args a) {
  using Tl = tile::Tile<S, true, false, false>;
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  constexpr int COLS = GATED ? Tl::BN / 2 : Tl::BN;
  const int out = GATED ? a.N / 2 : a.N, nt = ceil_div(out, COLS), stages = ceil_div(a.K, 128);
  int m, n;
  if (!tile::pick(blockIdx.x, list.total, nt * a.split, &m, &n)) return;
  const RowTile rt = list.at(m);
  const int part = n / nt, n0 = n % nt * COLS, rows = rt.end - rt.begin;
  const int k0 = stages * part / a.split * 128, k1 = min(stages * (part + 1) / a.split * 128, a.K);
  const tile::Operand A = rows_op<GATED>(a, rt, k0), B = weights_op<GATED>(a, rt, k0, n0);
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, k1 - k0, A, B, 0);
  Tl::template epilogue<GATED>(acc, lds, rows, [&](int r, int c, const auto& v) {
    if (n0 + c < out) put<GATED>(a, part, rt.begin + r, rt.group, n0 + c, v);
  });
}

// One row, 4096 x 28672 gated, in 22 us (5.3 TB/s of weights); 133 rows in 16
// groups, 1408 x 2048, in 12.
template <int NW, bool GATED>
__global__ __launch_bounds__(NW * 64) void gemm_i8_few_kernel(I8Args a) {
  using Fw = tile::Few<NW, true, false, GATED>;
  __shared__ __attribute__((aligned(1024))) char lds[Fw::LDS];
  const RowTiles list(a.off, a.G, a.T, Fw::BM);
  const int out = GATED ? a.N / 2 : a.N, nt = ceil_div(out, Fw::COLS), steps = a.K / Fw::KE;
  int m, n;
  if (!tile::pick(blockIdx.x, list.total, nt * a.split, &m, &n)) return;
  const RowTile rt = list.at(m);
  const int part = n / nt, n0 = n % nt * Fw::COLS;
  Fw::run(lds, rows_op<GATED>(a, rt, 0), weights_op<GATED>(a, rt, 0, n0), steps * part / a.split,
          steps * (part + 1) / a.split, rt.tiles == 1, [&](int r, int c, const auto& v) {
            if (n0 + c < out) put<GATED>(a, part, rt.begin + r, rt.group, n0 + c, v);
          });
}

// y from the partial sums: a wavefront takes 512 columns of a row
template <bool GATED>
__global__ __launch_bounds__(256) void gemm_i8_sum_kernel(I8Args a) {
  const int out = GATED ? a.N / 2 : a.N, i = blockIdx.x * 4 + (threadIdx.x >> 6);
  const RowTiles list(a.off, a.G, a.T, 1);
  if (i >= list.total) return;
  const RowTile rt = list.at(i);
  const int c = (blockIdx.y * 64 + (threadIdx.x & 63)) * 8;
  if (c >= out) return;
  uint32_t v[GATED ? 16 : 8] = {};
  for (int s = 0; s < a.split; ++s) {
    const int32_t* p = a.part + ((size_t)s * a.T + rt.begin) * a.N + c;
#pragma unroll
    for (int j = 0; j < (GATED ? 16 : 8); ++j) v[j] += (uint32_t)p[j / 8 * out + j % 8];
  }
  finish<GATED>(a, rt.begin, rt.group, c, v);
}

tile::Plan plan(const I8Args& a) {
  const bool gated = a.act != MOE_ACT_NONE;
  return tile::plan_of(a.T, a.G, gated ? a.N / 2 : a.N, gated ? 2 : 1, ceil_div(a.K, 128), true);
}

// Launches are for the most tiles that the groups can have.
template <bool GATED>
void launch(I8Args a, hipStream_t s) {
  const tile::Plan p = plan(a);
  a.split = p.split;
  const int out = GATED ? a.N / 2 : a.N;
  constexpr int per = GATED ? 2 : 1;
  const auto go = [&](auto kernel, int bm, int cols, int threads) {
    kernel<<<tile::grid_of(max_row_tiles(a.T, a.G, bm), ceil_div(out, cols) * a.split), threads, 0, s>>>(a);
  };
  using tile::Small, tile::Wide;
  using F4 = tile::Few<4, true, false, GATED>;
  using F8 = tile::Few<8, true, false, GATED>;
  switch (p.kind) {
    case tile::Plan::FEW4: go(gemm_i8_few_kernel<4, GATED>, F4::BM, F4::COLS, F4::THREADS); break;
    case tile::Plan::FEW8: go(gemm_i8_few_kernel<8, GATED>, F8::BM, F8::COLS, F8::THREADS); break;
    case tile::Plan::SMALL: go(gemm_i8_kernel<Small, GATED>, Small::BM, Small::BN / per, Small::THREADS); break;
    case tile::Plan::WIDE: go(gemm_i8_kernel<Wide, GATED>, Wide::BM, Wide::BN / per, Wide::THREADS); break;
  }
  if (a.split > 1) gemm_i8_sum_kernel<GATED><<<dim3(ceil_div(a.T, 4), ceil_div(out, 512)), 256, 0, s>>>(a);
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

I8Args args_of(const moe_gemm_i8_config* c) {
  I8Args a{};
  a.T = c->rows, a.K = c->depth, a.N = c->channels, a.G = c->n_groups, a.act = c->act;
  return a;
}

// Workspace: the partial sums of a split product, int32 [split][T][N].
size_t ws_size(const moe_gemm_i8_config* c) {
  const int s = plan(args_of(c)).split;
  return 256 + (s > 1 ? sizeof(int32_t) * (size_t)s * c->rows * c->channels : 0);
}

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
  // rows of up to 1024 values are a wavefront's each, four to a workgroup
  const auto kernel = cols <= 512     ? quantize_rows_kernel<64, 1>
                      : cols <= 1024  ? quantize_rows_kernel<64, 2>
                      : cols <= 2048  ? quantize_rows_kernel<256, 1>
                      : cols <= 4096  ? quantize_rows_kernel<256, 2>
                      : cols <= 8192  ? quantize_rows_kernel<256, 4>
                      : cols <= 16384 ? quantize_rows_kernel<256, 8>
                                      : quantize_rows_kernel<256, 16>;
  const int per = cols <= 1024 ? 4 : 1;
  kernel<<<ceil_div(rows, per), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(rows, cols, x, q, scale);
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
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 all(ceil_div(depth, QW_K), channels / QW_N, n_groups), each(ceil_div(channels, 256), n_groups);
  quantize_scales_kernel<<<each, 256, 0, s>>>(channels, q_channels, first, scale, 0);
  quantize_max_kernel<<<all, 256, 0, s>>>(depth, channels, q_channels, first, w, scale);
  quantize_weights_kernel<<<all, 256, 0, s>>>(depth, channels, q_channels, first, w, wq, scale);
  quantize_scales_kernel<<<each, 256, 0, s>>>(channels, q_channels, first, scale, 1);
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

moe_status moe_gemm_i8_plan_host(const moe_gemm_i8_config* cfg, moe_product_plan* out) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (!out) return fail(MOE_ERR_INVALID_ARG, "out is NULL");
  const tile::Plan p = plan(args_of(cfg));
  *out = {p.kind, p.split};
  return MOE_OK;
}

moe_status moe_gemm_i8(const moe_gemm_i8_config* cfg, const int8_t* xq, const float* x_scale, const int32_t* group_off,
                       const int8_t* wq, const float* w_scale, uint16_t* y, void* ws, size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!xq || !x_scale || !wq || !w_scale || !y) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!group_off && cfg->n_groups > 1) return fail(MOE_ERR_INVALID_ARG, "group_off is NULL with more than one group");
  if (reinterpret_cast<uintptr_t>(group_off) % 4) return fail(MOE_ERR_INVALID_ARG, "group_off is not aligned to its values");
  for (const void* p : {(const void*)xq, (const void*)x_scale, (const void*)wq, (const void*)w_scale, (const void*)y})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if (!ws || ws_bytes < ws_size(cfg))
    return fail(MOE_ERR_INVALID_ARG, "the workspace holds %zu of %zu bytes", ws ? ws_bytes : 0, ws_size(cfg));
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MOE_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  I8Args a = args_of(cfg);
  a.off = group_off;
  a.x = xq, a.w = wq, a.sx = x_scale, a.sw = w_scale, a.y = y;
  a.part = static_cast<int32_t*>(ws);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  a.act == MOE_ACT_NONE ? launch<false>(a, s) : launch<true>(a, s);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
