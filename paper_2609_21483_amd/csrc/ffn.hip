// The gated feed-forward block over row groups and its backward pass (moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "blocks.h"
#include "tile.h"

using namespace moe;

namespace {

struct FfnArgs {
  int T, H, F, G, act;
  const int32_t* off;
  const uint16_t *x, *w1, *w3, *w2, *gate, *up, *dy;
  uint16_t *h, *dgate, *dup;       // workspace
  uint16_t *kgate, *kup, *y;       // forward's outputs (kgate and kup may be NULL)
  uint16_t *dx, *dw1, *dw3, *dw2;  // backward's (dx, or the three dw, may be NULL)
  float* part;                     // partial sums [split][T][width] of a split product
  int split;
  float* dw_part;                  // and [dw_split][3][G][H F] of the weights' gradients
  int dw_split;
  int dx_blocks;                   // workgroups of dx, before those of the weights' gradients
};

__device__ __forceinline__ const char* bytes(const uint16_t* p) { return reinterpret_cast<const char*>(p); }

// The four products over rows.  UP: h = act(x W1) * (x W3), DOWN: y = h W2,
// DH: dh = dy W2^T and what follows from it, DX: dx = dgate W1^T + dup W3^T
// (one depth of 2 F).
enum Op { UP, DOWN, DH, DX };

template <Op OP>
constexpr bool GATED = OP == UP;
// columns of the output, depth, and columns of the partial sums
template <Op OP>
__host__ __device__ inline int cols_of(const FfnArgs& a) { return OP == UP || OP == DH ? a.F : a.H; }
template <Op OP>
__host__ __device__ inline int depth_of(const FfnArgs& a) { return OP == DOWN ? a.F : OP == DX ? 2 * a.F : a.H; }
template <Op OP>
__host__ __device__ inline int sums_of(const FfnArgs& a) { return OP == UP ? 2 * a.F : cols_of<OP>(a); }

__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4_t*>(p) = tile::pack8(v);
}

// 8 columns of a row from their fp32 sums (UP: v[8..15] the up projection's).
// h, d gate and d up are rounded to bf16 for the matrix instructions that take
// them: 2^-8 of each value at most, which their products' sums average out.
template <Op OP>
__device__ __forceinline__ void finish(const FfnArgs& a, size_t row, int col, const float* v) {
  const size_t at = row * cols_of<OP>(a) + col;
  float p[8], q[8], r[8];
  if constexpr (OP == UP) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = v[i];
      q[i] = v[8 + i];
      r[i] = act_of(p[i], a.act) * q[i];
    }
    store8(a.h + at, r);
    if (a.kgate) {
      store8(a.kgate + at, p);
      store8(a.kup + at, q);
    }
  } else if constexpr (OP == DH) {
    tile::unpack8(*reinterpret_cast<const u32x4_t*>(a.gate + at), p);
    tile::unpack8(*reinterpret_cast<const u32x4_t*>(a.up + at), q);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s, ds;
      act_grad(p[i], a.act, &s, &ds);
      r[i] = s * q[i];
      p[i] = v[i] * q[i] * ds;
      q[i] = v[i] * s;
    }
    store8(a.h + at, r);
    store8(a.dgate + at, p);
    store8(a.dup + at, q);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = v[i];
    store8((OP == DOWN ? a.y : a.dx) + at, p);
  }
}

// The same, or the partial sums where the product is split.
template <Op OP>
__device__ __forceinline__ void put(const FfnArgs& a, int part, size_t row, int col, const uint32_t* v) {
  constexpr int N = GATED<OP> ? 16 : 8;
  if (a.split > 1) {
    float* p = a.part + ((size_t)part * a.T + row) * sums_of<OP>(a) + col;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *reinterpret_cast<u32x4_t*>(p + i / 2 * a.F + i % 2 * 4) = u32x4_t{v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]};
    return;
  }
  float f[N];
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = __uint_as_float(v[i]);
  finish<OP>(a, row, col, f);
}

// Operands of a tile: rows of A from depth k on (elements), and W's columns
// from n0 on.  UP and DOWN read the weights transposed, DH and DX as they lie.
template <Op OP>
__device__ __forceinline__ tile::Operand rows_op(const FfnArgs& a, const RowTile& rt, int k) {
  const uint16_t* p = OP == UP ? a.x : OP == DOWN ? a.h : OP == DH ? a.dy : k < a.F ? a.dgate : a.dup - a.F;
  const int ld = OP == DX ? a.F : depth_of<OP>(a);
  return {bytes(p + (size_t)rt.begin * ld + k), nullptr, (uint32_t)ld * 2, rt.end - rt.begin, 0, 0};
}
template <Op OP>
__device__ __forceinline__ tile::Operand weights_op(const FfnArgs& a, const RowTile& rt, int k, int n0) {
  const size_t wo = (size_t)rt.group * a.H * a.F;
  if constexpr (OP == UP) {
    const size_t at = wo + (size_t)k * a.F;
    return {bytes(a.w1 + at), bytes(a.w3 + at), (uint32_t)a.F * 2, 0, n0, a.F};
  } else if constexpr (OP == DOWN) {
    return {bytes(a.w2 + wo + (size_t)k * a.H), nullptr, (uint32_t)a.H * 2, 0, n0, a.H};
  } else if constexpr (OP == DH) {
    return {bytes(a.w2 + wo + (size_t)n0 * a.H + k), nullptr, (uint32_t)a.H * 2, a.F - n0, 0, 0};
  } else {
    const uint16_t* w = k < a.F ? a.w1 : a.w3 - a.F;
    return {bytes(w + wo + (size_t)n0 * a.F + k), nullptr, (uint32_t)a.F * 2, a.H - n0, 0, 0};
  }
}

// The product OP's tile of workgroup `block`.  8192 rows, H = 4096, F = 14336:
// UP 1640 us (1.17 PFLOP/s), DOWN 770 (1.25), DH 970 (0.99, with three planes
// written), DX and the weights' gradients 3800 (1.27): see tile.h for what
// bounds them.  DH over 32 groups of 16384 rows, H = 2048, F = 768: 240 Wide
// tiles in one round, 102 us, of which the planes that all of them read and
// write at the end are a third.
template <Op OP, typename S>
__device__ __forceinline__ void rows_tile(const FfnArgs& a, int block, char* lds) {
  using Tl = tile::Tile<S, false, false, OP == UP || OP == DOWN>;
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  constexpr int COLS = GATED<OP> ? Tl::BN / 2 : Tl::BN;
  const int nt = ceil_div(cols_of<OP>(a), COLS), stages = depth_of<OP>(a) / 64;
  int m, n;
  if (!tile::pick(block, list.total, nt * a.split, &m, &n)) return;
  const RowTile rt = list.at(m);
  const int part = n / nt, n0 = n % nt * COLS, rows = rt.end - rt.begin;
  const int k0 = stages * part / a.split * 64, k1 = stages * (part + 1) / a.split * 64;
  // DX: the depth's second half is another pair of operands
  const int mid = OP == DX ? min(max(k0, a.F), k1) : k1;
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, rows_op<OP>(a, rt, k0), weights_op<OP>(a, rt, k0, n0), mid - k0, rows_op<OP>(a, rt, mid),
          weights_op<OP>(a, rt, mid, n0), k1 - mid);
  Tl::template epilogue<GATED<OP>>(acc, lds, rows, [&](int r, int c, const auto& v) {
    if (n0 + c < cols_of<OP>(a)) put<OP>(a, part, rt.begin + r, n0 + c, v);
  });
}

template <typename S>
constexpr int LDS_OF = tile::Tile<S, false, false, false>::LDS;

template <Op OP, typename S>
__global__ __launch_bounds__(S::THREADS) void ffn_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[LDS_OF<S>];
  rows_tile<OP, S>(a, blockIdx.x, lds);
}

template <Op OP, int NW>
using FewOf = tile::Few<NW, false, true, GATED<OP>>;

// One row, H = 4096, F = 14336: UP 48 us (4.9 TB/s of weights), DOWN 27 + 4 (4.3);
// 61 rows in 32 groups, H = 2048, F = 768: 36 + 17.
template <Op OP, int NW>
__global__ __launch_bounds__(NW * 64) void ffn_few_kernel(FfnArgs a) {
  using Fw = FewOf<OP, NW>;
  __shared__ __attribute__((aligned(1024))) char lds[Fw::LDS];
  const RowTiles list(a.off, a.G, a.T, Fw::BM);
  const int nt = cols_of<OP>(a) / Fw::COLS, steps = depth_of<OP>(a) / Fw::KE;
  int m, n;
  if (!tile::pick(blockIdx.x, list.total, nt * a.split, &m, &n)) return;
  const RowTile rt = list.at(m);
  const int part = n / nt, n0 = n % nt * Fw::COLS;
  Fw::run(lds, rows_op<OP>(a, rt, 0), weights_op<OP>(a, rt, 0, n0), steps * part / a.split, steps * (part + 1) / a.split,
          rt.tiles == 1, [&](int r, int c, const auto& v) { put<OP>(a, part, rt.begin + r, n0 + c, v); });
}

// The partial sums of a split product, added in order: bound by their bytes
// (dh of 2000 rows, F = 4096, two parts 27 us, 5.5 TB/s with the planes).
template <Op OP>
__global__ __launch_bounds__(256) void ffn_sum_kernel(FfnArgs a) {
  int b, e;
  covered_rows(a.off, a.G, a.T, &b, &e);
  const int width = cols_of<OP>(a);
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8, row = i / width, c = i % width;
  if (row < b || row >= e) return;
  float v[GATED<OP> ? 16 : 8] = {};
  for (int s = 0; s < a.split; ++s) {
    const float* at = a.part + ((size_t)s * a.T + row) * sums_of<OP>(a) + c;
#pragma unroll
    for (int j = 0; j < (GATED<OP> ? 16 : 8); ++j) v[j] += at[j / 8 * a.F + j % 8];
  }
  finish<OP>(a, row, (int)c, v);
}

// dW1 = x^T dgate, dW3 = x^T dup, dW2 = h^T dy, each group's: its rows are the
// depth, in stages of 64; a split takes runs of whole stages.
template <typename S>
__device__ __forceinline__ void dw_tile(const FfnArgs& a, int block, char* lds) {
  using Tl = tile::Tile<S, false, true, true>;
  static_assert(Tl::LDS <= LDS_OF<S>, "LDS");
  // Tiles of a group: those of dW1, of dW3, then of dW2.  Groups differ in
  // depth, so each XCD takes an eighth of every group's, and up to 64 groups
  // are taken in the order of their depths, the deepest first.  32 groups of 83
  // to 5286 rows, H = 2048, F = 768, us: 438 with runs of groups on each XCD,
  // 312 so; dx and these in one launch 430 -> 384 with the deepest first.
  const int hm = ceil_div(a.H, Tl::BM), fn = ceil_div(a.F, Tl::BN), fm = ceil_div(a.F, Tl::BM), hn = ceil_div(a.H, Tl::BN);
  const int t13 = hm * fn, per = 2 * t13 + fm * hn, run = ceil_div(per * a.dw_split, NXCD);
  const int slot = block / NXCD, w = block % NXCD * run + slot % run;
  if (w >= per * a.dw_split) return;
  const int part = w / per, i = w % per, which = i / t13 < 2 ? i / t13 : 2;
  int g = slot / run, b, e;
  if (a.off && a.G <= 64) g = ranked_group(a.off, a.T, a.G, g, &b, &e);
  else group_rows(a.off, a.T, g, &b, &e);
  const int stages = ceil_div(e - b, 64);
  const int k0 = stages * part / a.dw_split * 64, k1 = min(stages * (part + 1) / a.dw_split * 64, e - b);
  const uint16_t *p = which == 2 ? a.h : a.x, *q = which == 0 ? a.dgate : which == 1 ? a.dup : a.dy;
  const int M = which == 2 ? a.F : a.H, N = which == 2 ? a.H : a.F, mt = which == 2 ? fm : hm, nt = which == 2 ? hn : fn;
  const int j = i - which * t13, band = j / (tile::NEAR * nt), first = band * tile::NEAR;
  const int wide = min(tile::NEAR, mt - first), in = j - band * tile::NEAR * nt;
  const int m0 = (first + in % wide) * Tl::BM, n0 = in / wide * Tl::BN;
  const tile::Operand A{bytes(p + (size_t)(b + k0) * M), nullptr, (uint32_t)M * 2, 0, m0, M};
  const tile::Operand B{bytes(q + (size_t)(b + k0) * N), nullptr, (uint32_t)N * 2, 0, n0, N};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, k1 - k0, A, B, 0);
  const size_t at = ((size_t)g * M + m0) * N + n0, all = (size_t)a.G * a.H * a.F;
  uint16_t* out = (which == 0 ? a.dw1 : which == 1 ? a.dw3 : a.dw2) + at;
  float* sums = a.dw_part + (part * 3 + which) * all + at;
  Tl::template epilogue<false>(acc, lds, min(Tl::BM, M - m0), [&](int r, int c, const uint32_t (&v)[8]) {
    if (n0 + c >= N) return;
    if (a.dw_split > 1) {
      u32x4_t* o = reinterpret_cast<u32x4_t*>(sums + (size_t)r * N + c);
      o[0] = u32x4_t{v[0], v[1], v[2], v[3]};
      o[1] = u32x4_t{v[4], v[5], v[6], v[7]};
      return;
    }
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(v[j]);
    store8(out + (size_t)r * N + c, f);
  });
}

// dx and the weights' gradients in one launch (either may have no workgroups):
// the last tiles of the one run beside the first of the other.
template <typename S>
__global__ __launch_bounds__(S::THREADS) void ffn_grad_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[LDS_OF<S>];
  if ((int)blockIdx.x < a.dx_blocks) rows_tile<DX, S>(a, blockIdx.x, lds);
  else dw_tile<S>(a, blockIdx.x - a.dx_blocks, lds);
}

__global__ __launch_bounds__(256) void ffn_dw_sum_kernel(FfnArgs a) {
  const size_t all = (size_t)a.G * a.H * a.F, i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= 3 * all) return;
  float f[8] = {};
  for (int s = 0; s < a.dw_split; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] += a.dw_part[s * 3 * all + i + j];
  store8((i < all ? a.dw1 : i < 2 * all ? a.dw3 : a.dw2) + i % all, f);
}

// ---- host ---------------------------------------------------------------------
template <Op OP>
tile::Plan plan(const FfnArgs& a) {
  return tile::plan_of(a.T, a.G, cols_of<OP>(a), GATED<OP> ? 2 : 1, depth_of<OP>(a) / 64, OP == UP || OP == DOWN);
}
template <typename S>
int dw_tiles(const FfnArgs& a) {  // of a group
  return 2 * ceil_div(a.H, S::BM) * ceil_div(a.F, S::BN) + ceil_div(a.F, S::BM) * ceil_div(a.H, S::BN);
}
// The kind of tiles and the splits of dx and of the weights' gradients, which
// share a launch: its time is that of all their tiles, or of the deepest one
// (us per stage and per tile, and for a split, as in tile_plan).  The same
// whichever of them are asked for, so that results do not depend on it.
struct GradPlan {
  tile::Plan::Kind kind;
  int dx_split, dw_split;
};
template <typename S>
void grad_times(const FfnArgs& a, tile::Plan::Kind kind, GradPlan* best, double* least) {
  const bool wide = kind == tile::Plan::WIDE;
  const double cap = wide ? 256 : 512, busy = wide ? 2.0 : 1.25, alone = wide ? 1.85 : 1.0, over = wide ? 4 : 3;
  const double tx = tile::row_tiles(a.T, a.G, S::BM) * ceil_div(a.H, S::BN), tw = (double)a.G * dw_tiles<S>(a);
  const int sx = 2 * a.F / 64, sw = std::max(1, ceil_div(ceil_div(a.T, a.G), 64)), most = wide ? 1 : tile::MAX_SPLIT;
  for (int x = 1; x <= most && x <= sx; x *= 2)
    for (int w = 1; w <= most && w <= sw; w *= 2) {
      const int dx_stages = ceil_div(sx, x), dw_stages = ceil_div(sw, w);
      const double all = tx * x * (dx_stages * busy + over) + tw * w * (dw_stages * busy + over);
      const double deepest = std::max(dx_stages, dw_stages) * alone + 8;
      const double t = (tx * x + tw * w <= cap ? deepest : std::max(all / cap, deepest) + 0.35 * deepest) +
                       (x > 1 ? 6 + 8.0 * x * a.T * a.H / 6e6 : 0) + (w > 1 ? 6 + 24.0 * w * a.G * a.H * a.F / 6e6 : 0);
      if (t < *least) *least = t, *best = {kind, x, w};
    }
}
GradPlan grad_plan(const FfnArgs& a) {
  GradPlan p{};
  double least = 1e30;
  grad_times<tile::Wide>(a, tile::Plan::WIDE, &p, &least);
  grad_times<tile::Small>(a, tile::Plan::SMALL, &p, &least);
  return p;
}

// Launches are for the most tiles that the groups can have.
template <Op OP>
void launch(FfnArgs a, hipStream_t s) {
  const tile::Plan p = plan<OP>(a);
  a.split = p.split;
  const auto go = [&](auto kernel, int bm, int cols, int threads) {
    kernel<<<tile::grid_of(max_row_tiles(a.T, a.G, bm), ceil_div(cols_of<OP>(a), cols) * a.split), threads, 0, s>>>(a);
  };
  constexpr int per = GATED<OP> ? 2 : 1;
  if constexpr (OP == UP || OP == DOWN) {
    if (p.kind == tile::Plan::FEW4) go(ffn_few_kernel<OP, 4>, FewOf<OP, 4>::BM, FewOf<OP, 4>::COLS, FewOf<OP, 4>::THREADS);
    if (p.kind == tile::Plan::FEW8) go(ffn_few_kernel<OP, 8>, FewOf<OP, 8>::BM, FewOf<OP, 8>::COLS, FewOf<OP, 8>::THREADS);
  }
  using tile::Small, tile::Wide;
  if (p.kind == tile::Plan::SMALL) go(ffn_kernel<OP, Small>, Small::BM, Small::BN / per, Small::THREADS);
  if (p.kind == tile::Plan::WIDE) go(ffn_kernel<OP, Wide>, Wide::BM, Wide::BN / per, Wide::THREADS);
  if (a.split > 1) ffn_sum_kernel<OP><<<(int)(((long long)a.T * cols_of<OP>(a) / 8 + 255) / 256), 256, 0, s>>>(a);
}

void launch_grad(FfnArgs a, hipStream_t s) {
  const GradPlan p = grad_plan(a);
  a.split = p.dx_split, a.dw_split = p.dw_split;
  a.dw_part = a.part + (a.dx && a.split > 1 ? (size_t)a.split * a.T * a.H : 0);
  const auto go = [&](auto kernel, int bm, int bn, int threads, int tiles) {
    a.dx_blocks = a.dx ? tile::grid_of(max_row_tiles(a.T, a.G, bm), ceil_div(a.H, bn) * a.split) : 0;
    const int dw_blocks = a.dw1 ? a.G * ceil_div(tiles * a.dw_split, NXCD) * NXCD : 0;
    kernel<<<a.dx_blocks + dw_blocks, threads, 0, s>>>(a);
  };
  using tile::Small, tile::Wide;
  if (p.kind == tile::Plan::SMALL) go(ffn_grad_kernel<Small>, Small::BM, Small::BN, Small::THREADS, dw_tiles<Small>(a));
  else go(ffn_grad_kernel<Wide>, Wide::BM, Wide::BN, Wide::THREADS, dw_tiles<Wide>(a));
  if (a.dx && a.split > 1) ffn_sum_kernel<DX><<<(int)(((long long)a.T * a.H / 8 + 255) / 256), 256, 0, s>>>(a);
  if (a.dw1 && a.dw_split > 1) ffn_dw_sum_kernel<<<(int)((3LL * a.G * a.H * a.F / 8 + 255) / 256), 256, 0, s>>>(a);
}

moe_status check_cfg(const moe_ffn_config* c) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  if (c->rows < 0 || c->rows > (1 << 22)) return fail(MOE_ERR_INVALID_ARG, "rows must be in [0, 2^22]");
  if (c->hidden < 64 || c->hidden % 64 || c->hidden > 16384)
    return fail(MOE_ERR_INVALID_ARG, "hidden must be a multiple of 64 in [64, 16384]");
  if (c->ffn < 64 || c->ffn % 64 || c->ffn > 32768)
    return fail(MOE_ERR_INVALID_ARG, "ffn must be a multiple of 64 in [64, 32768]");
  if (c->n_groups < 1 || c->n_groups > MOE_MAX_GROUPS)
    return fail(MOE_ERR_INVALID_ARG, "n_groups must be in [1, %d]", MOE_MAX_GROUPS);
  if (c->act != MOE_ACT_SILU && c->act != MOE_ACT_GELU)
    return fail(MOE_ERR_INVALID_ARG, "act must be MOE_ACT_SILU or MOE_ACT_GELU");
  return MOE_OK;
}

FfnArgs args_of(const moe_ffn_config* c, const int32_t* off) {
  FfnArgs a{};
  a.T = c->rows, a.H = c->hidden, a.F = c->ffn, a.G = c->n_groups, a.act = c->act;
  a.off = off;
  return a;
}

// Workspace: bf16 [T][F] each of h (forward), or h, dgate and dup (backward);
// then the partial sums of the products that are split, one after the other.
size_t plane(const moe_ffn_config* c) { return align_up(sizeof(uint16_t) * (size_t)c->rows * c->ffn, 256); }
template <Op OP>
size_t part_bytes(const FfnArgs& a) {
  const int s = plan<OP>(a).split;
  return s > 1 ? sizeof(float) * (size_t)s * a.T * sums_of<OP>(a) : 0;
}
size_t ws_size(const moe_ffn_config* c, bool backward) {
  const FfnArgs a = args_of(c, nullptr);
  if (!backward) return 256 + plane(c) + std::max(part_bytes<UP>(a), part_bytes<DOWN>(a));
  const GradPlan p = grad_plan(a);
  const size_t grad = sizeof(float) * ((p.dx_split > 1 ? (size_t)p.dx_split * a.T * a.H : 0) +
                                       (p.dw_split > 1 ? 3 * (size_t)p.dw_split * a.G * a.H * a.F : 0));
  return 256 + 3 * plane(c) + std::max(part_bytes<DH>(a), grad);
}

moe_status check_ws(const moe_ffn_config* c, bool backward, const void* ws, size_t bytes) {
  const size_t need = ws_size(c, backward);
  if (!ws || bytes < need) return fail(MOE_ERR_INVALID_ARG, "the workspace holds %zu of %zu bytes", ws ? bytes : 0, need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MOE_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  return MOE_OK;
}

}  // namespace

extern "C" {

moe_status moe_ffn_workspace_size(const moe_ffn_config* cfg, int32_t backward, size_t* bytes) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = ws_size(cfg, backward != 0);
  return MOE_OK;
}

moe_status moe_ffn_plan_host(const moe_ffn_config* cfg, moe_ffn_plan* out) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (!out) return fail(MOE_ERR_INVALID_ARG, "out is NULL");
  const FfnArgs a = args_of(cfg, nullptr);
  const auto of = [](const tile::Plan& p) { return moe_product_plan{p.kind, p.split}; };
  const GradPlan g = grad_plan(a);
  *out = {of(plan<UP>(a)), of(plan<DOWN>(a)), of(plan<DH>(a)), {g.kind, g.dx_split}, {g.kind, g.dw_split}};
  return MOE_OK;
}

moe_status moe_ffn_forward(const moe_ffn_config* cfg, const uint16_t* x, const int32_t* group_off, const uint16_t* w1,
                           const uint16_t* w3, const uint16_t* w2, uint16_t* gate, uint16_t* up, uint16_t* y, void* ws,
                           size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!x || !w1 || !w3 || !w2 || !y) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!group_off && cfg->n_groups > 1) return fail(MOE_ERR_INVALID_ARG, "group_off is NULL with more than one group");
  if (reinterpret_cast<uintptr_t>(group_off) % 4) return fail(MOE_ERR_INVALID_ARG, "group_off is not aligned to its values");
  if (!gate != !up) return fail(MOE_ERR_INVALID_ARG, "gate and up are kept both or neither");
  for (const void* p : {(const void*)x, (const void*)w1, (const void*)w3, (const void*)w2, (const void*)gate,
                        (const void*)up, (const void*)y})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if ((st = check_ws(cfg, false, ws, ws_bytes)) != MOE_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FfnArgs a = args_of(cfg, group_off);
  a.x = x, a.w1 = w1, a.w3 = w3, a.w2 = w2;
  a.h = static_cast<uint16_t*>(ws), a.kgate = gate, a.kup = up, a.y = y;
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + plane(cfg));
  launch<UP>(a, s);
  launch<DOWN>(a, s);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_ffn_backward(const moe_ffn_config* cfg, const uint16_t* dy, const uint16_t* x, const int32_t* group_off,
                            const uint16_t* w1, const uint16_t* w3, const uint16_t* w2, const uint16_t* gate,
                            const uint16_t* up, uint16_t* dx, uint16_t* dw1, uint16_t* dw3, uint16_t* dw2, void* ws,
                            size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  // (without rows there is no dx, but the weights' gradients are written: zeros)
  if (cfg->rows > 0 && (!dy || !x || !w1 || !w3 || !w2 || !gate || !up)) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!group_off && cfg->n_groups > 1) return fail(MOE_ERR_INVALID_ARG, "group_off is NULL with more than one group");
  if (reinterpret_cast<uintptr_t>(group_off) % 4) return fail(MOE_ERR_INVALID_ARG, "group_off is not aligned to its values");
  if (!dw1 != !dw3 || !dw1 != !dw2) return fail(MOE_ERR_INVALID_ARG, "dw1, dw3 and dw2 are all wanted or none");
  for (const void* p : {(const void*)dy, (const void*)x, (const void*)w1, (const void*)w3, (const void*)w2,
                        (const void*)gate, (const void*)up, (const void*)dx, (const void*)dw1, (const void*)dw3,
                        (const void*)dw2})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if ((st = check_ws(cfg, true, ws, ws_bytes)) != MOE_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FfnArgs a = args_of(cfg, group_off);
  a.x = x, a.w1 = w1, a.w3 = w3, a.w2 = w2, a.gate = gate, a.up = up, a.dy = dy;
  char* at = static_cast<char*>(ws);
  a.h = reinterpret_cast<uint16_t*>(at);
  a.dgate = reinterpret_cast<uint16_t*>(at + plane(cfg));
  a.dup = reinterpret_cast<uint16_t*>(at + 2 * plane(cfg));
  a.part = reinterpret_cast<float*>(at + 3 * plane(cfg));
  a.dx = dx, a.dw1 = dw1, a.dw3 = dw3, a.dw2 = dw2;
  if (a.T == 0) a.dx = nullptr;
  if (a.T > 0 && (dx || dw1)) launch<DH>(a, s);
  if (a.dx || dw1) launch_grad(a, s);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
