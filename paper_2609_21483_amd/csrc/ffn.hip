// The gated feed-forward block over row groups and its backward pass (moe.h).
#include <hip/hip_runtime.h>

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
};

__device__ __forceinline__ const char* bytes(const uint16_t* p) { return reinterpret_cast<const char*>(p); }
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4_t*>(p) = tile::pack8(v);
}

// Forms of the tile: x W (weights transposed), d W^T, and x^T d
template <typename S>
using XW = tile::Tile<S, false, false, true>;
template <typename S>
using XWT = tile::Tile<S, false, false, false>;
template <typename S>
using XTD = tile::Tile<S, false, true, true>;

// h = act(x W1) * (x W3), and gate and up where they are kept
template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void ffn_up_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  constexpr int COLS = Tl::BN / 2;
  int m, n;
  if (!tile::pick(list.total, ceil_div(a.F, COLS), &m, &n)) return;
  const RowTile rt = list.at(m);
  const int n0 = n * COLS, rows = rt.end - rt.begin;
  const size_t wo = (size_t)rt.group * a.H * a.F;
  const tile::Operand A{bytes(a.x + (size_t)rt.begin * a.H), nullptr, (uint32_t)a.H * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.w1 + wo), bytes(a.w3 + wo), (uint32_t)a.F * 2, 0, n0, a.F};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.H, A, B, 0);
  Tl::template epilogue<true>(acc, lds, rows, [&](int r, int c, const uint32_t (&v)[16]) {
    if (n0 + c >= a.F) return;
    const size_t at = (size_t)(rt.begin + r) * a.F + n0 + c;
    float g[8], u[8], h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] = __uint_as_float(v[i]);
      u[i] = __uint_as_float(v[8 + i]);
      h[i] = act_of(g[i], a.act) * u[i];
    }
    store8(a.h + at, h);
    if (a.kgate) {
      store8(a.kgate + at, g);
      store8(a.kup + at, u);
    }
  });
}

// y = h W2
template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void ffn_down_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  int m, n;
  if (!tile::pick(list.total, ceil_div(a.H, Tl::BN), &m, &n)) return;
  const RowTile rt = list.at(m);
  const int n0 = n * Tl::BN, rows = rt.end - rt.begin;
  const tile::Operand A{bytes(a.h + (size_t)rt.begin * a.F), nullptr, (uint32_t)a.F * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.w2 + (size_t)rt.group * a.F * a.H), nullptr, (uint32_t)a.H * 2, 0, n0, a.H};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.F, A, B, 0);
  Tl::template epilogue<false>(acc, lds, rows, [&](int r, int c, const uint32_t (&v)[8]) {
    if (n0 + c < a.H) store8(a.y + (size_t)(rt.begin + r) * a.H + n0 + c, __builtin_bit_cast(float[8], v));
  });
}

// dh = dy W2^T, and from it h = act(gate) * up again, d gate and d up
template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void ffn_dh_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  int m, n;
  if (!tile::pick(list.total, ceil_div(a.F, Tl::BN), &m, &n)) return;
  const RowTile rt = list.at(m);
  const int n0 = n * Tl::BN, rows = rt.end - rt.begin;
  const tile::Operand A{bytes(a.dy + (size_t)rt.begin * a.H), nullptr, (uint32_t)a.H * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.w2 + ((size_t)rt.group * a.F + n0) * a.H), nullptr, (uint32_t)a.H * 2, a.F - n0, 0, 0};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.H, A, B, 0);
  Tl::template epilogue<false>(acc, lds, rows, [&](int r, int c, const uint32_t (&v)[8]) {
    if (n0 + c >= a.F) return;
    const size_t at = (size_t)(rt.begin + r) * a.F + n0 + c;
    float g[8], u[8], h[8];
    tile::unpack8(*reinterpret_cast<const u32x4_t*>(a.gate + at), g);
    tile::unpack8(*reinterpret_cast<const u32x4_t*>(a.up + at), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s, ds;
      act_grad(g[i], a.act, &s, &ds);
      const float d = __uint_as_float(v[i]);
      h[i] = s * u[i];
      g[i] = d * u[i] * ds;
      u[i] = d * s;
    }
    store8(a.h + at, h);
    store8(a.dgate + at, g);
    store8(a.dup + at, u);
  });
}

// dx = dgate W1^T + dup W3^T, one depth of 2 F
template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void ffn_dx_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const RowTiles list(a.off, a.G, a.T, Tl::BM);
  int m, n;
  if (!tile::pick(list.total, ceil_div(a.H, Tl::BN), &m, &n)) return;
  const RowTile rt = list.at(m);
  const int n0 = n * Tl::BN, rows = rt.end - rt.begin;
  const size_t ro = (size_t)rt.begin * a.F, wo = ((size_t)rt.group * a.H + n0) * a.F;
  const uint32_t ld = (uint32_t)a.F * 2;
  const tile::Operand A{bytes(a.dgate + ro), nullptr, ld, rows, 0, 0}, A2{bytes(a.dup + ro), nullptr, ld, rows, 0, 0};
  const tile::Operand B{bytes(a.w1 + wo), nullptr, ld, a.H - n0, 0, 0}, B2{bytes(a.w3 + wo), nullptr, ld, a.H - n0, 0, 0};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.F, A2, B2, a.F);
  Tl::template epilogue<false>(acc, lds, rows, [&](int r, int c, const uint32_t (&v)[8]) {
    if (n0 + c < a.H) store8(a.dx + (size_t)(rt.begin + r) * a.H + n0 + c, __builtin_bit_cast(float[8], v));
  });
}

// dW1 = x^T dgate, dW3 = x^T dup, dW2 = h^T dy, each group's
template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void ffn_dw_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  // tiles of a group: those of dW1, of dW3, then of dW2
  const int hm = ceil_div(a.H, Tl::BM), fn = ceil_div(a.F, Tl::BN), fm = ceil_div(a.F, Tl::BM), hn = ceil_div(a.H, Tl::BN);
  const int t13 = hm * fn, per = 2 * t13 + fm * hn, chunk = gridDim.x / NXCD;
  const int t = (blockIdx.x % NXCD) * chunk + blockIdx.x / NXCD;
  if (t >= per * a.G) return;
  const int g = t / per, i = t % per, which = i / t13 < 2 ? i / t13 : 2;
  int b, e;
  group_rows(a.off, a.T, g, &b, &e);
  const uint16_t *p = which == 2 ? a.h : a.x, *q = which == 0 ? a.dgate : which == 1 ? a.dup : a.dy;
  const int M = which == 2 ? a.F : a.H, N = which == 2 ? a.H : a.F, mt = which == 2 ? fm : hm, nt = which == 2 ? hn : fn;
  const int j = i - which * t13, band = j / (tile::NEAR * nt), first = band * tile::NEAR;
  const int wide = min(tile::NEAR, mt - first), in = j - band * tile::NEAR * nt;
  const int m0 = (first + in % wide) * Tl::BM, n0 = in / wide * Tl::BN;
  const tile::Operand A{bytes(p + (size_t)b * M), nullptr, (uint32_t)M * 2, 0, m0, M};
  const tile::Operand B{bytes(q + (size_t)b * N), nullptr, (uint32_t)N * 2, 0, n0, N};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, e - b, A, B, 0);
  uint16_t* out = (which == 0 ? a.dw1 : which == 1 ? a.dw3 : a.dw2) + ((size_t)g * M + m0) * N + n0;
  Tl::template epilogue<false>(acc, lds, min(Tl::BM, M - m0), [&](int r, int c, const uint32_t (&v)[8]) {
    if (n0 + c < N) store8(out + (size_t)r * N + c, __builtin_bit_cast(float[8], v));
  });
}

// Launches on the most tiles that the groups can have
#define LAUNCH(name, form, width)                                                                       \
  template <typename S>                                                                                   \
  void launch_##name(const FfnArgs& a, hipStream_t s) {                                                 \
    using Tl = form<S>;                                                                              \
    const int g = tile::grid_of(max_row_tiles(a.T, a.G, Tl::BM), width);                                \
    ffn_##name##_kernel<Tl><<<g, Tl::THREADS, 0, s>>>(a);                                               \
  }
LAUNCH(up, XW, ceil_div(a.F, Tl::BN / 2))
LAUNCH(down, XW, ceil_div(a.H, Tl::BN))
LAUNCH(dh, XWT, ceil_div(a.F, Tl::BN))
LAUNCH(dx, XWT, ceil_div(a.H, Tl::BN))
#undef LAUNCH
template <typename S>
void launch_dw(const FfnArgs& a, hipStream_t s) {
  using Tl = XTD<S>;
  const int per = 2 * ceil_div(a.H, Tl::BM) * ceil_div(a.F, Tl::BN) + ceil_div(a.F, Tl::BM) * ceil_div(a.H, Tl::BN);
  ffn_dw_kernel<Tl><<<tile::grid_of(a.G, per), Tl::THREADS, 0, s>>>(a);
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

// Workspace: bf16 [T][F] each of h (forward), or h, dgate and dup (backward).
size_t plane(const moe_ffn_config* c) { return align_up(sizeof(uint16_t) * (size_t)c->rows * c->ffn, 256); }
size_t ws_size(const moe_ffn_config* c, bool backward) { return 256 + plane(c) * (backward ? 3 : 1); }

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

moe_status moe_ffn_forward(const moe_ffn_config* cfg, const uint16_t* x, const int32_t* group_off, const uint16_t* w1,
                           const uint16_t* w3, const uint16_t* w2, uint16_t* gate, uint16_t* up, uint16_t* y, void* ws,
                           size_t ws_bytes, void* stream) {
  moe_status st = check_cfg(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!x || !w1 || !w3 || !w2 || !y) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!group_off && cfg->n_groups > 1) return fail(MOE_ERR_INVALID_ARG, "group_off is NULL with more than one group");
  if (!gate != !up) return fail(MOE_ERR_INVALID_ARG, "gate and up are kept both or neither");
  for (const void* p : {(const void*)x, (const void*)w1, (const void*)w3, (const void*)w2, (const void*)gate,
                        (const void*)up, (const void*)y})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if ((st = check_ws(cfg, false, ws, ws_bytes)) != MOE_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FfnArgs a{};
  a.T = cfg->rows, a.H = cfg->hidden, a.F = cfg->ffn, a.G = cfg->n_groups, a.act = cfg->act;
  a.off = group_off;
  a.x = x, a.w1 = w1, a.w3 = w3, a.w2 = w2;
  a.h = static_cast<uint16_t*>(ws), a.kgate = gate, a.kup = up, a.y = y;
  launch_up<tile::Wide>(a, s);
  launch_down<tile::Wide>(a, s);
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
  if (!dw1 != !dw3 || !dw1 != !dw2) return fail(MOE_ERR_INVALID_ARG, "dw1, dw3 and dw2 are all wanted or none");
  for (const void* p : {(const void*)dy, (const void*)x, (const void*)w1, (const void*)w3, (const void*)w2,
                        (const void*)gate, (const void*)up, (const void*)dx, (const void*)dw1, (const void*)dw3,
                        (const void*)dw2})
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  if ((st = check_ws(cfg, true, ws, ws_bytes)) != MOE_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  FfnArgs a{};
  a.T = cfg->rows, a.H = cfg->hidden, a.F = cfg->ffn, a.G = cfg->n_groups, a.act = cfg->act;
  a.off = group_off;
  a.x = x, a.w1 = w1, a.w3 = w3, a.w2 = w2, a.gate = gate, a.up = up, a.dy = dy;
  char* at = static_cast<char*>(ws);
  a.h = reinterpret_cast<uint16_t*>(at);
  a.dgate = reinterpret_cast<uint16_t*>(at + plane(cfg));
  a.dup = reinterpret_cast<uint16_t*>(at + 2 * plane(cfg));
  a.dx = dx, a.dw1 = dw1, a.dw3 = dw3, a.dw2 = dw2;
  if (a.T > 0 && (dx || dw1)) {
    launch_dh<tile::Wide>(a, s);
    if (dx) launch_dx<tile::Wide>(a, s);
  }
  if (dw1) launch_dw<tile::Wide>(a, s);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
