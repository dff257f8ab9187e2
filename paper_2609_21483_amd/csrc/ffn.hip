// The gated feed-forward block over row groups and its backward pass (moe.h).
#include <hip/hip_runtime.h>

#include "blocks.h"

using namespace moe;

namespace {

constexpr int TS = 64, KS = 16;  // tile and depth step

// acc[i][j] += sum_k a(m0 + ty + 16 i, k) b(k, n0 + tx + 16 j) over [0, Kd)
template <typename LA, typename LB>
__device__ void product(float (&acc)[4][4], int Kd, LA&& la, LB&& lb) {
  __shared__ float sa[KS][TS + 1], sb[KS][TS + 1];
  const int t = threadIdx.x, tx = t % 16, ty = t / 16;
  for (int k0 = 0; k0 < Kd; k0 += KS) {
    __syncthreads();
    for (int i = t; i < KS * TS; i += 256) {
      sa[i / TS][i % TS] = k0 + i / TS < Kd ? la(i % TS, k0 + i / TS) : 0.0f;
      sb[i / TS][i % TS] = k0 + i / TS < Kd ? lb(k0 + i / TS, i % TS) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < KS; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][ty + 16 * i] * sb[k][tx + 16 * j];
  }
}

template <typename Fn>
__device__ void each(int rows, int cols, Fn&& fn) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j)
      if (ty + 16 * i < rows && tx + 16 * j < cols) fn(i, j, ty + 16 * i, tx + 16 * j);
}

struct FfnArgs {
  int T, H, F, G, act;
  const int32_t* off;
  const uint16_t *x, *w1, *w3, *w2, *gate, *up, *dy, *h, *dgate, *dup;
  uint16_t *o0, *o1, *o2;
};

// h = act(x W1) * (x W3); o0 = h, o1, o2 = gate and up or NULL
__global__ __launch_bounds__(256) void ffn_up_kernel(FfnArgs a) {
  RowTile rt;
  int total;
  if (!row_tile(a.off, a.G, a.T, TS, blockIdx.y, &rt, &total)) return;
  const int n0 = blockIdx.x * TS, rows = rt.end - rt.begin;
  float g[4][4] = {}, u[4][4] = {};
  auto la = [&](int m, int k) { return m < rows ? bf16_to_f32(a.x[(size_t)(rt.begin + m) * a.H + k]) : 0.0f; };
  product(g, a.H, la, [&](int k, int n) { return bf16_to_f32(a.w1[((size_t)rt.group * a.H + k) * a.F + n0 + n]); });
  product(u, a.H, la, [&](int k, int n) { return bf16_to_f32(a.w3[((size_t)rt.group * a.H + k) * a.F + n0 + n]); });
  each(rows, a.F - n0, [&](int i, int j, int m, int n) {
    const size_t at = (size_t)(rt.begin + m) * a.F + n0 + n;
    a.o0[at] = f32_to_bf16(act_of(g[i][j], a.act) * u[i][j]);
    if (a.o1) a.o1[at] = f32_to_bf16(g[i][j]), a.o2[at] = f32_to_bf16(u[i][j]);
  });
}

// y = h W2
__global__ __launch_bounds__(256) void ffn_down_kernel(FfnArgs a) {
  RowTile rt;
  int total;
  if (!row_tile(a.off, a.G, a.T, TS, blockIdx.y, &rt, &total)) return;
  const int n0 = blockIdx.x * TS, rows = rt.end - rt.begin;
  float y[4][4] = {};
  product(y, a.F, [&](int m, int k) { return m < rows ? bf16_to_f32(a.h[(size_t)(rt.begin + m) * a.F + k]) : 0.0f; },
          [&](int k, int n) { return bf16_to_f32(a.w2[((size_t)rt.group * a.F + k) * a.H + n0 + n]); });
  each(rows, a.H - n0, [&](int i, int j, int m, int n) {
    a.o0[(size_t)(rt.begin + m) * a.H + n0 + n] = f32_to_bf16(y[i][j]);
  });
}

// dh = dy W2^T, and from it o0 = act(gate) * up, o1 = d gate, o2 = d up
__global__ __launch_bounds__(256) void ffn_dh_kernel(FfnArgs a) {
  RowTile rt;
  int total;
  if (!row_tile(a.off, a.G, a.T, TS, blockIdx.y, &rt, &total)) return;
  const int n0 = blockIdx.x * TS, rows = rt.end - rt.begin;
  float dh[4][4] = {};
  product(dh, a.H, [&](int m, int k) { return m < rows ? bf16_to_f32(a.dy[(size_t)(rt.begin + m) * a.H + k]) : 0.0f; },
          [&](int k, int n) { return bf16_to_f32(a.w2[((size_t)rt.group * a.F + n0 + n) * a.H + k]); });
  each(rows, a.F - n0, [&](int i, int j, int m, int n) {
    const size_t at = (size_t)(rt.begin + m) * a.F + n0 + n;
    const float g = bf16_to_f32(a.gate[at]), u = bf16_to_f32(a.up[at]);
    float v, dv;
    act_grad(g, a.act, &v, &dv);
    a.o0[at] = f32_to_bf16(v * u);
    a.o1[at] = f32_to_bf16(dh[i][j] * u * dv);
    a.o2[at] = f32_to_bf16(dh[i][j] * v);
  });
}

// dx = dgate W1^T + dup W3^T
__global__ __launch_bounds__(256) void ffn_dx_kernel(FfnArgs a) {
  RowTile rt;
  int total;
  if (!row_tile(a.off, a.G, a.T, TS, blockIdx.y, &rt, &total)) return;
  const int n0 = blockIdx.x * TS, rows = rt.end - rt.begin;
  float dx[4][4] = {};
  product(dx, a.F, [&](int m, int k) { return m < rows ? bf16_to_f32(a.dgate[(size_t)(rt.begin + m) * a.F + k]) : 0.0f; },
          [&](int k, int n) { return bf16_to_f32(a.w1[((size_t)rt.group * a.H + n0 + n) * a.F + k]); });
  product(dx, a.F, [&](int m, int k) { return m < rows ? bf16_to_f32(a.dup[(size_t)(rt.begin + m) * a.F + k]) : 0.0f; },
          [&](int k, int n) { return bf16_to_f32(a.w3[((size_t)rt.group * a.H + n0 + n) * a.F + k]); });
  each(rows, a.H - n0, [&](int i, int j, int m, int n) {
    a.o0[(size_t)(rt.begin + m) * a.H + n0 + n] = f32_to_bf16(dx[i][j]);
  });
}

// out[g] = p^T q over the group's rows; p [T][M], q [T][N]
__global__ __launch_bounds__(256) void ffn_dw_kernel(const int32_t* off, int T, const uint16_t* p, const uint16_t* q,
                                                     uint16_t* out, int M, int N) {
  const int g = blockIdx.z, m0 = blockIdx.y * TS, n0 = blockIdx.x * TS;
  int b, e;
  group_rows(off, T, g, &b, &e);
  float w[4][4] = {};
  product(w, e - b, [&](int m, int k) { return bf16_to_f32(p[(size_t)(b + k) * M + m0 + m]); },
          [&](int k, int n) { return bf16_to_f32(q[(size_t)(b + k) * N + n0 + n]); });
  each(M - m0, N - n0, [&](int i, int j, int m, int n) {
    out[((size_t)g * M + m0 + m) * N + n0 + n] = f32_to_bf16(w[i][j]);
  });
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
  uint16_t* h = static_cast<uint16_t*>(ws);
  a.h = h, a.o0 = h, a.o1 = gate, a.o2 = up;
  const int mt = max_row_tiles(a.T, a.G, TS);
  ffn_up_kernel<<<dim3(a.F / TS, mt), 256, 0, s>>>(a);
  a.o0 = y;
  ffn_down_kernel<<<dim3(a.H / TS, mt), 256, 0, s>>>(a);
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
  uint16_t* h = reinterpret_cast<uint16_t*>(at);
  uint16_t* dg = reinterpret_cast<uint16_t*>(at + plane(cfg));
  uint16_t* du = reinterpret_cast<uint16_t*>(at + 2 * plane(cfg));
  if (a.T > 0 && (dx || dw1)) {
    const int mt = max_row_tiles(a.T, a.G, TS);
    a.o0 = h, a.o1 = dg, a.o2 = du;
    ffn_dh_kernel<<<dim3(a.F / TS, mt), 256, 0, s>>>(a);
    if (dx) {
      a.dgate = dg, a.dup = du, a.o0 = dx;
      ffn_dx_kernel<<<dim3(a.H / TS, mt), 256, 0, s>>>(a);
    }
  }
  if (dw1) {
    ffn_dw_kernel<<<dim3(a.F / TS, a.H / TS, a.G), 256, 0, s>>>(a.off, a.T, x, dg, dw1, a.H, a.F);
    ffn_dw_kernel<<<dim3(a.F / TS, a.H / TS, a.G), 256, 0, s>>>(a.off, a.T, x, du, dw3, a.H, a.F);
    ffn_dw_kernel<<<dim3(a.H / TS, a.F / TS, a.G), 256, 0, s>>>(a.off, a.T, h, dy, dw2, a.F, a.H);
  }
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
