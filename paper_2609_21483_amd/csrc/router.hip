// The gate's logits and their gradients, and the routing's losses (moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "blocks.h"

using namespace moe;

namespace {

// ---- the gate's products ----------------------------------------------------------
struct GateArgs {
  int T, H, E, S;
  const int32_t* off;
  const uint16_t *x, *wg;
  const float *bias, *dlogits;
  float *logits, *dbias;
  uint16_t *dx, *dwg;
};

__device__ __forceinline__ float rounded(float v) { return bf16_to_f32((uint16_t)f32_to_bf16(v)); }

__global__ __launch_bounds__(256) void gate_logits_kernel(GateArgs a) {
  int b, e;
  covered_rows(a.off, a.S, a.T, &b, &e);
  const int t = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x;
  if (t < b || t >= e || n >= a.E) return;
  float v = 0;
  for (int h = 0; h < a.H; ++h) v += bf16_to_f32(a.x[(size_t)t * a.H + h]) * bf16_to_f32(a.wg[(size_t)h * a.E + n]);
  a.logits[(size_t)t * a.E + n] = a.bias ? v + a.bias[n] : v;
}

__global__ __launch_bounds__(256) void gate_dx_kernel(GateArgs a) {
  int b, e;
  covered_rows(a.off, a.S, a.T, &b, &e);
  const int t = blockIdx.x, h = blockIdx.y * 256 + threadIdx.x;
  if (t < b || t >= e || h >= a.H) return;
  float v = 0;
  for (int n = 0; n < a.E; ++n) v += rounded(a.dlogits[(size_t)t * a.E + n]) * bf16_to_f32(a.wg[(size_t)h * a.E + n]);
  a.dx[(size_t)t * a.H + h] = (uint16_t)f32_to_bf16(v);
}

// dwg, and dbias as one more row of it (h = H)
__global__ __launch_bounds__(256) void gate_dwg_kernel(GateArgs a) {
  int b, e;
  covered_rows(a.off, a.S, a.T, &b, &e);
  const int h = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x;
  if (n >= a.E || (h < a.H && !a.dwg)) return;  // (x may be missing where dwg is not wanted)
  float v = 0;
  for (int t = b; t < e; ++t) {
    const float d = a.dlogits[(size_t)t * a.E + n];
    v += h < a.H ? bf16_to_f32(a.x[(size_t)t * a.H + h]) * rounded(d) : d;
  }
  if (h == a.H) {
    if (a.dbias) a.dbias[n] = v;
  } else if (a.dwg) {
    a.dwg[(size_t)h * a.E + n] = (uint16_t)f32_to_bf16(v);
  }
}

// ---- the routing's losses ---------------------------------------------------------
struct LossArgs {
  int T, E, K, S, bm;  // bm: rows of a tile
  const int32_t *off, *idx;
  const float *logits, *topk_w, *dtopk_w, *dloss, *in_lse;
  const int32_t* in_counts;
  int32_t* counts;
  float *lse, *loss, *dlogits;
  float *part, *zpart, *seq;  // workspace: softmax sums [tiles][E], sums of lse^2 [tiles], [S][2]
  int32_t* cpart;             // and counts [tiles][E]
};

constexpr int PER = MAX_E / 64;  // experts of a lane: lane + 64 i

// A tile's rows are the four wavefronts' in turn.
__global__ __launch_bounds__(256) void route_loss_kernel(LossArgs a) {
  __shared__ int hist[MAX_E];
  __shared__ float sums[4][MAX_E], zs[4];
  const RowTiles list(a.off, a.S, a.T, a.bm);
  if ((int)blockIdx.x >= list.total) return;
  const RowTile rt = list.at(blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < MAX_E; i += 256) hist[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < (rt.end - rt.begin) * a.K; i += 256) {
    const int e = a.idx[(size_t)rt.begin * a.K + i];
    if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
  }
  float p[PER] = {}, z = 0;
  for (int row = rt.begin + wave; row < rt.end; row += 4) {
    float l[PER], top = -__builtin_inff(), total = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      l[i] = e < a.E ? a.logits[(size_t)row * a.E + e] : -__builtin_inff();
      top = fmaxf(top, l[i]);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (top == -__builtin_inff()) top = 0;  // nothing can be chosen: every exponential is 0
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      l[i] = __expf(l[i] - top);
      total += l[i];
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    const float lse = logf(total) + top, inv = total == 0 ? 0 : 1.0f / total;
    if (lane == 0) a.lse[row] = lse;
    z += total == 0 ? 0 : lse * lse;
#pragma unroll
    for (int i = 0; i < PER; ++i) p[i] += l[i] * inv;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) sums[wave][lane + 64 * i] = p[i];
  if (lane == 0) zs[wave] = z;
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += 256) {
    a.part[(size_t)blockIdx.x * a.E + e] = sums[0][e] + sums[1][e] + sums[2][e] + sums[3][e];
    a.cpart[(size_t)blockIdx.x * a.E + e] = hist[e];
  }
  if (threadIdx.x == 0) a.zpart[blockIdx.x] = zs[0] + zs[1] + zs[2] + zs[3];
}

// A sequence's counts and its parts of the losses, from its tiles in order.
__global__ __launch_bounds__(512) void route_loss_seq_kernel(LossArgs a) {
  __shared__ float red[2][8];
  const int g = blockIdx.x, e = threadIdx.x, lane = threadIdx.x & 63;
  const RowTiles list(a.off, a.S, a.T, a.bm);
  int b, end;
  group_rows(a.off, a.T, g, &b, &end);
  const int first = list.before(g), tiles = ceil_div(end - b, a.bm);
  float p = 0, z = 0;
  int c = 0;
  if (e < a.E) {
    for (int t = first; t < first + tiles; ++t) {
      p += a.part[(size_t)t * a.E + e];
      c += a.cpart[(size_t)t * a.E + e];
    }
    a.counts[(size_t)g * a.E + e] = c;
  }
  for (int t = first + threadIdx.x; t < first + tiles; t += 512) z += a.zpart[t];
  float v = p * (float)c;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    v += __shfl_xor(v, d);
    z += __shfl_xor(z, d);
  }
  if (lane == 0) red[0][e >> 6] = v, red[1][e >> 6] = z;
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 8; ++i) v += red[0][i], z += red[1][i];
  const float n = (float)(end - b);
  a.seq[2 * g] = tiles ? v * a.E / (a.K * n * n) : 0.0f;
  a.seq[2 * g + 1] = z;
}

__global__ __launch_bounds__(64) void route_loss_mean_kernel(LossArgs a) {
  int b, e;
  covered_rows(a.off, a.S, a.T, &b, &e);
  const int live = RowTiles(a.off, a.S, a.T, a.T).total;
  float v = 0, z = 0;
  for (int g = threadIdx.x; g < a.S; g += 64) v += a.seq[2 * g], z += a.seq[2 * g + 1];
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    v += __shfl_xor(v, d);
    z += __shfl_xor(z, d);
  }
  if (threadIdx.x) return;
  a.loss[0] = live ? v / live : 0.0f;
  a.loss[1] = live ? z / (e - b) : 0.0f;
}

__global__ __launch_bounds__(256) void route_loss_none_kernel(LossArgs a) {
  for (int i = threadIdx.x; i < a.S * a.E; i += 256) a.counts[i] = 0;
  if (threadIdx.x < 2) a.loss[threadIdx.x] = 0;
}

__global__ __launch_bounds__(256) void route_loss_grad_kernel(LossArgs a) {
  const RowTiles list(a.off, a.S, a.T, a.bm);
  if ((int)blockIdx.x >= list.total) return;
  const RowTile rt = list.at(blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int b, end, n0, n1;
  group_rows(a.off, a.T, rt.group, &b, &end);
  covered_rows(a.off, a.S, a.T, &n0, &n1);
  const float n = (float)(end - b), live = (float)RowTiles(a.off, a.S, a.T, a.T).total;
  const float db = a.dloss ? a.dloss[0] * a.E / (a.K * n * n * live) : 0.0f;
  const float dz = a.dloss ? 2.0f * a.dloss[1] / (n1 - n0) : 0.0f;
  float c[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
    c[i] = e < a.E ? (float)a.in_counts[(size_t)rt.group * a.E + e] * db : 0.0f;
  }
  for (int row = rt.begin + wave; row < rt.end; row += 4) {
    const float lse = a.in_lse[row];
    float p[PER], dot = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      // (a row of -inf alone: nothing can be chosen)
      p[i] = e < a.E && lse != -__builtin_inff() ? __expf(a.logits[(size_t)row * a.E + e] - lse) : 0.0f;
      dot += c[i] * p[i];
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) dot += __shfl_xor(dot, d);
    float wdw = 0;
    if (a.dtopk_w)
      for (int j = 0; j < a.K; ++j) wdw += a.topk_w[(size_t)row * a.K + j] * a.dtopk_w[(size_t)row * a.K + j];
    const float zl = lse == -__builtin_inff() ? 0.0f : dz * lse;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      float v = p[i] * (c[i] - dot + zl);
      if (a.dtopk_w)
        for (int j = 0; j < a.K; ++j)
          if (a.idx[(size_t)row * a.K + j] == e)
            v += a.topk_w[(size_t)row * a.K + j] * (a.dtopk_w[(size_t)row * a.K + j] - wdw);
      if (e < a.E) a.dlogits[(size_t)row * a.E + e] = v;
    }
  }
}

// ---- host ---------------------------------------------------------------------------
moe_status check_cfg(const moe_router_config* c) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "config is NULL");
  if (c->rows < 0 || c->rows > (1 << 22)) return fail(MOE_ERR_INVALID_ARG, "rows must be in [0, 2^22]");
  if (c->n_experts < 1 || c->n_experts > MAX_E) return fail(MOE_ERR_INVALID_ARG, "n_experts must be in [1, %d]", MAX_E);
  if (c->n_seqs < 1 || c->n_seqs > MOE_MAX_GROUPS)
    return fail(MOE_ERR_INVALID_ARG, "n_seqs must be in [1, %d]", MOE_MAX_GROUPS);
  return MOE_OK;
}
moe_status check_gate(const moe_router_config* c) {
  moe_status st = check_cfg(c);
  if (st != MOE_OK) return st;
  if (c->hidden < 64 || c->hidden % 64 || c->hidden > 16384)
    return fail(MOE_ERR_INVALID_ARG, "hidden must be a multiple of 64 in [64, 16384]");
  return MOE_OK;
}
moe_status check_loss(const moe_router_config* c) {
  moe_status st = check_cfg(c);
  if (st != MOE_OK) return st;
  if (c->top_k < 1 || c->top_k > MAX_TOPK || c->top_k > c->n_experts)
    return fail(MOE_ERR_INVALID_ARG, "top_k must be in [1, min(n_experts, %d)]", MAX_TOPK);
  return MOE_OK;
}
moe_status check_off(const moe_router_config* c, const int32_t* off) {
  if (!off && c->n_seqs > 1) return fail(MOE_ERR_INVALID_ARG, "seq_off is NULL with more than one sequence");
  if (reinterpret_cast<uintptr_t>(off) % 4) return fail(MOE_ERR_INVALID_ARG, "seq_off is not aligned to its values");
  return MOE_OK;
}
moe_status check_tensors(std::initializer_list<const void*> all) {
  for (const void* p : all)
    if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "a tensor does not start on a 16-byte boundary");
  return MOE_OK;
}
moe_status check_ws(const void* ws, size_t bytes, size_t need) {
  if (!ws || bytes < need) return fail(MOE_ERR_INVALID_ARG, "the workspace holds %zu of %zu bytes", ws ? bytes : 0, need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MOE_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  return MOE_OK;
}

GateArgs gate_args(const moe_router_config* c, const int32_t* off) {
  GateArgs a{};
  a.T = c->rows, a.H = c->hidden, a.E = c->n_experts, a.S = c->n_seqs, a.off = off;
  return a;
}

// About 1024 tiles of a long batch, whose sums fit the caches, and 16 rows at least
LossArgs loss_args(const moe_router_config* c, const int32_t* off) {
  LossArgs a{};
  a.T = c->rows, a.E = c->n_experts, a.K = c->top_k, a.S = c->n_seqs, a.off = off;
  a.bm = std::max(16, ceil_div(a.T, 1024));
  return a;
}

// Workspace: the tiles' sums and counts, their sums of lse^2, the sequences' losses.
struct LossSpace {
  size_t part, cpart, zpart, seq, total;
};
LossSpace loss_space(const LossArgs& a) {
  const size_t tiles = max_row_tiles(a.T, a.S, a.bm);
  LossSpace w{};
  w.cpart = align_up(tiles * a.E * sizeof(float), 256);
  w.zpart = w.cpart + align_up(tiles * a.E * sizeof(int32_t), 256);
  w.seq = w.zpart + align_up(tiles * sizeof(float), 256);
  w.total = w.seq + align_up(2 * a.S * sizeof(float), 256);
  return w;
}

size_t gate_ws(const moe_router_config*, bool) { return 256; }

}  // namespace

extern "C" {

moe_status moe_gate_workspace_size(const moe_router_config* cfg, int32_t backward, size_t* bytes) {
  moe_status st = check_gate(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = gate_ws(cfg, backward != 0);
  return MOE_OK;
}

moe_status moe_gate_logits(const moe_router_config* cfg, const uint16_t* x, const uint16_t* wg,
                           const float* logit_bias, const int32_t* seq_off, float* logits, void* ws, size_t ws_bytes,
                           void* stream) {
  moe_status st = check_gate(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!x || !wg || !logits) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if ((st = check_off(cfg, seq_off)) != MOE_OK) return st;
  if ((st = check_tensors({x, wg, logit_bias, logits})) != MOE_OK) return st;
  if ((st = check_ws(ws, ws_bytes, gate_ws(cfg, false))) != MOE_OK) return st;
  GateArgs a = gate_args(cfg, seq_off);
  a.x = x, a.wg = wg, a.bias = logit_bias, a.logits = logits;
  gate_logits_kernel<<<dim3(a.T, ceil_div(a.E, 256)), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_gate_backward(const moe_router_config* cfg, const float* dlogits, const uint16_t* x,
                             const uint16_t* wg, const int32_t* seq_off, uint16_t* dx, uint16_t* dwg, float* dbias,
                             void* ws, size_t ws_bytes, void* stream) {
  moe_status st = check_gate(cfg);
  if (st != MOE_OK) return st;
  // (without rows there is no dx, but the other gradients are written: zeros)
  if (cfg->rows > 0 && (!dlogits || (dwg && !x) || (dx && !wg))) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if ((st = check_off(cfg, seq_off)) != MOE_OK) return st;
  if ((st = check_tensors({dlogits, x, wg, dx, dwg, dbias})) != MOE_OK) return st;
  if ((st = check_ws(ws, ws_bytes, gate_ws(cfg, true))) != MOE_OK) return st;
  GateArgs a = gate_args(cfg, seq_off);
  a.x = x, a.wg = wg, a.dlogits = dlogits, a.dx = dx, a.dwg = dwg, a.dbias = dbias;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dx && a.T > 0) gate_dx_kernel<<<dim3(a.T, ceil_div(a.H, 256)), 256, 0, s>>>(a);
  if (dwg || dbias) gate_dwg_kernel<<<dim3(a.H + 1, ceil_div(a.E, 256)), 256, 0, s>>>(a);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_route_loss_workspace_size(const moe_router_config* cfg, size_t* bytes) {
  moe_status st = check_loss(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = loss_space(loss_args(cfg, nullptr)).total;
  return MOE_OK;
}

moe_status moe_route_loss(const moe_router_config* cfg, const float* logits, const int32_t* topk_idx,
                          const int32_t* seq_off, int32_t* counts, float* lse, float* loss, void* ws, size_t ws_bytes,
                          void* stream) {
  moe_status st = check_loss(cfg);
  if (st != MOE_OK) return st;
  // (without rows the counts and losses are written: zeros)
  if (!counts || !loss || (cfg->rows > 0 && (!logits || !topk_idx || !lse))) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if ((st = check_off(cfg, seq_off)) != MOE_OK) return st;
  if ((st = check_tensors({logits, topk_idx, counts, lse, loss})) != MOE_OK) return st;
  LossArgs a = loss_args(cfg, seq_off);
  const LossSpace w = loss_space(a);
  if ((st = check_ws(ws, ws_bytes, w.total)) != MOE_OK) return st;
  a.logits = logits, a.idx = topk_idx, a.counts = counts, a.lse = lse, a.loss = loss;
  char* at = static_cast<char*>(ws);
  a.part = reinterpret_cast<float*>(at + w.part), a.cpart = reinterpret_cast<int32_t*>(at + w.cpart);
  a.zpart = reinterpret_cast<float*>(at + w.zpart), a.seq = reinterpret_cast<float*>(at + w.seq);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (a.T == 0) {
    route_loss_none_kernel<<<1, 256, 0, s>>>(a);
  } else {
    route_loss_kernel<<<max_row_tiles(a.T, a.S, a.bm), 256, 0, s>>>(a);
    route_loss_seq_kernel<<<a.S, 512, 0, s>>>(a);
    route_loss_mean_kernel<<<1, 64, 0, s>>>(a);
  }
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

moe_status moe_route_loss_backward(const moe_router_config* cfg, const float* logits, const int32_t* topk_idx,
                                   const float* topk_w, const int32_t* seq_off, const int32_t* counts,
                                   const float* lse, const float* dloss, const float* dtopk_w, float* dlogits,
                                   void* stream) {
  moe_status st = check_loss(cfg);
  if (st != MOE_OK) return st;
  if (cfg->rows == 0) return MOE_OK;
  if (!logits || !topk_idx || !counts || !lse || !dlogits) return fail(MOE_ERR_INVALID_ARG, "NULL argument");
  if (!topk_w != !dtopk_w) return fail(MOE_ERR_INVALID_ARG, "topk_w and dtopk_w are given both or neither");
  if ((st = check_off(cfg, seq_off)) != MOE_OK) return st;
  if ((st = check_tensors({logits, topk_idx, topk_w, counts, lse, dtopk_w, dlogits})) != MOE_OK) return st;
  if (reinterpret_cast<uintptr_t>(dloss) % 4) return fail(MOE_ERR_INVALID_ARG, "dloss is not aligned to its values");
  LossArgs a = loss_args(cfg, seq_off);
  a.logits = logits, a.idx = topk_idx, a.topk_w = topk_w, a.in_counts = counts, a.in_lse = lse, a.dloss = dloss;
  a.dtopk_w = dtopk_w, a.dlogits = dlogits;
  route_loss_grad_kernel<<<max_row_tiles(a.T, a.S, a.bm), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
