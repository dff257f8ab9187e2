// The gate's logits and their gradients, and the routing's losses (moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

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
  int Ep;              // E rounded up to whole 16 bytes
  const int32_t *off, *idx;
  const float *logits, *topk_w, *dtopk_w, *dloss, *in_lse;
  const int32_t* in_counts;
  int32_t* counts;
  float *lse, *loss, *dlogits;
  // workspace: of each tile the sums of the softmax [tiles][Ep], the counts and the sum of lse^2; of each sequence and
  // 32 of its experts the part of the balance loss, and of each sequence the sum of lse^2; workgroups that are done
  float *part, *zpart, *seq, *zseq;
  int32_t *cpart, *done;
};

// The sequences' rows and tiles.  Every lane of the wavefront takes part and gets
// the same answers; each holds up to 8 consecutive sequences.
struct SeqTiles {
  const int32_t* off;
  int T, bm, g0, g1, first, before, n;  // first: where this lane's sequences start; before: the tiles ahead of its n
  int total, live, rows;                // tiles, sequences that have rows, and their rows
  struct Seq {
    int g, b, e, tile;  // rows [b, e) and the first tile
  };

  __device__ __forceinline__ SeqTiles(const int32_t* off_, int S, int T_, int bm_) : off(off_), T(T_), bm(bm_) {
    if (!off) {
      total = ceil_div(T, bm), live = 1, rows = T;
      return;
    }
    const int lane = threadIdx.x & 63, per = ceil_div(S, 64);
    g0 = min(lane * per, S), g1 = min(g0 + per, S);
    int m = 0;
    for (int g = g0; g < g1; ++g) m = max(m, clamp_off(off[g], T));
    const int own = g0 < S ? clamp_off(off[g0], T) : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(m, d);
      if (lane >= d) m = max(m, o);
    }
    m = __shfl_up(m, 1);
    first = max(lane ? m : 0, own);
    int at = first, sum = 0;  // tiles, and sequences with rows in the upper bits
    for (int g = g0; g < g1; ++g) {
      const int e = max(at, clamp_off(off[g + 1], T));
      sum += ceil_div(e - at, bm) + (e > at ? 1 << 21 : 0);
      at = e;
    }
    n = sum & ((1 << 21) - 1);
    // (this lane's last row: rows follow each other without gaps)
    const int last = (S - 1) / per;
    rows = __builtin_amdgcn_readlane(at, last) - __builtin_amdgcn_readfirstlane(first);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    before = (sum & ((1 << 21) - 1)) - n;
    sum = __builtin_amdgcn_readlane(sum, 63);
    total = sum & ((1 << 21) - 1);
    live = sum >> 21;
  }

  // the sequence for which `is` holds of its number and its tiles' range; one lane has it
  template <typename Fn>
  __device__ __forceinline__ Seq find(bool mine, Fn&& is) const {
    Seq s{};
    if (mine) {
      int at = first, tile = before;
      for (int g = g0; g < g1; ++g) {
        const int e = max(at, clamp_off(off[g + 1], T)), k = ceil_div(e - at, bm);
        if (is(g, tile, k)) s = {g, at, e, tile};
        at = e;
        tile += k;
      }
    }
    const int src = __ffsll((unsigned long long)__ballot(mine)) - 1;
    return {__builtin_amdgcn_readlane(s.g, src), __builtin_amdgcn_readlane(s.b, src), __builtin_amdgcn_readlane(s.e, src),
            __builtin_amdgcn_readlane(s.tile, src)};
  }
  __device__ __forceinline__ Seq of_tile(int t) const {  // t < total
    if (!off) return {0, 0, T, 0};
    return find(t >= before && t < before + n, [t](int, int tile, int k) { return t >= tile && t < tile + k; });
  }
  __device__ __forceinline__ Seq of(int g) const {
    if (!off) return {0, 0, T, 0};
    return find(g >= g0 && g < g1, [g](int i, int, int) { return i == g; });
  }
};

// A row of logits in the registers of LPR lanes, N values each: 16-byte pieces
// (VEC, where rows start on 16 bytes) or single values side by side.
template <int LPR_, int N_, bool VEC>
struct Row {
  static constexpr int LPR = LPR_, N = N_, AT_ONCE = 64 / LPR;  // AT_ONCE: rows of a wavefront
  static __device__ __forceinline__ int column(int l, int i) { return VEC ? (i / 4 * LPR + l) * 4 + i % 4 : i * LPR + l; }
  static __device__ __forceinline__ void load(float (&v)[N], const float* row, int l, int E, bool some) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        f32x4_t t{-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
        if (some && column(l, i) < E) t = *reinterpret_cast<const f32x4_t*>(row + column(l, i));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = t[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = some && column(l, i) < E ? row[column(l, i)] : -__builtin_inff();
    }
  }
  static __device__ __forceinline__ void store(const float (&v)[N], float* row, int l, int E) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < N; i += 4)
        if (column(l, i) < E) *reinterpret_cast<f32x4_t*>(row + column(l, i)) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (column(l, i) < E) row[column(l, i)] = v[i];
    }
  }
  static __device__ __forceinline__ float sum(float v) {
#pragma unroll
    for (int d = LPR / 2; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
  }
};

// A tile's rows are the four wavefronts' in turn; the next row's logits are loaded
// before a row is worked on.
template <typename R>
__global__ __launch_bounds__(256) void route_loss_kernel(LossArgs a) {
  __shared__ int hist[MAX_E];
  __shared__ float sums[256 * R::N], zs[4 * R::AT_ONCE];
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
  const SeqTiles list(a.off, a.S, a.T, a.bm);
  if ((int)blockIdx.x >= list.total) return;
  const SeqTiles::Seq seq = list.of_tile(blockIdx.x);
  const int begin = seq.b + ((int)blockIdx.x - seq.tile) * a.bm, end = min(begin + a.bm, seq.e);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % R::LPR, sub = lane / R::LPR;
  float p[R::N] = {}, z = 0, next[R::N];
  int base = begin + wave * R::AT_ONCE;
  R::load(next, a.logits + (size_t)(base + sub) * a.E, l, a.E, base + sub < end);
  for (int i = threadIdx.x; i < a.Ep; i += 256) hist[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < (end - begin) * a.K; i += 256) {
    const int e = a.idx[(size_t)begin * a.K + i];
    if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
  }
  for (; base < end; base += 4 * R::AT_ONCE) {
    const int row = base + sub, far = row + 4 * R::AT_ONCE;
    float v[R::N], top = -__builtin_inff(), total = 0;
#pragma unroll
    for (int i = 0; i < R::N; ++i) {
      v[i] = next[i];
      top = fmaxf(top, v[i]);
    }
    R::load(next, a.logits + (size_t)far * a.E, l, a.E, far < end);
#pragma unroll
    for (int d = R::LPR / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (top == -__builtin_inff()) top = 0;  // nothing can be chosen: every exponential is 0
#pragma unroll
    for (int i = 0; i < R::N; ++i) {
      v[i] = __expf(v[i] - top);
      total += v[i];
    }
    total = R::sum(total);
    const float lse = logf(total) + top, inv = total == 0 ? 0 : 1.0f / total;
    if (l == 0 && row < end) {
      a.lse[row] = lse;
      z += total == 0 ? 0 : lse * lse;
    }
#pragma unroll
    for (int i = 0; i < R::N; ++i) p[i] += v[i] * inv;
  }
  // [rows at once][column]
  constexpr int W = R::LPR * R::N;
#pragma unroll
  for (int i = 0; i < R::N; ++i) sums[(wave * R::AT_ONCE + sub) * W + R::column(l, i)] = p[i];
  if (l == 0) zs[wave * R::AT_ONCE + sub] = z;
  __syncthreads();
  for (int e = threadIdx.x; e < a.Ep; e += 256) {
    float v = sums[e];
#pragma unroll
    for (int i = 1; i < 4 * R::AT_ONCE; ++i) v += sums[i * W + e];
    a.part[(size_t)blockIdx.x * a.Ep + e] = v;
    a.cpart[(size_t)blockIdx.x * a.Ep + e] = hist[e];
  }
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < 4 * R::AT_ONCE; ++i) z += zs[i];
    a.zpart[blockIdx.x] = z;
  }
}

// Counts of a sequence's 32 experts from blockIdx.y * 32 on and their part of its
// balance loss, its tiles added in a fixed order: 8 threads side by side, 128 groups
// of them take the tiles in turn.  The last workgroup adds all parts up.
__global__ __launch_bounds__(1024) void route_loss_seq_kernel(LossArgs a) {
  __shared__ f32x4_t ps[128][8];
  __shared__ u32x4_t cs[128][8];
  __shared__ float zs[16], vs[16];
  __shared__ int last;
  const int g = blockIdx.x, q = threadIdx.x % 8, first = threadIdx.x / 8, c = blockIdx.y * 32 + q * 4;
  const SeqTiles list(a.off, a.S, a.T, a.bm);
  const SeqTiles::Seq seq = list.of(g);
  const int tiles = ceil_div(seq.e - seq.b, a.bm);
  f32x4_t p{0, 0, 0, 0};
  u32x4_t n{0, 0, 0, 0};
  if (c < a.Ep)
#pragma unroll 8
    for (int t = first; t < tiles; t += 128) {
      p += *reinterpret_cast<const f32x4_t*>(a.part + (size_t)(seq.tile + t) * a.Ep + c);
      n += *reinterpret_cast<const u32x4_t*>(a.cpart + (size_t)(seq.tile + t) * a.Ep + c);
    }
  float z = 0;
  if (blockIdx.y == 0)
    for (int t = threadIdx.x; t < tiles; t += 1024) z += a.zpart[seq.tile + t];
#pragma unroll
  for (int d = 32; d; d >>= 1) z += __shfl_xor(z, d);
  if (threadIdx.x % 64 == 0) zs[threadIdx.x / 64] = z;
  ps[first][q] = p;
  cs[first][q] = n;
  for (int k = 64; k; k >>= 1) {
    __syncthreads();
    if (first < k) {
      ps[first][q] += ps[first + k][q];
      cs[first][q] += cs[first + k][q];
    }
  }
  const float rows = (float)(seq.e - seq.b);
  if (threadIdx.x < 8) {
    float v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (c + j < a.E) a.counts[(size_t)g * a.E + c + j] = (int)cs[0][q][j];
      v += ps[0][q][j] * (float)cs[0][q][j];
    }
#pragma unroll
    for (int d = 4; d; d >>= 1) v += __shfl_xor(v, d);
    if (threadIdx.x == 0) {
      const auto put = [](float* at, float value) { __hip_atomic_store(at, value, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
      put(a.seq + g * gridDim.y + blockIdx.y, tiles ? v * a.E / (a.K * rows * rows) : 0.0f);
      if (blockIdx.y == 0) {
        for (int i = 1; i < 16; ++i) z += zs[i];
        put(a.zseq + g, z);
      }
      last = __hip_atomic_fetch_add(a.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)(gridDim.x * gridDim.y) - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  const auto get = [](const float* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  float v = 0;
  z = 0;
  for (int i = threadIdx.x; i < (int)(gridDim.x * gridDim.y); i += 1024) v += get(a.seq + i);
  if ((int)threadIdx.x < a.S) z = get(a.zseq + threadIdx.x);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    v += __shfl_xor(v, d);
    z += __shfl_xor(z, d);
  }
  if (threadIdx.x % 64 == 0) {
    vs[threadIdx.x / 64] = v;
    zs[threadIdx.x / 64] = z;
  }
  __syncthreads();
  if (threadIdx.x) return;
  for (int i = 1; i < 16; ++i) {
    v += vs[i];
    z += zs[i];
  }
  a.loss[0] = list.live ? v / list.live : 0.0f;
  a.loss[1] = list.live ? z / list.rows : 0.0f;
}

__global__ __launch_bounds__(256) void route_loss_none_kernel(LossArgs a) {
  for (int i = threadIdx.x; i < a.S * a.E; i += 256) a.counts[i] = 0;
  if (threadIdx.x < 2) a.loss[threadIdx.x] = 0;
}

template <typename R>
__global__ __launch_bounds__(256) void route_loss_grad_kernel(LossArgs a) {
  const SeqTiles list(a.off, a.S, a.T, a.bm);
  if ((int)blockIdx.x >= list.total) return;
  const SeqTiles::Seq seq = list.of_tile(blockIdx.x);
  const int begin = seq.b + ((int)blockIdx.x - seq.tile) * a.bm, end = min(begin + a.bm, seq.e);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % R::LPR, sub = lane / R::LPR;
  struct Given {  // what is read of a row: its logits, lse, and of choice l (where l < K) expert, weight and gradient
    float v[R::N], lse, w, dw;
    int e;
  };
  const auto load = [&](Given& r, int row) {
    const bool some = row < end;
    R::load(r.v, a.logits + (size_t)row * a.E, l, a.E, some);
    r.lse = some ? a.in_lse[row] : 0.0f;
    const bool choice = some && a.dtopk_w && l < a.K;
    r.e = choice ? a.idx[(size_t)row * a.K + l] : -1;
    r.w = choice ? a.topk_w[(size_t)row * a.K + l] : 0.0f;
    r.dw = choice ? a.dtopk_w[(size_t)row * a.K + l] : 0.0f;
  };
  Given next;
  int base = begin + wave * R::AT_ONCE;
  load(next, base + sub);
  const float n = (float)(seq.e - seq.b);
  const float db = a.dloss ? a.dloss[0] * a.E / (a.K * n * n * list.live) : 0.0f;
  const float dz = a.dloss ? 2.0f * a.dloss[1] / list.rows : 0.0f;
  float c[R::N];
#pragma unroll
  for (int i = 0; i < R::N; ++i) {
    const int e = R::column(l, i);
    c[i] = e < a.E ? (float)a.in_counts[(size_t)seq.g * a.E + e] * db : 0.0f;
  }
  for (; base < end; base += 4 * R::AT_ONCE) {
    const Given r = next;
    const int row = base + sub;
    load(next, row + 4 * R::AT_ONCE);
    const bool dead = r.lse == -__builtin_inff();  // a row of -inf alone: nothing can be chosen
    float p[R::N], dot = 0;
#pragma unroll
    for (int i = 0; i < R::N; ++i) {
      p[i] = dead ? 0.0f : __expf(r.v[i] - r.lse);
      dot += c[i] * p[i];
    }
    dot = R::sum(dot);
    const float rest = (dead ? 0.0f : dz * r.lse) - dot;
#pragma unroll
    for (int i = 0; i < R::N; ++i) p[i] *= c[i] + rest;
    if (a.dtopk_w) {
      // (choices are in the row's first 8 lanes)
      float all = r.w * r.dw;
#pragma unroll
      for (int d = 4; d; d >>= 1) all += __shfl_xor(all, d);
      const float t = r.w * (r.dw - all);
      for (int j = 0; j < a.K; ++j) {
        const float tj = __shfl(t, sub * R::LPR + j);
        const int ej = __shfl(r.e, sub * R::LPR + j);
#pragma unroll
        for (int i = 0; i < R::N; ++i) p[i] += R::column(l, i) == ej ? tj : 0.0f;
      }
    }
    if (row < end) R::store(p, a.dlogits + (size_t)row * a.E, l, a.E);
  }
}

// fn(a Row that holds E logits)
template <typename Fn>
void for_row(int E, Fn&& fn) {
  const auto of = [&](auto vec) {
    constexpr bool V = vec();
    if (E <= 32) fn(Row<8, 4, V>());
    else if (E <= 64) fn(Row<16, 4, V>());
    else if (E <= 128) fn(Row<32, 4, V>());
    else if (E <= 256) fn(Row<64, 4, V>());
    else fn(Row<64, 8, V>());
  };
  if (E % 4 == 0) of(std::true_type());
  else of(std::false_type());
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

// About 1024 tiles of a long batch, whose sums fit the caches; 32 rows at least
// (the four wavefronts' 4 to 32 at once).
LossArgs loss_args(const moe_router_config* c, const int32_t* off) {
  LossArgs a{};
  a.T = c->rows, a.E = c->n_experts, a.K = c->top_k, a.S = c->n_seqs, a.off = off;
  a.Ep = ceil_div(a.E, 4) * 4;
  a.bm = std::max(32, ceil_div(a.T, 1024));
  return a;
}

// Workspace: what LossArgs says, one after the other.
struct LossSpace {
  size_t part, cpart, zpart, seq, zseq, done, total;
};
LossSpace loss_space(const LossArgs& a) {
  const size_t tiles = max_row_tiles(a.T, a.S, a.bm);
  LossSpace w{};
  w.cpart = align_up(tiles * a.Ep * sizeof(float), 256);
  w.zpart = w.cpart + align_up(tiles * a.Ep * sizeof(int32_t), 256);
  w.seq = w.zpart + align_up(tiles * sizeof(float), 256);
  w.zseq = w.seq + align_up(ceil_div(a.Ep, 32) * a.S * sizeof(float), 256);
  w.done = w.zseq + align_up(a.S * sizeof(float), 256);
  w.total = w.done + 256;
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
  a.zseq = reinterpret_cast<float*>(at + w.zseq), a.done = reinterpret_cast<int32_t*>(at + w.done);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (a.T == 0) {
    route_loss_none_kernel<<<1, 256, 0, s>>>(a);
  } else {
    for_row(a.E, [&](auto row) { route_loss_kernel<decltype(row)><<<max_row_tiles(a.T, a.S, a.bm), 256, 0, s>>>(a); });
    route_loss_seq_kernel<<<dim3(a.S, ceil_div(a.Ep, 32)), 1024, 0, s>>>(a);
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
  for_row(a.E, [&](auto row) {
    route_loss_grad_kernel<decltype(row)>
        <<<max_row_tiles(a.T, a.S, a.bm), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  });
  HIP_TRY(hipGetLastError());
  return MOE_OK;
}

}  // extern "C"
