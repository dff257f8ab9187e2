// What the products over row groups share: the groups' rows, the activations
// of the gated block, and the host's checks (ffn.hip, int8.hip).
#pragma once

#include "common.h"
#include "host.h"

namespace moe {

// ---- row groups -------------------------------------------------------------
// Offsets are the caller's device data and are not trusted: offset i counts as
// the running maximum of the offsets up to i, each clamped to [0, T], so that
// groups never overlap and stay inside the tensors whatever the array holds.

struct RowTile {
  int group, begin, end;  // the tile's rows: [begin, end) of its group
  int tiles;              // row tiles of the group
};

__device__ __forceinline__ int clamp_off(int v, int T) { return v < 0 ? 0 : (v > T ? T : v); }

// The rows of group g (every lane of the wavefront calls it and gets the same).
__device__ __forceinline__ void group_rows(const int32_t* off, int T, int g, int* begin, int* end) {
  if (!off) {
    *begin = 0;
    *end = T;
    return;
  }
  int m = 0;
  for (int i = threadIdx.x & 63; i <= g; i += 64) m = max(m, clamp_off(off[i], T));
#pragma unroll
  for (int d = 32; d; d >>= 1) m = max(m, __shfl_xor(m, d));
  *begin = __builtin_amdgcn_readfirstlane(m);
  *end = __builtin_amdgcn_readfirstlane(max(m, clamp_off(off[g + 1], T)));
}

// The list of all groups' row tiles of `bm` rows, in group order (an empty
// group has none).  Every lane of the wavefront takes part and gets the same
// answers; each holds up to 8 consecutive groups (MOE_MAX_GROUPS / 64).
struct RowTiles {
  const int32_t* off;
  int T, bm, g0, g1, first, incl, n;  // first: where this lane's groups start; n: their tiles, incl: and those before
  int total;

  __device__ __forceinline__ RowTiles(const int32_t* off_, int G, int T_, int bm_) : off(off_), T(T_), bm(bm_) {
    if (!off) {
      total = ceil_div(T, bm);
      return;
    }
    const int lane = threadIdx.x & 63, per = ceil_div(G, 64);
    g0 = min(lane * per, G), g1 = min(g0 + per, G);
    int m = 0;  // the largest offset so far, over the lanes before and this lane's
    for (int g = g0; g < g1; ++g) m = max(m, clamp_off(off[g], T));
    const int own = g0 < G ? clamp_off(off[g0], T) : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(m, d);
      if (lane >= d) m = max(m, o);
    }
    m = __shfl_up(m, 1);
    first = max(lane ? m : 0, own);
    n = 0;
    for (int g = g0, at = first; g < g1; ++g) {
      const int e = max(at, clamp_off(off[g + 1], T));
      n += ceil_div(e - at, bm);
      at = e;
    }
    incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    total = __builtin_amdgcn_readlane(incl, 63);
  }

  // tile t < total
  __device__ __forceinline__ RowTile at(int t) const {
    if (!off) return {0, t * bm, min((t + 1) * bm, T), total};
    int group = 0, begin = 0, end = 0, tiles = 0, left = t - (incl - n);
    const bool mine = left >= 0 && left < n;
    if (mine)
      for (int g = g0, a = first; g < g1; ++g) {
        const int e = max(a, clamp_off(off[g + 1], T)), k = ceil_div(e - a, bm);
        if (left >= 0 && left < k) {
          group = g;
          tiles = k;
          begin = a + left * bm;
          end = min(begin + bm, e);
        }
        left -= k;
        a = e;
      }
    const int src = __ffsll((unsigned long long)__ballot(mine)) - 1;
    return {__builtin_amdgcn_readlane(group, src), __builtin_amdgcn_readlane(begin, src),
            __builtin_amdgcn_readlane(end, src), __builtin_amdgcn_readlane(tiles, src)};
  }
};

// The group of rank r by its number of rows, the largest first (equal ones in
// order), and its rows; up to 64 groups, one a lane.  About 0.3 us.
__device__ __forceinline__ int ranked_group(const int32_t* off, int T, int G, int r, int* begin, int* end) {
  const int lane = threadIdx.x & 63;
  int b = lane < G ? clamp_off(off[lane], T) : 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(b, d);
    if (lane >= d) b = max(b, o);
  }
  const int e = lane < G ? max(b, clamp_off(off[lane + 1], T)) : b, n = e - b;
  int rank = 0;
  for (int j = 0; j < G; ++j) {
    const int other = __builtin_amdgcn_readlane(n, j);
    rank += other > n || (other == n && j < lane);
  }
  const int src = __ffsll((unsigned long long)__ballot(lane < G && rank == r)) - 1;
  *begin = __builtin_amdgcn_readlane(b, src);
  *end = __builtin_amdgcn_readlane(e, src);
  return src;
}

// The rows that some group has: [begin, end).
__device__ __forceinline__ void covered_rows(const int32_t* off, int G, int T, int* begin, int* end) {
  int e;
  group_rows(off, T, 0, begin, &e);
  if (G > 1) group_rows(off, T, G - 1, &e, end);
  else *end = e;
}

// Most row tiles a list can have: one for each group that has rows, whose
// first row it holds, and one for every bm of the other rows.
__host__ __device__ inline int max_row_tiles(int T, int G, int bm) {
  const int some = G < T ? G : T;
  return some + (T - some) / bm;
}

// ---- the gated block's activation ---------------------------------------------
// Both forms are v * s(z), s the logistic function: z = v for SiLU, and for
// the tanh form z = 2 c (v + 0.044715 v^3), c = sqrt(2/pi), since
// (1 + tanh(u)) / 2 = s(2u).  The exponential is the hardware's of z log2(e),
// whose rounding in fp32 makes e^-z off by up to |z| 2^-24 of itself, and the
// roundings of a cubic z add as many each: up to 6 |z| 2^-24, 3e-5 at |z| = 88,
// beyond which e^-z leaves fp32.  Every result is rounded to bf16 next, up to
// 4e-3 of itself.
constexpr float GELU_2C = 1.5957691216057308f, GELU_A = 0.044715f;

__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

__device__ __forceinline__ float act_of(float v, int act) {
  const float z = act == MOE_ACT_GELU ? GELU_2C * (v + GELU_A * v * v * v) : v;
  return v * logistic(z);
}

// d/dv [v s(z)] = s + v s (1 - s) z'
__device__ __forceinline__ void act_grad(float v, int act, float* a, float* da) {
  const bool gelu = act == MOE_ACT_GELU;
  const float z = gelu ? GELU_2C * (v + GELU_A * v * v * v) : v;
  const float s = logistic(z), t = s * (1.0f - s);
  const float dz = gelu ? GELU_2C * (1.0f + 3.0f * GELU_A * v * v) : 1.0f;
  *a = v * s;
  // (t is 0 where s is 0 or 1, and dz may be infinite there)
  *da = t == 0.0f ? s : s + v * t * dz;
}

// ---- host checks ----------------------------------------------------------------
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace moe
