// The gate's logits and their gradients, and the routing's losses (moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "blocks.h"
#include "tile.h"

using namespace moe;

namespace {

// ---- the gate's products ----------------------------------------------------------
// logits = x wg, dx = d wg^T and dwg = x^T d on the tiles of the products over row
// groups, over the rows that some sequence has.  The tiles want whole 16 bytes, so
// a gate whose rows are none is copied with zeros behind each row; dlogits are
// rounded to bf16 for both products that take them, with zeros up to a multiple of
// 64, the depth of a stage.  The matrix instructions multiply bf16 by bf16, as x and
// the gate are: dlogits as two bf16 terms would be the products of twice the experts
// (32768 x 4096, E = 128 : 256, all gradients 135 : 200 us).  One term puts each of a
// sum's terms off by up to 2^-8: dx and dwg by 2.3e-3 of their 2-norm where nothing
// cancels, 1.7e-3 of it their own rounding.  A caller has both terms by two calls.
struct GateArgs {
  int T, H, E, S;
  int Ep;  // columns of the gate as the product reads it
  const int32_t* off;
  const uint16_t *x, *wg;
  const float *bias, *dlogits;
  float *logits, *dbias;
  uint16_t *dx, *dwg;
  uint16_t *gate, *d;  // workspace: the gate [H][Ep] where it is copied, dlogits [T][Ep]
  float *part, *bpart;  // partial sums: of a split product, and of dbias [dbias_parts][E]
  int split, bias_parts;
  int dx_split, dx_blocks, dwg_blocks;  // strips' parts of the rows; workgroups of dx and of dwg in one launch
};

__device__ __forceinline__ const char* bytes(const uint16_t* p) { return reinterpret_cast<const char*>(p); }

// The rows that some sequence has: from the first offset to the largest.
struct Rows {
  int b, e;
  __device__ __forceinline__ explicit Rows(const GateArgs& a) : b(0), e(a.T) {
    if (!a.off) return;
    const int lane = threadIdx.x & 63;
    int first = 0, most = 0;
    for (int i = lane; i <= a.S; i += 64) {
      const int v = clamp_off(a.off[i], a.T);
      if (i == 0) first = v;
      most = max(most, v);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, __shfl_xor(most, d));
    b = __builtin_amdgcn_readfirstlane(first);
    e = __builtin_amdgcn_readfirstlane(most);
  }
};

// Piece i of the gate's copy with rows of Ep values
__device__ __forceinline__ void copy_gate(const GateArgs& a, int i) {
  const int h = i / (a.Ep / 8), c = i % (a.Ep / 8) * 8;
  if (h >= a.H) return;
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = c + 2 * j < a.E ? a.wg[(size_t)h * a.E + c + 2 * j] : 0;
    const uint32_t hi = c + 2 * j + 1 < a.E ? a.wg[(size_t)h * a.E + c + 2 * j + 1] : 0;
    w[j] = lo | hi << 16;
  }
  *reinterpret_cast<u32x4_t*>(a.gate + (size_t)h * a.Ep + c) = u32x4_t{w[0], w[1], w[2], w[3]};
}
__global__ __launch_bounds__(256) void gate_copy_kernel(GateArgs a) { copy_gate(a, blockIdx.x * 256 + threadIdx.x); }

// What the gradients' products start from: dlogits in bf16 with rows of Ep values
// (where dx or dwg is wanted), and the parts of dbias; a workgroup takes 64 columns
// and its share of the rows, 16 threads side by side with 4 columns each.  The
// workgroups behind copy the gate.
__global__ __launch_bounds__(256) void gate_round_kernel(GateArgs a) {
  __shared__ f32x4_t red[16][16];
  const int part = blockIdx.x % a.bias_parts, strip = blockIdx.x / a.bias_parts;
  if (strip * 64 >= a.Ep) {
    copy_gate(a, (blockIdx.x - a.bias_parts * (a.Ep / 64)) * 256 + threadIdx.x);
    return;
  }
  const Rows r(a);
  const int n = ceil_div(r.e - r.b, a.bias_parts);
  const int begin = r.b + part * n, end = min(begin + n, r.e);
  const int c = strip * 64 + threadIdx.x % 16 * 4, first = threadIdx.x / 16;
  f32x4_t sum{0, 0, 0, 0};
#pragma unroll 4
  for (int row = begin + first; row < end; row += 16) {
    const float* p = a.dlogits + (size_t)row * a.E + c;
    f32x4_t v{0, 0, 0, 0};
    if (a.E % 4 == 0) {
      if (c < a.E) v = *reinterpret_cast<const f32x4_t*>(p);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.E) v[j] = p[j];
    }
    sum += v;
    if (a.d) *reinterpret_cast<uint2*>(a.d + (size_t)row * a.Ep + c) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
  if (!a.dbias) return;
  red[first][threadIdx.x % 16] = sum;
  __syncthreads();
  if (threadIdx.x >= 16) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += red[i][threadIdx.x];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < a.E) a.bpart[(size_t)part * a.E + c + j] = sum[j];
}

// 8 logits of a row from column c on, from their sums
__device__ __forceinline__ void put_logits(const GateArgs& a, size_t row, int c, const float* v) {
  float* out = a.logits + row * a.E + c;
  if (a.E % 4 == 0) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      if (c + i >= a.E) break;
      f32x4_t t{v[i], v[i + 1], v[i + 2], v[i + 3]};
      if (a.bias) t += *reinterpret_cast<const f32x4_t*>(a.bias + c + i);
      *reinterpret_cast<f32x4_t*>(out + i) = t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.E) out[i] = a.bias ? v[i] + a.bias[c + i] : v[i];
  }
}
// The same, or the partial sums [split][T][Ep] where the product is split.
__device__ __forceinline__ void put(const GateArgs& a, int part, size_t row, int c, const uint32_t* v) {
  if (c >= a.Ep) return;
  if (a.split > 1) {
    float* p = a.part + ((size_t)part * a.T + row) * a.Ep + c;
    reinterpret_cast<u32x4_t*>(p)[0] = u32x4_t{v[0], v[1], v[2], v[3]};
    reinterpret_cast<u32x4_t*>(p)[1] = u32x4_t{v[4], v[5], v[6], v[7]};
    return;
  }
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i]);
  put_logits(a, row, c, f);
}

template <typename S>
__global__ __launch_bounds__(S::THREADS) void gate_logits_kernel(GateArgs a) {
  using Tl = tile::Tile<S, false, false, true>;
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const Rows r(a);
  const int nt = ceil_div(a.Ep, Tl::BN), stages = a.H / 64;
  int m, n;
  if (!tile::pick(blockIdx.x, ceil_div(r.e - r.b, Tl::BM), nt * a.split, &m, &n)) return;
  const int part = n / nt, n0 = n % nt * Tl::BN, row = r.b + m * Tl::BM, rows = min(r.e - row, Tl::BM);
  const int k0 = stages * part / a.split * 64, k1 = stages * (part + 1) / a.split * 64;
  const tile::Operand A{bytes(a.x + (size_t)row * a.H + k0), nullptr, (uint32_t)a.H * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.gate + (size_t)k0 * a.Ep), nullptr, (uint32_t)a.Ep * 2, 0, n0, a.Ep};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, k1 - k0, A, B, 0);
  Tl::template epilogue<false>(acc, lds, rows, [&](int i, int c, const auto& v) { put(a, part, row + i, n0 + c, v); });
}

using Stream = tile::Shape<4, 2, 1, 2>;  // 128 x 128, 8 waves

// x comes from memory once, the gate from the L2, three stages of 32 KB under way in
// each CU; parts of the depth where there are fewer tiles than CUs.  A row tile starts at a stage of its own: rows are a power of
// two apart, and tiles that start together would read from the same memory channels
// all along (32768 x 4096 x 128: 71 us so, 58 with turns, 5.0 TB/s; two stages of
// Small tiles in two workgroups a CU, the depth in two parts, 81 + 12).
__global__ __launch_bounds__(Stream::THREADS) void gate_logits_stream_kernel(GateArgs a) {
  using Tl = tile::Tile<Stream, false, false, true>;
  __shared__ __attribute__((aligned(1024))) char lds[Tl::RING_LDS<4>];
  const Rows r(a);
  const int nt = ceil_div(a.Ep, Tl::BN), stages = a.H / 64;
  int m, n;
  if (!tile::pick(blockIdx.x, ceil_div(r.e - r.b, Tl::BM), nt * a.split, &m, &n)) return;
  const int part = n / nt, n0 = n % nt * Tl::BN, row = r.b + m * Tl::BM, rows = min(r.e - row, Tl::BM);
  const int s0 = stages * part / a.split, s1 = stages * (part + 1) / a.split;
  const tile::Operand A{bytes(a.x + (size_t)row * a.H + s0 * 64), nullptr, (uint32_t)a.H * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.gate + (size_t)s0 * 64 * a.Ep), nullptr, (uint32_t)a.Ep * 2, 0, n0, a.Ep};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::ring<4>(acc, lds, A, B, (s1 - s0) * 64, 1, m % (s1 - s0));
  Tl::template epilogue<false>(acc, lds, rows, [&](int i, int c, const auto& v) { put(a, part, row + i, n0 + c, v); });
}

template <int NW>
__global__ __launch_bounds__(NW * 64) void gate_logits_few_kernel(GateArgs a) {
  using Fw = tile::Few<NW, false, true, false>;
  __shared__ __attribute__((aligned(1024))) char lds[Fw::LDS];
  const Rows r(a);
  const int nt = ceil_div(a.Ep, Fw::COLS), steps = a.H / Fw::KE, mt = ceil_div(r.e - r.b, Fw::BM);
  int m, n;
  if (!tile::pick(blockIdx.x, mt, nt * a.split, &m, &n)) return;
  const int part = n / nt, n0 = n % nt * Fw::COLS, row = r.b + m * Fw::BM;
  const tile::Operand A{bytes(a.x + (size_t)row * a.H), nullptr, (uint32_t)a.H * 2, min(r.e - row, Fw::BM), 0, 0};
  const tile::Operand B{bytes(a.gate), nullptr, (uint32_t)a.Ep * 2, 0, n0, a.Ep};
  Fw::run(lds, A, B, steps * part / a.split, steps * (part + 1) / a.split, mt == 1,
          [&](int i, int c, const auto& v) { put(a, part, row + i, n0 + c, v); });
}

__global__ __launch_bounds__(256) void gate_logits_sum_kernel(GateArgs a) {
  const Rows r(a);
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8, row = i / a.Ep, c = i % a.Ep;
  if (row < r.b || row >= r.e) return;
  float v[8] = {};
  for (int s = 0; s < a.split; ++s) {
    const float* p = a.part + ((size_t)s * a.T + row) * a.Ep + c;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += p[j];
  }
  put_logits(a, row, (int)c, v);
}

__device__ __forceinline__ void store8(uint16_t* p, const uint32_t* v) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i]);
  *reinterpret_cast<u32x4_t*>(p) = tile::pack8(f);
}

template <typename S>
__global__ __launch_bounds__(S::THREADS) void gate_dx_kernel(GateArgs a) {
  using Tl = tile::Tile<S, false, false, false>;
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const Rows r(a);
  int m, n;
  if (!tile::pick(blockIdx.x, ceil_div(r.e - r.b, Tl::BM), ceil_div(a.H, Tl::BN), &m, &n)) return;
  const int n0 = n * Tl::BN, row = r.b + m * Tl::BM, rows = min(r.e - row, Tl::BM);
  const tile::Operand A{bytes(a.d + (size_t)row * a.Ep), nullptr, (uint32_t)a.Ep * 2, rows, 0, 0};
  const tile::Operand B{bytes(a.gate + (size_t)n0 * a.Ep), nullptr, (uint32_t)a.Ep * 2, a.H - n0, 0, 0};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, a.Ep, A, B, 0);
  Tl::template epilogue<false>(acc, lds, rows, [&](int i, int c, const auto& v) {
    if (n0 + c < a.H) store8(a.dx + (size_t)(row + i) * a.H + n0 + c, v);
  });
}

// dx where the depth is 64 to 256 (KC times 64): nothing but dx itself comes from or
// goes to memory, so a wave keeps its 64 columns of the gate in registers and passes
// over rows.  Eight waves share strips of 64 rows of dlogits, which come from the
// caches into a ring of three in LDS (k-contiguous, granules as in tile.h), two
// ahead; four wide by two deep, a wave multiplies 32 rows by its columns.  The
// columns are dealt to the matrix instruction so that a lane's 32 results are
// consecutive; they pass through 4 KB of LDS of the wave's own and leave as whole
// lines.  32768 x 128 x 4096 alone: 49 to 57 us, 5 TB/s of writes; on 256 x 256 tiles 85;
// with dlogits loaded straight into registers 89 (a lane's 16 bytes are a row's, 32
// rows a load).
template <int KC>
__device__ __forceinline__ void dx_strips(const GateArgs& a, int block, char* lds) {
  constexpr int STRIP = KC * 8192, RING = 3;  // and 8 * 4096 bytes behind them
  const Rows r(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int panels = ceil_div(a.H, 256), run = ceil_div(panels * a.dx_split, NXCD);
  const int w = block % NXCD * run + block / NXCD;
  if (block / NXCD >= run || w >= panels * a.dx_split) return;
  const int part = w / panels, n0 = w % panels * 256 + wave % 4 * 64, deep = wave / 4 * 32;
  const int strips = ceil_div(r.e - r.b, 64);  // dealt to the parts in turn
  if (part >= strips) return;
  const bool active = n0 < a.H;
  const int half = lane >> 5, i = lane & 31;
  const auto swz = [](int row) { return (row >> 1) & 7; };
  // row i of the instruction's first operand: lane half h of its results holds the rows 8 q + 4 h + j, which are the
  // columns 32 h + 16 nb + 4 q + j
  bf16x8_t g[2][KC * 4];
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int k = 0; k < KC * 4; ++k) {
      const int col = min(n0, a.H - 64) + 32 * (i >> 2 & 1) + 16 * nb + 4 * (i >> 3) + (i & 3);
      g[nb][k] = *reinterpret_cast<const bf16x8_t*>(a.gate + (size_t)col * a.Ep + k * 16 + half * 8);
    }
  const uint32_t l0 = tile::lds_u32(lds) + wave * 1024;
  const char* d0 = tile::uniform_ptr(bytes(a.d) + (size_t)r.b * a.Ep * 2);
  const int in = wave * 8 + lane / 8, rows = r.e - r.b;
  int slot_in = 0;
  const auto issue = [&](int strip) {  // a wave loads 8 rows of the strip
    const uint32_t o = (uint32_t)min(strip * 64 + in, rows - 1) * (uint32_t)(a.Ep * 2) + (uint32_t)(((lane & 7) ^ swz(in)) * 16);
#pragma unroll
    for (int k = 0; k < KC; ++k) tile::dma16(d0, o + k * 128, l0 + slot_in * STRIP + k * 8192);
    slot_in = slot_in == RING - 1 ? 0 : slot_in + 1;
  };
  char* mine = lds + RING * STRIP + wave * 4096;
  tile::wait_vm<0>();  // (the gate's loads: only strips and stores are counted from here)
  issue(part);
  if (part + a.dx_split < strips) issue(part + a.dx_split);
  int slot = 0, turn = 0;
  for (int strip = part; strip < strips; strip += a.dx_split, slot = slot == RING - 1 ? 0 : slot + 1, ++turn) {
    // behind this strip's loads are the next one's and two strips' stores, 4 each
    tile::compiler_fence();
    if (strip + a.dx_split >= strips) tile::wait_vm<0>();
    else if (active && turn >= 2) tile::wait_vm<KC + 8>();
    else tile::wait_vm<KC>();
    tile::lds_barrier();
    if (strip + 2 * a.dx_split < strips) issue(strip + 2 * a.dx_split);
    if (!active) continue;
    const char* st = lds + slot * STRIP + (deep + i) * 128;
    f32x16_t acc[2];
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[0][j] = acc[1][j] = 0;
#pragma unroll
    for (int k = 0; k < KC * 4; ++k) {
      const bf16x8_t d = *reinterpret_cast<const bf16x8_t*>(st + k / 4 * 8192 + ((k % 4 * 2 + half) ^ swz(deep + i)) * 16);
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g[nb][k], d, acc[nb], 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // 8 columns of row i each, 16-byte granules at position c ^ (row & 7)
      const f32x16_t& v = acc[q / 2];
      const int o = q % 2 * 8;
      *reinterpret_cast<u32x4_t*>(mine + i * 128 + ((half * 4 + q) ^ (i & 7)) * 16) =
          u32x4_t{pack_bf16x2(v[o], v[o + 1]), pack_bf16x2(v[o + 2], v[o + 3]), pack_bf16x2(v[o + 4], v[o + 5]),
                  pack_bf16x2(v[o + 6], v[o + 7])};
    }
    tile::compiler_fence();
    const int row0 = r.b + strip * 64 + deep;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = q * 8 + lane / 8, c = lane % 8;
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(mine + row * 128 + (c ^ (row & 7)) * 16);
      if (row0 + row < r.e) *reinterpret_cast<u32x4_t*>(a.dx + (size_t)(row0 + row) * a.H + n0 + c * 8) = v;
    }
  }
}

// A tile's sums, as one of the parts [split][H][Ep] of dwg
template <typename Tl>
__device__ __forceinline__ void put_dwg(const GateArgs& a, const typename Tl::Acc& acc, char* lds, int part, int m0, int n0) {
  float* sums = a.part + (size_t)part * a.H * a.Ep;
  Tl::template epilogue<false>(acc, lds, min(Tl::BM, a.H - m0), [&](int i, int c, const uint32_t (&v)[8]) {
    c += n0;
    if (c >= a.Ep) return;
    u32x4_t* o = reinterpret_cast<u32x4_t*>(sums + (size_t)(m0 + i) * a.Ep + c);
    o[0] = u32x4_t{v[0], v[1], v[2], v[3]};
    o[1] = u32x4_t{v[4], v[5], v[6], v[7]};
  });
}

// dwg: tiles of 128 columns of x by 128 or 256 experts, the rows their depth, in stages of
// 64 that are dealt to the parts in turn.  Tiles of one part follow each other: they
// read the same rows of dlogits and run on one XCD.  32768 x 4096 x 128 in 256
// workgroups: 57 us alone, 5 TB/s; behind dx, whose writes are still on their way to
// memory, 78, with parts of consecutive rows 84, and on two stages of Small tiles 85.
template <bool BROAD>
using DwTile = tile::Tile<std::conditional_t<BROAD, tile::Shape<2, 4, 2, 2>, Stream>, false, true, true>;
template <bool BROAD>
constexpr int DW_RING = BROAD ? 3 : 4;  // stages of 48 or 32 KB
template <bool BROAD>
__device__ __forceinline__ void dwg_tile(const GateArgs& a, int block, char* lds) {
  using Tl = DwTile<BROAD>;
  const Rows r(a);
  const int mt = ceil_div(a.H, Tl::BM), nt = ceil_div(a.E, Tl::BN), per = mt * nt, run = ceil_div(per * a.split, NXCD);
  const int w = block % NXCD * run + block / NXCD;
  if (block / NXCD >= run || w >= per * a.split) return;
  const int part = w / per, m0 = w % per % mt * Tl::BM, n0 = w % per / mt * Tl::BN;
  const int stages = ceil_div(r.e - r.b, 64), mine = stages > part ? (stages - part - 1) / a.split + 1 : 0;
  const int depth = mine * 64 - (mine && (stages - 1) % a.split == part ? stages * 64 - (r.e - r.b) : 0);
  const size_t row = r.b + part * 64;
  const tile::Operand A{bytes(a.x + row * a.H), nullptr, (uint32_t)a.H * 2, 0, m0, a.H};
  const tile::Operand B{bytes(a.d + row * a.Ep), nullptr, (uint32_t)a.Ep * 2, 0, n0, a.Ep};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::template ring<DW_RING<BROAD>>(acc, lds, A, B, depth, a.split, 0);
  put_dwg<Tl>(a, acc, lds, part, m0, n0);
}

// The same on 256 x 256 tiles, whose operands come through the L2 half as often;
// parts of the rows follow each other.
__global__ __launch_bounds__(512) void gate_dwg_wide_kernel(GateArgs a) {
  using Tl = tile::Tile<tile::Wide, false, true, true>;
  __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
  const Rows r(a);
  const int mt = ceil_div(a.H, Tl::BM), nt = ceil_div(a.E, Tl::BN), per = mt * nt, run = ceil_div(per * a.split, NXCD);
  const int w = blockIdx.x % NXCD * run + blockIdx.x / NXCD;
  if ((int)blockIdx.x / NXCD >= run || w >= per * a.split) return;
  const int part = w / per, m0 = w % per % mt * Tl::BM, n0 = w % per / mt * Tl::BN;
  const int stages = ceil_div(r.e - r.b, 64);
  const int k0 = stages * part / a.split * 64, k1 = min(stages * (part + 1) / a.split * 64, r.e - r.b);
  const tile::Operand A{bytes(a.x + (size_t)(r.b + k0) * a.H), nullptr, (uint32_t)a.H * 2, 0, m0, a.H};
  const tile::Operand B{bytes(a.d + (size_t)(r.b + k0) * a.Ep), nullptr, (uint32_t)a.Ep * 2, 0, n0, a.Ep};
  typename Tl::Acc acc;
  Tl::zero(acc);
  Tl::run(acc, lds, A, B, k1 - k0, A, B, 0);
  put_dwg<Tl>(a, acc, lds, part, m0, n0);
}

// dx, which is written, and dwg, for which x is read, in one launch, in turn by eight
// workgroups (one for each XCD): either may have none.  32768 rows, H = 4096, E = 128:
// 117 to 136 us for 0.55 GB, about a copy's rate; one after the other 57 + 78.
template <int KC, bool BROAD>
__global__ __launch_bounds__(512, 2) void gate_grad_kernel(GateArgs a) {
  constexpr int LDS = std::max(DwTile<BROAD>::template RING_LDS<DW_RING<BROAD>>, KC ? 3 * KC * 8192 + 8 * 4096 : 0);
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  const int eights = std::min(a.dx_blocks, a.dwg_blocks) / NXCD, turn = blockIdx.x / NXCD, x = blockIdx.x % NXCD;
  const bool mixed = turn < 2 * eights;
  const bool dx = mixed ? turn % 2 == 0 : a.dx_blocks > a.dwg_blocks;
  const int block = (mixed ? turn / 2 : turn - eights) * NXCD + x;
  if (KC && dx) dx_strips<KC ? KC : 1>(a, block, lds);
  else if (!dx) dwg_tile<BROAD>(a, block, lds);
}

// dwg from its parts, 4 columns a thread, and behind it dbias: 16 columns a
// workgroup, 16 threads each.
__global__ __launch_bounds__(256) void gate_sum_kernel(GateArgs a, int dwg_blocks) {
  __shared__ float red[16][16];
  if ((int)blockIdx.x >= dwg_blocks) {
    const int q = threadIdx.x % 16, c = (blockIdx.x - dwg_blocks) * 16 + q, first = threadIdx.x / 16;
    float v = 0;
    if (c < a.E)
#pragma unroll 8
      for (int i = first; i < a.bias_parts; i += 16) v += a.bpart[(size_t)i * a.E + c];
    red[first][q] = v;
    __syncthreads();
    if (first || c >= a.E) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) v += red[i][q];
    a.dbias[c] = v;
    return;
  }
  const int i = blockIdx.x * 256 + threadIdx.x, h = i / (a.Ep / 4), c = i % (a.Ep / 4) * 4;
  if (h >= a.H || c >= a.E) return;
  f32x4_t v{0, 0, 0, 0};
#pragma unroll 8
  for (int s = 0; s < a.split; ++s) v += *reinterpret_cast<const f32x4_t*>(a.part + ((size_t)s * a.H + h) * a.Ep + c);
  uint16_t* out = a.dwg + (size_t)h * a.E + c;
  if (a.E % 4 == 0) {
    *reinterpret_cast<uint2*>(out) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < a.E) out[j] = (uint16_t)f32_to_bf16(v[j]);
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
// before a row is worked on.  Bound by memory (131072 x 512 in 62 us with the sums, 4.4
// TB/s) or, below 32768 rows of 128, by two launches of a few latencies each (16).
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

// A batch whose softmax fits the LDS, by one workgroup: 333 rows of 8 experts in 6.2
// us, against 4.8 + 6.6 by the two kernels above, each a chain of memory latencies.
constexpr int SMALL_ROWS = 1024, SMALL_P = 16384, SMALL_COUNTS = 4096;
template <typename R>
__global__ __launch_bounds__(1024) void route_loss_small_kernel(LossArgs a) {
  __shared__ float p[SMALL_P];  // [row][Ep]
  __shared__ int hist[SMALL_COUNTS], start[MOE_MAX_GROUPS + 1];
  __shared__ float vs[16], zs[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % R::LPR, sub = lane / R::LPR;
  const SeqTiles list(a.off, a.S, a.T, a.bm);
  int begin = 0;
  if (a.off) {
    begin = __builtin_amdgcn_readfirstlane(list.first);
    if (wave == 0) {
      int at = list.first;
      for (int g = list.g0; g < list.g1; ++g) {
        start[g] = at;
        at = max(at, clamp_off(a.off[g + 1], a.T));
      }
    }
  } else if (threadIdx.x == 0) {
    start[0] = 0;
  }
  const int end = begin + list.rows;
  if (threadIdx.x == 0) start[a.S] = end;
  for (int i = threadIdx.x; i < a.S * a.Ep; i += 1024) hist[i] = 0;
  float z = 0;
  for (int base = begin + wave * R::AT_ONCE; base < end; base += 16 * R::AT_ONCE) {
    const int row = base + sub;
    float v[R::N], top = -__builtin_inff(), total = 0;
    R::load(v, a.logits + (size_t)row * a.E, l, a.E, row < end);
#pragma unroll
    for (int i = 0; i < R::N; ++i) top = fmaxf(top, v[i]);
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
    if (row >= end) continue;
    if (l == 0) {
      a.lse[row] = lse;
      z += total == 0 ? 0 : lse * lse;
    }
#pragma unroll
    for (int i = 0; i < R::N; ++i)
      if (R::column(l, i) < a.Ep) p[(row - begin) * a.Ep + R::column(l, i)] = v[i] * inv;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (end - begin) * a.K; i += 1024) {
    const int e = a.idx[(size_t)begin * a.K + i], row = begin + i / a.K;
    int g = 0;  // the last sequence that starts at or before the row (those without rows start where the next one does)
    for (int d = 256; d; d >>= 1)
      if (g + d < a.S && start[g + d] <= row) g += d;
    if (e >= 0 && e < a.E) atomicAdd(&hist[g * a.Ep + e], 1);
  }
  __syncthreads();
  // 8 threads a sequence and expert, each over every eighth row
  float v = 0;
  for (int q = threadIdx.x / 8; q < a.S * a.Ep; q += 128) {
    const int g = q / a.Ep, e = q % a.Ep, first = start[g], rows = start[g + 1] - first;
    float sum = 0;
#pragma unroll 4
    for (int row = threadIdx.x % 8; row < rows; row += 8) sum += p[(first - begin + row) * a.Ep + e];
    if (e < a.E && threadIdx.x % 8 == 0) a.counts[(size_t)g * a.E + e] = hist[q];
    const float n = (float)rows;
    if (rows) v += sum * (float)hist[q] * (a.E / (a.K * n * n));
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    v += __shfl_xor(v, d);
    z += __shfl_xor(z, d);
  }
  if (lane == 0) {
    vs[wave] = v;
    zs[wave] = z;
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
bool is_small(const LossArgs& a) {
  return a.T <= SMALL_ROWS && a.T * a.Ep <= SMALL_P && a.S * a.Ep <= SMALL_COUNTS;
}

__global__ __launch_bounds__(256) void route_loss_none_kernel(LossArgs a) {
  for (int i = threadIdx.x; i < a.S * a.E; i += 256) a.counts[i] = 0;
  if (threadIdx.x < 2) a.loss[threadIdx.x] = 0;
}

// 32768 rows, E = 128: 13.5 us, 6 of them a launch, the offsets and the first loads, the
// others at memory's rate; 131072 x 512 116 us, 4.7 TB/s.
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
      // (choices are in the row's first 8 lanes; of a dead row routing's weights are NaN)
      float all = r.w * r.dw;
#pragma unroll
      for (int d = 4; d; d >>= 1) all += __shfl_xor(all, d);
      const float t = dead ? 0.0f : r.w * (r.dw - all);
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

// About 1024 tiles of a long batch, whose sums fit the caches; at least as many rows as
// the four wavefronts take in two turns (one, where they take 32 at once).  E = 256, 8 rows
// against 32, losses and gradient, us: 512 rows 12.6 : 16.1, 9.0 : 11.7; 8192 16.4 : 17.9,
// 9.2 : 14.3; E = 128, 16 against 32, 512 rows 12.6 : 13.5.
LossArgs loss_args(const moe_router_config* c, const int32_t* off) {
  LossArgs a{};
  a.T = c->rows, a.E = c->n_experts, a.K = c->top_k, a.S = c->n_seqs, a.off = off;
  a.Ep = ceil_div(a.E, 4) * 4;
  const int turns = 2 * 4 * (a.E <= 64 ? 4 : a.E <= 128 ? 2 : 1);
  a.bm = std::max(turns, ceil_div(a.T, 1024));
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

// How the gate's products are computed, from the config alone.
struct GatePlan {
  int Ep;           // columns of the gate
  bool copied;      // the gate is copied to have them
  bool stream;      // logits by a ring of stages; dx by strips
  tile::Plan prod;  // the tiles of logits, or of dx, where they are not; parts of logits' depth
  int dx_split;     // parts of the rows that strips are dealt to
  bool dwg_wide, dwg_broad;   // dwg on 256 x 256 tiles, on 128 x 256
  int dwg_split, bias_parts;  // dwg's and dbias's parts of the rows
};
GatePlan logits_plan(const moe_router_config* c) {
  GatePlan p{};
  p.Ep = ceil_div(c->n_experts, 8) * 8;
  p.copied = p.Ep != c->n_experts;
  // x, which is long, is what the time is spent on, so this has a rule of its own: the
  // ring, or tiles of few rows, in the number of parts whose estimate is lowest.  us,
  // fitted to 130 sizes (64 to 32768 rows, H = 1024 to 8192): a ring's stage 0.5; a CU's
  // pass over a tile of few rows 0.0016 to 0.0024 for each step of the depth; x from
  // memory as far as it passes 50 MB, overlapped better by the ring; parts a launch and
  // their sums.  Ring : few rows, us, H = 4096: E = 128, 4096 rows 37, 20 in four parts :
  // 14; 8192 37, 26 in four : 24; 16384 48, 42 in two : 65; 32768 58 : 122; E = 8, 32768
  // rows 51 : 69; E = 256, 8192 rows 39, 34 in two : 42; H = 8192, E = 64, 2048 rows 67, 19
  // in eight : 22, 14 in four.  The rule that the products over row groups have took 12
  // and 33 for 2048 rows of that (E = 64, 512), 32 for E = 128, 8192 rows, 50 for 16384.
  const int stages = c->hidden / 64, few = ceil_div(c->rows, 32) * ceil_div(p.Ep, 64);
  const int tiles = ceil_div(c->rows, Stream::BM) * ceil_div(p.Ep, Stream::BN);
  const double far = std::max(0.0, 2.0 * c->rows * c->hidden - 50e6);
  // More tiles of the ring than CUs: of one column it is the best all the same; of more,
  // the other tiles (E = 512, 32768 rows 183 : 124; E = 256, 20000 rows 79 : 69)
  if (tiles > 256 && p.Ep > Stream::BN) {
    p.prod = tile::plan_of(c->rows, 1, p.Ep, 1, stages, false);
    return p;
  }
  double best = 1e30;
  const auto take = [&](bool stream, tile::Plan plan, double us) {
    if (plan.split > 1) us += 4 + 0.25 * plan.split + 4.0 * plan.split * c->rows * p.Ep / 2.2e6;
    if (us < best) best = us, p.stream = stream, p.prod = plan;
  };
  for (int s = 1; s <= tile::MAX_SPLIT && (s == 1 || 4 * s <= stages); s *= 2) {
    if (s == 1 || tiles * s <= 256)
      take(true, {tile::Plan::SMALL, s}, 4.5 + ceil_div(tiles * s, 256) * 0.5 * stages / s + far / 9e6);
    if (s == 1 || few * s <= 256)
      take(false, {few * s <= 256 ? tile::Plan::FEW8 : tile::Plan::FEW4, s},
           4 + ceil_div(few * s, 256) * (double)c->hidden / s * (1.6e-3 + 0.8e-3 * std::min(p.Ep, 64) / 64) + far / 5e6);
  }
  return p;
}
GatePlan grad_plan(const moe_router_config* c, bool with_dwg = true) {
  GatePlan p{};
  p.Ep = ceil_div(c->n_experts, 64) * 64;
  p.copied = p.Ep != c->n_experts;
  p.prod = tile::plan_of(c->rows, 1, c->hidden, 1, p.Ep / 64, false);
  p.prod.split = 1;
  // Strips as far as the gate's columns fit a wave's registers (E = 256: 128 of them).
  // Strips against tiles, us: H = 4096, 32768 rows, dx alone, E = 128 60 : 88, E = 256 87 :
  // 122; all gradients, E = 256, 8192 rows 68 : 75, 2048 28 : 34, 512 21 : 29, H = 1024,
  // 2048 rows 20 : 29; E = 128, 2048 21 : 28.
  p.stream = p.Ep <= 256;
  const int stages = std::max(1, ceil_div(c->rows, 64));
  // Wide tiles where each of 256 workgroups has 20 stages or more.  Wide against 128 x
  // 128, us with the launches around them: H = 4096, 32768 rows, E = 512 (64 stages)
  // 152 : 201, E = 300 (64) 132 : 193, E = 256 (32) 103 : 109; 8192 rows, E = 300 (16)
  // 51 : 55, E = 512 (16) 62 : 60, E = 256 (8) 48 : 38.
  p.dwg_wide = p.Ep > 128 &&
               stages * ceil_div(c->hidden, tile::Wide::BM) * ceil_div(c->n_experts, tile::Wide::BN) >= 20 * 256;
  // One workgroup a CU: half of the CUs each where both are in one launch.  128 + 128
  // workgroups against 256 + 256 and 64 + 128 of dx and dwg, us: H = 4096, E = 128, 32768
  // rows 135 : 144 : 171, 4531 29 : 37 : 35; H = 2048, E = 60, 4531 rows 20 : 24 : 22.  dx
  // alone takes them all, for its bits do not depend on its parts; dwg's do, and are
  // the same whatever else is asked for (alone 102 where 256 parts take 75).
  const bool together = p.stream && !p.dwg_wide;
  // Broad tiles read x once, which pays where it is long; of fewer rows their parts are
  // more, and of more experts there are too few.  Broad against 128 x 128, us: E = 256, 8192
  // x 4096 60 : 67, 4096 x 7168 58 : 64, 32768 x 1024 68 : 73, 16384 x 1024 41 : 42, 8192 x
  // 2048 39 : 35; E = 192 56 : 65, 54 : 63, 61 : 70, 38 : 38, 33 : 32; E = 512, 4096 x 2048 46 : 42.
  p.dwg_broad = !p.dwg_wide && p.Ep > 128 && p.Ep <= 256 && (long long)c->rows * c->hidden >= 24 << 20;
  const int bm = p.dwg_wide ? 256 : 128, bn = p.dwg_wide || p.dwg_broad ? 256 : 128;
  const auto parts = [&](int most, int tiles) { return std::max(1, std::min(stages, most / tiles)); };
  p.dwg_split = parts(together ? 128 : 256, ceil_div(c->hidden, bm) * ceil_div(c->n_experts, bn));
  p.dx_split = parts(together && with_dwg ? 128 : 256, ceil_div(c->hidden, 256));
  p.bias_parts = std::max(1, std::min(512, ceil_div(c->rows, 16)));
  return p;
}

// Workspace: the gate's copy, dlogits in bf16, dbias's parts, then the products' partial sums.
struct GateSpace {
  size_t gate, d, bpart, part, total;
};
GateSpace gate_space(const moe_router_config* c, bool backward) {
  const GatePlan p = backward ? grad_plan(c) : logits_plan(c);
  GateSpace w{};
  w.d = p.copied ? align_up(sizeof(uint16_t) * c->hidden * p.Ep, 256) : 0;
  w.bpart = w.d + (backward ? align_up(sizeof(uint16_t) * (size_t)c->rows * p.Ep, 256) : 0);
  w.part = w.bpart + (backward ? align_up(sizeof(float) * p.bias_parts * c->n_experts, 256) : 0);
  const size_t logits = p.prod.split > 1 ? sizeof(float) * (size_t)p.prod.split * c->rows * p.Ep : 0;
  w.total = w.part + (backward ? sizeof(float) * (size_t)p.dwg_split * c->hidden * p.Ep : logits) + 256;
  return w;
}
size_t gate_ws(const moe_router_config* c, bool backward) { return gate_space(c, backward).total; }

GateArgs gate_args(const moe_router_config* c, const int32_t* off, const uint16_t* wg, bool backward, void* ws) {
  const GatePlan p = backward ? grad_plan(c) : logits_plan(c);
  const GateSpace w = gate_space(c, backward);
  char* at = static_cast<char*>(ws);
  GateArgs a{};
  a.T = c->rows, a.H = c->hidden, a.E = c->n_experts, a.S = c->n_seqs, a.off = off;
  a.Ep = p.Ep, a.wg = wg;
  a.d = reinterpret_cast<uint16_t*>(at + w.d);
  a.bpart = reinterpret_cast<float*>(at + w.bpart), a.part = reinterpret_cast<float*>(at + w.part);
  a.bias_parts = p.bias_parts;
  a.gate = p.copied ? reinterpret_cast<uint16_t*>(at) : const_cast<uint16_t*>(wg);
  return a;
}

}  // namespace

extern "C" {

moe_status moe_gate_workspace_size(const moe_router_config* cfg, int32_t backward, size_t* bytes) {
  moe_status st = check_gate(cfg);
  if (st != MOE_OK) return st;
  if (!bytes) return fail(MOE_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = gate_ws(cfg, backward != 0);
  return MOE_OK;
}

moe_status moe_gate_plan_host(const moe_router_config* cfg, moe_gate_plan* out) {
  moe_status st = check_gate(cfg);
  if (st != MOE_OK) return st;
  if (!out) return fail(MOE_ERR_INVALID_ARG, "out is NULL");
  const GatePlan l = logits_plan(cfg), g = grad_plan(cfg);
  out->logits = {l.stream ? (int)MOE_TILES_RING : (int)l.prod.kind, l.prod.split};
  out->dx = {g.stream ? (int)MOE_TILES_STRIPS : (int)g.prod.kind, g.stream ? g.dx_split : 1};
  out->dwg = {g.dwg_wide ? MOE_TILES_WIDE : g.dwg_broad ? MOE_TILES_BROAD : MOE_TILES_RING, g.dwg_split};
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
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  GateArgs a = gate_args(cfg, seq_off, wg, false, ws);
  a.x = x, a.bias = logit_bias, a.logits = logits;
  const GatePlan p = logits_plan(cfg);
  a.split = p.prod.split;
  if (p.copied) gate_copy_kernel<<<ceil_div(a.H * (a.Ep / 8), 256), 256, 0, s>>>(a);
  const auto go = [&](auto kernel, int bm, int bn, int threads) {
    kernel<<<tile::grid_of(ceil_div(a.T, bm), ceil_div(a.Ep, bn) * a.split), threads, 0, s>>>(a);
  };
  using tile::Small, tile::Wide;
  if (p.stream) go(gate_logits_stream_kernel, Stream::BM, Stream::BN, Stream::THREADS);
  else switch (p.prod.kind) {
    case tile::Plan::FEW4: go(gate_logits_few_kernel<4>, 32, 64, 256); break;
    case tile::Plan::FEW8: go(gate_logits_few_kernel<8>, 32, 64, 512); break;
    case tile::Plan::SMALL: go(gate_logits_kernel<Small>, Small::BM, Small::BN, Small::THREADS); break;
    case tile::Plan::WIDE: go(gate_logits_kernel<Wide>, Wide::BM, Wide::BN, Wide::THREADS); break;
  }
  if (a.split > 1) gate_logits_sum_kernel<<<(int)(((long long)a.T * a.Ep / 8 + 255) / 256), 256, 0, s>>>(a);
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
  if (dx && (dx == x || dx == wg)) return fail(MOE_ERR_INVALID_ARG, "dx is x or wg");
  if (dwg && (dwg == wg || dwg == x)) return fail(MOE_ERR_INVALID_ARG, "dwg is wg or x");
  if ((st = check_ws(ws, ws_bytes, gate_ws(cfg, true))) != MOE_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (!dx && !dwg && !dbias) return MOE_OK;
  if (cfg->rows == 0) dx = nullptr;
  GateArgs a = gate_args(cfg, seq_off, wg, true, ws);
  a.x = x, a.dlogits = dlogits, a.dx = dx, a.dwg = dwg, a.dbias = dbias;
  if (!dx && !dwg) a.d = nullptr;
  const GatePlan p = grad_plan(cfg, dwg != nullptr);
  const int copies = p.copied && dx ? ceil_div(a.H * (a.Ep / 8), 256) : 0;
  gate_round_kernel<<<a.bias_parts * (a.Ep / 64) + copies, 256, 0, s>>>(a);
  if (dx && !p.stream) {
    using tile::Small, tile::Wide;
    const auto go = [&](auto kernel, int bm, int bn, int threads) {
      kernel<<<tile::grid_of(ceil_div(a.T, bm), ceil_div(a.H, bn)), threads, 0, s>>>(a);
    };
    if (p.prod.kind == tile::Plan::WIDE) go(gate_dx_kernel<Wide>, Wide::BM, Wide::BN, Wide::THREADS);
    else go(gate_dx_kernel<Small>, Small::BM, Small::BN, Small::THREADS);
  }
  a.split = p.dwg_split, a.dx_split = p.dx_split;
  const auto eights = [](int n) { return ceil_div(n, NXCD) * NXCD; };
  a.dx_blocks = dx && p.stream ? eights(ceil_div(a.H, 256) * a.dx_split) : 0;
  if (dwg && p.dwg_wide)
    gate_dwg_wide_kernel<<<eights(ceil_div(a.H, tile::Wide::BM) * ceil_div(a.E, tile::Wide::BN) * a.split), 512, 0, s>>>(a);
  else if (dwg)
    a.dwg_blocks = eights(ceil_div(a.H, 128) * ceil_div(a.E, p.dwg_broad ? 256 : 128) * a.split);
  const auto go = [&](auto kernel, decltype(kernel) broad = nullptr) {
    (p.dwg_broad ? broad : kernel)<<<a.dx_blocks + a.dwg_blocks, 512, 0, s>>>(a);
  };
  if (a.dx_blocks + a.dwg_blocks) switch (a.dx_blocks ? a.Ep : 0) {
    case 0: go(gate_grad_kernel<0, false>, gate_grad_kernel<0, true>); break;
    case 64: go(gate_grad_kernel<1, false>); break;
    case 128: go(gate_grad_kernel<2, false>); break;
    case 192: go(gate_grad_kernel<3, false>, gate_grad_kernel<3, true>); break;
    case 256: go(gate_grad_kernel<4, false>, gate_grad_kernel<4, true>); break;
  }
  const int sums = dwg ? ceil_div(a.H * (a.Ep / 4), 256) : 0;
  if (dwg || dbias) gate_sum_kernel<<<sums + (dbias ? ceil_div(a.E, 16) : 0), 256, 0, s>>>(a, sums);
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
  } else if (is_small(a)) {
    for_row(a.E, [&](auto row) { route_loss_small_kernel<decltype(row)><<<1, 1024, 0, s>>>(a); });
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
