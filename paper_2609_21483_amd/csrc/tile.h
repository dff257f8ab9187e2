// Matrix-core tiles of the products over row groups (ffn.hip, int8.hip):
// C[BM x BN] = A[BM x K] B[K x BN], bf16 or int8 operands read where they lie.
//
// An operand is k-contiguous (rows of the tile, each a run of the depth) or
// transposed (rows of the depth, each a run of the tile's rows or columns):
// weights [H][F] are the latter for x W and the former for d W^T, and both
// operands of x^T d are.  No pass over the weights lays them out first.
//
// A stage of the depth is 128 bytes of it: 64 bf16 or 128 int8 values, BM * 128
// and BN * 128 bytes, loaded straight into LDS (global_load_lds_dwordx4), two
// stages in turn.  LDS images, in 16-byte granules:
//  - k-contiguous: row r at r * 128 bytes, granule c at position c ^ (r / 2) % 8.
//    A fragment (lane: row l % 32, 16 bytes of the depth) is one ds_read_b128,
//    and the 16 rows read together lie on different banks (c ^ r % 8: every
//    read took twice the cycles).
//  - transposed (bf16): two panels of half the tile's width, each 64 depth rows
//    of PW columns; granule c of row k at position c ^ swz(k).  A fragment is
//    two ds_read_b64_tr_b16: 16 lanes address 4 depth rows x 16 columns, lane
//    i at row i / 4, columns 4 (i % 4), and lane i receives column i of all 4.
//    The swizzle puts the four rows' 64-byte pieces (32 columns) on different
//    banks.
// Panels also let a gated tile take half of its columns from each matrix: a
// wave's first NB / 2 column blocks lie in panel 0 and the others, the same
// columns, in panel 1.
//
// WM x WN waves, each MB x NB blocks of 32 x 32 (v_mfma_f32_32x32x16_bf16,
// v_mfma_i32_32x32x32_i8).  Row block b of the tile belongs to wave row
// b % WM.  B is the first operand of the instruction, so that a lane's
// accumulators are 4 consecutive columns of one row: column 8 (r / 4) + 4 (l /
// 32) + r % 4 of row l % 32 in register r.
//
// What bounds Wide tiles (x W of 8192 x 4096 x 28672, 1640 us): the loads alone
// take 1340 (13 TB/s over all CUs, 80% of it L2 hits), the LDS reads and
// products alone 1475, at a clock that falls to 1.65 GHz (int8: 2.0).  A ring of
// five 64-byte steps, three to four ahead, took 5 to 12% longer (half lines of
// the k-contiguous operand, twice the barriers); four waves of 128 x 128 1 to 8%
// longer; uniform branches around a partly filled tile's empty row blocks 8%
// longer on full ones and no shorter on ragged groups.
#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "blocks.h"
#include "gemm.h"

namespace moe {
namespace tile {

using gemm::compiler_fence;
using gemm::dma16;
using gemm::lds_barrier;
using gemm::lds_u32;
using gemm::uniform_ptr;
using gemm::wait_vm;

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((__vector_size__(4 * sizeof(short))));

constexpr int DEPTH = 128;  // bytes of the depth per stage

// One operand's matrix as a tile sees it: `p` and, for the second panel, `p2`
// (the same matrix, or the up projection's) are the addresses of depth 0; ld
// the bytes between rows.  k-contiguous: `valid` rows exist from p on, rows
// from half the tile on are read at p2 (gated) or behind p (p2 = NULL).
// Transposed: columns [col, cols) of the matrix exist, a panel starts at col
// (+ PW in panel 1 unless p2 is given).
struct Operand {
  const char *p, *p2;
  uint32_t ld;
  int valid, col, cols;
};

template <int WM_, int WN_, int MB_, int NB_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_;
  static constexpr int BM = WM * MB * 32, BN = WN * NB * 32, THREADS = WM * WN * 64;
};
using Wide = Shape<2, 4, 4, 2>;   // 256 x 256
using Small = Shape<2, 2, 2, 2>;  // 128 x 128

template <typename S, bool I8_, bool AT_, bool BT_>
struct Tile {
  static constexpr int WM = S::WM, WN = S::WN, MB = S::MB, NB = S::NB;
  static constexpr bool I8 = I8_, AT = AT_, BT = BT_;
  static constexpr int NW = WM * WN, BM = WM * MB * 32, BN = WN * NB * 32;
  static constexpr int A_BYTES = BM * DEPTH, B_BYTES = BN * DEPTH, STAGE = A_BYTES + B_BYTES;
  static constexpr int AI = BM / 8 / NW, BI = BN / 8 / NW, INSTR = AI + BI;  // DMA instructions of a wave per stage
  static constexpr int THREADS = NW * 64;
  static constexpr int EPI = WM * 32 * BN * 4;  // bytes of one staged set of row blocks (fp32)
  static constexpr int LDS = 2 * STAGE > 2 * EPI ? 2 * STAGE : 2 * EPI;
  static_assert(AI * NW * 8 == BM && BI * NW * 8 == BN && NB % 2 == 0, "tile shape");
  static_assert(!I8 || (!AT && !BT), "int8 operands are k-contiguous");
  using Acc1 = std::conditional_t<I8, i32x16_t, f32x16_t>;
  typedef Acc1 Acc[MB][NB];
  using Frag = std::conditional_t<I8, i32x4_t, bf16x8_t>;

  // Byte offsets of a wave's DMA lanes from the operand's base; `last` the
  // valid depth rows of the stage (transposed operands; 64 except in the end)
  template <bool TR, int ROWS, int N>
  static __device__ __forceinline__ void offsets(uint32_t (&o)[N], const Operand& m, int wave, int lane, int last) {
    if constexpr (TR) {
      constexpr int PW = ROWS / 2, RPI = 512 / PW, IPP = 64 / RPI, GR = PW / 8;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j = wave * N + i, panel = j / IPP, k = (j % IPP) * RPI + lane / GR;
        const int c = (lane % GR) ^ swz<PW>(k);
        const int col = m.col + c * 8 + (m.p2 ? 0 : panel * PW);
        o[i] = (uint32_t)min(k, last - 1) * m.ld + (uint32_t)min(col, m.cols - 8) * 2u;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (wave * N + i) * 8 + (lane >> 3);
        const int rr = m.p2 && r >= ROWS / 2 ? r - ROWS / 2 : r;
        o[i] = (uint32_t)min(rr, m.valid - 1) * m.ld + (uint32_t)(granule<N>(i, wave, lane) * 16);
      }
    }
  }
  // the granule of its row that a lane's k-contiguous load i takes
  template <int N>
  static __device__ __forceinline__ int granule(int i, int wave, int lane) {
    return (lane & 7) ^ swz_row((wave * N + i) * 8 + (lane >> 3));
  }
  static __device__ __forceinline__ int swz_row(int r) { return (r >> 1) & 7; }
  template <int PW>
  static __device__ __forceinline__ int swz(int k) {
    return PW == 128 ? 4 * (k & 3) : 4 * ((k >> 1) & 1);
  }
  // the base a wave's DMA reads from (its instructions are all of one panel)
  template <int ROWS, int N>
  static __device__ __forceinline__ const char* base_of(const Operand& m, int wave) {
    static_assert((ROWS / 16) % N == 0, "a wave's DMA stays in one half");
    return uniform_ptr(m.p2 && wave * N * 8 >= ROWS / 2 ? m.p2 : m.p);
  }

  struct FragOffs {
    uint32_t a[AT ? MB : 4], b[BT ? NB : 4];
  };
  static __device__ __forceinline__ FragOffs frag_offsets(int wm, int wn, int lane) {
    FragOffs f;
    if constexpr (AT) {
      constexpr int PW = BM / 2;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const int row = (mb * WM + wm) * 32;
        f.a[mb] = tr_offset<PW>(row / PW, row % PW, lane);
      }
    } else {
      const int r = wm * 32 + (lane & 31);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) f.a[kk] = (uint32_t)(r * DEPTH + ((kk * 2 + (lane >> 5)) ^ swz_row(r)) * 16);
    }
    if constexpr (BT) {
      constexpr int PW = BN / 2;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        f.b[nb] = A_BYTES + tr_offset<PW>(nb / (NB / 2), (wn * (NB / 2) + nb % (NB / 2)) * 32, lane);
    } else {
      const int r = wn * (NB / 2) * 32 + (lane & 31);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        f.b[kk] = (uint32_t)(A_BYTES + r * DEPTH + ((kk * 2 + (lane >> 5)) ^ swz_row(r)) * 16);
    }
    return f;
  }
  template <int PW>
  static __device__ __forceinline__ uint32_t tr_offset(int panel, int col, int lane) {
    const int k = (lane >> 5) * 8 + ((lane & 15) >> 2);
    const int c = (col >> 3) + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    return (uint32_t)(panel * 64 * PW * 2 + k * PW * 2 + (c ^ swz<PW>(k)) * 16 + (lane & 1) * 8);
  }
  template <int PW>
  static __device__ __forceinline__ Frag read_tr(const char* st, uint32_t off, int kk) {
    typedef __attribute__((address_space(3))) s16x4_t* P;
    const char* p = st + off + kk * 16 * PW * 2;
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * PW * 2));
    return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // byte distance of column block nb from a wave's first (k-contiguous B)
  static constexpr int nb_bytes(int nb) { return (nb / (NB / 2) * (BN / 2) + nb % (NB / 2) * 32) * DEPTH; }

  // fragment u of slice kk: B's blocks, then A's
  static constexpr int FRAGS = NB + MB;
  static __device__ __forceinline__ void load_frag(int u, const char* st, int kk, const FragOffs& f, Frag (&a)[MB], Frag (&b)[NB]) {
    if (u < NB) {
      if constexpr (BT) b[u] = read_tr<BN / 2>(st, f.b[u], kk);
      else b[u] = *reinterpret_cast<const Frag*>(st + f.b[kk] + nb_bytes(u));
    } else {
      const int mb = u - NB;
      if constexpr (AT) a[mb] = read_tr<BM / 2>(st, f.a[mb], kk);
      else a[mb] = *reinterpret_cast<const Frag*>(st + f.a[kk] + mb * WM * 32 * DEPTH);
    }
  }
  static __device__ __forceinline__ void load_frags(const char* st, int kk, const FragOffs& f, Frag (&a)[MB], Frag (&b)[NB]) {
#pragma unroll
    for (int u = 0; u < FRAGS; ++u) load_frag(u, st, kk, f, a, b);
  }
  // The products of one slice, with next(u) for u in [0, FRAGS), the loads of
  // the next slice's fragments, and dma(i) for i in [0, INSTR) between them,
  // in this order: left to itself the compiler loads each fragment right
  // before the product that takes it, and every product waits for LDS (4 to 9%
  // of the time of large products).
  template <typename Next, typename Dma>
  static __device__ __forceinline__ void multiply(Acc& acc, const Frag (&a)[MB], const Frag (&b)[NB], Next&& next, Dma&& dma) {
    constexpr int P = MB * NB;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int mb = i / NB, nb = i % NB;
      if constexpr (I8) acc[mb][nb] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[nb], a[mb], acc[mb][nb], 0, 0, 0);
      else acc[mb][nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[nb], a[mb], acc[mb][nb], 0, 0, 0);
#pragma unroll
      for (int u = i * FRAGS / P; u < (i + 1) * FRAGS / P; ++u) next(u);
#pragma unroll
      for (int j = i * INSTR / P; j < (i + 1) * INSTR / P; ++j) dma(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // acc += A B over the depth in [0, n1), and of a second pair of operands
  // (A2, B2: same shapes) over n2 more; depths in elements.  Depths are
  // multiples of 64 (int8: the second half of a last stage is not multiplied)
  // or, where both operands are transposed, any (the rows behind the end are
  // cleared in LDS, so that whatever lies there, NaN too, adds nothing).
  static __device__ __forceinline__ void run(Acc& acc, char* lds, const Operand& A, const Operand& B, int n1,
                                             const Operand& A2, const Operand& B2, int n2) {
    constexpr int KE = I8 ? 128 : 64;  // depth elements of a stage
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int half = (n1 + KE - 1) / KE, ns = half + (n2 + KE - 1) / KE;
    if (ns == 0) return;
    uint32_t oa[AI], ob[BI];
    offsets<AT, BM, AI>(oa, A, wave, lane, 64);
    offsets<BT, BN, BI>(ob, B, wave, lane, 64);
    const char *pa = base_of<BM, AI>(A, wave), *pb = base_of<BN, BI>(B, wave);
    const char *pa2 = n2 ? base_of<BM, AI>(A2, wave) : nullptr, *pb2 = n2 ? base_of<BN, BI>(B2, wave) : nullptr;
    const size_t sa = AT ? (size_t)A.ld * 64 : DEPTH, sb = BT ? (size_t)B.ld * 64 : DEPTH;
    const uint32_t la = lds_u32(lds) + wave * AI * 1024, lb = lds_u32(lds) + A_BYTES + wave * BI * 1024;
    const int rest = n1 % KE;  // depth of the last stage, 0: whole (only without a second pair)
    // instruction i of stage s (its operands' addresses at, its offsets and LDS)
    auto issue_one = [&](int i, const char* a, const char* b, uint32_t so, uint32_t back) {
      if (i < AI) {
        const uint32_t o = oa[i < AI ? i : 0];
        dma16(a, I8 && (granule<AI>(i, wave, lane) & 4) ? o - back : o, la + so + i * 1024);
      } else {
        const uint32_t o = ob[i < AI ? 0 : i - AI];
        dma16(b, I8 && (granule<BI>(i - AI, wave, lane) & 4) ? o - back : o, lb + so + (i - AI) * 1024);
      }
    };
    const auto base_a = [&](int s) { return s < half ? pa + s * sa : pa2 + (s - half) * sa; };
    const auto base_b = [&](int s) { return s < half ? pb + s * sb : pb2 + (s - half) * sb; };
    // (int8: a last stage of 64 has no granules 4..7; they are read as 0..3)
    const auto back_of = [&](int s) -> uint32_t {
      return I8 && rest && s == ns - 1 ? 64 : 0;
    };
    auto issue = [&](int s) {
      const uint32_t so = (s & 1) * STAGE, back = back_of(s);
      const char *a = base_a(s), *b = base_b(s);
      if ((AT && BT) && rest && s == ns - 1) {
        uint32_t ta[AI], tb[BI];
        offsets<AT, BM, AI>(ta, A, wave, lane, rest);
        offsets<BT, BN, BI>(tb, B, wave, lane, rest);
#pragma unroll
        for (int i = 0; i < AI; ++i) dma16(a, ta[i], la + so + i * 1024);
#pragma unroll
        for (int i = 0; i < BI; ++i) dma16(b, tb[i], lb + so + i * 1024);
        return;
      }
#pragma unroll
      for (int i = 0; i < INSTR; ++i) issue_one(i, a, b, so, back);
    };
    // clears the depth rows from `rest` on of a stage of transposed operands
    auto clear = [&](char* st) {
      if constexpr (AT && BT) {
        for (int i = threadIdx.x; i < STAGE / 16; i += THREADS) {
          constexpr int RA = BM / 2 * 2 / 16, RB = BN / 2 * 2 / 16;  // granules per depth row of a panel
          const int k = i < A_BYTES / 16 ? i / RA % 64 : (i - A_BYTES / 16) / RB % 64;
          if (k >= rest) *reinterpret_cast<u32x4_t*>(st + i * 16) = u32x4_t{0, 0, 0, 0};
        }
        lds_barrier();
      }
    };
    const FragOffs f = frag_offsets(wm, wn, lane);
    Frag a0[MB], b0[NB], a1[MB], b1[NB];
    issue(0);
    if (ns > 1) {
      issue(1);
      wait_vm<INSTR>();
    } else {
      wait_vm<0>();
    }
    __builtin_amdgcn_s_barrier();
    compiler_fence();
    if ((AT && BT) && rest && ns == 1) clear(lds);
    load_frags(lds, 0, f, a0, b0);
    const auto none = [](int) {};
    const auto from = [&](const char* st, int kk, Frag (&a)[MB], Frag (&b)[NB]) {
      return [&, st, kk](int u) { load_frag(u, st, kk, f, a, b); };
    };
    // this wave's reads of a stage have arrived and so has its part of the
    // next one: after the barrier everyone's have, and the stage is free
    const auto meet = [] {
      compiler_fence();
      __builtin_amdgcn_s_waitcnt(7 << 4);  // vmcnt(0) lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      compiler_fence();
    };
    // steady state: the stage after the next one is whole and loaded
    const int steady = rest ? ns - 3 : ns - 2;
    int s = 0;
    for (; s < steady; ++s) {
      const char* st = lds + (s & 1) * STAGE;
      const char* nx = lds + (~s & 1) * STAGE;
      multiply(acc, a0, b0, from(st, 1, a1, b1), none);
      multiply(acc, a1, b1, from(st, 2, a0, b0), none);
      multiply(acc, a0, b0, from(st, 3, a1, b1), none);
      meet();
      const char *pan = base_a(s + 2), *pbn = base_b(s + 2);
      const uint32_t so = (s & 1) * STAGE;
      multiply(acc, a1, b1, from(nx, 0, a0, b0), [&](int i) { issue_one(i, pan, pbn, so, 0); });
    }
    const int whole = I8 && rest ? ns - 1 : ns;
    for (; s < whole; ++s) {
      const char* st = lds + (s & 1) * STAGE;
      char* nx = lds + (~s & 1) * STAGE;
      multiply(acc, a0, b0, from(st, 1, a1, b1), none);
      multiply(acc, a1, b1, from(st, 2, a0, b0), none);
      multiply(acc, a0, b0, from(st, 3, a1, b1), none);
      meet();
      if (s + 2 < ns) issue(s + 2);
      if (s + 1 < ns) {
        if ((AT && BT) && rest && s + 2 == ns) clear(nx);
        load_frags(nx, 0, f, a0, b0);
      }
      multiply(acc, a1, b1, none, none);
    }
    if (I8 && whole < ns) {  // half a stage
      multiply(acc, a0, b0, from(lds + (whole & 1) * STAGE, 1, a1, b1), none);
      multiply(acc, a1, b1, none, none);
    }
    lds_barrier();
  }

  // run() of one pair of operands over a ring of NS stages, NS - 1 of them in
  // flight: for operands that come from memory once and are multiplied by little,
  // where two stages (a stage's latency each) leave the memory idle.  Stages lie
  // `apart` times their length apart and are taken from `turn` on, around, so that
  // workgroups that start together need not read from the same memory channels all
  // along.
  template <int NS>
  static constexpr int RING_LDS = NS * STAGE > 2 * EPI ? NS * STAGE : 2 * EPI;
  template <int NS>
  static __device__ __forceinline__ void ring(Acc& acc, char* lds, const Operand& A, const Operand& B, int n, int apart, int turn) {
    static_assert(!I8 && NS >= 3 && NS <= 5, "ring");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM, ns = (n + 63) / 64, rest = AT && BT ? n % 64 : 0;
    if (ns == 0) return;
    uint32_t oa[AI], ob[BI];
    offsets<AT, BM, AI>(oa, A, wave, lane, 64);
    offsets<BT, BN, BI>(ob, B, wave, lane, 64);
    const char *pa = base_of<BM, AI>(A, wave), *pb = base_of<BN, BI>(B, wave);
    const size_t sa = (AT ? (size_t)A.ld * 64 : DEPTH) * apart, sb = (BT ? (size_t)B.ld * 64 : DEPTH) * apart;
    const uint32_t la = lds_u32(lds) + wave * AI * 1024, lb = lds_u32(lds) + A_BYTES + wave * BI * 1024;
    int slot_in = 0;  // where the next stage goes
    auto issue = [&](int s) {
      const uint32_t so = slot_in * STAGE;
      slot_in = slot_in + 1 == NS ? 0 : slot_in + 1;
      const int st = s + turn < ns ? s + turn : s + turn - ns;
      const char *a = pa + st * sa, *b = pb + st * sb;
      if ((AT && BT) && rest && st == ns - 1) {
        uint32_t ta[AI], tb[BI];
        offsets<AT, BM, AI>(ta, A, wave, lane, rest);
        offsets<BT, BN, BI>(tb, B, wave, lane, rest);
#pragma unroll
        for (int i = 0; i < AI; ++i) dma16(a, ta[i], la + so + i * 1024);
#pragma unroll
        for (int i = 0; i < BI; ++i) dma16(b, tb[i], lb + so + i * 1024);
        return;
      }
#pragma unroll
      for (int i = 0; i < AI; ++i) dma16(a, oa[i], la + so + i * 1024);
#pragma unroll
      for (int i = 0; i < BI; ++i) dma16(b, ob[i], lb + so + i * 1024);
    };
    const FragOffs f = frag_offsets(wm, wn, lane);
    Frag a0[MB], b0[NB], a1[MB], b1[NB];
    const auto none = [](int) {};
    const int ahead = ns < NS - 1 ? ns : NS - 1;
    for (int s = 0; s < ahead; ++s) issue(s);
    int slot = 0;
    for (int s = 0; s < ns; ++s, slot = slot + 1 == NS ? 0 : slot + 1) {
      // this wave's part of the stage has arrived, and its reads of the one before
      // are done; after the barrier so are everyone's
      compiler_fence();
      const int young = ns - 1 - s;  // stages behind this one, of which NS - 2 are in flight
      if (young >= NS - 2) wait_vm<(NS - 2) * INSTR>();
      else if (NS > 4 && young == 2) wait_vm<2 * INSTR>();
      else if (NS > 3 && young == 1) wait_vm<INSTR>();
      else wait_vm<0>();
      __builtin_amdgcn_s_waitcnt((3 << 14) | (7 << 4) | 15);  // lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      compiler_fence();
      char* st = lds + slot * STAGE;
      if constexpr (AT && BT) {
        if (rest && (s + turn < ns ? s + turn : s + turn - ns) == ns - 1) {  // the rows behind the end are cleared
          for (int i = threadIdx.x; i < STAGE / 16; i += THREADS) {
            constexpr int RA = BM / 2 * 2 / 16, RB = BN / 2 * 2 / 16;
            const int k = i < A_BYTES / 16 ? i / RA % 64 : (i - A_BYTES / 16) / RB % 64;
            if (k >= rest) *reinterpret_cast<u32x4_t*>(st + i * 16) = u32x4_t{0, 0, 0, 0};
          }
          lds_barrier();
        }
      }
      if (s + NS - 1 < ns) issue(s + NS - 1);
      const auto from = [&](int kk, Frag (&a)[MB], Frag (&b)[NB]) {
        return [&, kk](int u) { load_frag(u, st, kk, f, a, b); };
      };
      load_frags(st, 0, f, a0, b0);
      multiply(acc, a0, b0, from(1, a1, b1), none);
      multiply(acc, a1, b1, from(2, a0, b0), none);
      multiply(acc, a0, b0, from(3, a1, b1), none);
      multiply(acc, a1, b1, none, none);
    }
    lds_barrier();
  }

  static __device__ __forceinline__ void zero(Acc& acc) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mb][nb][r] = 0;
  }

  // Hands out the tile by rows: fn(row, col, v) for every 8 consecutive
  // columns of a row, row < rows.  col counts the tile's columns; GATED: the
  // columns of panel 0, v[0..7] theirs and v[8..15] panel 1's.  Accumulators
  // pass through LDS one set of WM row blocks at a time (two buffers, one
  // barrier each), 16-byte granules at position c ^ (row & 15).
  template <bool GATED, typename Fn>
  static __device__ __forceinline__ void epilogue(const Acc& acc, char* lds, int rows, Fn&& fn) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    constexpr int SET = WM * 32, PPR = (GATED ? BN / 2 : BN) / 8;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      if (mb * SET >= rows) break;
      char* buf = lds + (mb & 1) * EPI;
      const int sr = wm * 32 + (lane & 31);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = nb / (NB / 2) * (BN / 2) + (wn * (NB / 2) + nb % (NB / 2)) * 32 + q * 8 + (lane >> 5) * 4;
          u32x4_t v;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if constexpr (I8) v[r] = (uint32_t)acc[mb][nb][q * 4 + r];
            else v[r] = __float_as_uint(acc[mb][nb][q * 4 + r]);
          }
          *reinterpret_cast<u32x4_t*>(buf + sr * BN * 4 + ((col / 4) ^ (sr & 15)) * 16) = v;
        }
      lds_barrier();
#pragma unroll
      for (int i = 0; i < SET * PPR / THREADS; ++i) {
        const int piece = (int)threadIdx.x + i * THREADS, r = piece / PPR, c = piece % PPR * 8;
        if (mb * SET + r < rows) {
          uint32_t v[GATED ? 16 : 8];
#pragma unroll
          for (int p = 0; p < (GATED ? 4 : 2); ++p) {
            const int g = (c + p / 2 * (BN / 2)) / 4 + p % 2;
            *reinterpret_cast<u32x4_t*>(v + p * 4) =
                *reinterpret_cast<const u32x4_t*>(buf + r * BN * 4 + (g ^ (r & 15)) * 16);
          }
          fn(mb * SET + r, c, v);
        }
      }
    }
  }
};

// dma16 for lines that are read once: they do not displace what the L2 holds
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_once(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// ---------------------------------------------------------------------------
// Few rows: up to 32 rows x 64 columns (gated: 64 of each matrix), whose time
// is that of streaming the weights.  The four or eight waves share the columns
// and take the steps of the depth (64 bytes: 32 bf16 or 64 int8 values) in turn,
// each with slots of LDS of its own, so the loop has no barrier: a wave waits
// for its oldest slot, multiplies it and loads a later step into it.  The
// waves' sums are added in a fixed order at the end.
// LDS images of a slot: weights, k-contiguous as rows of 64 bytes, granule c
// at c ^ (r / 4) % 4, or transposed as 32 depth rows of 64 columns per matrix
// (a panel of PW = 64, as above); then the 32 rows of A, k-contiguous.
// ---------------------------------------------------------------------------
template <int NW_, bool I8_, bool BT_, bool GATED_>
struct Few {
  static constexpr bool I8 = I8_, BT = BT_, GATED = GATED_;
  static constexpr int NW = NW_, THREADS = NW * 64, BM = 32, COLS = 64, STEP = 64, KE = I8 ? 64 : 32;
  static constexpr int NB = GATED ? 4 : 2, W_BYTES = NB * 2048, SLOT = W_BYTES + 2048, SLOTS = GATED ? 2 : 3;
  static constexpr int WI = W_BYTES / 1024, INSTR = SLOT / 1024, SUMS = 32 * NB * 32 * 4;  // bytes of a wave's sums
  static constexpr int LDS = NW * SLOTS * SLOT;
  static_assert(NW * SUMS <= LDS, "the sums fit");
  static_assert(!I8 || !BT, "int8 operands are k-contiguous");
  using Acc1 = std::conditional_t<I8, i32x16_t, f32x16_t>;
  using Frag = std::conditional_t<I8, i32x4_t, bf16x8_t>;
  using Big = Tile<Small, I8, false, BT>;  // the transposed reads, which are the same

  // fn(row, col, v) for every 8 consecutive columns of each row, v[8..15] the
  // second matrix's where gated: the sums over steps [s0, s1) of the depth.
  // Rows of A past A.valid are read as the last and not handed out.  once: no
  // other row tile reads these weights.
  template <typename Fn>
  static __device__ __forceinline__ void run(char* lds, const Operand& A, const Operand& B, int s0, int s1, bool once,
                                             Fn&& fn) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t ow[WI], ox[2];
#pragma unroll
    for (int i = 0; i < WI; ++i) {
      if constexpr (BT) {
        const int k = i % 4 * 8 + (lane >> 3), c = (lane & 7) ^ Big::template swz<64>(k);
        ow[i] = (uint32_t)k * B.ld + (uint32_t)min(B.col + c * 8, B.cols - 8) * 2u;
      } else {
        const int r = i % 4 * 16 + (lane >> 2);
        ow[i] = (uint32_t)min(r, B.valid - 1) * B.ld + (uint32_t)(((lane & 3) ^ ((r >> 2) & 3)) * 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = i * 16 + (lane >> 2);
      ox[i] = (uint32_t)min(r, A.valid - 1) * A.ld + (uint32_t)(((lane & 3) ^ ((r >> 2) & 3)) * 16);
    }
    const char *pa = uniform_ptr(A.p), *pb = uniform_ptr(B.p), *pb2 = GATED ? uniform_ptr(B.p2) : nullptr;
    const size_t sb = BT ? (size_t)B.ld * 32 : STEP;
    char* mine = lds + wave * SLOTS * SLOT;
    const uint32_t l0 = lds_u32(mine);
    const int n = (s1 - s0 - wave + NW - 1) / NW;  // this wave's steps
    auto issue = [&](int j) {
      const size_t s = s0 + wave + j * NW;
      const uint32_t l = l0 + j % SLOTS * SLOT;
#pragma unroll
      for (int i = 0; i < WI; ++i) {
        const char* w = (GATED && i >= 4 ? pb2 : pb) + s * sb;
        // transposed weights come in whole lines: past the L2 where no other
        // tile reads them (8 to 10% of the time; 50% more where two do).  A step
        // of k-contiguous ones is half of each line, which the next one reads
        if (BT && once) dma16_once(w, ow[i], l + i * 1024);
        else dma16(w, ow[i], l + i * 1024);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) dma16(pa + s * STEP, ox[i], l + W_BYTES + i * 1024);
    };
    uint32_t fw[2], fx[2];  // fragment offsets (k-contiguous: of slice 0 and 1; transposed: of column block 0 and 1)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = lane & 31;
      fx[i] = (uint32_t)(r * STEP + ((i * 2 + (lane >> 5)) ^ ((r >> 2) & 3)) * 16);
      fw[i] = BT ? Big::template tr_offset<64>(0, i * 32, lane) : fx[i];
    }
    Acc1 acc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[nb][r] = 0;
#pragma unroll
    for (int j = 0; j < SLOTS; ++j)
      if (j < n) issue(j);
    for (int j = 0; j < n; ++j) {
      if (j + SLOTS <= n) wait_vm<(SLOTS - 1) * INSTR>();
      else if (SLOTS > 2 && j + 2 == n) wait_vm<INSTR>();
      else wait_vm<0>();
      compiler_fence();
      const char* st = mine + j % SLOTS * SLOT;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const Frag x = *reinterpret_cast<const Frag*>(st + W_BYTES + fx[kk]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          Frag w;
          if constexpr (BT) w = Big::template read_tr<64>(st + nb / 2 * 4096, fw[nb % 2], kk);
          else w = *reinterpret_cast<const Frag*>(st + nb * 2048 + fw[kk]);
          if constexpr (I8) acc[nb] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, acc[nb], 0, 0, 0);
          else acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x, acc[nb], 0, 0, 0);
        }
      }
      // the slot's reads are done before it is loaded again
      compiler_fence();
      __builtin_amdgcn_s_waitcnt((3 << 14) | (7 << 4) | 15);  // lgkmcnt(0)
      if (j + SLOTS < n) issue(j + SLOTS);
    }
    lds_barrier();
    // [wave][row][column], granules of 4 columns at position c ^ (row & 15)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = lane & 31, g = nb * 8 + q * 2 + (lane >> 5);
        u32x4_t v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (I8) v[r] = (uint32_t)acc[nb][q * 4 + r];
          else v[r] = __float_as_uint(acc[nb][q * 4 + r]);
        }
        *reinterpret_cast<u32x4_t*>(lds + wave * SUMS + row * (NB * 128) + (g ^ (row & 15)) * 16) = v;
      }
    lds_barrier();
    if (threadIdx.x >= 256) return;
    const int row = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
    if (row >= A.valid) return;
    uint32_t v[NB * 4];
#pragma unroll
    for (int p = 0; p < NB; ++p) {
      const int g = (c + p / 2 * 64) / 4 + p % 2;
      const char* at = lds + row * (NB * 128) + (g ^ (row & 15)) * 16;
      u32x4_t t = *reinterpret_cast<const u32x4_t*>(at);
#pragma unroll
      for (int w = 1; w < NW; ++w) {
        const u32x4_t o = *reinterpret_cast<const u32x4_t*>(at + w * SUMS);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (I8) t[r] += o[r];
          else t[r] = __float_as_uint(__uint_as_float(t[r]) + __uint_as_float(o[r]));
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) v[p * 4 + r] = t[r];
    }
    fn(row, c, v);
  }
};

// ---------------------------------------------------------------------------
// Which tiles a product is computed by, and in how many parts its depth is
// split (a kernel behind it adds the parts' sums, in order).
// ---------------------------------------------------------------------------
struct Plan {
  enum Kind { FEW4 = MOE_TILES_FEW4, FEW8 = MOE_TILES_FEW8, SMALL = MOE_TILES_SMALL, WIDE = MOE_TILES_WIDE } kind;
  int split;
};
constexpr int MAX_SPLIT = 16;

// Small or Wide tiles, from how many there are of each: rounds of workgroups
// (one Wide or two Small per CU) times the time of one.  Measured, us per
// stage: Wide 1.85 to 2.2; Small 0.85 to 1.1 (and 8 at the ends) with one
// workgroup per CU and 1.2 to 1.4 with two.  So Wide tiles take 1.3 times less
// where they fill the chip, and Small ones win where Wide ones leave CUs idle:
// dh of 2000 rows, H = F = 4096, 128 Wide tiles 123, 512 Small 89; of 4000 rows
// 147 : 179; int8, 6007 rows in 16 groups, 2048 x 2816, 352 Wide tiles 71, 1210 Small 60.  A split costs a
// launch (6 with its gap) and the sums' way out and back, `sum_bytes` per part
// (6 TB/s): dx of 333 rows in 4 groups, H = 1024, F = 2816 (40 Small tiles, 88
// stages), 80 : 52 : 33 : 25 in 1, 2, 4 and 8 parts; dh of the same rows (88
// tiles, 16 stages) 27 : 21; dh of 2000 rows above, 89 against 83 + 27 in two.
struct Timed {
  Plan plan;
  double us;
};
inline Timed tile_plan(double wide, double small, int stages, double sum_bytes, double weight_bytes) {
  // the weights once (1 row, the down projection of F = 14336 in 16 parts: 10 us
  // longer than tiles of few rows where nothing is left in the caches)
  const double stream = weight_bytes / 3.8e6;
  Timed best{{Plan::WIDE, 1}, std::max(std::ceil(wide / 256) * (stages * 2.0 + 4), stream)};
  for (int s = 1; s <= MAX_SPLIT && s <= std::max(stages, 1); s *= 2) {
    const double w = small * s, rounds = w <= 512 ? 1 : w / 512 + 0.35;
    const double t = std::max(rounds * (w <= 256 ? ceil_div(stages, s) * 1.0 + 8 : ceil_div(stages, s) * 1.25 + 3), stream) +
                     (s > 1 ? 6 + 2 * s * sum_bytes / 6e6 : 0);
    if (t < best.us) best = {{Plan::SMALL, s}, t};
  }
  return best;
}

// Tiles of few rows: a wave's steps (0.7 to 1.2 us: a load's latency over the
// slots) behind 5 of ends, or the weights' stream where that is longer, once
// from memory (5 TB/s) and for further row tiles mostly out of the caches (9).
// Few rows against Small, us: H = 4096, F = 14336, up and down projection, 32
// rows 49 + 33 : 57 + 56, 64 rows 77 + 46 : 60 + 57; H = 2048, F = 1408, 256 rows
// 14 + 8 : 17 + 17; 16 groups of 32 rows on average 43 + 27 : 46 + 27, of 64 rows
// 60 + 37 : 49 + 34.
// Eight waves share the depth where one workgroup per CU holds all tiles (the
// most there can be: 264 of 8 waves take two rounds), else four.  Parts cost 6
// (a launch with its gap) and their sums' way out and back, `sum_bytes` each: 1
// row, H = 4096, down projection of F = 14336 (64 tiles, 448 steps) 60, 39 in two
// parts, 31 in four; 2 rows, H = 3008, F = 192 (3 gated tiles, 94 steps) 20, 13 in
// four.
inline Timed few_plan(long long most, double tiles, int steps, double sum_bytes, double weight_bytes,
                      double streamed_bytes) {
  Timed best{{Plan::FEW4, 1}, 1e30};
  for (int s = 1; s <= MAX_SPLIT && (s == 1 || (most * s <= 512 && s * 4 <= steps)); s *= 2) {
    const int waves = most * s <= 256 ? 8 : 4;
    const double rounds = std::ceil(tiles * s / (waves == 8 ? 256 : 512));
    const double stream = weight_bytes / 5e6 + std::max(0.0, streamed_bytes - weight_bytes) / 9e6;
    const double t = 5 + std::max(rounds * ceil_div(steps, s * waves), stream) +
                     (s > 1 ? 6 + 2 * s * sum_bytes / 5e6 : 0);
    if (t < best.us) best = {{waves == 8 ? Plan::FEW8 : Plan::FEW4, s}, t};
  }
  return best;
}

// Row tiles of T rows in G groups to expect: the last of a group is half full,
// and every group that has rows has one (T rows leave exp(-T / G) of them empty).
inline double row_tiles(int T, int G, int bm) {
  if (G == 1) return ceil_div(T, bm);
  return std::min((double)T, std::max((double)T / bm + 0.5 * G, G * (1 - std::exp(-(double)T / G))));
}

// The plan of a product of T rows in G groups: `cols` columns of the output
// from `per` (2 where gated) columns of weights each, a depth of `stages`.
inline Plan plan_of(int T, int G, int cols, int per, int stages, bool can_be_few) {
  const double column = (double)DEPTH * stages * per, groups = G == 1 ? 1 : G * (1 - std::exp(-(double)T / G));
  const double weights = groups * cols * column, sums = 4.0 * T * cols * per;
  const Timed t = tile_plan(row_tiles(T, G, Wide::BM) * ceil_div(cols * per, Wide::BN),
                            row_tiles(T, G, Small::BM) * ceil_div(cols * per, Small::BN), stages, sums, weights);
  if (!can_be_few) return t.plan;
  const int nt = ceil_div(cols, 64);
  const double few = row_tiles(T, G, 32);
  const Timed f = few_plan((long long)max_row_tiles(T, G, 32) * nt, few * nt, stages * 2, sums, weights,
                           few * cols * column);
  return f.us <= t.us ? f.plan : t.plan;
}

__device__ __forceinline__ u32x4_t pack8(const float (&v)[8]) {
  return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void unpack8(u32x4_t w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}

// The tile of workgroup `block` among mt row tiles x nt column tiles: workgroup i
// runs on XCD i % 8, and each XCD takes a run of consecutive tiles, ordered so
// that 8 row tiles share each column tile's operand while it is in the XCD's
// L2.  False: no tile (the grid is sized for the most row tiles there can be).
constexpr int NEAR = 8;
__device__ __forceinline__ bool pick(int block, int mt, int nt, int* m, int* n) {
  const int total = mt * nt, chunk = ceil_div(total, NXCD), t = block % NXCD * chunk + block / NXCD;
  if (block / NXCD >= chunk || t >= total) return false;
  const int band = t / (NEAR * nt), first = band * NEAR, wide = min(NEAR, mt - first), in = t - band * NEAR * nt;
  *m = first + in % wide;
  *n = in / wide;
  return true;
}
inline int grid_of(long long mt, int nt) { return (int)((mt * nt + NXCD - 1) / NXCD * NXCD); }

}  // namespace tile
}  // namespace moe
