// Tile products of the block operators on the gfx950 matrix cores (bf16, fp32 and
// 8-bit integers), fed by direct HBM -> LDS loads.
//
// A workgroup of WGM x WGN waves owns a BM x BN tile of C[m][n] = sum_k a(m, k)
// b(n, k); a wave owns (BM / WGM) x (BN / WGN) of it in 16 x 16 MFMA tiles
// (v_mfma_f32_16x16x32_bf16, v_mfma_i32_16x16x64_i8: both take 16 bytes per lane
// and operand; fp32: the 16 bytes are the operands of four v_mfma_f32_16x16x4_f32,
// which between them take 16 of k in an order of their own, the same for both
// operands).  k advances by a step of 128 bytes of k per row (64 bf16, 32 fp32, 128
// 8-bit values) through a ring of ST LDS stages; 16 bytes per lane go straight
// from global memory into LDS (no registers).
//
// Each operand lies in memory in one of two ways:
//   k along the rows ("KC": weights [out, in], activations [rows, in]).  A stage
//     holds 128 bytes of every tile row; the 16-byte piece c of row r sits in
//     slot c ^ ((r >> 1) & 7), so the 16 rows of a fragment spread over all LDS
//     banks.
//   k across the rows ("KR": the operands of the gradients, contracted over
//     tokens or over output features).  A stage holds 64 (fp32: 32) rows of the tile's
//     columns.  A lane reads the same N neighbouring columns of its 8 (4) rows k and
//     joins the halves of bf16 dwords by v_perm, which gives it 8 k of N columns,
//     the operands of N MFMAs: fragment j of such a group has columns j, N + j,
//     2 N + j ...  For N = 2 (4-byte reads) the 64-byte piece p of row k sits in
//     piece p ^ f, f = (k >> 3) & 3, so that the four rows of a read lie in different
//     banks.  (ds_read_b64_tr_b16 would turn the block by itself, but the compiler
//     lets such a read wait for every load into LDS that is on its way.)
//
// Loop over the steps (a step is two half-steps of one MFMA depth): the MFMAs of
// half-step h run while the fragments of h + 1 are read -- the a fragments into
// the other register set, each b fragment in place once its column is done --
// and the workgroup meets once per step, after the first of half-step 1's columns,
// when every fragment of the stage is in registers; then the stage is refilled
// and the next stage's fragments are read under the remaining columns.  (Meeting
// before the first column or halfway, and raising the waves' priority around the
// MFMAs, measured within 2 % of it.)
//
// Measured, operands of 4096 x 10240 x 4096 and so much work that the clock falls
// to 1.7 GHz: both projections of the gated block 515 - 530 us (1.30 - 1.33 PFLOP/s,
// MFMA busy in 68 % of the cycles; a library product of 8192^3 reaches 1.37), dx 510 -
// 580 (1.18 - 1.35; the library with k across b's rows 1.21), dW 585 - 640 (1.07 -
// 1.18; k across both 1.08); 8 bits at 4096 x 4096 x 12288 168 - 179 us (2.3 - 2.45
// POP/s; 2.11); fp32 at 4096 x 9216 x 1152 608 us (143 TFLOP/s; 154).  At K = 1152 the
// first loads and the epilogue take a fifth to a half of a tile's time, see kTiles.
//
// fp32 operands whose rows do not lie in whole, aligned 16-byte pieces (U) are loaded
// by the same 16 bytes per lane from addresses that are multiples of 4, and 4 bytes
// per lane, four times the instructions, where a piece would reach past a row's end:
// KC in the last step, KR in a tile that is wider than the matrix.
//
// Few tiles of a long contraction leave most CUs idle and each busy one waiting for its
// own loads: there KG groups of waves share a tile, each with a slice of the steps and
// a ring of its own, and the groups' sums are added through LDS in a fixed order.
//
// Sizes: tile rows behind the operand's last are read as that row (KC), columns as
// its last ones (KR): what comes of them is not stored.  k behind the end is read as
// zeros (KC: by an offset behind the resource, KR: by the resource's bound) and
// adds nothing.
#pragma once

#include <type_traits>

#include "block_ops.h"

namespace t2i {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// s_waitcnt with only vmcnt constrained (low bits [3:0], high bits [15:14])
template <int N>
__device__ __forceinline__ void tile_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
// at most `younger` load rounds of B instructions outstanding
template <int B>
__device__ __forceinline__ void tile_wait(int younger) {
  switch (younger) {
    case 0: tile_vmcnt<0>(); break;
    case 1: tile_vmcnt<(B < 64 ? B : 0)>(); break;
    case 2: tile_vmcnt<(2 * B < 64 ? 2 * B : 0)>(); break;
    default: tile_vmcnt<(3 * B < 64 ? 3 * B : 0)>(); break;
  }
}
// this wave's LDS accesses done, then the barrier; outstanding loads go on
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("s_barrier" ::: "memory");
}

// BYTES per lane from global memory into LDS at the wave-uniform address lds
template <int BYTES>
__device__ __forceinline__ void tile_load(__amdgpu_buffer_rsrc_t r, char* lds, uint32_t voff, int soff) {
  auto* d = (__attribute__((address_space(3))) void*)lds;
  if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, d, 16, voff, soff, 0, 0);
  else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, d, 4, voff, soff, 0, 0);
}

// consecutive workgroups of one XCD (they are dealt out in turn over 8) get
// consecutive tiles
__device__ __forceinline__ int tile_of_block(int b, int nb) {
  const int q = nb >> 3, r = nb & 7, x = b & 7, j = b >> 3;
  return (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + j;
}

// One operand of a product.  `p` (and `p2`) in bytes.
struct TileOperand {
  const char* p;
  const char* p2;    // second matrix (two: see TileProduct), else unused
  uint32_t ld;       // bytes from row to row
  int rows;          // KC: rows of the matrix; KR: rows of the contraction
  int cols;          // KR: columns that may be read (whole pieces of a load)
};

struct TileShape {
  int tiles_m, tiles_n, group_m;
  int steps;         // k steps in all
  int kbytes;        // KC: bytes of a row that hold k
  int half;          // steps in the first matrix of a two-matrix contraction
  int first;         // the first step (a KC operand's resource starts there, too)
};

// The tile of a workgroup: tiles of one XCD are consecutive and walk group_m row
// blocks down before moving one column block right, sharing both operands in its L2
__device__ __forceinline__ void tile_place(const TileShape& s, int block, int blocks, int& tm, int& tn) {
  const int tile = tile_of_block(block, blocks);
  const int per_group = s.group_m * s.tiles_n, grp = tile / per_group, first = grp * s.group_m;
  const int rows_in = min(s.tiles_m - first, s.group_m), in_grp = tile - grp * per_group;
  tm = first + in_grp % rows_in;
  tn = in_grp / rows_in;
}

constexpr uint32_t kTileOff = 0x80000000u;   // behind every resource: reads as zero

// KG groups of WGM x WGN waves share a tile, each with a slice of the contraction and
// a ring of its own
template <int BM_, int BN_, int WGM_, int WGN_, int ST_, int KG_ = 1>
struct TileDims {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, ST = ST_, KG = KG_;
  static constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  static constexpr int STAGE = (BM + BN) * 128, RING = ST * STAGE, THREADS = KG * NW * 64;
  static constexpr int LOADS = (BM + BN) / 8 / NW;   // load instructions per wave and step
  static_assert((BM + BN) / 8 % NW == 0 && BM / 8 % NW == 0, "whole load rounds per operand");
  static_assert(WM % 16 == 0 && WN % 16 == 0 && ST >= 2 && ST <= 5 && (ST - 1) * LOADS < 64, "tile shape");
};

enum TileElem { ELEM_BF16, ELEM_I8, ELEM_F32 };

// the row of operand a (a KC one) that a tile's row is: the next ones from the first
struct NextRows {
  __device__ __forceinline__ int operator()(int row, int rows, int first) const { return min(row, rows - 1 - first); }
};
// what a product's accumulators start from: zeros
struct FromZero {
  template <class A>
  __device__ __forceinline__ void operator()(A&) const {}
};

// E: element type.  AKR, BKR: operand layouts.  DUAL: b is two matrices side by side,
// p for the first half of the tile's columns and p2 for the second, so that a wave
// holds both of an output.  SEGS (BKR): the contraction runs over p's rows, then p2's.
// U: operand rows anywhere (fp32).
template <class D, TileElem E, bool AKR, bool BKR, bool DUAL, bool SEGS, bool U = false>
struct TileProduct {
  static_assert(!U || E == ELEM_F32, "rows off 16 bytes");
  static constexpr int LOADS = D::LOADS;
  static constexpr bool I8 = E == ELEM_I8;
  static constexpr int EB = E == ELEM_F32 ? 4 : I8 ? 1 : 2;   // bytes of an element
  static constexpr int KROWS = 128 / EB;                      // k of a step
  using Acc = typename std::conditional<I8, i32x4, f32x4>::type;
  static constexpr int BM = D::BM, BN = D::BN, TM = D::TM, TN = D::TN, ST = D::ST;

  // columns per group of a KR operand (see above): a's whole set, two of b's
  static constexpr int NA = AKR ? TM : 1, NB = BKR ? 2 : 1;
  static_assert(!AKR || TM == 2 || TM == 4 || (TM == 8 && EB == 2), "fragments per wave");
  static_assert(!BKR || TN % 2 == 0, "fragments per wave");

  // f of the rows k with (k >> 3) & 3 = g (see above; counted by SQ_LDS_BANK_CONFLICT:
  // none so, a half of the LDS cycles with the bits of g swapped for every N)
  template <int N>
  static __device__ __forceinline__ int kr_swap(int g) { return EB == 2 && N == 2 ? g : 0; }
  // the (row, column) of a KR tile of W columns that byte `at` of its stage holds
  template <int W, int N>
  static __device__ __forceinline__ void kr_source(int at, int& row, int& col) {
    constexpr int RB = W * EB, MASK = W >= 128 ? 3 : W / 32 - 1;
    row = at / RB;
    const int o = at % RB, f = kr_swap<N>((row >> 3) & 3) & MASK;
    col = ((o >> 6) ^ f) * (64 / EB) + (o & 63) / EB;
  }

  // tile row (column) that index x = 0 .. 15 of fragment i (j) of a wave stands for
  static __device__ __forceinline__ int row_of(int i, int x) { return i / NA * NA * 16 + x * NA + i % NA; }
  static __device__ __forceinline__ int col_of(int j, int x) { return j / NB * NB * 16 + x * NB + j % NB; }

  // the tile product: acc[i][j][r] belongs to the wave's row row_of(i, lane & 15)
  // and column col_of(j, 4 (lane >> 4) + r).  `from` may add to the accumulators before the
  // first step, while the ring's first loads are under way; `pick` says which rows of a the
  // tile's are, counted from m0.
  template <class F = FromZero, class R = NextRows>
  static __device__ __forceinline__ void run(char* smem, const TileOperand& a, const TileOperand& b, const TileShape& s,
                                             int m0, int n0, Acc (&acc)[TM][TN], const F& from = F(),
                                             const R& pick = R()) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane((tid >> 6) % D::NW);
    const int wm = wave / D::WGN, wn = wave % D::WGN, fr = lane & 15, g = lane >> 4;
    constexpr int LA = BM / 8 / D::NW;
    const int KT = s.steps;

    // ---- sources: this lane's offset of each load.  Load i takes KB block wave + i
    // waves of the stage, a's blocks first; byte `at` of that operand's stage.
    auto block_of = [&](int i) { return wave + (i < LA ? i : i - LA) * D::NW; };
    auto at_of = [&](int i) { return block_of(i) * 1024 + lane * 16; };
    // KC: row and byte of k (within the step) of a place in the stage
    auto kc_row = [](int at) { return at >> 7; };
    auto kc_byte = [](int at) { return ((((at >> 4) & 7) ^ ((at >> 8) & 7)) << 4) | (at & 15); };
    // offset of the `bytes` that belong at byte `at`
    auto source = [&](bool is_a, int at, int bytes) -> uint32_t {
      const TileOperand& o = is_a ? a : b;
      if (is_a ? AKR : BKR) {
        int row, col;
        if (is_a) kr_source<BM, NA>(at, row, col);
        else kr_source<BN, NB>(at, row, col);
        return (uint32_t)row * o.ld + EB * (uint32_t)min((is_a ? m0 : n0) + col, o.cols - bytes / EB);
      }
      // rows from the tile's first, not behind the last (DUAL: within the half)
      const int r0 = is_a ? m0 : n0, lr = kc_row(at);
      const int rr = !is_a && DUAL && lr >= BN / 2 ? lr - BN / 2 : lr;
      return (uint32_t)(is_a ? pick(rr, o.rows, r0) : min(rr, o.rows - 1 - r0)) * o.ld + kc_byte(at);
    };
    uint32_t src[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) src[i] = source(i < LA, at_of(i), 16);
    const bool ragged_k = !I8 && (s.first + s.steps) * 128 > s.kbytes;   // KC: places of the last step lie behind k
    // KC: rows at fixed offsets from the tile's first, k as the scalar offset.
    // KR: the step's first row as the base, the resource ends with its last row.
    auto kc_res = [](const char* p, size_t off) {
      return __builtin_amdgcn_make_buffer_rsrc((void*)(p + off), 0, 0x7fffffff, 0x00020000);
    };
    auto kr_res = [&](const TileOperand& o, int t, bool segs) {
      t += s.first;
      const bool second = segs && t >= s.half;
      const int row0 = (second ? t - s.half : t) * KROWS;
      // (a step may lie wholly behind the rows: nothing to read)
      const int left = min(o.rows - row0, KROWS);
      return __builtin_amdgcn_make_buffer_rsrc((void*)((second ? o.p2 : o.p) + (size_t)row0 * o.ld), 0,
                                               left > 0 ? (left - 1) * (int)o.ld + EB * o.cols : 0, 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t ra_kc = kc_res(a.p, AKR ? 0 : (size_t)m0 * a.ld + (size_t)s.first * 128);
    const __amdgpu_buffer_rsrc_t rb_kc = kc_res(b.p, BKR ? 0 : (size_t)n0 * b.ld + (size_t)s.first * 128);
    const __amdgpu_buffer_rsrc_t rb2_kc = kc_res(DUAL ? b.p2 : b.p, BKR ? 0 : (size_t)n0 * b.ld + (size_t)s.first * 128);
    auto res_a = [&](int t) { return AKR ? kr_res(a, t, false) : ra_kc; };
    auto res_b = [&](int t) { return BKR ? kr_res(b, t, SEGS) : rb_kc; };
    // U: whether a load of step t takes 4 bytes at a time (a KR operand a is the
    // gradients' workspace: whole pieces)
    auto fine = [&](bool is_a, int t) {
      if (is_a ? AKR : BKR) return !is_a && n0 + BN > b.cols;
      return ragged_k && t == KT - 1;
    };
    auto issue = [&](int i, int t, uint32_t slot, const __amdgpu_buffer_rsrc_t& ra,
                     const __amdgpu_buffer_rsrc_t& rb) {
      const bool is_a = i < LA;
      const int blk = block_of(i);
      char* const dst = smem + slot + (is_a ? 0 : BM * 128) + blk * 1024;
      const bool up = DUAL && !is_a && blk * 8 >= BN / 2;
      const __amdgpu_buffer_rsrc_t& r = is_a ? ra : up ? rb2_kc : rb;
      const bool kr = is_a ? AKR : BKR;
      const int soff = kr ? 0 : t * 128;
      auto behind = [&](int at) {   // KC: k behind the end
        return !kr && ragged_k && t == KT - 1 && (s.first + t) * 128 + kc_byte(at) >= s.kbytes;
      };
      if (U && fine(is_a, t)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int at = blk * 1024 + q * 256 + lane * 4;
          tile_load<4>(r, dst + q * 256, behind(at) ? kTileOff : source(is_a, at, 4), soff);
        }
      } else {
        tile_load<16>(r, dst, behind(at_of(i)) ? kTileOff : src[i], soff);
      }
    };

    // ---- fragments
    const uint32_t kc = fr * 128 + ((g ^ ((fr >> 1) & 7)) << 4);   // half-step 1: ^ 64
    auto read_kc = [&](bool is_a, uint32_t slot, int kk, int i) -> i32x4 {
      int row = is_a ? wm * D::WM + i * 16 : wn * D::WN + i * 16;
      if (!is_a && DUAL)
        row = i < TN / 2 ? wn * (D::WN / 2) + i * 16 : BN / 2 + wn * (D::WN / 2) + (i - TN / 2) * 16;
      return *(const i32x4*)(smem + slot + (is_a ? 0 : BM * 128) + row * 128 + (kc ^ (kk ? 64u : 0u)));
    };
    // N fragments of a KR tile of W columns from column c0 on, its rows from `base`
    auto read_kr = [&](auto n, auto w, uint32_t base, int kk, int c0, i32x4* f) {
      constexpr int N = decltype(n)::value, W = decltype(w)::value, MASK = W >= 128 ? 3 : W / 32 - 1;
      constexpr int LK = 16 / EB, DW = N * EB / 4;   // k of a lane, dwords of its read
      typedef int raw_t __attribute__((ext_vector_type(DW > 1 ? DW : 2)));
      const int o = (c0 + N * fr) * EB;
      const char* at = smem + base + (kk * (KROWS / 2) + g * LK) * W * EB +
                       (((o >> 6) ^ (kr_swap<N>(g) & MASK)) << 6) + (o & 63);
      int raw[LK][DW];
#pragma unroll
      for (int k = 0; k < LK; ++k) {
        if constexpr (DW == 1) {
          raw[k][0] = *(const int*)(at + k * W * EB);
        } else {
          const raw_t v = *(const raw_t*)(at + k * W * EB);
#pragma unroll
          for (int p = 0; p < DW; ++p) raw[k][p] = v[p];
        }
      }
      if constexpr (EB == 4) {
#pragma unroll
        for (int p = 0; p < N; ++p)
#pragma unroll
          for (int k = 0; k < 4; ++k) f[p][k] = raw[k][p];
      } else {
#pragma unroll
        for (int p = 0; p < DW; ++p)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            f[2 * p][d] = __builtin_amdgcn_perm(raw[2 * d + 1][p], raw[2 * d][p], 0x05040100);
            f[2 * p + 1][d] = __builtin_amdgcn_perm(raw[2 * d + 1][p], raw[2 * d][p], 0x07060302);
          }
      }
    };
    auto read_a = [&](uint32_t slot, int kk, i32x4 (&av)[TM]) {
      if constexpr (AKR) {
        read_kr(std::integral_constant<int, TM>(), std::integral_constant<int, BM>(), slot, kk, wm * D::WM, av);
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i) av[i] = read_kc(true, slot, kk, i);
      }
    };
    i32x4 a0[TM], a1[TM], bf[TN];
    // the b fragments that column j completes: j's own, or its pair's
    auto read_b = [&](uint32_t slot, int kk, int j) {
      if constexpr (BKR) {
        if (j % 2 == 1)
          read_kr(std::integral_constant<int, 2>(), std::integral_constant<int, BN>(), slot + BM * 128, kk,
                  wn * D::WN + (j - 1) * 16, bf + (j - 1));
      } else {
        bf[j] = read_kc(false, slot, kk, j);
      }
    };
    auto column = [&](int j, const i32x4 (&av)[TM]) {
      if constexpr (E == ELEM_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(bf[j][k]), __int_as_float(av[i][k]),
                                                             acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if constexpr (I8)
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[j], av[i], acc[i][j], 0, 0, 0);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, bf[j]),
                                                               __builtin_bit_cast(bf16x8, av[i]), acc[i][j], 0, 0, 0);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = Acc{0, 0, 0, 0};

    // ---- loop
    constexpr int S = TN / 3;                                   // columns before the barrier
    constexpr int LPC = (LOADS + TN - S - 1) / (TN - S);        // loads per column after it
#pragma unroll
    for (int t = 0; t < ST; ++t)
      if (t < KT) {
        const __amdgpu_buffer_rsrc_t ra = res_a(t), rb = res_b(t);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) issue(i, t, t * D::STAGE, ra, rb);
      }
    from(acc);
    tile_wait<LOADS>(min(ST, KT) - 1);
    tile_barrier();
    read_a(0, 0, a0);
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(0, 0, j);
    auto half0 = [&](uint32_t slot) {
      read_a(slot, 1, a1);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        column(j, a0);
        read_b(slot, 1, j);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < S; ++j) column(j, a1);
      __builtin_amdgcn_sched_barrier(0);
    };
    uint32_t slot = 0;
#pragma unroll 1
    for (int t = 0; t < KT - 1; ++t) {
      half0(slot);
      if constexpr (ST == 2) tile_vmcnt<0>();
      else tile_wait<LOADS>(min(ST - 2, KT - 2 - t));   // stage t + 1 landed
      tile_barrier();
      const uint32_t next = slot == (ST - 1) * D::STAGE ? 0 : slot + D::STAGE;
      const bool more = t + ST < KT;
      const __amdgpu_buffer_rsrc_t ra = res_a(more ? t + ST : 0), rb = res_b(more ? t + ST : 0);
      read_a(next, 0, a0);
#pragma unroll
      for (int j = 0; j < S; ++j) read_b(next, 0, j);
#pragma unroll
      for (int j = S; j < TN; ++j) {
        column(j, a1);
        read_b(next, 0, j);
        if (more) {
#pragma unroll
          for (int q = 0; q < LPC; ++q)
            if ((j - S) * LPC + q < LOADS) issue((j - S) * LPC + q, t + ST, slot, ra, rb);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      slot = next;
    }
    half0(slot);
#pragma unroll
    for (int j = S; j < TN; ++j) column(j, a1);
  }

  // the same by KG groups of waves; the sum, in ascending group order, is the first
  // group's, whose accumulators `from` adds to.  Returns whether this wave is of that group
  // (the others have no outputs).
  template <class F = FromZero, class R = NextRows>
  static __device__ __forceinline__ bool run_groups(char* smem, const TileOperand& a, const TileOperand& b, TileShape s,
                                                    int m0, int n0, Acc (&acc)[TM][TN], const F& from = F(),
                                                    const R& pick = R()) {
    if constexpr (D::KG == 1) {
      run(smem, a, b, s, m0, n0, acc, from, pick);
      return true;
    } else {
      const int kg = __builtin_amdgcn_readfirstlane((int)threadIdx.x / (D::NW * 64)), t = threadIdx.x % (D::NW * 64);
      const int total = s.steps, per = (total + D::KG - 1) / D::KG;
      s.first = kg * total / D::KG;
      s.steps = (kg + 1) * total / D::KG - s.first;
      run(smem + kg * D::RING, a, b, s, m0, n0, acc, [&](Acc (&c)[TM][TN]) {
        if (kg == 0) from(c);
      }, pick);
      // (every group meets as often: slices differ by a step)
      for (int x = s.steps; x < per; ++x) tile_barrier();
      tile_barrier();
      Acc* const part = (Acc*)smem + t;
      if (kg > 0) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) part[(((kg - 1) * TM + i) * TN + j) * D::NW * 64] = acc[i][j];
      }
      tile_barrier();
      if (kg == 0) {
#pragma unroll
        for (int x = 0; x < D::KG - 1; ++x)
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] += part[((x * TM + i) * TN + j) * D::NW * 64];
      }
      return kg == 0;
    }
  }
};

}  // namespace t2i
