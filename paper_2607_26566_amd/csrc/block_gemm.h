// What the block operators' products share beside the tiles of gemm_tile.h: tile shapes
// and their choice, epilogue parts, contractions in slices.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "gemm_tile.h"

namespace t2i {

// ---- tile shapes.  `per_cu` workgroups of a shape share a CU.  A launch of n
// tiles takes rounds of 256 per_cu; a round takes `full` us per k step and `end` us
// for its first loads and its epilogue, the last one `alone` per step if it has 256
// tiles or fewer, and in between what lies between.
struct TileChoice { int bm, bn, per_cu; float alone, full, end; };
struct TilePick { int shape; float us; };
inline TilePick choose_tile(const TileChoice* c, int shapes, long rows, long cols, int steps, float end_scale,
                            int slices = 1) {
  TilePick best{0, 0.f};
  for (int i = 0; i < shapes; ++i) {
    const long tiles = ((rows + c[i].bm - 1) / c[i].bm) * ((cols + c[i].bn - 1) / c[i].bn) * slices;
    const long slots = 256L * c[i].per_cu, rest = tiles % slots;
    const float end = c[i].end * end_scale, more = rest <= 256 ? 0.f : (float)(rest - 256) / (float)(slots - 256);
    const float us = (float)(tiles / slots) * (c[i].full * steps + end) +
                     (rest == 0 ? 0.f : (c[i].alone + (c[i].full - c[i].alone) * more) * steps + end);
    if (i == 0 || us < best.us) best = {i, us};
  }
  return best;
}

// rows of fp32 values that the epilogue needs, fetched into registers before the
// main loop (older than its loads, whose waits count younger ones) and put into
// LDS behind the ring after it: the epilogue's stores then wait for no load
template <int N, int THREADS, class F>
struct Staged {
  static constexpr int PER = (N + THREADS - 1) / THREADS;
  float v[PER];
  __device__ __forceinline__ void fetch(const F& f) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = (int)threadIdx.x + i * THREADS;
      v[i] = x < N ? f(x) : 0.f;
    }
  }
  __device__ __forceinline__ void put(float* lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = (int)threadIdx.x + i * THREADS;
      if (x < N) lds[x] = v[i];
    }
  }
};

// four consecutive values of a row, to memory as T: one store at any alignment of T
// (odd widths: fp32 dW of 9238 x 2385 82 -> 36 us, 8 bits 4032 x 9343 x 632 90 -> 66)
template <typename T>
__device__ __forceinline__ void store4(T* p, int left, const float (&v)[4]) {
  typedef T any4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (left >= 4) {
    *(any4*)p = any4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) p[r] = from_f32<T>(v[r]);
  }
}

template <typename T>
constexpr TileElem elem_of() { return sizeof(T) == 4 ? ELEM_F32 : ELEM_BF16; }

// The gradients' products.  b is a KR operand: a pair of fragments holds 8
// neighbouring columns of a row (bf16: all of them exist).  Stored in the operands'
// type (row stride ldc), or as fp32 partial sums (row stride Split::ld) where the
// contraction is split.
template <class D, class P, typename T>
__device__ __forceinline__ void store_tile(const typename P::Acc (&acc)[D::TM][D::TN], T* C, int ldc, int m0,
                                           int n0, int M, int N) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const int mw = m0 + (wave / D::WGN) * D::WM, nw = n0 + (wave % D::WGN) * D::WN;
#pragma unroll
  for (int i = 0; i < D::TM; ++i) {
    const int m = mw + P::row_of(i, fr);
    if (m >= M) continue;
#pragma unroll
    for (int j = 0; j < D::TN; j += 2) {
      const int n = nw + P::col_of(j, g * 4);
      if (n >= N) continue;
      T* p = C + (size_t)m * ldc + n;
      if constexpr (sizeof(T) == 2) {
        bf16x8 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[2 * r] = (bf16)acc[i][j][r], v[2 * r + 1] = (bf16)acc[i][j + 1][r];
        *(bf16x8*)p = v;
      } else {
        const float lo[4] = {acc[i][j][0], acc[i][j + 1][0], acc[i][j][1], acc[i][j + 1][1]};
        const float hi[4] = {acc[i][j][2], acc[i][j + 1][2], acc[i][j][3], acc[i][j + 1][3]};
        store4(p, N - n, lo);
        store4(p + 4, N - n - 4, hi);
      }
    }
  }
}

// First column of column block tn.  U: the last block ends with the matrix (if that is
// not narrower than a tile) and does some columns over again, the same sums in the
// same order, so that no load reaches past a row's end.
template <class D, bool U>
__device__ __forceinline__ int first_column(int tn, int cols) {
  return U && cols >= D::BN ? min(tn * D::BN, cols - D::BN) : tn * D::BN;
}

// A contraction split over gridDim.y slices of `per` steps: slice y writes fp32
// partial sums [rows][ld] behind those of the slices before it, which
// split_sum_kernel adds up in order.
struct Split {
  float* partial;   // NULL: not split
  int per, ld;      // ld: the output's columns in whole 16-byte pieces
};
__device__ __forceinline__ void take_slice(const Split& sp, TileShape& s) {
  s.first = (int)blockIdx.y * sp.per;
  s.steps = min(sp.per, s.steps - s.first);
}

// out (rows [0, half) to o0, the others to o1) = the sum of the slices' partials
// [rows][ldp], in ascending slice order; one thread per 4 columns
template <typename T>
__global__ __launch_bounds__(256) void split_sum_kernel(const float* __restrict__ partial, int slices, long rows,
                                                        long half, int cols, int ldp, T* o0, T* o1, int ld) {
  const long x = blockIdx.x * 256L + threadIdx.x, n4 = ldp / 4;
  if (x >= rows * n4) return;
  const long r = x / n4;
  const int c = (int)(x - r * n4) * 4;
  const float* p = partial + r * ldp + c;
  f32x4 a = *(const f32x4*)p;
#pragma unroll 4
  for (int i = 1; i < slices; ++i) a += *(const f32x4*)(p + i * rows * ldp);
  const float v[4] = {a[0], a[1], a[2], a[3]};
  store4((r < half ? o0 + r * ld : o1 + (r - half) * ld) + c, cols - c, v);
}

// Shapes of the bf16 and 8-bit products: times measured on products of 4096 x 20480 x
// 4096 (full), 333 rows (alone) and K = 1152 (end; with bf16 outputs for every column
// of the tile, half of it for the gated block), then moved by up to a quarter to
// choose best for 104 drawn products (1.5 % above each one's fastest shape in the
// mean, 12 % at most).  Two stages and several workgroups per CU where the tiles fill
// the chip -- the epilogue of one then runs beside the loop of another --, three or
// four stages where they do not: 7531 x 4608 x 1152 in 8 bits 84 us on 256 x 256, 63 on
// 128 x 128 with two stages, 89 with four; 600 x 1152 x 4608 57, 28 and 21, 16 on 64 x
// 128 with three.  Three stages on 64 and 32 rows, two workgroups per CU, beat four
// where there are more than 256 tiles (gated 200 x 4608 x 1152 15.4 -> 11.2 us) and
// lose where the weights of few rows stream from memory (1 x 10240 x 4096 33.5 and 36.3
// us on 32 rows).
using Tile256 = TileDims<256, 256, 2, 4, 2>;
using Tile128 = TileDims<128, 128, 2, 4, 2>;
using Tile128d = TileDims<128, 128, 2, 4, 4>;
using Tile64 = TileDims<64, 128, 2, 4, 2>;
using Tile64d = TileDims<64, 128, 2, 4, 3>;
using Tile32 = TileDims<32, 128, 1, 4, 4>;
using Tile32d = TileDims<32, 128, 1, 4, 3>;
using Tile32k = TileDims<32, 64, 2, 2, 3, 2>;
using Tile16k = TileDims<16, 32, 1, 1, 3, 4>;
constexpr TileChoice kTiles[] = {{256, 256, 1, 1.60f, 1.60f, 13.f}, {128, 128, 2, 0.72f, 1.02f, 4.8f},
                                 {128, 128, 1, 0.55f, 0.55f, 5.f},  {64, 128, 3, 0.60f, 1.01f, 3.f},
                                 {64, 128, 2, 0.48f, 1.00f, 2.85f}, {32, 128, 2, 0.44f, 0.78f, 2.f},
                                 {32, 64, 2, 0.155f, 0.37f, 2.2f},  {16, 32, 2, 0.073f, 0.17f, 2.5f}};
// Shapes with groups of waves, for few tiles: their launch takes up to 2048 threads for 64
// x 64 outputs (the others at most 512), so that it stays below 2^32 only up to here.
inline bool few_tiles(long rows, long cols) { return ((rows + 63) / 64) * ((cols + 63) / 64) < 1 << 21; }
constexpr int kGradTiles = 6, kTile32 = 5, kTile32k = 6, kTile16k = 7, kStream = 8;
// The products without slices (8-bit layer, gated forward) have two more shapes for few
// tiles of a long contraction: groups of waves share the steps of a tile.  us on the
// shapes before them, on Tile32k and on Tile16k: 8 bits 4 x 775 x 7447 20.5, 10.9, 9;
// F = 488 at 5 rows of K = 8896 35, 21, 11.7; F = 6488 at 21 rows of 2824 -, 13.4, 20.1.
// (Eight groups of 16 x 32 leave no room for a second workgroup: F = 1232 9.1 -> 8.2, F =
// 4256 17.0 -> 18.9.)  Tile32 takes one block of rows whose weights stream from memory.
inline int tile_index(long rows, long cols, int steps, float end_scale) {
  const bool groups = steps >= 4 && few_tiles(rows, cols);
  const int shape = choose_tile(kTiles, groups ? kGradTiles + 2 : kGradTiles, rows, cols, steps, end_scale).shape;
  return shape >= kTile32 && rows <= 32 && cols > 128 * 128 ? kStream : shape;
}

// fp32 (sizes: rows x columns of g | u x K): bound by the matrix cores (154 TFLOP/s: 1.7
// us per step of 128 x 128), so that two stages are enough and several workgroups share
// a CU (4096 x 9216 x 1152: 143 TFLOP/s on 128 x 128, 139 on 64 x 64, 134 and 128 with
// four stages).  Costs from 36 to 9216 tiles of 36 steps: 22.7 us for up to 256 of 64 x
// 64, 17.1 for every 256 more; 70.5 and 67 on 128 x 128.  A wave's step is 32 MFMAs of
// 32 cycles on 64 x 64, 16 on 32 x 64, where a chain of steps is what takes the time: 33
// x 2304 x 1152 22.3 and 14.9 us (three stages; two stages of 32 x 32 per wave 4 - 10 us
// more, four stages 0.5 - 2); 517 x 2832 x 1152 38 and 32; 1024 x 9216 x 1152 160 and 174.
using Tile64s = TileDims<64, 64, 2, 2, 2>;
using Tile32s = TileDims<32, 64, 2, 2, 3>;
constexpr TileChoice kTilesF32[] = {{128, 128, 1, 1.88f, 1.79f, 3.f}, {64, 64, 1, 0.605f, 0.455f, 0.9f},
                                    {32, 64, 1, 0.404f, 0.25f, 0.7f}, {32, 64, 1, 0.32f, 0.25f, 1.2f},
                                    {16, 32, 2, 0.10f, 0.18f, 3.f}};
// dW: a's fragments are turned in twos at least, which 16 rows per wave do not have.
// The last two, with groups of waves, for the gated forward: a step of 16 x 32 is 16
// MFMAs instead of 64 of the CU (23 x 9238 x 2385 32.9 us on 32 x 64, 25.6 with two
// groups; 1 x 4608 x 7496 80, 69 and 26 on 16 x 32; 82 x 4512 x 1792 22, 19, 23).
constexpr int kF32DwTiles = 2, kF32DxTiles = 3, kF32Groups = 3;
inline int tile_index_f32(long rows, long cols, int steps) {
  const bool groups = steps >= 4 && few_tiles(rows, cols);
  return choose_tile(kTilesF32, groups ? kF32Groups + 2 : kF32Groups, rows, cols, steps, 0.5f).shape;
}
constexpr int kMaxSlices = 16;

// group_m 8: eight row blocks share a column block's operand in an XCD's L2
template <class D>
inline TileShape tile_shape(int rows, int cols, int steps, int kbytes, int half) {
  TileShape s;
  s.tiles_m = (rows + D::BM - 1) / D::BM;
  s.tiles_n = (cols + D::BN - 1) / D::BN;
  s.group_m = 8;
  s.steps = steps;
  s.kbytes = kbytes;
  s.half = half;
  s.first = 0;
  return s;
}

#define T2I_TILES(SHAPE, CALL)                    \
  switch (SHAPE) {                                \
    case 0: { using D = Tile256; CALL; break; }   \
    case 1: { using D = Tile128; CALL; break; }   \
    case 2: { using D = Tile128d; CALL; break; }  \
    case 3: { using D = Tile64; CALL; break; }    \
    case 4: { using D = Tile64d; CALL; break; }   \
    default: { using D = Tile32d; CALL; break; }  \
  }
#define T2I_TILES_FWD(SHAPE, CALL)                        \
  switch (SHAPE) {                                        \
    case kTile32k: { using D = Tile32k; CALL; break; }    \
    case kTile16k: { using D = Tile16k; CALL; break; }    \
    case kStream: { using D = Tile32; CALL; break; }      \
    default: T2I_TILES(SHAPE, CALL)                       \
  }

#define T2I_TILES_F32_DW(SHAPE, CALL)            \
  switch (SHAPE) {                               \
    case 0: { using D = Tile128; CALL; break; }  \
    default: { using D = Tile64s; CALL; break; } \
  }
#define T2I_TILES_F32_DX(SHAPE, CALL)            \
  switch (SHAPE) {                               \
    case 2: { using D = Tile32s; CALL; break; }  \
    default: T2I_TILES_F32_DW(SHAPE, CALL)       \
  }
#define T2I_TILES_F32_FWD(SHAPE, CALL)                       \
  switch (SHAPE) {                                           \
    case kF32Groups: { using D = Tile32k; CALL; break; }     \
    case kF32Groups + 1: { using D = Tile16k; CALL; break; } \
    default: T2I_TILES_F32_DX(SHAPE, CALL)                   \
  }

// whether these sizes and strides of fp32 values, and pointers, are whole 16-byte pieces
inline bool f32_pieces(std::initializer_list<int> sizes, std::initializer_list<const void*> ptrs) {
  uintptr_t bits = 0;
  for (int n : sizes) bits |= (uintptr_t)n * 4;
  for (const void* p : ptrs) bits |= (uintptr_t)p;
  return bits % 16 == 0;
}

// Tile shape and slices of a gradient's product: as few slices as keep the time
// least, counting 4 us for the second launch and the partial sums' way out and back
// at 4 TB/s (1024 x 9216 x 1152: 63 us on 144 64 x 128 tiles, 41 in slices).
struct SplitPick { int shape, slices, per; };
inline SplitPick choose_split(const TileChoice* tiles, int shapes, long rows, long cols, int steps) {
  SplitPick best{0, 1, steps};
  float least = 0.f;
  for (int n = 1; n <= kMaxSlices; ++n) {
    const int per = (steps + n - 1) / n, slices = (steps + per - 1) / per;
    if (slices != n || (n > 1 && per < 4)) continue;
    const TilePick p = choose_tile(tiles, shapes, rows, cols, per, n > 1 ? 2.f : 1.f, n);
    const float us = p.us + (n > 1 ? 4.f + (float)n * rows * cols * 8 / 4e6f : 0.f);
    if (n == 1 || us < least) least = us, best = {p.shape, n, per};
  }
  return best;
}

// (adapter.hip: shapes of the layer beside adapters, of which three are its own, and of dx)
constexpr int kTile192 = 9, kTile16n = 11;
int adapter_tile(bool is_bf16, int M, int N, int K);
SplitPick adapter_dx_pick(bool is_bf16, int M, int N, int K);

inline long whole4(long cols) { return (cols + 3) / 4 * 4; }
inline SplitPick split_dx(bool is_bf16, long rows, long cols, int k) {
  return is_bf16 ? choose_split(kTiles, kGradTiles, rows, cols, (k + 63) / 64)
                 : choose_split(kTilesF32, kF32DxTiles, rows, cols, (k + 31) / 32);
}
inline SplitPick split_dw(bool is_bf16, long rows, long cols, int k) {
  return is_bf16 ? choose_split(kTiles, kGradTiles, rows, cols, (k + 63) / 64)
                 : choose_split(kTilesF32, kF32DwTiles, rows, cols, (k + 31) / 32);
}

template <typename T>
inline void split_sum(const Split& sp, int slices, long rows, long half, int cols, T* o0, T* o1, int ld,
                      hipStream_t st) {
  hipLaunchKernelGGL((split_sum_kernel<T>), dim3((unsigned)((rows * (sp.ld / 4) + 255) / 256)), dim3(256), 0, st,
                     sp.partial, slices, rows, half, cols, sp.ld, o0, o1, ld);
}

}  // namespace t2i
