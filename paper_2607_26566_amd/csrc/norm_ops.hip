// The residual's addition with an RMS norm, its output in the operands' type or in 8
// bits, and the gradients (gfx950).  All of them are bound by HBM: a row's pieces are
// read once, 16 bytes per lane, held in registers while its sum is taken, and each
// output is written once.  With a large copy at 4.84 TB/s: 7531 rows of 1152 with an fp32
// residual 18.4 us (104 MB, 5.7 TB/s, part of it in the cache), 8192 of 4096 43 in bf16, 49
// to 8 bits (4.8), gradients of 4096 of 10240 69 + 5 (4.9).
#include <algorithm>
#include <type_traits>

#include "row_ops.h"

namespace t2i {

// sum over the TPR threads of a row, the same in each of them; `red` [TPR / 64] of the row
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[(threadIdx.x % TPR) >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v += red[i];
  }
  return v;
}

// the same of NV values per thread, each wave's sums of one after the other in the order of
// the row: the same result for any TPR NV; `red` [NV TPR / 64]
template <int TPR, int NV>
__device__ __forceinline__ float row_sum_in_order(float (&v)[NV], float* red) {
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v[i] += __shfl_xor(v[i], o, kWave);
  float s = 0.f;
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) red[i * NW + ((threadIdx.x % TPR) >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV * NW; ++i) s += red[i];
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) s += v[i];
  }
  return s;
}

// ---------------------------------------------------------------------------
// Forward: h = resid + x, rounded to resid's type R, which the norm then takes:
//   r = (mean h^2 + eps)^-1/2,  y = h r w.
// 8 bits: t = h w, T = max |t| over the row; y = t r, so that r leaves the quotient of
// the scale s = T r / 127 and an element alone: q = 127 t / T to the nearest whole
// number, ties to even, of the exact quotient.
//
// t of bf16 factors is exact in fp32 (but for its smallest values), that of fp32 ones in fp64.  127 t / T takes no
// division: m = fma(t, 127 / T, 1.5 2^23) leaves the nearest whole number n in its low
// bits; the factor, t and the product are off by 2^-24 of themselves each, so that n may
// be wrong only where the quotient is within 127 3 2^-24 < 2^-15 of a half.  Pieces that
// hold such a value (an element in 2^14) are settled by the sign of 127 t - (n +- 1/2) T:
// of bf16 factors r = fma(-n, T, 127 t) is exact (127 t has 23 bits, r, at most about T /
// 2, no more than 24 above the last place of t), of fp32 ones fp64 products with what their
// rounding leaves are.  (Settled by an fp64 division, one element after the other, 333 rows
// of 1051 took 11.2 us instead of 8.1, 8192 of 4096 53 instead of 48.)

constexpr float kMagic = 12582912.f;   // 1.5 2^23

// the nearest whole number to 127 t / T, ties to even, from an n that is it or next to it
__device__ __forceinline__ float settle(float n, float t, float T) {
  const float r2 = 2.f * fmaf(-n, T, 127.f * t);
  const bool odd = ((int)n & 1) != 0;
  return r2 > T || (r2 == T && odd) ? n + 1.f : r2 < -T || (r2 == -T && odd) ? n - 1.f : n;
}
// the same where neither 127 t nor the products with T need be exact
__device__ __forceinline__ double settle(double n, double t, double T) {
  const double p = 127. * t, pe = fma(127., t, -p);
  auto beside = [&](double c) {
    const double q = c * T;
    return (p - q) + (pe - fma(c, T, -q));
  };
  const bool odd = ((int)n & 1) != 0;
  const double up = beside(n + 0.5), down = beside(n - 0.5);
  return up > 0. || (up == 0. && odd) ? n + 1. : down < 0. || (down == 0. && odd) ? n - 1. : n;
}

// T: x, w and y; R: resid and h.  TPR threads per row, NV pieces per thread in
// registers; longer rows take their pieces of h (or x) again from memory.
template <typename T, typename R, int TPR, int NV, bool I8>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void add_rms_norm_kernel(NormFwd a) {
  constexpr int RPB = TPR > 256 ? 1 : 256 / TPR, NW = TPR / 64;
  constexpr bool WIDE = I8 && sizeof(R) == 4;   // products past fp32
  __shared__ float red_s[RPB][NV * NW];
  __shared__ uint32_t red_m[RPB][NW];
  __shared__ double red_d[RPB][NW];
  __shared__ float red_l[RPB][NW];
  const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
  const int row = blockIdx.x * RPB + rl, K = a.K;
  const bool live = row < a.rows;
  const size_t at = live ? row : 0;
  const T* const x = (const T*)a.x + at * a.ldx;
  const R* const resid = a.resid ? (const R*)a.resid + at * a.ldr : nullptr;
  R* const h = a.resid ? (R*)a.h + at * a.ldh : nullptr;
  const T* const w = (const T*)a.w;
  const int pieces = (K + 7) / 8, all = I8 ? (K + 127) / 128 * 16 : pieces;
  const int rounds = (pieces + TPR * NV - 1) / (TPR * NV);

  float v[NV][8];
  // the values of h in this thread's pieces of round r
  auto load = [&](int r, bool first) {
    Piece<T> px[NV];
    Piece<R> pr[NV];
    const bool sum = resid && first;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = ((r * NV + i) * TPR + t) * 8;
      px[i].clear();
      pr[i].clear();
      if (k < K) {
        if (!resid || first) load_piece(x, k, K, px[i]);
        if (resid) load_piece(sum ? resid : (const R*)h, k, K, pr[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = !resid ? px[i].get(j) : sum ? (float)(R)(pr[i].get(j) + px[i].get(j)) : pr[i].get(j);
    if (sum && live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = ((r * NV + i) * TPR + t) * 8;
        if (k < K) store_piece(h + k, K - k, v[i]);
      }
    }
  };
  // w of a piece (1 where there is none)
  auto weight = [&](int k, float (&o)[8]) {
    Piece<T> p;
    if (w && k < K) {
      load_piece(w, k, K, p);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = p.get(j);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = 1.f;
    }
  };

  double total = 0.;   // (over rounds; a round's squares in fp32)
  float ss[NV];        // a piece's each
  uint32_t top = 0;    // bits of the largest |h w|, which order as it does, infinity and NaN above
  double topd = 0.;
  for (int r = 0; r < rounds; ++r) {
    load(r, true);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      ss[i] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss[i] = fmaf(v[i][j], v[i][j], ss[i]);
      if constexpr (I8) {
        float wv[8];
        weight(((r * NV + i) * TPR + t) * 8, wv);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          top = max(top, __float_as_uint(v[i][j] * wv[j]) & 0x7fffffffu);
          if constexpr (WIDE) topd = fmax(topd, fabs((double)v[i][j] * (double)wv[j]));
        }
      }
    }
    if (rounds > 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) total += (double)ss[i];
  }
  if (rounds > 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) ss[i] = i == 0 ? (float)total : 0.f;
  if constexpr (I8) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      top = max(top, (uint32_t)__shfl_xor((int)top, o, kWave));
      if constexpr (WIDE) topd = fmax(topd, __shfl_xor(topd, o, kWave));
    }
    if constexpr (TPR > 64) {
      if ((t & 63) == 0) {
        red_m[rl][t >> 6] = top;
        if constexpr (WIDE) red_d[rl][t >> 6] = topd;
      }
    }
  }
  const float squares = row_sum_in_order<TPR, NV>(ss, red_s[rl]);
  if constexpr (I8 && TPR > 64) {
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      top = max(top, red_m[rl][i]);
      if constexpr (WIDE) topd = fmax(topd, red_d[rl][i]);
    }
  }
  const float rs = rsqrtf(fmaf(squares, 1.f / (float)K, a.eps));
  if (!live) return;

  if constexpr (!I8) {
    T* const y = (T*)a.y + at * a.ldy;
    for (int r = 0; r < rounds; ++r) {
      if (rounds > 1) load(r, false);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = ((r * NV + i) * TPR + t) * 8;
        if (k >= K) break;
        float wv[8];
        weight(k, wv);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * rs * wv[j];
        store_piece(y + k, K - k, v[i]);
      }
    }
  } else {
    const bool finite = top < 0x7f800000u && rs == rs;
    const float most = __uint_as_float(top);
    int8_t* const q = (int8_t*)a.y + at * a.ldy;
    if constexpr (!WIDE) {
      // Products of bf16 factors up to 2^-90 may have lost bits in fp32, which holds 2^160 times
      // them (from 2^-266): codes by division, settled as below.  (Apart, from memory once more,
      // so that other rows keep their registers.)
      if (most <= 0x1p-90f) {   // (the same for all threads of the row)
        const R* const from = resid ? (const R*)h : (const R*)x;
        auto products = [&](int c, float (&p)[8]) {
          Piece<R> hv;
          float wv[8];
          load_piece(from, c * 8, K, hv);
          weight(c * 8, wv);
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = (float)((double)hv.get(j) * (double)wv[j] * 0x1p160);
        };
        float large = 0.f;
#pragma unroll 1
        for (int c = t; c < pieces; c += TPR) {
          float p[8];
          products(c, p);
#pragma unroll
          for (int j = 0; j < 8; ++j) large = fmaxf(large, fabsf(p[j]));
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) large = fmaxf(large, __shfl_xor(large, o, kWave));
        if constexpr (TPR > 64) {
          if ((t & 63) == 0) red_l[rl][t >> 6] = large;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < NW; ++i) large = fmaxf(large, red_l[rl][i]);
        }
        if (t == 0) a.scale[at] = (float)((double)large * 0x1p-160 * (double)rs / 127.);
#pragma unroll 1
        for (int c = t; c < all; c += TPR) {
          uint64_t codes = 0;
          if (c < pieces && large > 0.f) {
            float p[8];
            products(c, p);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              codes |= (uint64_t)(uint8_t)(int)settle(rintf(127.f * p[j] / large), p[j], large) << (8 * j);
          }
          *(uint64_t*)(q + (size_t)c * 8) = codes;
        }
        return;
      }
    }
    // (factors past fp32's range, or products that have lost bits there: in fp64)
    const bool plain = most > 0x1p-90f && most < 0x1p120f;
    const float inv = plain ? 127.f / most : 0.f;
    const double exact = WIDE ? topd : (double)most;
    if (t == 0)
      a.scale[at] = !finite ? __uint_as_float(0x7fc00000u) : plain ? most * rs / 127.f : (float)(exact * (double)rs / 127.);
    const int qrounds = (all + TPR * NV - 1) / (TPR * NV);
    for (int r = 0; r < qrounds; ++r) {
      if (rounds > 1) load(r, false);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (r * NV + i) * TPR + t;
        if (c >= all) break;
        uint32_t b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (finite && exact > 0. && c < pieces && r < rounds) {
          float wv[8], far = 0.f;
          weight(c * 8, wv);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float p = v[i][j] * wv[j], m = fmaf(p, inv, kMagic);
            far = fmaxf(far, fabsf(fmaf(p, inv, kMagic - m)));
            b[j] = __float_as_uint(m);
          }
          if (far >= 0.5f - 0x1p-14f || !plain) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float n = __uint_as_float(b[j]) - kMagic;
              if (!WIDE && plain) {
                b[j] = (uint32_t)(int)settle(n, v[i][j] * wv[j], most);
              } else {
                const double p = (double)v[i][j] * (double)wv[j];
                b[j] = (uint32_t)(int)settle(plain ? (double)n : rint(127. * p / exact), p, exact);
              }
            }
          }
        }
        uint32_t o[2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
          o[g] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * g + 3], b[4 * g + 2], 0x0c0c0400),
                                       __builtin_amdgcn_perm(b[4 * g + 1], b[4 * g], 0x0c0c0400), 0x05040100);
        *(uint2*)(q + (size_t)c * 8) = uint2{o[0], o[1]};
      }
    }
  }
}

template <typename T, typename R, bool I8>
static void norm_any(const NormFwd& a, hipStream_t st) {
#define T2I_N(TPR, NV)                                                                                       \
  hipLaunchKernelGGL((add_rms_norm_kernel<T, R, TPR, NV, I8>),                                               \
                     dim3((unsigned)((a.rows + (TPR > 64 ? 0L : 3L)) / (TPR > 64 ? 1 : 4))),                 \
                     dim3(TPR > 64 ? TPR : 256), 0, st, a)
  // One wave per row up to 2048 elements, whose sums need no LDS, a workgroup for longer
  // rows, as few threads as hold theirs in two or three pieces each.  34 million elements, to
  // bf16 and to 8 bits: rows of 1152 45 and 55 us, 51 and 72 with 256 threads; 2048 45 and
  // 52, 44 and 51; 2560 44 and 52, 49 and 66 with 512; 5000 45 and 57, 54 and 71 with 1024;
  // 16384 46 and 54, 46 and 58 with 512 of four pieces.
  // Few rows, which leave CUs idle: a piece per thread (two of the longest).  16 rows of 1152
  // 4.0 and 7.5 us, 2.9 and 4.2 with 256 threads; 333 of 1051 5.4 and 8.6, 4.1 and 5.1; 1500 of
  // 1000 4.3 and 6.5, 4.7 and 6.4, of 1152 5.0 and 8.0, 4.9 and 6.7, of 2048 6.5 and 10.2, 5.6
  // and 7.4; 700 of 4096 5.8 and 7.8, 5.5 and 7.1 with 512; 100 of 8192
  // 4.1 and 6.5, 4.1 and 5.8 with 1024, 333 5.9 and 8.3, 6.2 and 8.2.
  if (a.K <= 512) T2I_N(64, 1);
  else if (a.K <= 2048 && a.rows <= (a.K <= 1024 ? 1024 : 2048)) T2I_N(256, 1);
  else if (a.K <= 1024) T2I_N(64, 2);
  else if (a.K <= 1536) T2I_N(64, 3);
  else if (a.K <= 2048) T2I_N(64, 4);
  else if (a.K <= 4096 && a.rows <= 1024) T2I_N(512, 1);
  else if (a.K <= 4096) T2I_N(256, 2);
  else if (a.K <= 8192 && a.rows <= 256) T2I_N(1024, 1);
  else if (a.K <= 8192) T2I_N(512, 2);
  else if (a.K <= 12288 && a.rows > 256) T2I_N(512, 3);
  else T2I_N(1024, 2);
#undef T2I_N
}

hipError_t launch_add_rms_norm(bool is_bf16, bool resid_bf16, bool to_i8, const NormFwd& a, hipStream_t st) {
  if (is_bf16 && resid_bf16) to_i8 ? norm_any<bf16, bf16, true>(a, st) : norm_any<bf16, bf16, false>(a, st);
  else if (is_bf16) to_i8 ? norm_any<bf16, float, true>(a, st) : norm_any<bf16, float, false>(a, st);
  else to_i8 ? norm_any<float, float, true>(a, st) : norm_any<float, float, false>(a, st);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Backward, with d = dy w, n = h r:
//   dsum = dh + r (d - n mean(d n)),  dw = sum over rows of dy n.
// A fixed number of workgroups walks the rows; a thread keeps its columns of w and of
// dw, which adds up over the thread's own rows (at most kChain), in fp64 over the waves of a
// workgroup that have the same columns and in fp64 over the workgroups
// (norm_weight_grad_kernel): a fixed order.  A thread's and a workgroup's sums are fp32 where
// the result is bf16, fp64 where it is fp32 (16000 rows of 512: error of dw 8.9e-8 with sums
// in fp32, 200000 of 64 1.6e-7; a result's own rounding and its products' are 5 to 6e-8), from
// three pieces per thread in LDS, for registers hold no more.
constexpr int kChain = 64;
template <typename T>
using ColumnSum = std::conditional_t<sizeof(T) == 4, double, float>;
__device__ __forceinline__ void store_sums(float* p, int n, const float (&v)[8]) { store_piece(p, n, v); }
__device__ __forceinline__ void store_sums(double* p, int n, const double (&v)[8]) {
  typedef double any2 __attribute__((ext_vector_type(2), aligned(8)));
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    if (i + 2 <= n) *(any2*)(p + i) = any2{v[i], v[i + 1]};
    else if (i < n) p[i] = v[i];
  }
}

template <typename T, typename R, int TPR, int NV>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void add_rms_norm_bwd_kernel(
    NormBwd a, ColumnSum<T>* __restrict__ partial) {
  using S = ColumnSum<T>;
  constexpr int RPB = TPR > 256 ? 1 : 256 / TPR, NW = TPR / 64;
  constexpr bool IN_LDS = sizeof(S) == 8 && NV >= 3;
  __shared__ float red[2][2][RPB][NW];
  __shared__ S cols[RPB > 1 ? RPB : 1][RPB > 1 ? TPR * NV * 8 : 1];
  __shared__ S kept[IN_LDS ? NV : 1][IN_LDS ? 8 : 1][IN_LDS ? TPR : 1];   // a thread's own each
  const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR, K = a.K;
  S dw[IN_LDS ? 1 : NV][8];
  Piece<T> w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int k = (i * TPR + t) * 8;
    w[i].clear();
    if (k < K) {
      if (a.w) load_piece((const T*)a.w, k, K, w[i]);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) w[i].set(j, (T)1.f);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if constexpr (IN_LDS) kept[i][j][t] = 0;
      else dw[i][j] = 0;
  }
  int parity = 0;
  for (int r0 = blockIdx.x * RPB; r0 < a.rows; r0 += gridDim.x * RPB, parity ^= 1) {
    const int row = r0 + rl;
    const bool live = row < a.rows;
    const size_t at = live ? row : 0;
    Piece<T> dy[NV];
    Piece<R> h[NV], dh[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = (i * TPR + t) * 8;
      dy[i].clear();
      h[i].clear();
      dh[i].clear();
      if (live && k < K) {
        load_piece((const T*)a.dy + at * a.lddy, k, K, dy[i]);
        load_piece((const R*)a.h + at * a.ldh, k, K, h[i]);
        if (a.dh) load_piece((const R*)a.dh + at * a.lddh, k, K, dh[i]);
      }
    }
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float hv = h[i].get(j);
        ss = fmaf(hv, hv, ss);
        dot = fmaf(dy[i].get(j) * w[i].get(j), hv, dot);
      }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      ss += __shfl_xor(ss, o, kWave);
      dot += __shfl_xor(dot, o, kWave);
    }
    if constexpr (TPR > 64) {
      if ((t & 63) == 0) {
        red[parity][0][rl][t >> 6] = ss;
        red[parity][1][rl][t >> 6] = dot;
      }
      __syncthreads();   // (the other parity's values may still be read)
      ss = dot = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        ss += red[parity][0][rl][i];
        dot += red[parity][1][rl][i];
      }
    }
    const float rk = 1.f / (float)K, r = rsqrtf(fmaf(ss, rk, a.eps)), c = dot * r * rk;
    if (live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int k = (i * TPR + t) * 8;
        if (k >= K) break;
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float n = h[i].get(j) * r, d = dy[i].get(j);
          if constexpr (IN_LDS) kept[i][j][t] += (S)(d * n);
          else if constexpr (sizeof(S) == 8) dw[i][j] += (S)(d * n);
          else dw[i][j] = fmaf(d, n, dw[i][j]);
          o[j] = fmaf(r, fmaf(-n, c, d * w[i].get(j)), dh[i].get(j));
        }
        store_piece((T*)a.dx + at * a.lddx + k, K - k, o);
        if (a.dresid) store_piece((R*)a.dresid + at * a.lddr + k, K - k, o);
      }
    }
  }
  // (one workgroup: its sums are dw)
  T* const whole = gridDim.x == 1 ? (T*)a.dw : nullptr;
  if (!partial && !whole) return;
  S* const p = partial + (size_t)blockIdx.x * K;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) cols[rl][(i * TPR + t) * 8 + j] = dw[i][j];
    __syncthreads();
    for (int k = threadIdx.x; k < K; k += 256) {
      double s = 0.;
#pragma unroll
      for (int g = 0; g < RPB; ++g) s += (double)cols[g][k];
      if (whole) whole[k] = from_f32<T>((float)s);
      else p[k] = (S)s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = (i * TPR + t) * 8;
      if (k >= K) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if constexpr (IN_LDS) dw[0][j] = kept[i][j][t];
      const S(&o)[8] = dw[IN_LDS ? 0 : i];
      if (whole) {
        const float v[8] = {(float)o[0], (float)o[1], (float)o[2], (float)o[3],
                            (float)o[4], (float)o[5], (float)o[6], (float)o[7]};
        store_piece(whole + k, K - k, v);
      } else {
        store_sums(p + k, K - k, o);
      }
    }
  }
}

// rows longer than registers hold: a workgroup per row reads its pieces twice and keeps r;
// dw by a kernel of its own
template <typename T, typename R>
__global__ __launch_bounds__(1024) void add_rms_norm_bwd_long_kernel(NormBwd a, float* __restrict__ rstd) {
  __shared__ float red[2][16];
  const int row = blockIdx.x, K = a.K;
  const T* const dy = (const T*)a.dy + (size_t)row * a.lddy;
  const R* const h = (const R*)a.h + (size_t)row * a.ldh;
  auto weight = [&](int k, Piece<T>& p) {
    if (a.w) load_piece((const T*)a.w, k, K, p);
    else {
      p.clear();
#pragma unroll
      for (int j = 0; j < 8; ++j) p.set(j, (T)1.f);
    }
  };
  double sd = 0., dd = 0.;
  for (int k = threadIdx.x * 8; k < K; k += 8192) {
    Piece<T> pd, pw;
    Piece<R> ph;
    load_piece(dy, k, K, pd);
    load_piece(h, k, K, ph);
    weight(k, pw);
    float s = 0.f, d = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float hv = ph.get(j);
      s = fmaf(hv, hv, s);
      d = fmaf(pd.get(j) * pw.get(j), hv, d);
    }
    sd += (double)s;
    dd += (double)d;
  }
  const float ss = row_sum<1024>((float)sd, red[0]), dot = row_sum<1024>((float)dd, red[1]);
  const float rk = 1.f / (float)K, r = rsqrtf(fmaf(ss, rk, a.eps)), c = dot * r * rk;
  if (rstd && threadIdx.x == 0) rstd[row] = r;
  for (int k = threadIdx.x * 8; k < K; k += 8192) {
    Piece<T> pd, pw;
    Piece<R> ph, pg;
    load_piece(dy, k, K, pd);
    load_piece(h, k, K, ph);
    weight(k, pw);
    pg.clear();
    if (a.dh) load_piece((const R*)a.dh + (size_t)row * a.lddh, k, K, pg);
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = fmaf(r, fmaf(-(ph.get(j) * r), c, pd.get(j) * pw.get(j)), pg.get(j));
    store_piece((T*)a.dx + (size_t)row * a.lddx + k, K - k, o);
    if (a.dresid) store_piece((R*)a.dresid + (size_t)row * a.lddr + k, K - k, o);
  }
}
// (after the rows': dx may not lie over dy or h)
template <typename T, typename R>
__global__ __launch_bounds__(256) void add_rms_norm_dw_long_kernel(NormBwd a, const float* __restrict__ rstd,
                                                                   ColumnSum<T>* __restrict__ partial) {
  using S = ColumnSum<T>;
  const int k = (blockIdx.y * 256 + threadIdx.x) * 8, K = a.K;
  if (k >= K) return;
  S dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Piece<T> pd;
    Piece<R> ph;
    load_piece((const T*)a.dy + (size_t)row * a.lddy, k, K, pd);
    load_piece((const R*)a.h + (size_t)row * a.ldh, k, K, ph);
    const float r = rstd[row];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if constexpr (sizeof(S) == 8) dw[j] += (S)(pd.get(j) * (ph.get(j) * r));
      else dw[j] = fmaf(pd.get(j), ph.get(j) * r, dw[j]);
  }
  store_sums(partial + (size_t)blockIdx.x * K + k, K - k, dw);
}

template <typename T>
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(const ColumnSum<T>* __restrict__ partial,
                                                                int blocks, int K, T* __restrict__ dw) {
  const int c = blockIdx.x * 16 + threadIdx.x % 16;
  const double v = column_sum(partial, blocks, (size_t)K, c, c < K);
  if (threadIdx.x < 16 && c < K) dw[c] = from_f32<T>((float)v);
}

constexpr int kNormRegisters = 16384;   // elements of a row that a workgroup holds
// a wave per row, four rows at a time, up to 1024 elements (longer: 4451 rows of 1152 22
// us, 18.4 with a workgroup per row)
static int norm_rows_at_once(int K) { return K <= 1024 ? 4 : 1; }
// Workgroups: as few as keep the memory busy, for their sums of columns go out and back
// (4451 x 1152 19.2 us with 512, 18.5 with 768; 8192 x 4096 51.6, 54; 4096 x 10240 73 with
// 256, 80 with 512; 2000 x 8192 52.5, 57.8).  fp64 sums of the longest rows, whose kernel has
// several workgroups to a row, from 64 (600 x 20000 in fp32 61 us, 76 with 256).
int norm_bwd_blocks(bool is_bf16, int rows, int K) {
  const int per = norm_rows_at_once(K);
  const long units = ((long)rows + per - 1) / per;
  // few rows: one workgroup, whose sums need no second launch
  if (units <= 4 && K <= kNormRegisters) return 1;
  const int most = K <= 1024 ? 512 : K <= 2048 ? 768 : K <= 4096 ? 512 : K <= kNormRegisters || is_bf16 ? 256 : 64;
  return (int)std::max(std::min<long>(units, most), (units + kChain - 1) / kChain);
}

template <typename T, typename R>
static void norm_bwd_any(const NormBwd& a, float* ws, hipStream_t st) {
  const int blocks = norm_bwd_blocks(sizeof(T) == 2, a.rows, a.K);
  if (norm_bwd_ws_bytes(a.rows, a.K) == 0) ws = nullptr;
  // rows' factors first, then the workgroups' sums of columns
  float* const rstd = ws;
  using S = ColumnSum<T>;
  S* const partial = ws ? (S*)(ws + ((size_t)a.rows + 63) / 64 * 64) : nullptr;
#define T2I_N(TPR, NV)                                                                                  \
  hipLaunchKernelGGL((add_rms_norm_bwd_kernel<T, R, TPR, NV>), dim3((unsigned)blocks),                  \
                     dim3(TPR > 256 ? TPR : 256), 0, st, a, partial)
  if (a.K <= 512) T2I_N(64, 1);
  else if (a.K <= 1024) T2I_N(64, 2);
  else if (a.K <= 2048) T2I_N(256, 1);
  else if (a.K <= 4096) T2I_N(256, 2);
  else if (a.K <= 8192) T2I_N(512, 2);
  else if (a.K <= 12288) T2I_N(512, 3);
  else if (a.K <= kNormRegisters) T2I_N(512, 4);
  else {
    hipLaunchKernelGGL((add_rms_norm_bwd_long_kernel<T, R>), dim3((unsigned)a.rows), dim3(1024), 0, st, a, rstd);
    if (partial)
      hipLaunchKernelGGL((add_rms_norm_dw_long_kernel<T, R>), dim3((unsigned)blocks, (unsigned)((a.K + 2047) / 2048)),
                         dim3(256), 0, st, a, rstd, partial);
  }
#undef T2I_N
  if (partial)
    hipLaunchKernelGGL((norm_weight_grad_kernel<T>), dim3((unsigned)((a.K + 15) / 16)), dim3(1024), 0, st, partial, blocks,
                       a.K, (T*)a.dw);
}

hipError_t launch_add_rms_norm_bwd(bool is_bf16, bool resid_bf16, const NormBwd& a, float* ws, hipStream_t st) {
  if (is_bf16 && resid_bf16) norm_bwd_any<bf16, bf16>(a, ws, st);
  else if (is_bf16) norm_bwd_any<bf16, float>(a, ws, st);
  else norm_bwd_any<float, float>(a, ws, st);
  return hipGetLastError();
}

size_t norm_bwd_ws_bytes(int rows, int K) {
  const size_t low = norm_bwd_blocks(true, rows, K), full = norm_bwd_blocks(false, rows, K);
  if (low == 1 && K <= kNormRegisters) return 0;
  return (((size_t)rows + 63) / 64 * 64 + std::max(low, 2 * full) * K) * 4;   // (for either type)
}

}  // namespace t2i
