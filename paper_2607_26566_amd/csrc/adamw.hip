// An AdamW step over many tensors at once (gfx950), bound by HBM: weights, gradients and
// moments are read once and weights and moments written once, 16 bytes per lane and
// load, one piece of eight elements per thread.  Up to 64 tensors, whose pointers travel
// as kernel arguments, take one launch.
//
//   g' = c g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p -= lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd p)
//
// in fp32.  bf16 weights are the rounded copies of fp32 masters, which hold what a step
// adds below bf16's half step.
//
// 28 bytes an element with bf16 weights and gradients: 42 million of them 224 us, 5.3 TB/s
// read and written (a large copy: 4.84); the counted step's factors, worked out by each
// workgroup while its loads are under way, add 1 (before them: 6).  2.1 million elements
// of 168 small tensors: three launches of 7 us, which the last waves' latency bounds.
#include "row_ops.h"

namespace t2i {

template <typename T, typename G>
__global__ __launch_bounds__(256) void adamw_kernel(AdamGroup a, AdamScalars s) {
  constexpr bool LOW = sizeof(T) == 2;
  __shared__ float factors[2];
  // the tensor of this workgroup: as many as end before it
  const int lane = threadIdx.x & 63;
  const int which = __builtin_amdgcn_readfirstlane(
      (int)__popcll(__ballot(lane < a.n && a.first[lane + 1] <= (int)blockIdx.x)));
  const int64_t n = a.numel[which], at = ((int64_t)((int)blockIdx.x - a.first[which]) * 256 + threadIdx.x) * 8;
  const int k = n - at < 8 ? (int)(n - at) : 8;   // (<= 0: none)
  float* const master = LOW ? a.master[which] + at : (float*)a.p[which] + at;
  float* const m = a.m[which] + at;
  float* const v = a.v[which] + at;
  Piece<float> pp, pm, pv;
  Piece<G> pg;
  if (k > 0) {
    load_piece(master, 0, k, pp);
    load_piece((const G*)a.g[which] + at, 0, k, pg);
    load_piece(m, 0, k, pm);
    load_piece(v, 0, k, pv);
  }
  float r1 = s.r1, r2 = s.r2, lr = s.lr;
  if (s.step) {   // (on the device: a graph's replays count on; while the loads are under way)
    if (threadIdx.x == 0) {
      const double t = (double)*s.step;
      factors[0] = (float)(1. / (1. - pow(s.beta1, t)));
      factors[1] = (float)(1. / (1. - pow(s.beta2, t)));
    }
    __syncthreads();
    r1 = factors[0], r2 = factors[1];
  }
  if (s.lr_dev) lr = *s.lr_dev;
  const float c = s.grad_scale ? *s.grad_scale : 1.f;
  if (k <= 0) return;
  float np[8], nm[8], nv[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float g = pg.get(i) * c;
    nm[i] = fmaf(s.b1, pm.get(i), s.c1 * g);
    nv[i] = fmaf(s.b2, pv.get(i), s.c2 * g * g);
    np[i] = pp.get(i) - lr * fmaf(s.wd, pp.get(i), nm[i] * r1 / (sqrtf(nv[i] * r2) + s.eps));
  }
  store_piece(master, k, np);
  store_piece(m, k, nm);
  store_piece(v, k, nv);
  if constexpr (LOW) store_piece((T*)a.p[which] + at, k, np);
}

hipError_t launch_adamw(bool low, bool grad_bf16, const AdamGroup& a, const AdamScalars& s, hipStream_t st) {
  const dim3 grid((unsigned)a.first[a.n]);
  if (low && grad_bf16) hipLaunchKernelGGL((adamw_kernel<bf16, bf16>), grid, dim3(256), 0, st, a, s);
  else if (low) hipLaunchKernelGGL((adamw_kernel<bf16, float>), grid, dim3(256), 0, st, a, s);
  else if (grad_bf16) hipLaunchKernelGGL((adamw_kernel<float, bf16>), grid, dim3(256), 0, st, a, s);
  else hipLaunchKernelGGL((adamw_kernel<float, float>), grid, dim3(256), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace t2i
