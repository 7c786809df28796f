// Entry point of the AdamW step: argument checks, then a launch per group of tensors.
#include <cmath>
#include <cstring>

#include "block_ops.h"

using namespace t2i;

namespace {

bool bad_dtype(int32_t d) { return d != T2I_F32 && d != T2I_BF16; }
bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
bool fraction(double b) { return b >= 0. && b < 1.; }

}  // namespace

extern "C" {

t2i_status t2i_op_adamw_step(int32_t param_dtype, int32_t grad_dtype, int32_t n, const int64_t* numel,
                             void* const* params, const void* const* grads, float* const* exp_avg,
                             float* const* exp_avg_sq, float* const* masters, double lr, double beta1, double beta2,
                             double eps, double weight_decay, int64_t step, const float* lr_device,
                             const int32_t* step_device, const float* grad_scale, void* stream) {
  if (bad_dtype(param_dtype) || bad_dtype(grad_dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (n < 1) return ops_fail(T2I_ERR_SHAPE, "no tensors");
  if (!numel || !params || !grads || !exp_avg || !exp_avg_sq) return ops_fail(T2I_ERR_INVALID_ARG, "NULL array");
  const bool low = param_dtype == T2I_BF16;
  if (low != (masters != nullptr)) return ops_fail(T2I_ERR_INVALID_ARG, "bf16 weights, and only they, have fp32 masters");
  if (!fraction(beta1) || !fraction(beta2)) return ops_fail(T2I_ERR_INVALID_ARG, "betas must be in [0, 1)");
  if (!(eps >= 0.) || !std::isfinite(eps) || !std::isfinite(weight_decay) || (!lr_device && !std::isfinite(lr)))
    return ops_fail(T2I_ERR_INVALID_ARG, "lr, eps and weight_decay must be finite, eps >= 0");
  if (!step_device && step < 1) return ops_fail(T2I_ERR_INVALID_ARG, "steps count from 1");
  if (off(lr_device, 4) || off(step_device, 4) || off(grad_scale, 4))
    return ops_fail(T2I_ERR_INVALID_ARG, "lr, step and grad_scale need 4-byte alignment");
  const size_t pe = low ? 2 : 4, ge = grad_dtype == T2I_BF16 ? 2 : 4;
  for (int32_t i = 0; i < n; ++i) {
    if (numel[i] < 0 || numel[i] > 1LL << 33) return ops_fail(T2I_ERR_SHAPE, "a tensor has 0 .. 2^33 elements");
    if (numel[i] == 0) continue;
    if (!params[i] || !grads[i] || !exp_avg[i] || !exp_avg_sq[i] || (low && !masters[i]))
      return ops_fail(T2I_ERR_INVALID_ARG, "NULL tensor");
    if (off(params[i], pe) || off(grads[i], ge) || off(exp_avg[i], 4) || off(exp_avg_sq[i], 4) ||
        (low && off(masters[i], 4)))
      return ops_fail(T2I_ERR_INVALID_ARG, "tensors need the alignment of their type");
  }
  AdamScalars s;
  std::memset(&s, 0, sizeof(s));
  s.beta1 = beta1;
  s.beta2 = beta2;
  s.b1 = (float)beta1;
  s.b2 = (float)beta2;
  s.c1 = (float)(1. - beta1);
  s.c2 = (float)(1. - beta2);
  s.lr = (float)lr;
  s.eps = (float)eps;
  s.wd = (float)weight_decay;
  if (!step_device) {
    s.r1 = (float)(1. / (1. - std::pow(beta1, (double)step)));
    s.r2 = (float)(1. / (1. - std::pow(beta2, (double)step)));
  }
  s.lr_dev = lr_device;
  s.step = step_device;
  s.grad_scale = grad_scale;
  AdamGroup a;
  a.n = 0;
  a.first[0] = 0;
  hipError_t err = hipSuccess;
  auto flush = [&]() {
    if (a.n && err == hipSuccess) err = launch_adamw(low, grad_dtype == T2I_BF16, a, s, (hipStream_t)stream);
    a.n = 0;
  };
  for (int32_t i = 0; i < n && err == hipSuccess; ++i) {
    if (numel[i] == 0) continue;
    // workgroups of 2048 elements; a launch has fewer than 2^32 threads
    const int64_t blocks = (numel[i] + 2047) / 2048;
    if (a.n == kAdamTensors || (a.n && a.first[a.n] + blocks >= 1 << 23)) flush();
    a.p[a.n] = params[i];
    a.g[a.n] = grads[i];
    a.m[a.n] = exp_avg[i];
    a.v[a.n] = exp_avg_sq[i];
    a.master[a.n] = low ? masters[i] : nullptr;
    a.numel[a.n] = numel[i];
    a.first[a.n + 1] = a.first[a.n] + (int32_t)blocks;
    ++a.n;
  }
  flush();
  return err == hipSuccess ? T2I_OK : ops_fail(T2I_ERR_DEVICE, hipGetErrorString(err));
}

}  // extern "C"
