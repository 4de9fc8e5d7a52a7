// The AdamW update of one element, shared by the step over many tensors (adamw.cu) and the server's apply kernels.
//
//   m = b1 m + (1 - b1) g        v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// In fp32.  The moments' operations are rounded one by one (no fused multiply-adds): the same bits on whatever path an element takes, which
// is what lets the 8-bit moments' codes be tested for equality.  The square root and the quotient, which only the step depends on, are the
// fast ones (sqrt.approx, div.approx: off by 2^-23 and 2 ulp); with the rounded ones the ordered server step, 37 updates of 813,258 weights,
// took 86 us, and the many-tensor step with 8-bit moments, 400 M elements, 1,528 us.  The constants are made in fp64 and rounded once.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

namespace psk {

struct AdamScalars {
  float b1, a1, b2, a2;      // beta and 1 - beta
  float eps, step_size;      // lr / (1 - b1^t)
  float rs2;                 // 1 / sqrt(1 - b2^t)
  float factor;              // of the gradient: its scale, and the clipping
};

// What the constants are made from.
struct AdamHyper {
  double lr, beta1, beta2, eps;
};

// beta^t by repeated squaring
__host__ __device__ inline double pow_steps(double beta, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r *= beta;
    beta *= beta;
  }
  return r;
}

__host__ __device__ inline AdamScalars adam_scalars(const AdamHyper& h, int64_t t, double factor) {
  AdamScalars s;
  s.b1 = (float)h.beta1; s.a1 = (float)(1.0 - h.beta1);
  s.b2 = (float)h.beta2; s.a2 = (float)(1.0 - h.beta2);
  s.eps = (float)h.eps;
  s.step_size = (float)(h.lr / (1.0 - pow_steps(h.beta1, t)));
  s.rs2 = (float)(1.0 / sqrt(1.0 - pow_steps(h.beta2, t)));
  s.factor = (float)factor;
  return s;
}

// The factor 1 - lr wd that the decoupled decay multiplies a weight with.
__host__ __device__ inline float adam_decay(double lr, double wd) {
#ifdef __CUDA_ARCH__
  return (float)__dsub_rn(1.0, __dmul_rn(lr, wd));
#else
  return (float)(1.0 - lr * wd);
#endif
}

#ifdef __CUDACC__
__device__ __forceinline__ void adam_update(float& p, float g, float& m, float& v, const AdamScalars& s, float decay) {
  m = __fadd_rn(__fmul_rn(m, s.b1), __fmul_rn(g, s.a1));
  v = __fadd_rn(__fmul_rn(v, s.b2), __fmul_rn(__fmul_rn(g, s.a2), g));
  float root;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
  const float d = fmaf(root, s.rs2, s.eps);      // at least 2^-126: within the fast quotient's range
  p = fmaf(-s.step_size, __fdividef(m, d), __fmul_rn(p, decay));
}
#endif

}  // namespace psk
