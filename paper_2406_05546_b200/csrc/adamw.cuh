// The AdamW update of one element, shared by the step over many tensors (adamw.cu) and the server's apply kernels.
//
//   m = b1 m + (1 - b1) g        v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// In fp32.  The moments' operations are rounded one by one (no fused multiply-adds): the same bits on whatever path an element takes, which
// is what lets the 8-bit moments' codes be tested for equality.  The square root and the quotient, which only the step depends on, are the
// approximate ones (off by 2^-23 and 2 ulp), and two elements share an instruction where there is one for pairs.  us of the ordered server step,
// 37 updates of 813,258 weights, and of the many-tensor step with 8-bit moments, 400 M elements: all rounded 86 and 1,528; approximate 39 and
// 1,400; in pairs 36 and 1,283.  The constants are made in fp64 and rounded once.
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
  float minus_zero;          // what adam_update2 adds to a product to have it rounded
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
  s.minus_zero = -0.0f;
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
// Pairs of elements in 64-bit registers: two operations an instruction.
__device__ __forceinline__ unsigned long long adam_pair(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void adam_unpair(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ unsigned long long add_pair(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// A rounded product.  The assembler joins a mul.rn.f32x2 and an add.rn.f32x2 behind it into one multiply-add; one that adds a -0 which it does not
// know at compile time stays by itself, and a + -0 is a for every a.
__device__ __forceinline__ unsigned long long mul_pair(unsigned long long a, unsigned long long b, const AdamScalars& s) {
  return fma_pair(a, b, adam_pair(s.minus_zero, s.minus_zero));
}
// The reciprocal of sqrt(v) * rs2 + eps.  The root is taken of at least 2^-126 (a smaller v, that of gradients below 4e-18, has roots below 1e-19), so
// that neither it nor the sum, which lies in 2^-126 .. 2^92, needs the slower forms for subnormal values.  NaN stays.
__device__ __forceinline__ float adam_root(float v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(1.17549435e-38f));
  asm("sqrt.approx.ftz.f32 %0, %0;" : "+f"(r));
  return r;
}
__device__ __forceinline__ float adam_reciprocal(float d) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return r;
}
// Two elements; g: the gradient, factor included.
__device__ __forceinline__ void adam_update2(float& p0, float& p1, float g0, float g1, float& m0, float& m1, float& v0, float& v1, const AdamScalars& s, float decay) {
  const unsigned long long g = adam_pair(g0, g1);
  const unsigned long long m = add_pair(mul_pair(adam_pair(m0, m1), adam_pair(s.b1, s.b1), s), mul_pair(g, adam_pair(s.a1, s.a1), s));
  const unsigned long long v = add_pair(mul_pair(adam_pair(v0, v1), adam_pair(s.b2, s.b2), s), mul_pair(mul_pair(g, adam_pair(s.a2, s.a2), s), g, s));
  adam_unpair(v, v0, v1);
  adam_unpair(m, m0, m1);
  float d0, d1;
  adam_unpair(fma_pair(adam_pair(adam_root(v0), adam_root(v1)), adam_pair(s.rs2, s.rs2), adam_pair(s.eps, s.eps)), d0, d1);
  const unsigned long long q = mul_pair(m, adam_pair(adam_reciprocal(d0), adam_reciprocal(d1)), s);
  adam_unpair(fma_pair(adam_pair(-s.step_size, -s.step_size), q, mul_pair(adam_pair(p0, p1), adam_pair(decay, decay), s)), p0, p1);
}
#endif

}  // namespace psk
