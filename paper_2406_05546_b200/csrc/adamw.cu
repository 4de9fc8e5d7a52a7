// One AdamW step over many tensors at once (ps_adamw_* in include/ps.h): every tensor is cut into pieces of PIECE elements, and one
// launch covers the pieces of all of them, whatever their sizes.
//
// Bytes per element: weight, gradient, copy and the moments, each read or written once: 28 with everything in fp32, 16 with a bf16
// gradient and copy and moments in 8 bits.  Nothing is computed twice and nothing is reused, so HBM is the bound; a thread takes eight
// consecutive elements with one load of 32 (fp32), 16 or 8 bytes per array, and enough CTAs are resident to keep the memory busy.
// Clipping by global norm needs the norm before the first update: it reads the gradients once more, in a kernel of its own.
//
// Moments in 8 bits: blocks of 256 elements (one warp: eight elements a lane) with a power-of-two scale each, so that scaling rounds
// nothing.  The first moment is held in e4m3, rounded to nearest even.  The second is held in e5m2 (its square needs the range) and
// rounded stochastically: a step changes it by 1 - b2, a thousandth, where neighbouring codes are 14 to 25 % apart, so to nearest it would
// never fall again; with sixteen random bits (Philox, the repository's generator) it follows in the mean.  A positive second moment is never
// rounded to zero: the next step would divide by eps alone.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <type_traits>
#include <vector>

#include "adamw.cuh"
#include "device_common.cuh"
#include "error.h"
#include "kernels.h"
#include "ps.h"

namespace psk {

namespace {

constexpr int TPB = 256, PER = 8, PIECE = TPB * PER;      // 2,048 elements: eight blocks of 8-bit moments
constexpr int BLOCK8 = 32 * PER;                          // elements that share a scale
constexpr int NORM_CTAS = 148 * 8;
constexpr int64_t MAX_ELEMENTS = (int64_t)1 << 40;

struct DevTensor {
  void* p; const void* g; void* copy; void* m; void* v;
  uint8_t *m_scale, *v_scale;
  int64_t n;
  double wd;
  int32_t wide_g, wide;      // may the gradient / all arrays be read in vectors?
};

// Where the pieces lie: piece `i` of the call is piece i - first of `tensor`.
struct PieceRef { int32_t tensor, piece; };

// Device-side state of an optimizer.
struct DevState {
  AdamScalars s;
  double lr;                 // as used by the step under way
  int64_t step;              // steps taken, where the device counts them; the step under way
  int64_t counted;
  int64_t skipped;
  int32_t skip;
  float norm;
  uint32_t ticket;
};

struct Call {
  AdamScalars s;             // where the host knows them all
  AdamHyper h;
  double grad_scale, clip;
  const float* lr_dev;
  int64_t step;              // 0: the device counts
  uint64_t seed;
  int32_t skip_nonfinite;
};

__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }

// Eight consecutive values: 32 bytes of fp32 in one access, 16 of the narrow types, 8 of codes.  Streamed: none of it is used again.
__device__ __forceinline__ void load8(const float* p, float (&x)[PER]) {
  asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[PER]) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
// Eight values as they are loaded.
template <typename T> struct Raw8 { uint4 w; };
template <> struct Raw8<float> { float x[PER]; };
__device__ __forceinline__ void load8(const float* p, Raw8<float>& r) { load8(p, r.x); }
template <typename T> __device__ __forceinline__ void load8(const T* p, Raw8<T>& r) { r.w = __ldcs(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&x)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = r.x[i];
}
template <typename T> __device__ __forceinline__ void widen8(const Raw8<T>& r, float (&x)[PER]) {
  T t[PER];
  memcpy(t, &r.w, 16);
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = as_float(t[i]);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[PER]) {
  T t[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) t[i] = from_float<T>(x[i]);
  uint4 w;
  memcpy(&w, t, 16);
  *reinterpret_cast<uint4*>(p) = w;
}
// n of eight values from i0 on, the others zero / left alone
__device__ __forceinline__ void load_some(const float* p, int64_t i0, int n, Raw8<float>& r) {
#pragma unroll
  for (int i = 0; i < PER; ++i) r.x[i] = i < n ? p[i0 + i] : 0.f;
}
template <typename T> __device__ __forceinline__ void load_some(const T* p, int64_t i0, int n, Raw8<T>& r) {
  T t[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) t[i] = i < n ? p[i0 + i] : from_float<T>(0.f);
  memcpy(&r.w, t, 16);
}
template <typename T> __device__ __forceinline__ void store_some(T* p, int64_t i0, int n, const float (&x)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i < n) p[i0 + i] = from_float<T>(x[i]);
}

// ---- moments in 8 bits
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }            // 2^(byte - 127), byte 1 .. 254; 0: 0
__device__ __forceinline__ float inverse_scale_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ void decode_e4m3(uint2 codes, float scale, float (&x)[PER]) {
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) {
    const uint16_t two = (uint16_t)((i < 2 ? codes.x : codes.y) >> (16 * (i & 1)));
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(two));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    x[2 * i] = f.x * scale;
    x[2 * i + 1] = f.y * scale;
  }
}
__device__ __forceinline__ void decode_e5m2(uint2 codes, float scale, float (&x)[PER]) {      // a half whose low byte is zero
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) {
    const uint32_t h2 = prmt(i < 2 ? codes.x : codes.y, 0u, i & 1 ? 0x3424u : 0x1404u);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    x[2 * i] = f.x * scale;
    x[2 * i + 1] = f.y * scale;
  }
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
// The largest magnitude of eight values, NaN if one of them is.
__device__ __forceinline__ float most_of(const float (&x)[PER]) {
  float m = fabsf(x[0]);
#pragma unroll
  for (int i = 1; i < PER; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(x[i])));
  return m;
}
__device__ __forceinline__ uint32_t finite_most_of(const float (&x)[PER]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) most = max(most, finite(x[i]) ? __float_as_uint(x[i]) & 0x7FFFFFFFu : 0u);
  return most;
}
// The scale that puts a block's largest (its bits) at 1.75 * 2^top at most, the types' largest values.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most, int top) { return (uint32_t)min(max((int)((most + 0x1FFFFFu) >> 23) - top, 1), 254); }
template <bool CHECK>
__device__ __forceinline__ uint2 encode_e4m3(const float (&x)[PER], float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) {
    const float nan = __uint_as_float(0x7FFFFFFFu);
    const float lo = !CHECK || finite(x[2 * i]) ? x[2 * i] * inv : nan, hi = !CHECK || finite(x[2 * i + 1]) ? x[2 * i + 1] * inv : nan;
    uint16_t two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(hi), "f"(lo));
    w[i >> 1] |= (uint32_t)two << (16 * (i & 1));
  }
  return make_uint2(w[0], w[1]);
}
// random16: added below the two bits of the mantissa that stay
__device__ __forceinline__ uint32_t encode_e5m2(float x, float inv, uint32_t random16) {
  if (!finite(x)) return 0x7Fu;
  const float u = x * inv;      // 0 .. 57,344
  // below 2^-14 the codes are evenly spaced: adding 2^-14 brings them to the places of one binade
  const bool low = u < 6.103515625e-05f;
  const uint32_t bits = __float_as_uint(low ? __fadd_rn(u, 6.103515625e-05f) : u) + (random16 << 5);
  return max((bits >> 21) - (low ? 113u * 4u : 112u * 4u), min(__float_as_uint(u), 1u));      // a positive value is not rounded to zero
}
// Eight second moments of a block with scale byte `scale`.  Where all eight are ordinary (above 2^-14 of the scale, which is nearly always), the
// scale only moves the exponent: a code is the upper byte of bits * 8 + random * 256 - (112 + scale - 127) * 2^26, three instructions with its
// share of the packing instead of fifteen.
__device__ __forceinline__ uint2 encode_e5m2(const float (&v)[PER], uint32_t scale, const uint4& r) {
  const uint32_t words[4] = {r.x, r.y, r.z, r.w};
  uint32_t least = __float_as_uint(v[0]), most = least;
#pragma unroll
  for (int i = 1; i < PER; ++i) {
    least = min(least, __float_as_uint(v[i]));
    most = max(most, __float_as_uint(v[i]));
  }
  uint32_t w[2] = {0u, 0u};
  if (scale > 15u && least >= (scale - 14u) << 23 && most < 0x7F800000u) {
    const uint32_t minus = 0u - ((scale - 15u) << 2);      // in its lowest byte: what takes the exponent's excess away
    uint32_t y[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) y[i] = (__float_as_uint(v[i]) << 3) + (prmt(words[i >> 1], minus, i & 1 ? 0x4320u : 0x4100u) & 0xFFFFFF00u);
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = prmt(prmt(y[4 * i], y[4 * i + 1], 0x0073u), prmt(y[4 * i + 2], y[4 * i + 3], 0x0073u), 0x5410u);
  } else {
    const float inv = inverse_scale_of(scale);
#pragma unroll
    for (int i = 0; i < PER; ++i) w[i >> 2] |= encode_e5m2(v[i], inv, (words[i >> 1] >> (16 * (i & 1))) & 0xFFFFu) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}

// ---- one step
// What a thread loads of a piece, and where it goes.
template <typename P, typename G, int BITS> struct Loaded;
template <typename P, typename G> struct Loaded<P, G, 32> { Raw8<P> p; Raw8<G> g; Raw8<float> m, v; };
template <typename P, typename G> struct Loaded<P, G, 8> { Raw8<P> p; Raw8<G> g; uint2 m, v; uint32_t sm, sv; };

// A CTA takes PIECES pieces, all of whose loads come before the first one's work: one with moments in 32 bits, two with 8, whose loads are half the
// bytes.  us for 200 M elements (bf16 gradient and copy): 32 bits 830, more than the copy rate; 8 bits with one piece 570, two 546, two and
// registers for four CTAs on an SM 500, 98 % of the copy rate.  (Copies into a ring in shared memory two pieces ahead, by cp.async: 950 to 1,010.)
template <typename P, typename G, typename C, bool HAS_COPY, int BITS, int PIECES>
__global__ void __launch_bounds__(TPB, BITS == 8 ? 4 : 1) adamw_step(const DevTensor* __restrict__ tensors, const PieceRef* __restrict__ pieces, int n_pieces, Call call, const DevState* state) {
  pdl_enter();
  AdamScalars s = call.s;
  double lr = call.h.lr;
  uint32_t step = (uint32_t)call.step;
  if (state) {
    if (state->skip) return;
    s = state->s;
    lr = state->lr;
    step = (uint32_t)state->step;
  }
  PieceRef ref[PIECES];
  Loaded<P, G, BITS> x[PIECES];
#pragma unroll
  for (int k = 0; k < PIECES; ++k) ref[k] = (int)blockIdx.x * PIECES + k < n_pieces ? pieces[blockIdx.x * PIECES + k] : PieceRef{-1, 0};
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    if (PIECES > 1 && ref[k].tensor < 0) break;
    const DevTensor& t = tensors[ref[k].tensor];
    const int64_t i0 = (int64_t)ref[k].piece * PIECE + threadIdx.x * PER;
    const int n = (int)min((int64_t)PER, max((int64_t)0, t.n - i0));
    if (t.wide && n == PER) {
      load8(reinterpret_cast<const P*>(t.p) + i0, x[k].p);
      load8(reinterpret_cast<const G*>(t.g) + i0, x[k].g);
      if constexpr (BITS == 32) {
        load8(reinterpret_cast<const float*>(t.m) + i0, x[k].m);
        load8(reinterpret_cast<const float*>(t.v) + i0, x[k].v);
      } else {
        x[k].m = __ldcs(reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(t.m) + i0));
        x[k].v = __ldcs(reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(t.v) + i0));
      }
    } else {
      load_some(reinterpret_cast<const P*>(t.p), i0, n, x[k].p);
      load_some(reinterpret_cast<const G*>(t.g), i0, n, x[k].g);
      if constexpr (BITS == 32) {
        load_some(reinterpret_cast<const float*>(t.m), i0, n, x[k].m);
        load_some(reinterpret_cast<const float*>(t.v), i0, n, x[k].v);
      } else {
        const uint8_t *pm = reinterpret_cast<const uint8_t*>(t.m) + i0, *pv = reinterpret_cast<const uint8_t*>(t.v) + i0;
        x[k].m = x[k].v = make_uint2(0u, 0u);
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (i < n) {
            (i < 4 ? x[k].m.x : x[k].m.y) |= (uint32_t)pm[i] << (8 * (i & 3));
            (i < 4 ? x[k].v.x : x[k].v.y) |= (uint32_t)pv[i] << (8 * (i & 3));
          }
      }
    }
    if constexpr (BITS == 8) {
      const int64_t block = i0 / BLOCK8;
      const bool there = block * BLOCK8 < t.n;      // the same for a warp
      x[k].sm = there ? t.m_scale[block] : 0;
      x[k].sv = there ? t.v_scale[block] : 0;
    }
  }
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    if (PIECES > 1 && ref[k].tensor < 0) break;
    const DevTensor& t = tensors[ref[k].tensor];
    const int64_t i0 = (int64_t)ref[k].piece * PIECE + threadIdx.x * PER, block = i0 / BLOCK8;
    const int n = (int)min((int64_t)PER, max((int64_t)0, t.n - i0));
    if (BITS == 32 ? n == 0 : block * BLOCK8 >= t.n) continue;
    const bool vec = t.wide && n == PER;
    const float decay = adam_decay(lr, t.wd);
    float p[PER], g[PER], m[PER], v[PER];
    widen8(x[k].p, p);
    widen8(x[k].g, g);
    if constexpr (BITS == 32) {
      widen8(x[k].m, m);
      widen8(x[k].v, v);
    } else {
      decode_e4m3(x[k].m, scale_of(x[k].sm), m);
      decode_e5m2(x[k].v, scale_of(x[k].sv), v);
    }
#pragma unroll
    for (int i = 0; i < PER; i += 2) adam_update2(p[i], p[i + 1], __fmul_rn(g[i], s.factor), __fmul_rn(g[i + 1], s.factor), m[i], m[i + 1], v[i], v[i + 1], s, decay);
    if (vec) store8(reinterpret_cast<P*>(t.p) + i0, p);
    else store_some(reinterpret_cast<P*>(t.p), i0, n, p);
    if constexpr (HAS_COPY) {
      if (vec) store8(reinterpret_cast<C*>(t.copy) + i0, p);
      else store_some(reinterpret_cast<C*>(t.copy), i0, n, p);
    }
    if constexpr (BITS == 32) {
      if (vec) {
        store8(reinterpret_cast<float*>(t.m) + i0, m);
        store8(reinterpret_cast<float*>(t.v) + i0, v);
      } else {
        store_some(reinterpret_cast<float*>(t.m), i0, n, m);
        store_some(reinterpret_cast<float*>(t.v), i0, n, v);
      }
    } else {
      // lanes past the tensor's end hold zero moments: they had zero gradients and moments
      const uint64_t j = (uint64_t)(i0 / PER);
      const uint4 r = philox4x32_10(make_uint4((uint32_t)j, (uint32_t)(j >> 32), (uint32_t)ref[k].tensor, step),
                                    make_uint2((uint32_t)call.seed, (uint32_t)(call.seed >> 32)));
      uint32_t most_m = __reduce_max_sync(0xffffffffu, __float_as_uint(most_of(m))), most_v = __reduce_max_sync(0xffffffffu, __float_as_uint(most_of(v)));
      const bool all_finite = max(most_m, most_v) < 0x7F800000u;
      if (!all_finite) {
        most_m = __reduce_max_sync(0xffffffffu, finite_most_of(m));
        most_v = __reduce_max_sync(0xffffffffu, finite_most_of(v));
      }
      const uint32_t sm = scale_byte(most_m, 8), sv = scale_byte(most_v, 15);
      const float inv_m = inverse_scale_of(sm);
      const uint2 cm = all_finite ? encode_e4m3<false>(m, inv_m) : encode_e4m3<true>(m, inv_m), cv = encode_e5m2(v, sv, r);
      uint8_t *pm = reinterpret_cast<uint8_t*>(t.m) + i0, *pv = reinterpret_cast<uint8_t*>(t.v) + i0;
      if (vec) {
        *reinterpret_cast<uint2*>(pm) = cm;
        *reinterpret_cast<uint2*>(pv) = cv;
      } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (i < n) {
            pm[i] = (uint8_t)((i < 4 ? cm.x : cm.y) >> (8 * (i & 3)));
            pv[i] = (uint8_t)((i < 4 ? cv.x : cv.y) >> (8 * (i & 3)));
          }
      }
      if ((threadIdx.x & 31) == 0) {
        t.m_scale[block] = (uint8_t)sm;
        t.v_scale[block] = (uint8_t)sv;
      }
    }
  }
}

// What the device has to find out before the step: the norm, and the constants of a step that it counts itself.
__device__ void finish_state(double total, bool has_norm, const Call& call, DevState* st) {
  double factor = call.grad_scale;
  bool skip = false;
  if (has_norm) {
    const double norm = fabs(call.grad_scale) * sqrt(total);
    st->norm = (float)norm;
    skip = call.skip_nonfinite && !isfinite(norm);
    if (call.clip > 0.0) factor *= isnan(norm) ? norm : fmin(1.0, call.clip / norm);      // a zero gradient keeps its factor (clip / 0 = inf)
  }
  st->skip = skip ? 1 : 0;
  if (skip) { st->skipped += 1; return; }
  if (call.step == 0) st->counted += 1;
  st->step = call.step == 0 ? st->counted : call.step;
  AdamHyper h = call.h;
  if (call.lr_dev) h.lr = (double)*call.lr_dev;
  st->lr = h.lr;
  st->s = adam_scalars(h, st->step, factor);
}

// has_norm: of no gradients at all, zero
__global__ void adamw_begin(bool has_norm, Call call, DevState* st) {
  pdl_enter();
  finish_state(0.0, has_norm, call, st);
}

// The sum of all gradients' squares in fp64 (squares of fp32 values are exact in it), in an order that depends on the sizes alone; the CTA
// that finishes last adds the CTAs' sums in their order and makes the step's constants.
template <typename G>
__global__ void __launch_bounds__(TPB) adamw_norm(const DevTensor* __restrict__ tensors, const PieceRef* __restrict__ pieces, int64_t n_pieces, Call call,
                                                  double* partial, DevState* st) {
  __shared__ double warp_sum[TPB / 32];
  __shared__ bool last;
  pdl_enter();
  double acc[2] = {0.0, 0.0};
  for (int64_t c = blockIdx.x; c < n_pieces; c += gridDim.x) {
    const PieceRef ref = pieces[c];
    const DevTensor& t = tensors[ref.tensor];
    const int64_t i0 = (int64_t)ref.piece * PIECE + threadIdx.x * PER;
    const int n = (int)min((int64_t)PER, max((int64_t)0, t.n - i0));
    Raw8<G> x;
    if (t.wide_g && n == PER) load8(reinterpret_cast<const G*>(t.g) + i0, x);
    else load_some(reinterpret_cast<const G*>(t.g), i0, n, x);
    float g[PER];
    widen8(x, g);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i & 1] = fma((double)g[i], (double)g[i], acc[i & 1]);
  }
  auto cta_sum = [&](double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = x;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int w = 0; w < TPB / 32; ++w) r += warp_sum[w];
    return r;
  };
  const double mine = cta_sum(acc[0] + acc[1]);
  if (threadIdx.x == 0) {
    partial[blockIdx.x] = mine;
    __threadfence();
    last = atomicAdd(&st->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double x = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += TPB) x += __ldcg(partial + i);
  const double total = cta_sum(x);
  if (threadIdx.x == 0) {
    st->ticket = 0;
    finish_state(total, true, call, st);
  }
}

uint64_t align256(uint64_t v) { return (v + 255) / 256 * 256; }
size_t type_size(int32_t t) { return t == PS_TYPE_FP32 ? 4 : 2; }
bool known_type(int32_t t) { return t == PS_TYPE_FP32 || t == PS_TYPE_BF16 || t == PS_TYPE_FP16; }
// eight values of `size` bytes in one access (32, 16 or 8 bytes)
bool wide_ok(const void* p, size_t size) { return ((uintptr_t)p & (size * PER - 1)) == 0; }

}  // namespace

}  // namespace psk

struct ps_adamw {
  ps_adamw_config cfg;
  cudaStream_t st;
  int device = 0;
  bool copies = false;
  int64_t n_pieces = 0;
  std::vector<psk::DevTensor> host;
  psk::DevTensor* tensors;
  psk::PieceRef* pieces;
  double* partial;
  psk::DevState* state;
};

namespace psk {
namespace {

bool has_copies(const ps_adamw_tensor* t, int32_t n) {      // as the first tensor with anything in it
  for (int32_t i = 0; i < n; ++i)
    if (t[i].n > 0) return t[i].copy != nullptr;
  return false;
}

int32_t check(const ps_adamw_config* c, const ps_adamw_tensor* t, int32_t n, bool pointers, int64_t* pieces_out) {
  if (!c || !t) return fail(PS_ERR_BAD_ARG, "NULL argument");
  if (n < 1 || n > PS_ADAMW_MAX_TENSORS) return fail(PS_ERR_BAD_ARG, "n_tensors must be 1..%d", PS_ADAMW_MAX_TENSORS);
  if (!known_type(c->param_type) || !known_type(c->grad_type)) return fail(PS_ERR_BAD_ARG, "unknown param_type or grad_type");
  if (c->state_bits != 32 && c->state_bits != 8) return fail(PS_ERR_BAD_ARG, "state_bits must be 32 or 8");
  const bool copies = has_copies(t, n);
  if (copies && (c->param_type != PS_TYPE_FP32 || (c->copy_type != PS_TYPE_BF16 && c->copy_type != PS_TYPE_FP16)))
    return fail(PS_ERR_BAD_ARG, "copies are BF16 or FP16, of FP32 weights");
  int64_t pieces = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].n < 0 || t[i].n > MAX_ELEMENTS) return fail(PS_ERR_BAD_ARG, "tensor %d has %lld elements", i, (long long)t[i].n);
    if (!(t[i].weight_decay >= 0.0) || !std::isfinite(t[i].weight_decay)) return fail(PS_ERR_BAD_ARG, "weight_decay of tensor %d must be >= 0", i);
    pieces += (t[i].n + PIECE - 1) / PIECE;
    if (!pointers || t[i].n == 0) continue;
    if (!t[i].param || !t[i].grad || !t[i].m || !t[i].v) return fail(PS_ERR_BAD_ARG, "tensor %d lacks a buffer", i);
    if (c->state_bits == 8 && (!t[i].m_scale || !t[i].v_scale)) return fail(PS_ERR_BAD_ARG, "tensor %d lacks its scales", i);
    if ((t[i].copy != nullptr) != copies) return fail(PS_ERR_BAD_ARG, "either every tensor has a copy or none");
    const size_t state = c->state_bits == 32 ? 4 : 1;
    if ((uintptr_t)t[i].param % type_size(c->param_type) || (uintptr_t)t[i].grad % type_size(c->grad_type) || (uintptr_t)t[i].m % state ||
        (uintptr_t)t[i].v % state || (copies && (uintptr_t)t[i].copy % 2))
      return fail(PS_ERR_BAD_ARG, "a buffer of tensor %d is not aligned to its type", i);
  }
  if (pieces > 0x7FFFFFFFll) return fail(PS_ERR_BAD_ARG, "too many elements");
  *pieces_out = pieces;
  return PS_OK;
}

// Two pieces that write the same memory would race: a tensor given twice, moments that two tensors share.
int32_t check_written(const ps_adamw_config* c, const ps_adamw_tensor* t, int32_t n) {
  struct Range { uintptr_t first, end; int32_t tensor; };
  std::vector<Range> list;
  try {
    list.reserve((size_t)n * (c->state_bits == 8 ? 6 : 4));
  } catch (const std::exception&) {
    return fail(PS_ERR_BAD_ARG, "out of host memory");
  }
  const size_t state = c->state_bits == 32 ? 4 : 1;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    auto add = [&](const void* p, size_t bytes) { if (p) list.push_back(Range{(uintptr_t)p, (uintptr_t)p + bytes, i}); };
    const size_t count = (size_t)t[i].n, blocks = (count + BLOCK8 - 1) / BLOCK8;
    add(t[i].param, count * type_size(c->param_type));
    add(t[i].copy, count * 2);
    add(t[i].m, count * state);
    add(t[i].v, count * state);
    if (c->state_bits == 8) {
      add(t[i].m_scale, blocks);
      add(t[i].v_scale, blocks);
    }
  }
  std::sort(list.begin(), list.end(), [](const Range& a, const Range& b) { return a.first < b.first; });
  for (size_t i = 1; i < list.size(); ++i)
    if (list[i].first < list[i - 1].end) return fail(PS_ERR_BAD_ARG, "weights, copies or moments of tensors %d and %d share memory", list[i - 1].tensor, list[i].tensor);
  return PS_OK;
}

uint64_t arena_layout(ps_adamw* o, void* base, int32_t n, int64_t pieces) {
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t a = (uint64_t)base + at; at = align256(at + bytes); return a; };
  const uint64_t a = take(sizeof(DevTensor) * (uint64_t)n), b = take(sizeof(PieceRef) * (uint64_t)pieces), c = take(sizeof(double) * NORM_CTAS), d = take(sizeof(DevState));
  if (o) {
    o->tensors = (DevTensor*)a; o->pieces = (PieceRef*)b; o->partial = (double*)c; o->state = (DevState*)d;
  }
  return at;
}

void set_wide(const ps_adamw_config& c, DevTensor& t) {
  const size_t state = c.state_bits == 32 ? 4 : 1;
  t.wide_g = wide_ok(t.g, type_size(c.grad_type)) ? 1 : 0;
  t.wide = t.wide_g && wide_ok(t.p, type_size(c.param_type)) && wide_ok(t.m, state) && wide_ok(t.v, state) && (!t.copy || wide_ok(t.copy, 2));
}

int32_t upload_tensors(ps_adamw* o) {      // the copy's source is pageable: it has been read when the call returns
  const cudaError_t e = cudaMemcpyAsync(o->tensors, o->host.data(), o->host.size() * sizeof(DevTensor), cudaMemcpyHostToDevice, o->st);
  return e == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "table upload: %s", cudaGetErrorString(e));
}

int32_t check_device(const ps_adamw* o) {
  int device = -1;
  if (cudaGetDevice(&device) == cudaSuccess && device == o->device) return PS_OK;
  return fail(PS_ERR_BAD_ARG, "the optimizer lives on device %d, the current one is %d", o->device, device);
}

template <typename P, typename G, typename C, bool HAS_COPY>
void launch_step(const ps_adamw* o, const Call& call, const DevState* state) {
  const int n = (int)o->n_pieces;
  if (o->cfg.state_bits == 32) launch_pdl(adamw_step<P, G, C, HAS_COPY, 32, 1>, dim3((unsigned)n), TPB, 0, o->st, o->tensors, o->pieces, n, call, state);
  else launch_pdl(adamw_step<P, G, C, HAS_COPY, 8, 2>, dim3((unsigned)((n + 1) / 2)), TPB, 0, o->st, o->tensors, o->pieces, n, call, state);
}
template <typename P, typename G>
void launch_copy(const ps_adamw* o, const Call& call, const DevState* state) {
  if constexpr (std::is_same<P, float>::value) {
    if (o->copies && o->cfg.copy_type == PS_TYPE_BF16) return launch_step<P, G, __nv_bfloat16, true>(o, call, state);
    if (o->copies) return launch_step<P, G, __half, true>(o, call, state);
  }
  launch_step<P, G, float, false>(o, call, state);
}
template <typename P>
void launch_grad(const ps_adamw* o, const Call& call, const DevState* state) {
  if (o->cfg.grad_type == PS_TYPE_FP32) launch_copy<P, float>(o, call, state);
  else if (o->cfg.grad_type == PS_TYPE_BF16) launch_copy<P, __nv_bfloat16>(o, call, state);
  else launch_copy<P, __half>(o, call, state);
}
template <typename G>
void launch_norm(const ps_adamw* o, const Call& call) {
  launch_pdl(adamw_norm<G>, dim3((unsigned)std::min<int64_t>(o->n_pieces, NORM_CTAS)), TPB, 0, o->st, o->tensors, o->pieces, o->n_pieces, call, o->partial, o->state);
}

}  // namespace

int32_t check_adamw_hyper(const ps_adamw_hyper* h) {
  if (!h) return fail(PS_ERR_BAD_ARG, "hyper is NULL");
  if (!std::isfinite(h->lr)) return fail(PS_ERR_BAD_ARG, "lr must be finite");
  if (!(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0)) return fail(PS_ERR_BAD_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!((float)h->eps >= 1.17549435e-38f) || !std::isfinite((float)h->eps)) return fail(PS_ERR_BAD_ARG, "eps must be a normal positive fp32 value");
  if (!(h->clip_norm >= 0.0)) return fail(PS_ERR_BAD_ARG, "clip_norm must be >= 0");
  if (h->step < 0) return fail(PS_ERR_BAD_ARG, "step must be >= 0");
  return PS_OK;
}

}  // namespace psk

using namespace psk;

extern "C" {

int32_t ps_adamw_query_bytes(const ps_adamw_config* cfg, const ps_adamw_tensor* tensors, int32_t n_tensors, uint64_t* arena_bytes) {
  int64_t pieces = 0;
  int32_t rc = check(cfg, tensors, n_tensors, false, &pieces);
  if (rc != PS_OK) return rc;
  if (!arena_bytes) return fail(PS_ERR_BAD_ARG, "NULL argument");
  *arena_bytes = arena_layout(nullptr, nullptr, n_tensors, pieces);
  return PS_OK;
}

int32_t ps_adamw_create(const ps_adamw_config* cfg, const ps_adamw_tensor* tensors, int32_t n_tensors, ps_adamw** out) {
  int64_t n_pieces = 0;
  int32_t rc = check(cfg, tensors, n_tensors, true, &n_pieces);
  if (rc != PS_OK) return rc;
  if ((rc = check_written(cfg, tensors, n_tensors)) != PS_OK) return rc;
  if (!out) return fail(PS_ERR_BAD_ARG, "NULL argument");
  if (!cfg->arena || ((uint64_t)cfg->arena & 255) != 0) return fail(PS_ERR_BAD_ARG, "arena must be a 256-byte aligned device pointer");
  const uint64_t need = arena_layout(nullptr, nullptr, n_tensors, n_pieces);
  if (cfg->arena_bytes < need) return fail(PS_ERR_ARENA_TOO_SMALL, "arena has %llu bytes, %llu needed", (unsigned long long)cfg->arena_bytes, (unsigned long long)need);
  ps_adamw* o = nullptr;
  std::vector<PieceRef> pieces;
  try {
    o = new ps_adamw();
    o->host.resize((size_t)n_tensors);
    pieces.reserve((size_t)n_pieces);
  } catch (const std::exception&) {
    delete o;
    return fail(PS_ERR_BAD_ARG, "out of host memory");
  }
  o->cfg = *cfg;
  o->st = (cudaStream_t)cfg->stream;
  o->copies = has_copies(tensors, n_tensors);
  o->n_pieces = n_pieces;
  arena_layout(o, cfg->arena, n_tensors, n_pieces);
  for (int32_t i = 0; i < n_tensors; ++i) {
    const ps_adamw_tensor& t = tensors[i];
    DevTensor& d = o->host[(size_t)i];
    d.p = t.param; d.g = t.grad; d.copy = t.copy; d.m = t.m; d.v = t.v; d.m_scale = t.m_scale; d.v_scale = t.v_scale;
    d.n = t.n; d.wd = t.weight_decay;
    set_wide(o->cfg, d);
    for (int64_t c = 0; c * PIECE < t.n; ++c) pieces.push_back(PieceRef{i, (int32_t)c});
  }
  cudaError_t e = cudaGetDevice(&o->device);
  rc = PS_OK;
  if (e == cudaSuccess) rc = upload_tensors(o);
  if (rc == PS_OK && e == cudaSuccess && n_pieces) e = cudaMemcpyAsync(o->pieces, pieces.data(), pieces.size() * sizeof(PieceRef), cudaMemcpyHostToDevice, o->st);
  if (rc == PS_OK && e == cudaSuccess) e = cudaMemsetAsync(o->state, 0, sizeof(DevState), o->st);
  if (rc == PS_OK && e == cudaSuccess) e = cudaStreamSynchronize(o->st);
  if (rc != PS_OK || e != cudaSuccess) {
    delete o;
    return rc != PS_OK ? rc : fail(PS_ERR_CUDA, "ps_adamw_create: %s", cudaGetErrorString(e));
  }
  *out = o;
  return PS_OK;
}

int32_t ps_adamw_destroy(ps_adamw* o) {
  if (!o) return fail(PS_ERR_BAD_ARG, "optimizer is NULL");
  const cudaError_t e = cudaStreamSynchronize(o->st);
  delete o;
  return e == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "ps_adamw_destroy: %s", cudaGetErrorString(e));
}

int32_t ps_adamw_set_grads(ps_adamw* o, const void* const* grads) {
  if (!o || !grads) return fail(PS_ERR_BAD_ARG, "NULL argument");
  const size_t size = type_size(o->cfg.grad_type);
  for (size_t i = 0; i < o->host.size(); ++i)
    if (o->host[i].n > 0 && (!grads[i] || (uintptr_t)grads[i] % size)) return fail(PS_ERR_BAD_ARG, "gradient %zu is NULL or not aligned to its type", i);
  int32_t rc = check_device(o);
  if (rc != PS_OK) return rc;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(o->st, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone)
    return fail(PS_ERR_BAD_ARG, "ps_adamw_set_grads is not to be captured into a graph");
  std::vector<DevTensor> now;
  try {
    now = o->host;
  } catch (const std::exception&) {
    return fail(PS_ERR_BAD_ARG, "out of host memory");
  }
  for (size_t i = 0; i < now.size(); ++i) {
    now[i].g = grads[i];
    set_wide(o->cfg, now[i]);
  }
  now.swap(o->host);
  rc = upload_tensors(o);
  if (rc != PS_OK) now.swap(o->host);
  return rc;
}

int32_t ps_adamw_step(ps_adamw* o, const ps_adamw_hyper* h) {
  if (!o) return fail(PS_ERR_BAD_ARG, "optimizer is NULL");
  int32_t rc = check_adamw_hyper(h);
  if (rc != PS_OK) return rc;
  if (!std::isfinite(h->grad_scale)) return fail(PS_ERR_BAD_ARG, "grad_scale must be finite");
  if ((rc = check_device(o)) != PS_OK) return rc;
  Call c;
  c.h = AdamHyper{h->lr, h->beta1, h->beta2, h->eps};
  c.grad_scale = h->grad_scale; c.clip = h->clip_norm; c.lr_dev = h->lr_dev; c.step = h->step; c.seed = h->seed;
  c.skip_nonfinite = h->skip_nonfinite;
  const bool norm = h->clip_norm > 0.0 || h->skip_nonfinite, on_device = norm || h->step == 0 || h->lr_dev;
  c.s = on_device ? AdamScalars{} : adam_scalars(c.h, h->step, h->grad_scale);
  if (norm && o->n_pieces) {
    if (o->cfg.grad_type == PS_TYPE_FP32) launch_norm<float>(o, c);
    else if (o->cfg.grad_type == PS_TYPE_BF16) launch_norm<__nv_bfloat16>(o, c);
    else launch_norm<__half>(o, c);
  } else if (on_device) {
    launch_pdl(adamw_begin, dim3(1), 1, 0, o->st, norm, c, o->state);
  }
  const DevState* state = on_device ? o->state : nullptr;
  if (o->n_pieces) {      // the steps of a list without elements are counted, and that is all
    if (o->cfg.param_type == PS_TYPE_FP32) launch_grad<float>(o, c, state);
    else if (o->cfg.param_type == PS_TYPE_BF16) launch_grad<__nv_bfloat16>(o, c, state);
    else launch_grad<__half>(o, c, state);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "adamw launch: %s", cudaGetErrorString(e));
}

int32_t ps_adamw_read_info(ps_adamw* o, ps_adamw_info* out) {
  if (!o || !out) return fail(PS_ERR_BAD_ARG, "NULL argument");
  DevState s;
  cudaError_t e = cudaMemcpyAsync(&s, o->state, sizeof(s), cudaMemcpyDeviceToHost, o->st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(o->st);
  if (e != cudaSuccess) return fail(PS_ERR_CUDA, "ps_adamw_read_info: %s", cudaGetErrorString(e));
  out->counted_steps = s.counted;
  out->skipped_steps = s.skipped;
  out->grad_norm = s.norm;
  out->grad_factor = s.s.factor;
  return PS_OK;
}

}  // extern "C"
