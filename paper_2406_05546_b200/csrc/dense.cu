// The dense layer of W workers with ragged mini-batches (workers_dense_forward / workers_dense_backward in include/ps.h), on the
// fifth-generation tensor cores: BF16 or FP16 operands, FP32 accumulation.
//   forward          pre[m][n] = sum_k x[m][k] W[n][k] + b[n] ;  y = act(pre) + r         (rows m of the workers that hold W)
//   input gradient   dx[m][k]  = sum_n dy[m][n] W[n][k] + dx_add ;  dx_pre = dx * act'(x_pre)
//   weight gradient  dW[n][k]  = sum_m dy[m][n] x[m][k]                                   (m = the rows of one worker)
// Every operand is read as it lies, with k contiguous or its row index contiguous (128-byte swizzle, blocks of 64), and every result is
// rounded once, in the epilogue that also does everything elementwise.
//
// Tiles, by the work there is (the rules are in plan_rows and plan_weights):
//   Pair   256 x 256 by two CTAs that share each MMA (cta_group::2): half of the right operand each, so that a CTA brings in 32 KB for
//          128 x 256 x 64 products.  Two accumulators of 256 columns are used in turn: one is read out while the other fills.
//   Single 128 x 256 by one CTA: workers with less than 256 rows.
//   Thin   128 x 128, two CTAs on an SM, for reductions so short that writing bounds them.
//   Split  128 x 128, the blocks of k dealt out over a cluster of CTAs whose partial tiles are added through distributed shared memory
//          in a fixed order: few tiles.
//   Few    weights as the left operand, 128 of their rows x 16, 32 or 64 rows of a worker, split likewise: bound by reading the weights.
// Pair, Single and Thin run as many CTAs (pairs) as the SMs hold, which walk over the tiles; the others one cluster per tile.
//
// What bounds it, by size (us a call, cold; in brackets the library's product alone, without anything elementwise):
//   16,384 x 4096 x 4096, BF16   the tensor pipe (80 % of its cycles; weight gradient 72 %): forward 338 (317), in FP32 392, input gradient 343 (320),
//                                weight gradient 376 (332), in FP32 412, added to what is there 423; with GELU's derivative, a matrix added and
//                                two results the input gradient 410, which moves 670 MB
//   16,384 x 1568 -> 512         128 tiles on 74 pairs of SMs, two waves, and 7,700 of 52,000 clocks before the first operands: 36 (17 at the copy rate)
//   41 rows on 16 of 4096 x 4096 reading the weights: 404 MB, 74, 5.4 TB/s
//   8,192 x 200 -> 4999          the epilogue, two bytes a lane: with everything on 120 (38 at the copy rate), backward 159
//   1 row, 1568 -> 512           the host's call, 5 to 7
//
// Precision: the accumulators drop low bits with every instruction (16 products), of each of its terms and always towards zero: of products of both signs
// (n - 1) / 2 times 1.3e-8 to 1.6e-8 after n instructions (bf16x3.cuh), of products of one sign 1.7e-7 to 2.0e-7.  So the sums over a bounded number of
// values of k are handed to registers and added there, rounded: over 512 for results in FP32 (2.6e-6 is lost at most, whatever the length), over
// 8,192 in FP16 and 65,536 in BF16 (5.2e-5 and 4e-4: a fifth of what their own rounding takes at least, 2^-12 and 2^-9).
//
// Ragged reductions (weight gradient): a tile's last block of 64 rows may reach into the next worker's.  Those rows are zeroed in shared
// memory, in both operands (a NaN times zero would stay), before the MMA reads them.
//
// Every wait on an mbarrier is bounded; a CTA that gives up counts itself in a word that workers_dense_status reads.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <mutex>
#include <type_traits>

#include "device_common.cuh"
#include "error.h"
#include "kernels.h"
#include "ps.h"
#include "tc5_common.cuh"

namespace psk {

namespace {

namespace cg = cooperative_groups;

enum { D_FWD = 0, D_DX = 1, D_DW = 2 };
constexpr int BM = 128, BK = 64;
// Reductions up to this length are bound by what they write: Thin tiles.  us, Pair or Single -> Thin: forward, 8,192 rows -> 4096 with residual and GELU, K =
// 64 53 -> 44, 256 57 -> 52, 384 61 -> 57, 512 65 -> 64, 768 72 -> 76; weight gradient, 16 workers of 1568 x 512 in FP32, 64 rows each 16.6 -> 13.2,
// 300 20.6 -> 19.5, 500 24.7 -> 26.3, 8 workers of 2048 x 2048, 300 rows 30 -> 33;
// a few larger workers among small ones (16 workers, 290 rows the most of 1,024: 23.6 -> 21.5, 480 of 930: 25.6 -> 23.6; 600 of 1,340: no gain; half with
// 400, half with 100: 27.7 -> 31.7).  Results of 16 bits, half the writing, and wider ones gain less or nothing: 64 workers of 512 x 1568, 200 rows each, FP32
// 72 -> 70, BF16 49 -> 53; 16 of 2048 x 2048, 64 rows each, 66 -> 70 and 35 -> 37.  The input gradient, which reads two matrices more, has not the
// registers for it (64 -> 117).
constexpr int THIN_RED_FWD = 384, THIN_RED_DW = 256, THIN_MOST_DW = 512, THIN_MEAN_DW = 128;
constexpr int DRAIN_FP32 = 8, DRAIN_FP16 = 128, DRAIN_BF16 = 1024;      // blocks of k whose sums share an accumulator, by the result's type
constexpr int SMEM_MOST = 227 * 1024, BARRIER_BYTES = 256;

template <int OP_, int CTAS_, int BN_, int STAGES_, bool SPLIT_, bool FEW_, bool DRAIN_, int PER_SM_ = 1> struct DenseShape {
  static constexpr int OP = OP_, CTAS = CTAS_, BN = BN_, STAGES = STAGES_, TM = BM * CTAS;
  // DRAIN: the sums of a bounded part of the reduction go to registers, 128 a lane (64 for Split, which has 128 columns).  With what the epilogue reads ahead
  // that is more than there is: 90 bytes (weight gradient) to 330 (forward, input gradient) of a thread spill.  us, 16,384 x 4096 x 4096, 16-bit result with
  // one accumulator -> FP32: forward 338 -> 392, weight gradient 376 -> 412.
  static constexpr bool SPLIT = SPLIT_, FEW = FEW_, DRAIN = DRAIN_;
  static constexpr int PER_SM = PER_SM_;      // CTAs that an SM holds
  static constexpr bool A_MN = FEW ? OP == D_DX : OP == D_DW, B_MN = !FEW && OP != D_FWD;      // is the operand's row index contiguous?
  static constexpr int B_ROWS = BN / CTAS;
  static constexpr int A_BYTES = BM * BK * 2, B_BYTES = B_ROWS * BK * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int BUFS = SPLIT ? 1 : 2, ACC = BN < 32 ? 32 : BN;
  static constexpr int EPI_WARPS = FEW ? 4 : 8, THREADS = 64 + 32 * EPI_WARPS, COLS = BN / (EPI_WARPS / 4);
  // May pieces of rows change lanes?  Not where there are no registers left for it: the sums of a drained accumulator (weight gradient in FP32, 16,384 x
  // 4096 x 4096 457 -> 641 us), two CTAs on an SM (forward, 8,192 x 64 -> 4096 with everything on 64 -> 91).
  static constexpr bool TURN = !DRAIN && PER_SM == 1;
  static constexpr int OUT_BYTES = SPLIT ? 0 : EPI_WARPS * 4096;      // a 32 x 32 block per warp on its way to whole rows
  static constexpr int SMEM = 1024 + STAGES * STAGE + OUT_BYTES + BARRIER_BYTES;
  static constexpr int PART_PITCH = FEW ? BM + 4 : BN + 4, PART_BYTES = (FEW ? BN : BM) * PART_PITCH * 4;
  static_assert(SMEM <= SMEM_MOST && STAGE % 1024 == 0 && ACC * BUFS <= 512, "tile shape");
  static_assert(!SPLIT || PART_BYTES <= STAGES * STAGE, "the partial tile takes the operands' place");
  static_assert(!SPLIT || CTAS == 1, "a pair's tile is not split");
};
template <int OP, bool DRAIN> using Pair = DenseShape<OP, 2, 256, 6, false, false, DRAIN>;
template <int OP, bool DRAIN> using Single = DenseShape<OP, 1, 256, 4, false, false, DRAIN>;
template <int OP> using Thin = DenseShape<OP, 1, 128, 2, false, false, false, 2>;
static_assert(THIN_RED_FWD <= DRAIN_FP32 * BK && THIN_MOST_DW <= DRAIN_FP32 * BK, "Thin tiles do not drain their accumulators");
template <int OP> using Split = DenseShape<OP, 1, 128, 6, true, false, true>;
template <int OP, int BN> using Few = DenseShape<OP, 1, BN, BN == 64 ? 4 : 5, true, true, true>;

// Forward and input gradient: groups of rows [row0[g], row1[g]), those with the same weights next to each other (a run), cut into blocks of rows;
// blk0: prefix sums of their blocks.  Weight gradient: the workers' rows.
struct DenseTab {
  int32_t groups, runs;
  int32_t row0[PS_MAX_WORKERS], row1[PS_MAX_WORKERS], blk0[PS_MAX_WORKERS + 1];
  int32_t run_blk0[PS_MAX_WORKERS + 1], run_pair0[PS_MAX_WORKERS + 1];      // a run's first block, and first pair of blocks
  uint16_t w[PS_MAX_WORKERS], run_w[PS_MAX_WORKERS];
};

// What the epilogue adds and where it writes (pitches in elements).  forward: in0 bias, in1 residual, out0 y, out1 pre; input gradient: in1
// dx_add, in2 x_pre, out0 dx, out1 dx_pre; weight gradient: out0 dW.
struct DenseEpi {
  const void *in0, *in1, *in2;
  void *out0, *out1;
  int64_t in0_stride, in1_pitch, in2_pitch, out0_pitch, out0_stride, out1_pitch;
  int32_t act, bf16, out0_fp32, accumulate;
  int32_t pairs, quads, rows, wide;      // may two values, four, 16 bytes, 32 bytes be moved at once, in every matrix there is?
};

// The kernels of one backward call read nothing of one another's.  The first enters as every kernel does (pdl_enter); the others need not wait for it,
// whose entry says that all work before the call is done: they start when it has started, and wait for the one before them where they
// have brought in all they will, so that what follows the call, which waits for its last kernel only, finds all of them done.  A kernel starts only when every
// CTA of the one before it has its SM, shared memory and tensor memory: none waits for a CTA that has no place.
// us a call in a row, db, dx and dw one after another -> so: 16 ragged workers of 1,024 rows 1568 -> 512 33.5 -> 27, 4,096 x 1024 x 1024 43 -> 36, x 2048 x
// 2048 75 -> 66, 16,384 x 4096 x 4096 970 -> 965.
enum { JOIN_FIRST = 0, JOIN_BETWEEN = 1, JOIN_LAST = 2 };

struct DenseArgs {
  int32_t n_tiles, m_tiles, n_side, n_tiles_n;      // tiles; along the left side; length and tiles of the right side (Few: of the left)
  int32_t m_side;                                   // weight gradient: length of the left side
  int32_t red;                                      // reduction length (weight gradient: the group's rows)
  int32_t rows;                                     // of all groups
  int32_t chunk;                                    // blocks of k per accumulator
  uint32_t idesc;
  int32_t join;                                     // JOIN_*
  int64_t limit;                                    // clocks that a wait may last
};

// CTAs whose wait gave up, on this device: these entry points have no context to keep it in.  It is never written by a reader, so that none takes a
// failure away from another, or loses one that comes while it reads.
__device__ uint32_t g_dense_failures;

__global__ void __launch_bounds__(32) dense_wait_probe(long long limit) {
  __shared__ uint64_t never;
  if (threadIdx.x == 0) {
    mbar_init(&never, 1);      // one arrival expected; nobody ever arrives
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  const bool ok = __all_sync(0xffffffffu, mbar_wait(&never, 0, limit));
  if (!ok && threadIdx.x == 0) atomicAdd(&g_dense_failures, 1u);
}

struct DenseMaps { CUtensorMap a, b; };

// ---- element types -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float widen(uint32_t half_word, int bf16) {
  return bf16 ? __uint_as_float(half_word << 16) : __half2float(__ushort_as_half((unsigned short)half_word));
}
__device__ __forceinline__ uint32_t narrow2(float lo, float hi, int bf16) {
  if (bf16) return bf16_pair(lo, hi);
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// ---- elementwise, two values at a time ---------------------------------------------------------------------------------------
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// The normal distribution function of two values, and e = exp(-z^2 / 2), which it shares with the density.  Its tail at |z| is e t P(t) with
// t = 1 / (1 + 0.3046 |z|), the form of Abramowitz and Stegun 7.1.26, but with a P of degree 7, fitted here for the least largest relative error over 0 .. 14
// (9.0e-8, by reweighted least squares; 7.1.26 keeps erf to 1.5e-7 of its largest value, which is nothing of a tail).  In fp32 the tail is off by
// 2^-20 + z^2 2^-23 of itself at most, the rest from the exponent's roundings.  NaN stays.
// GELU's error in fp32, of z in -4 .. -3, -1 .. 0 and 1 .. 2: 2.3e-9, 0.7e-7 and 1.3e-7 at most (with 7.1.26 and the tail taken from 1/2: 2.6e-7,
// 1.1e-7 and 2.8e-7; z (1 + erf) / 2 in fp32: 0.6e-7, 0.3e-7 and 1.6e-7).  us with the published polynomial of degree 4 -> so: forward with everything on,
// 11,776 x 2048 -> 5000 206 -> 210, 16,384 x 4096 -> 4096 376 -> 380, 8,192 x 200 -> 5000 112 -> 116; input gradient 16,384 x 4096 x 4096 407 -> 410.
__device__ __forceinline__ u64 normal_cdf2(u64 z, u64& e) {
  float z0, z1, a0, a1, b0, b1;
  unpack2(z, z0, z1);
  const u64 t = pack2(reciprocal_fast(fmaf(0.3046f, fabsf(z0), 1.f)), reciprocal_fast(fmaf(0.3046f, fabsf(z1), 1.f)));
  unpack2(mul2(mul2(z, z), both(-0.72134752f)), a0, a1);      // -log2(e) / 2
  e = pack2(exp2_fast(a0), exp2_fast(a1));
  u64 q = ffma2(t, both(0.036764886f), both(-0.15391697f));
  q = ffma2(t, q, both(0.1883008f));
  q = ffma2(t, q, both(-0.040023267f));
  q = ffma2(t, q, both(0.12202316f));
  q = ffma2(t, q, both(0.103026144f));
  q = ffma2(t, q, both(0.12234751f));
  q = ffma2(t, q, both(0.12147778f));
  const u64 tail = mul2(mul2(q, t), e);
  unpack2(tail, a0, a1);
  unpack2(ffma2(tail, both(-1.f), both(1.f)), b0, b1);
  return pack2(z0 < 0.f ? a0 : b0, z1 < 0.f ? a1 : b1);
}
__device__ __forceinline__ u64 logistic2(u64 z) {
  float a0, a1;
  unpack2(mul2(z, both(-1.44269504f)), a0, a1);
  unpack2(add2(pack2(exp2_fast(a0), exp2_fast(a1)), both(1.f)), a0, a1);
  return pack2(reciprocal_fast(a0), reciprocal_fast(a1));
}
template <int ACT>
__device__ __forceinline__ u64 activate2(u64 z) {
  if (ACT == PS_ACT_RELU) {      // NaN stays
    float z0, z1;
    unpack2(z, z0, z1);
    return pack2(z0 < 0.f ? 0.f : z0, z1 < 0.f ? 0.f : z1);
  }
  if (ACT == PS_ACT_GELU) {
    u64 e;
    const u64 c = normal_cdf2(z, e);
    return mul2(z, c);
  }
  return mul2(z, logistic2(z));      // SiLU
}
// d * act'(z)
template <int ACT>
__device__ __forceinline__ u64 through2(u64 d, u64 z) {
  if (ACT == PS_ACT_RELU) {
    float z0, z1, d0, d1;
    unpack2(z, z0, z1);
    unpack2(d, d0, d1);
    return pack2(z0 > 0.f ? d0 : 0.f, z1 > 0.f ? d1 : 0.f);
  }
  if (ACT == PS_ACT_GELU) {
    u64 e;
    const u64 c = normal_cdf2(z, e);
    return mul2(d, ffma2(mul2(z, both(0.39894228f)), e, c));
  }
  const u64 q = logistic2(z);
  return mul2(mul2(d, q), ffma2(z, ffma2(q, both(-1.f), both(1.f)), both(1.f)));
}
// f(activation as a constant)
template <typename F> __device__ __forceinline__ void with_activation(int act, F f) {
  if (act == PS_ACT_RELU) f(std::integral_constant<int, PS_ACT_RELU>());
  else if (act == PS_ACT_GELU) f(std::integral_constant<int, PS_ACT_GELU>());
  else if (act == PS_ACT_SILU) f(std::integral_constant<int, PS_ACT_SILU>());
}

// f(whether the operands are BF16, as a constant): asked once for a chunk of a tile
template <typename F> __device__ __forceinline__ void with_type(int bf16, F f) {
  if (bf16) f(std::true_type());
  else f(std::false_type());
}
template <bool BF16> __device__ __forceinline__ u64 widen2(uint32_t w) {
  if (BF16) return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return pack2(f.x, f.y);
}
template <bool BF16> __device__ __forceinline__ uint32_t narrow_pair(u64 v) {
  float a, b;
  unpack2(v, a, b);
  return narrow2(a, b, BF16);
}

// 32 bytes of a lane in one access, first out of L2 again: what the epilogue moves is not needed there, what the products read is (8,192 x 2048 -> 5120
// with everything on 154 -> 141 us).
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.L1::no_allocate.L2::evict_first.L2::256B.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void store_words(void* p, const uint32_t* w) {
  asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// ---- the elementwise part of a tile ------------------------------------------------------------------------------------------
// which: the weight matrix (forward) or the worker (weight gradient).
template <int OP> __device__ __forceinline__ int64_t out0_at(const DenseEpi& e, int64_t row, int col, int which) {
  return (OP == D_DW ? (int64_t)which * e.out0_stride : 0) + row * e.out0_pitch + col;
}

// Rows: a lane has 32 consecutive columns of a row of its own.  Where 32 bytes can be moved at once it loads and stores them straight from and to
// global memory.  Where only 16 can, a lane alone would write half sectors, and the rest of each in another access: there four lanes
// move 64 consecutive bytes of a row, and pieces of 16 bytes change lanes in shared memory (11,776 x 2048 -> 5000 with everything on 284 -> 236 us).
// What is read is loaded a chunk ahead.
template <int OP> struct RowIn { uint32_t a[OP == D_DW ? 1 : 16], b[OP == D_DX ? 16 : 1]; };
// TURN: may pieces change lanes?  Then every lane of the warp comes along, and the existence of its rows is asked where they are moved; if not, only
// lanes with a row come at all.
template <bool TURN> struct RowPlace {
  int row0, end, lane;      // the warp's first row; the rows' end
  uint8_t* turn;            // 2 KB of shared memory
  __device__ __forceinline__ int row() const { return row0 + lane; }
  __device__ __forceinline__ int piece_row(int i) const { return row0 + 8 * i + (lane >> 2); }      // of a lane's piece i, where four lanes share a row
};
__device__ __forceinline__ uint4* turn_at(const RowPlace<true>& p, int row, int piece) {      // without conflicts, by rows and by pieces
  return reinterpret_cast<uint4*>(p.turn + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4));
}
// 64 bytes of a row per lane -> pieces, and back
__device__ __forceinline__ void to_pieces(const RowPlace<true>& p, uint32_t* w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *turn_at(p, p.lane, i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *turn_at(p, 8 * i + (p.lane >> 2), p.lane & 3);
    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
  }
  __syncwarp();
}
__device__ __forceinline__ void to_rows(const RowPlace<true>& p, uint32_t* w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *turn_at(p, 8 * i + (p.lane >> 2), p.lane & 3) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *turn_at(p, p.lane, i);
    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
  }
  __syncwarp();
}
template <bool TURN> __device__ __forceinline__ void loaded(const RowPlace<TURN>& p, int wide, uint32_t* w) {
  if constexpr (TURN)
    if (!wide) to_rows(p, w);
}
// 64 bytes of each row from `base` on, pitch in bytes; as pieces where not wide.
template <bool TURN>
__device__ __forceinline__ void load_row(const void* base, int64_t pitch, const RowPlace<TURN>& p, int wide, uint32_t (&w)[16]) {
  const uint8_t* b = reinterpret_cast<const uint8_t*>(base);
  if (wide) {
    if (!TURN || p.row() < p.end) {
      load_words(b + p.row() * pitch, *reinterpret_cast<uint32_t (*)[8]>(&w[0]));
      load_words(b + p.row() * pitch + 32, *reinterpret_cast<uint32_t (*)[8]>(&w[8]));
    }
  } else if (!TURN) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(b + p.row() * pitch + 16 * i);
      w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p.piece_row(i) < p.end) {
        const uint4 v = *reinterpret_cast<const uint4*>(b + p.piece_row(i) * pitch + 16 * (p.lane & 3));
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
  }
}
template <bool TURN>
__device__ __forceinline__ void store_row(void* base, int64_t pitch, const RowPlace<TURN>& p, int wide, uint32_t* w) {
  uint8_t* b = reinterpret_cast<uint8_t*>(base);
  if (wide) {
    if (!TURN || p.row() < p.end) {
      store_words(b + p.row() * pitch, w);
      store_words(b + p.row() * pitch + 32, w + 8);
    }
  } else if constexpr (!TURN) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(b + p.row() * pitch + 16 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
    to_pieces(p, w);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p.piece_row(i) < p.end) *reinterpret_cast<uint4*>(b + p.piece_row(i) * pitch + 16 * (p.lane & 3)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}
template <bool BF16, bool TURN>
__device__ __forceinline__ void store_row16(void* base, int64_t pitch, const RowPlace<TURN>& p, int col, int wide, const u64 (&v)[16]) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = narrow_pair<BF16>(v[i]);
  store_row(reinterpret_cast<uint16_t*>(base) + col, 2 * pitch, p, wide, w);
}
// add: to what is there
template <bool TURN>
__device__ __forceinline__ void store_row32(void* base, int64_t pitch, const RowPlace<TURN>& p, int col, int wide, int add, u64 (&v)[16]) {
  float* at = reinterpret_cast<float*>(base) + col;
  if (add) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t o[16];
      load_row(at + 16 * h, 4 * pitch, p, wide, o);
      loaded(p, wide, o);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[8 * h + i] = add2(v[8 * h + i], pack2(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1])));
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[2 * i] = (uint32_t)v[8 * h + i];
      w[2 * i + 1] = (uint32_t)(v[8 * h + i] >> 32);
    }
    store_row(at + 16 * h, 4 * pitch, p, wide, w);
  }
}
template <int OP, bool TURN>
__device__ __forceinline__ void row_ahead(const DenseEpi& e, const RowPlace<TURN>& p, int col, RowIn<OP>& x) {
  if constexpr (OP != D_DW) {
    if (e.in1) load_row(reinterpret_cast<const uint16_t*>(e.in1) + col, 2 * e.in1_pitch, p, e.wide, x.a);
    if constexpr (OP == D_DX)
      if (e.out1) load_row(reinterpret_cast<const uint16_t*>(e.in2) + col, 2 * e.in2_pitch, p, e.wide, x.b);
  }
}
// bias: 32 floats in shared memory
template <int OP, bool BF16, bool TURN>
__device__ __forceinline__ void finish_row_of(const DenseEpi& e, const RowPlace<TURN>& p, int col, int which, const float* bias, RowIn<OP>& x, u64 (&v)[16]) {
  if constexpr (OP == D_FWD) {
    if (e.in0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 b = reinterpret_cast<const float4*>(bias)[i];
        v[2 * i] = add2(v[2 * i], pack2(b.x, b.y));
        v[2 * i + 1] = add2(v[2 * i + 1], pack2(b.z, b.w));
      }
    }
    if (e.out1) store_row16<BF16>(e.out1, e.out1_pitch, p, col, e.wide, v);
    with_activation(e.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = activate2<decltype(act)::value>(v[i]);
    });
  }
  if constexpr (OP != D_DW) {
    if (e.in1) {
      loaded(p, e.wide, x.a);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = add2(v[i], widen2<BF16>(x.a[i]));
    }
  }
  if constexpr (OP == D_FWD) {
    if (e.out0_fp32) store_row32(e.out0, e.out0_pitch, p, col, e.wide, 0, v);
    else store_row16<BF16>(e.out0, e.out0_pitch, p, col, e.wide, v);
  } else if constexpr (OP == D_DX) {
    if (e.out0) store_row16<BF16>(e.out0, e.out0_pitch, p, col, e.wide, v);
    if (e.out1) {
      loaded(p, e.wide, x.b);
      with_activation(e.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = through2<decltype(act)::value>(v[i], widen2<BF16>(x.b[i]));
      });
      store_row16<BF16>(e.out1, e.out1_pitch, p, col, e.wide, v);
    }
  } else {
    const int64_t first = (int64_t)which * e.out0_stride;
    if (e.out0_fp32) {
      float* out = reinterpret_cast<float*>(e.out0) + first;
      store_row32(out, e.out0_pitch, p, col, e.wide, e.accumulate, v);
    } else {
      uint16_t* out = reinterpret_cast<uint16_t*>(e.out0) + first;
      if (e.accumulate) {
        uint32_t o[16];
        load_row(out + col, 2 * e.out0_pitch, p, e.wide, o);
        loaded(p, e.wide, o);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = add2(v[i], widen2<BF16>(o[i]));
      }
      store_row16<BF16>(out, e.out0_pitch, p, col, e.wide, v);
    }
  }
}

template <int OP, bool TURN>
__device__ __forceinline__ void finish_row(const DenseEpi& e, const RowPlace<TURN>& p, int col, int which, const float* bias, RowIn<OP>& x, u64 (&v)[16]) {
  with_type(e.bf16, [&](auto bf16) { finish_row_of<OP, decltype(bf16)::value, TURN>(e, p, col, which, bias, x, v); });
}

// Columns, for matrices of any alignment and at their right edge: a lane has W = 1, 2 or 4 consecutive columns of R rows, row0 + i * step, of which
// those below `end` exist.  Its values are in pairs, of columns (W > 1) or of rows.
// Value h (0 or 1) of pair p: its row and its column.
template <int W> __host__ __device__ constexpr int pair_row(int p, int h) { return W == 1 ? 2 * p + h : 2 * p / W; }
template <int W> __host__ __device__ constexpr int pair_col(int p, int h) { return W == 1 ? 0 : 2 * p % W + h; }
template <int W> __device__ __forceinline__ void load_few(const void* base, int64_t i, uint32_t (&w)[(W + 1) / 2]) {      // W values of 16 bits
  const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + i;
  if constexpr (W == 1) w[0] = *p;
  else if constexpr (W == 2) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
}
template <int W> __device__ __forceinline__ void load_few_f32(const void* base, int64_t i, uint32_t (&w)[W]) {
  const float* p = reinterpret_cast<const float*>(base) + i;
  if constexpr (W == 1) w[0] = __float_as_uint(*p);
  else if constexpr (W == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
  else { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
}
template <int OP, int R, int W> struct ColumnIn { uint32_t a[R][OP == D_DW ? W : (W + 1) / 2], b[OP == D_DX ? R : 1][(W + 1) / 2]; };
// f(i) for the rows that exist; FULL: all R do.  Nothing else is asked for a row: a branch a row took longer than the row.
template <int R, bool FULL, typename F> __device__ __forceinline__ void each_row(int64_t row0, int step, int64_t end, F f) {
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (FULL || row0 + i * step < end) f(i);
}
template <int OP, int R, int W, bool FULL>
__device__ __forceinline__ void columns_ahead_of(const DenseEpi& e, int64_t row0, int step, int64_t end, int col, int which, ColumnIn<OP, R, W>& x) {
  if constexpr (OP == D_DW) {
    if (e.accumulate) {
      const int64_t at = out0_at<OP>(e, row0, col, which), down = step * e.out0_pitch;
      if (e.out0_fp32) each_row<R, FULL>(row0, step, end, [&](int i) { load_few_f32<W>(e.out0, at + i * down, x.a[i]); });
      else each_row<R, FULL>(row0, step, end, [&](int i) { load_few<W>(e.out0, at + i * down, *reinterpret_cast<uint32_t (*)[(W + 1) / 2]>(&x.a[i])); });
    }
  } else {
    if (e.in1) {
      const int64_t at = row0 * e.in1_pitch + col, down = step * e.in1_pitch;
      each_row<R, FULL>(row0, step, end, [&](int i) { load_few<W>(e.in1, at + i * down, x.a[i]); });
    }
    if constexpr (OP == D_DX)
      if (e.out1) {
        const int64_t at = row0 * e.in2_pitch + col, down = step * e.in2_pitch;
        each_row<R, FULL>(row0, step, end, [&](int i) { load_few<W>(e.in2, at + i * down, x.b[i]); });
      }
  }
}
template <int OP, int R, int W>
__device__ __forceinline__ void columns_ahead(const DenseEpi& e, int64_t row0, int step, int64_t end, int col, int which, ColumnIn<OP, R, W>& x) {
  if (row0 + (R - 1) * step < end) columns_ahead_of<OP, R, W, true>(e, row0, step, end, col, which, x);
  else columns_ahead_of<OP, R, W, false>(e, row0, step, end, col, which, x);
}
// Pair p of what was loaded as 16 bits.
template <int R, int W, bool BF16, int N> __device__ __forceinline__ u64 pair_of(const uint32_t (&x)[R][N], int p) {
  if constexpr (W == 1) return widen2<BF16>(x[2 * p][0] | (x[2 * p + 1][0] << 16));
  else return widen2<BF16>(x[pair_row<W>(p, 0)][pair_col<W>(p, 0) / 2]);
}
// at: the first row's element
template <int R, int W, bool BF16, bool FULL>
__device__ __forceinline__ void store_columns(void* base, int64_t pitch, int64_t at, int64_t row0, int step, int64_t end, int fp32, const u64 (&v)[R * W / 2]) {
  const int64_t down = step * pitch;
  if (fp32) {
    each_row<R, FULL>(row0, step, end, [&](int i) {
      float* p = reinterpret_cast<float*>(base) + at + i * down;
      if constexpr (W == 1) {
        *p = __uint_as_float(i & 1 ? (uint32_t)(v[i / 2] >> 32) : (uint32_t)v[i / 2]);
      } else if constexpr (W == 2) {
        *reinterpret_cast<u64*>(p) = v[i];
      } else {
        *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(v[2 * i], v[2 * i + 1]);
      }
    });
  } else {
    uint32_t w[R * W / 2];
#pragma unroll
    for (int p = 0; p < R * W / 2; ++p) w[p] = narrow_pair<BF16>(v[p]);
    each_row<R, FULL>(row0, step, end, [&](int i) {
      uint16_t* p = reinterpret_cast<uint16_t*>(base) + at + i * down;
      if constexpr (W == 1) *p = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
      else if constexpr (W == 2) *reinterpret_cast<uint32_t*>(p) = w[i];
      else *reinterpret_cast<uint2*>(p) = make_uint2(w[2 * i], w[2 * i + 1]);
    });
  }
}
// One kind of work for all rows, then the next.  bias: of the lane's columns.
template <int OP, int R, int W, bool BF16, bool FULL>
__device__ __forceinline__ void finish_columns_of(const DenseEpi& e, int64_t row0, int step, int64_t end, int col, int which, const float (&bias)[W], const ColumnIn<OP, R, W>& x,
                                                  u64 (&v)[R * W / 2]) {
  constexpr int N = R * W / 2;
  auto store = [&](void* base, int64_t pitch, int fp32) { store_columns<R, W, BF16, FULL>(base, pitch, row0 * pitch + col, row0, step, end, fp32, v); };
  if constexpr (OP == D_FWD) {
#pragma unroll
    for (int p = 0; p < N; ++p) v[p] = add2(v[p], pack2(bias[pair_col<W>(p, 0)], bias[pair_col<W>(p, 1)]));
    if (e.out1) store(e.out1, e.out1_pitch, 0);
    with_activation(e.act, [&](auto act) {
#pragma unroll
      for (int p = 0; p < N; ++p) v[p] = activate2<decltype(act)::value>(v[p]);
    });
  }
  if constexpr (OP != D_DW) {
    if (e.in1) {
#pragma unroll
      for (int p = 0; p < N; ++p) v[p] = add2(v[p], pair_of<R, W, BF16>(x.a, p));
    }
  }
  if constexpr (OP == D_FWD) {
    store(e.out0, e.out0_pitch, e.out0_fp32);
  } else if constexpr (OP == D_DX) {
    if (e.out0) store(e.out0, e.out0_pitch, 0);
    if (e.out1) {
      with_activation(e.act, [&](auto act) {
#pragma unroll
        for (int p = 0; p < N; ++p) v[p] = through2<decltype(act)::value>(v[p], pair_of<R, W, BF16>(x.b, p));
      });
      store(e.out1, e.out1_pitch, 0);
    }
  } else {
    if (e.accumulate) {
      if (e.out0_fp32) {
#pragma unroll
        for (int p = 0; p < N; ++p)
          v[p] = add2(v[p], pack2(__uint_as_float(x.a[pair_row<W>(p, 0)][pair_col<W>(p, 0)]), __uint_as_float(x.a[pair_row<W>(p, 1)][pair_col<W>(p, 1)])));
      } else {
#pragma unroll
        for (int p = 0; p < N; ++p) v[p] = add2(v[p], pair_of<R, W, BF16>(x.a, p));
      }
    }
    store_columns<R, W, BF16, FULL>(e.out0, e.out0_pitch, out0_at<OP>(e, row0, col, which), row0, step, end, e.out0_fp32, v);
  }
}
template <int OP, int R, int W>
__device__ __forceinline__ void finish_columns(const DenseEpi& e, int64_t row0, int step, int64_t end, int col, int which, const float (&bias)[W], const ColumnIn<OP, R, W>& x,
                                               u64 (&v)[R * W / 2]) {
  with_type(e.bf16, [&](auto bf16) {
    if (row0 + (R - 1) * step < end) finish_columns_of<OP, R, W, decltype(bf16)::value, true>(e, row0, step, end, col, which, bias, x, v);
    else finish_columns_of<OP, R, W, decltype(bf16)::value, false>(e, row0, step, end, col, which, bias, x, v);
  });
}
template <int OP, int W>
__device__ __forceinline__ void load_bias(const DenseEpi& e, int col, int which, float (&b)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) b[j] = 0.f;
  if (OP == D_FWD && e.in0) {
#pragma unroll
    for (int j = 0; j < W; ++j) b[j] = widen(reinterpret_cast<const uint16_t*>(e.in0)[(int64_t)which * e.in0_stride + col + j], e.bf16);
  }
}

// pdl_enter's two halves (JOIN_*).
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- pairs of CTAs ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// A barrier's address in the pair's first CTA.
__device__ __forceinline__ uint32_t leaders(const uint64_t* bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(bar)));
  return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool cluster_try(uint32_t addr, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done) : "r"(addr), "r"(parity) : "memory");
  return done != 0;
}
// The bounded wait of a whole warp for arrivals from both CTAs.
__device__ __forceinline__ bool pair_wait(uint64_t* bar, uint32_t parity, const volatile uint32_t* abort_flag, long long limit) {
  const uint32_t addr = smem_u32(bar);
  bool done = cluster_try(addr, parity);
  if (!done) {
    const long long t0 = clock64();
    do {
      done = cluster_try(addr, parity);
    } while (!done && clock64() - t0 <= limit);
  }
  return __all_sync(0xffffffffu, done && !*abort_flag);
}
// The wait for a ragged block of a warp that passes over the blocks before it, perhaps a second's worth and more: the limit starts anew whenever the
// CTA's copying warp, whose own waits are bounded, has brought in another block.
__device__ __forceinline__ bool tail_wait(uint64_t* bar, uint32_t parity, const volatile uint32_t* abort_flag, const volatile uint32_t* copied, long long limit) {
  const uint32_t addr = smem_u32(bar);
  uint32_t seen = *copied;
  long long t0 = clock64();
  bool done;
  while (!(done = mbar_try(addr, parity)) && !*abort_flag) {
    const uint32_t now = *copied;
    if (now != seen) {
      seen = now;
      t0 = clock64();
    } else if (clock64() - t0 > limit) {
      break;
    }
  }
  return __all_sync(0xffffffffu, done && !*abort_flag);
}
// Copies and their byte counts, issued by a whole warp that has stayed together, as the MMAs are: one lane of it issues.  From a single lane's
// branch every copy's operands went through vector registers, about 150 clocks each, and with four copies to a stage (weight gradient) the producer
// was what the kernel waited for: 934 clocks per stage; 16,384 x 4096 x 4096 576 -> 382 us.
// PAIR: into this CTA's shared memory, completing on the barrier of the pair's first CTA.
template <bool PAIR>
__device__ __forceinline__ void tma_load_warp(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
        "@q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
        "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void expect_tx_warp(uint32_t bar, uint32_t bytes) {
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void umma_f16_pair(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n\t}"
      ::"r"(tmem_d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier of both CTAs when the pair's MMAs so far are done.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t.reg .b16 m;\n\telect.sync _|q, 0xffffffff;\n\tmov.b16 m, 3;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}" ::"r"(smem_u32(bar)) : "memory");
}

// Shared-memory descriptors.  k contiguous: rows of 128 bytes, groups of eight rows 1,024 apart.  Row index contiguous: one k = 128 bytes
// (64 rows), groups of eight k 1,024 apart, the next 64 rows 8 KB further.  128-byte swizzle (type 2) in both.
constexpr uint32_t DESC_HI = (1024 >> 4) | (1u << 14) | (2u << 29);
template <bool MN> __device__ __forceinline__ uint32_t tile_desc_lo(uint32_t addr) {
  return ((addr & 0x3FFFF) >> 4) | ((MN ? (BK * 128) >> 4 : 1u) << 16);
}
template <bool MN> __host__ __device__ constexpr uint32_t tile_k_step() { return MN ? 16 * 128 / 16 : 32 / 16; }      // sixteen k further, in 16-byte units

struct DenseTile {
  int w;                 // the weight matrix; weight gradient: the worker
  int m0, m_end;         // left side: first row of this CTA's part, end of the rows that count
  int n0, n_end;         // right side, of the whole tile
  int red0, red;         // reduction: first index, length
};

// The last of `n` ascending starts that is not above `at`: of equal ones, the one that is not empty.
__device__ __forceinline__ int find_start(const int32_t* start, int n, int at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

// Tile t of m_tiles x n_tiles: bands of eight along the left side, so that tiles under way together share operands in L2.
__device__ __forceinline__ void in_bands(int t, int m_tiles, int n_tiles, int& m, int& n) {
  const int per = 8 * n_tiles, band = t / per, in = min(8, m_tiles - 8 * band), l = t - band * per;
  m = 8 * band + l % in;
  n = l / in;
}

template <class S>
__device__ __forceinline__ void decode_tile(const DenseArgs& a, const DenseTab& tab, int t, int rank, DenseTile& c) {
  if (S::OP == D_DW) {
    const int per = a.m_tiles * a.n_tiles_n, g = t / per, l = t - g * per;
    c.w = g;
    int m, n;
    in_bands(l, a.m_tiles, a.n_tiles_n, m, n);
    c.m0 = m * S::TM + rank * BM; c.m_end = a.m_side;
    c.n0 = n * S::BN; c.n_end = a.n_side;
    c.red0 = tab.row0[g]; c.red = tab.row1[g] - c.red0;
    return;
  }
  c.red0 = 0; c.red = a.red;
  if (S::FEW) {      // the blocks of a run that share a piece of the weights lie together
    const int r = find_start(tab.run_pair0, tab.runs, t), l = t - tab.run_pair0[r], blocks = tab.run_blk0[r + 1] - tab.run_blk0[r];
    const int blk = tab.run_blk0[r] + l % blocks, g = find_start(tab.blk0, tab.groups, blk);
    c.w = tab.run_w[r];
    c.m0 = (l / blocks) * BM; c.m_end = a.n_side;
    c.n0 = tab.row0[g] + (blk - tab.blk0[g]) * S::BN; c.n_end = tab.row1[g];
    return;
  }
  int m, n;
  in_bands(t, a.m_tiles, a.n_tiles_n, m, n);
  c.n0 = n * S::BN; c.n_end = a.n_side;
  int blk = m;
  if (S::CTAS == 2) {
    const int r = find_start(tab.run_pair0, tab.runs, m);
    blk = tab.run_blk0[r] + 2 * (m - tab.run_pair0[r]) + rank;
    c.w = tab.run_w[r];
    if (blk >= tab.run_blk0[r + 1]) {      // the run's blocks are odd in number: nothing to bring in but zeros, nothing to write
      c.m0 = c.m_end = a.rows;
      return;
    }
  }
  const int g = find_start(tab.blk0, tab.groups, blk);
  c.w = tab.w[g];
  c.m0 = tab.row0[g] + (blk - tab.blk0[g]) * BM; c.m_end = tab.row1[g];
}

__device__ __forceinline__ int blocks_of(int red) { return (red + BK - 1) / BK; }

template <class S>
__global__ void __launch_bounds__(S::THREADS, S::PER_SM) dense_gemm(const __grid_constant__ DenseMaps maps, const __grid_constant__ DenseArgs a,
                                                            const __grid_constant__ DenseEpi epi, const __grid_constant__ DenseTab tab) {
  constexpr int STAGES = S::STAGES, BUFS = S::BUFS, EPI = S::EPI_WARPS;
  constexpr bool PAIR = S::CTAS == 2, RAGGED = S::OP == D_DW;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* tiles = smem_raw + (base - smem_u32(smem_raw));
  uint8_t* out_stage = tiles + STAGES * S::STAGE;
  uint64_t* full = reinterpret_cast<uint64_t*>(out_stage + S::OUT_BYTES);      // [STAGES] copies -> MMA (of the pair's first CTA)
  uint64_t* empty = full + STAGES;           // [STAGES] MMA -> copies
  uint64_t* acc_full = empty + STAGES;       // [BUFS] MMA -> epilogue
  uint64_t* acc_empty = acc_full + BUFS;     // [BUFS] epilogue (of both CTAs) -> MMA
  uint64_t* tail_full = acc_empty + BUFS;    // [STAGES] copies of a ragged last block -> the warp that zeroes what is not this worker's
  uint64_t* tail_ready = tail_full + STAGES; // [STAGES] the second CTA's such warp -> MMA
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail_ready + STAGES);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  volatile uint32_t* copied = tmem_slot + 2;      // blocks that the copying warp has asked for (a pair's second CTA, ragged reductions)
  const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
  const uint32_t rank = PAIR ? cluster_rank() : 0u;
  const int first_tile = PAIR ? blockIdx.x >> 1 : blockIdx.x, tile_step = S::SPLIT ? a.n_tiles : (PAIR ? gridDim.x >> 1 : gridDim.x);
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); mbar_init(&tail_full[s], 1); mbar_init(&tail_ready[s], 1); }
    for (int i = 0; i < BUFS; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], EPI * S::CTAS); }
    *abort_flag = 0;
    *copied = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(BUFS * S::ACC) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(BUFS * S::ACC) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cg::this_cluster().sync();
  tc_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  if (a.join == JOIN_FIRST) pdl_enter();
  else if (a.join == JOIN_BETWEEN) pdl_next();

  // this CTA's blocks of k of a tile with `n` of them
  auto block_range = [&](int n, int& b0, int& b1) {
    b0 = 0; b1 = n;
    if (S::SPLIT) {
      b0 = (int)((int64_t)n * (int)blockIdx.z / (int)gridDim.z);
      b1 = (int)((int64_t)n * ((int)blockIdx.z + 1) / (int)gridDim.z);
    }
  };

  if (warp == 0) {
    // ---------------- copies
    const uint32_t full0 = smem_u32(full), full_of_pair = PAIR ? leaders(full) : full0, tail0 = smem_u32(tail_full);
    int s = 0;
    uint32_t use = 0, blocks = 0;
    bool ok = true;
    for (int t = first_tile; t < a.n_tiles && ok; t += tile_step) {
      DenseTile c;
      decode_tile<S>(a, tab, t, (int)rank, c);
      int b0, b1;
      block_range(blocks_of(c.red), b0, b1);
      const int am = c.m0, bn = c.n0 + (int)rank * S::B_ROWS;
      for (int kb = b0; kb < b1; ++kb) {
        if (use > 0 && !warp_wait(&empty[s], (use - 1) & 1, abort_flag, a.limit)) { *abort_flag = 1; ok = false; break; }
        const uint32_t A = base + s * S::STAGE, B = A + S::A_BYTES;
        const int k0 = kb * BK, r0 = c.red0 + k0;
        auto load = [&](auto remote, uint32_t bar) {
          constexpr bool R = decltype(remote)::value;
          if (S::A_MN) {
#pragma unroll
            for (int i = 0; i < BM / 64; ++i) tma_load_warp<R>(A + i * BK * 128, &maps.a, bar, am + 64 * i, r0, S::FEW ? c.w : 0);
          } else {
            tma_load_warp<R>(A, &maps.a, bar, k0, am, S::FEW ? c.w : 0);
          }
          if (S::B_MN) {
#pragma unroll
            for (int i = 0; i < S::B_ROWS / 64; ++i) tma_load_warp<R>(B + i * BK * 128, &maps.b, bar, bn + 64 * i, r0, S::OP == D_DX ? c.w : 0);
          } else {
            tma_load_warp<R>(B, &maps.b, bar, k0, bn, S::FEW ? 0 : c.w);
          }
        };
        if (!PAIR) {
          expect_tx_warp(full0 + 8 * s, S::STAGE);
          load(std::false_type(), full0 + 8 * s);
        } else if (RAGGED && c.red - k0 < BK) {      // each CTA of a pair cleans up its own
          if (rank == 0) expect_tx_warp(full0 + 8 * s, 0);
          expect_tx_warp(tail0 + 8 * s, S::STAGE);
          load(std::false_type(), tail0 + 8 * s);
        } else {
          if (rank == 0) expect_tx_warp(full0 + 8 * s, 2 * S::STAGE);
          load(std::true_type(), full_of_pair + 8 * s);
        }
        if (PAIR && RAGGED && rank != 0) *copied = ++blocks;
        if (++s == STAGES) { s = 0; ++use; }
      }
    }
    if (a.join != JOIN_FIRST) pdl_wait();
    if (a.join == JOIN_LAST) pdl_next();
  } else if (warp == 1) {
    // ---------------- MMA (a pair's: by its first CTA; the second's warp cleans up its own ragged blocks)
    // zeroes k rows [valid, next multiple of sixteen) of a stage whose operands both have k as their rows
    auto clean = [&](int s, int valid) {
      const int upto = (valid + 15) & ~15;
      uint8_t* st = tiles + s * S::STAGE;
      for (int i = lane; i < (upto - valid) * 8; i += 32) {
        const int at = (valid + (i >> 3)) * 128 + (i & 7) * 16;
#pragma unroll
        for (int b = 0; b < S::STAGE / (BK * 128); ++b) *reinterpret_cast<uint4*>(st + b * (BK * 128) + at) = make_uint4(0u, 0u, 0u, 0u);
      }
      fence_proxy_async_smem();
      __syncwarp();
    };
    int s = 0, lead = 0;
    uint32_t parity = 0, tails = 0;          // tails: a bit per stage, the parity of its next ragged block
    bool ok = true;
    for (int t = first_tile; t < a.n_tiles && ok; t += tile_step) {
      DenseTile c;
      decode_tile<S>(a, tab, t, (int)rank, c);
      int b0, b1;
      block_range(blocks_of(c.red), b0, b1);
      if (PAIR && rank != 0) {
        if (RAGGED && c.red % BK != 0) {
          const int at = (s + b1 - 1) % STAGES;
          if (!tail_wait(&tail_full[at], (tails >> at) & 1, abort_flag, copied, a.limit)) { *abort_flag = 1; break; }
          tails ^= 1u << at;
          clean(at, c.red % BK);
          if (lane == 0) arrive_at(leaders(&tail_ready[at]));
        }
        s = (s + b1) % STAGES;
        continue;
      }
      for (int kb = b0; kb < b1; ++kb) {
        const bool first = (kb - b0) % a.chunk == 0, last = (kb - b0) % a.chunk == a.chunk - 1 || kb + 1 == b1;
        if (first && lead >= BUFS) {
          const uint32_t p = ((lead / BUFS) - 1) & 1;
          if (!(PAIR ? pair_wait(&acc_empty[lead % BUFS], p, abort_flag, a.limit) : warp_wait(&acc_empty[lead % BUFS], p, abort_flag, a.limit))) { *abort_flag = 1; ok = false; break; }
        }
        if (!(PAIR ? pair_wait(&full[s], parity, abort_flag, a.limit) : warp_wait(&full[s], parity, abort_flag, a.limit))) { *abort_flag = 1; ok = false; break; }
        const int valid = min(BK, c.red - kb * BK);
        if (RAGGED && valid < BK) {
          if (PAIR && !warp_wait(&tail_full[s], (tails >> s) & 1, abort_flag, a.limit)) { *abort_flag = 1; ok = false; break; }
          clean(s, valid);
          if (PAIR && !pair_wait(&tail_ready[s], (tails >> s) & 1, abort_flag, a.limit)) { *abort_flag = 1; ok = false; break; }
          tails ^= 1u << s;
        }
        tc_fence_after();
        const uint32_t a_lo = tile_desc_lo<S::A_MN>(base + s * S::STAGE), b_lo = tile_desc_lo<S::B_MN>(base + s * S::STAGE + S::A_BYTES);
        const uint32_t d = tmem + (lead % BUFS) * S::ACC;
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
          if (k * 16 < valid) {
            const uint32_t ka = a_lo + k * tile_k_step<S::A_MN>(), kbb = b_lo + k * tile_k_step<S::B_MN>(), acc = k ? 1u : (first ? 0u : 1u);
            if (PAIR) umma_f16_pair(d, ka, DESC_HI, kbb, DESC_HI, a.idesc, acc);
            else umma_f16(d, ka, DESC_HI, kbb, DESC_HI, a.idesc, acc);
          }
        if (PAIR) umma_commit_pair(&empty[s]); else umma_commit(&empty[s]);
        if (last) {
          if (PAIR) umma_commit_pair(&acc_full[lead % BUFS]); else umma_commit(&acc_full[lead % BUFS]);
          ++lead;
        }
        if (++s == STAGES) { s = 0; parity ^= 1; }
      }
    }
  } else {
    // ---------------- epilogue
    const int quarter = warp & 3, col0 = S::FEW ? 0 : ((warp - 2) >> 2) * S::COLS;
    const uint32_t t_lane = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col0;
    auto release = [&](int buf) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) arrive_at(leaders(&acc_empty[buf]));
        else mbar_arrive(&acc_empty[buf]);
      }
    };
    int lead = 0;
    for (int t = first_tile; t < a.n_tiles; t += tile_step) {
      DenseTile c;
      decode_tile<S>(a, tab, t, (int)rank, c);
      int b0, b1;
      block_range(blocks_of(c.red), b0, b1);
      const int m_base = c.m0 + quarter * 32;
      // a warp's 4 KB of shared memory: the bias of its columns and 2 KB where pieces of rows change lanes, or a 32 x 32 block on its way from rows to columns
      float* stage = reinterpret_cast<float*>(out_stage + (warp - 2) * 4096);
      const RowPlace<S::TURN> place{m_base, c.m_end, lane, reinterpret_cast<uint8_t*>(stage) + 2048};
      auto by_rows = [&](int j0) { return epi.rows && c.n_end - (c.n0 + col0 + j0) >= 32; };
      if (S::OP == D_FWD && !S::SPLIT && epi.in0 && by_rows(0)) {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < S::COLS; j += 32) {
          const int col = c.n0 + col0 + j + lane;
          stage[j + lane] = col < c.n_end ? widen(reinterpret_cast<const uint16_t*>(epi.in0)[(int64_t)c.w * epi.in0_stride + col], epi.bf16) : 0.f;
        }
        __syncwarp();
      }
      auto read_ahead = [&](RowIn<S::OP>& x, int j0) {
        if (by_rows(j0) && (S::TURN || place.row() < place.end)) row_ahead<S::OP>(epi, place, c.n0 + col0 + j0, x);
      };
      auto write_out = [&](u64 (&v)[16], int j0, RowIn<S::OP>& x) {
        const int col = c.n0 + col0 + j0;
        if (by_rows(j0)) {
          if (S::TURN || place.row() < place.end) finish_row<S::OP>(epi, place, col, c.w, stage + j0, x, v);
        } else if (col < c.n_end) {
          // W columns of every 32 / W lanes, rows W at a time side by side; everything is loaded before the block is turned round
          auto columns = [&](auto width) {
            constexpr int W = decltype(width)::value, R = S::DRAIN ? 8 / W : 8;
            const int at = lane % (32 / W) * W, sub = lane / (32 / W), here = col + at;
            const bool mine = here < c.n_end;
            float bias[W];
            ColumnIn<S::OP, R, W> in;
            if (mine) {
              load_bias<S::OP, W>(epi, here, c.w, bias);
              columns_ahead<S::OP, R, W>(epi, m_base + sub, W, c.m_end, here, c.w, in);
            }
            __syncwarp();      // the bias, if it lies there, has been read: no more whole chunks follow
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              float lo, hi;
              unpack2(v[j], lo, hi);
              stage[lane * 32 + ((2 * j) ^ lane)] = lo;
              stage[lane * 32 + ((2 * j + 1) ^ lane)] = hi;
            }
            __syncwarp();
            if (mine) {
#pragma unroll 1
              for (int r0 = sub; r0 < 32 && m_base + r0 < c.m_end; r0 += R * W) {
                if (r0 != sub) columns_ahead<S::OP, R, W>(epi, m_base + r0, W, c.m_end, here, c.w, in);
                u64 u[R * W / 2];
#pragma unroll
                for (int p = 0; p < R * W / 2; ++p) {
                  const int r = r0 + W * pair_row<W>(p, 0), r2 = r0 + W * pair_row<W>(p, 1);
                  u[p] = pack2(stage[r * 32 + ((at + pair_col<W>(p, 0)) ^ r)], stage[r2 * 32 + ((at + pair_col<W>(p, 1)) ^ r2)]);
                }
                finish_columns<S::OP, R, W>(epi, m_base + r0, W, c.m_end, here, c.w, bias, in, u);
              }
            }
            __syncwarp();
          };
          if (epi.pairs) columns(std::integral_constant<int, 2>());
          else columns(std::integral_constant<int, 1>());
        }
      };
      if constexpr (S::DRAIN) {
        float sum[S::COLS];
#pragma unroll
        for (int j = 0; j < S::COLS; ++j) sum[j] = 0.f;
        bool ok = true;
        for (int kb = b0; kb < b1; kb += a.chunk) {
          const int buf = lead % BUFS;
          if (!warp_wait(&acc_full[buf], (lead / BUFS) & 1, abort_flag, a.limit)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int j0 = 0; j0 < S::COLS; j0 += 32) {
            uint32_t r[2][16];
            tmem_ld16(t_lane + buf * S::ACC + j0, r[0]);
            if (j0 + 16 < S::COLS) tmem_ld16(t_lane + buf * S::ACC + j0 + 16, r[1]);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j0 + j < S::COLS) sum[j0 + j] += __uint_as_float(r[j / 16][j % 16]);
          }
          release(buf);
          ++lead;
        }
        if (!ok) { *abort_flag = 1; break; }
        if constexpr (S::SPLIT) {      // all copies have landed and been read: the partial tile takes their place
          float* part = reinterpret_cast<float*>(tiles);
          if (S::FEW) {
#pragma unroll
            for (int j = 0; j < S::COLS; ++j) part[j * S::PART_PITCH + quarter * 32 + lane] = sum[j];
          } else {
            float4* d = reinterpret_cast<float4*>(part + (quarter * 32 + lane) * S::PART_PITCH + col0);
#pragma unroll
            for (int j = 0; j < S::COLS / 4; ++j) d[j] = make_float4(sum[4 * j], sum[4 * j + 1], sum[4 * j + 2], sum[4 * j + 3]);
          }
        } else {
#pragma unroll
          for (int j0 = 0; j0 < S::COLS; j0 += 32) {
            RowIn<S::OP> x;
            read_ahead(x, j0);
            u64 v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = pack2(sum[j0 + 2 * j], sum[j0 + 2 * j + 1]);
            write_out(v, j0, x);
          }
        }
      } else {
        const int buf = lead % BUFS;
        const bool empty_sum = b1 == b0;      // a worker without rows: its weight gradient is zero
        RowIn<S::OP> now, next;
        read_ahead(now, 0);
        if (!empty_sum) {
          if (!warp_wait(&acc_full[buf], (lead / BUFS) & 1, abort_flag, a.limit)) { *abort_flag = 1; break; }
          tc_fence_after();
        }
#pragma unroll 1
        for (int j0 = 0; j0 < S::COLS; j0 += 32) {
          uint32_t r[32];
          if (j0 + 32 < S::COLS) read_ahead(next, j0 + 32);
          if (empty_sum) {
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = 0u;
          } else {
            tmem_ld32(t_lane + buf * S::ACC + j0, r);
          }
          if (j0 + 32 >= S::COLS && !empty_sum) release(buf);
          u64 v[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = pack2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
          write_out(v, j0, now);
          now = next;
        }
        if (!empty_sum) ++lead;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag)      // copies and products already issued end before the memory that they write is given up
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  if (PAIR) cg::this_cluster().sync();      // no CTA leaves while the other may still arrive at its barriers
  if (warp == 1) {
    tc_fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(BUFS * S::ACC) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(BUFS * S::ACC) : "memory");
  }
  if constexpr (S::SPLIT) {
    DenseTile c;
    decode_tile<S>(a, tab, blockIdx.x, 0, c);
    cg::cluster_group cl = cg::this_cluster();
    const int ranks = gridDim.z, me = blockIdx.z;
    const int rows = S::FEW ? min(S::BN, c.n_end - c.n0) : min(BM, c.m_end - c.m0);
    const int row0 = S::FEW ? c.n0 : c.m0, column0 = S::FEW ? c.m0 : c.n0, end = S::FEW ? c.m_end : c.n_end;
    const float* part = reinterpret_cast<const float*>(tiles);
    // a thread keeps its columns and goes down the rows, R at a time, what is read for the next ones under way (for the first, while the cluster's
    // CTAs wait for one another)
    auto finish = [&](auto width) {
      constexpr int W = decltype(width)::value, R = W == 4 ? 4 : 8;
      const int across = (min(S::FEW ? BM : S::BN, end - column0) + W - 1) / W, at_once = S::THREADS / across, step = ranks * at_once;      // threads to a row; rows of a CTA at once
      const int q = tid % across, col = column0 + W * q, first = me * at_once + tid / across;
      const bool active = tid < at_once * across && first < rows;
      float bias[W];
      ColumnIn<S::OP, R, W> in, next;
      if (active) {
        load_bias<S::OP, W>(epi, col, c.w, bias);
        columns_ahead<S::OP, R, W>(epi, row0 + first, step, row0 + rows, col, c.w, in);
      }
      cl.sync();
      if (!active) return;
#pragma unroll 1
      for (int r0 = first; r0 < rows; r0 += R * step) {
        if (r0 + R * step < rows) columns_ahead<S::OP, R, W>(epi, row0 + r0 + R * step, step, row0 + rows, col, c.w, next);
        float u[R][W];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int j = 0; j < W; ++j) u[i][j] = 0.f;
        for (int k = 0; k < ranks; ++k) {
          const float* from = (ranks == 1 ? part : cl.map_shared_rank(part, k)) + r0 * S::PART_PITCH + W * q;
          auto take = [&](int i) {
            uint32_t w[W];
            load_few_f32<W>(from, i * step * S::PART_PITCH, w);
#pragma unroll
            for (int j = 0; j < W; ++j) u[i][j] += __uint_as_float(w[j]);
          };
          if (r0 + (R - 1) * step < rows) each_row<R, true>(r0, step, rows, take);
          else each_row<R, false>(r0, step, rows, take);
        }
        u64 v[R * W / 2];
#pragma unroll
        for (int p = 0; p < R * W / 2; ++p) v[p] = pack2(u[pair_row<W>(p, 0)][pair_col<W>(p, 0)], u[pair_row<W>(p, 1)][pair_col<W>(p, 1)]);
        finish_columns<S::OP, R, W>(epi, row0 + r0, step, row0 + rows, col, c.w, bias, in, v);
        in = next;
      }
    };
    if (epi.quads) finish(std::integral_constant<int, 4>());
    else finish(std::integral_constant<int, 1>());
    cl.sync();                               // a CTA's shared memory outlives its readers
  }
  if (tid == 0 && *abort_flag) atomicAdd(&g_dense_failures, 1u);
}

// ---- the bias gradient: column sums of each worker's rows ------------------------------------------------------------------
// A CTA sums 64 columns (128 bytes of a row) over its share of a worker's rows, eight rows' loads of a thread under way at once; the CTAs of a
// cluster share a worker's rows and add their sums in order.
// 16,384 x 4096 45 us, 2.9 TB/s: a row gives a CTA 128 bytes at a time.  (Beside the products it hides nowhere: they hold every SM.)
constexpr int CSUM_TPB = 256, CSUM_COLS = 64, CSUM_ROWS = CSUM_TPB / (CSUM_COLS / 8);      // rows that a CTA reads at once
struct ColumnSumArgs {
  const void* dy; void* db;
  int64_t pitch, db_stride;
  int32_t N, bf16, db_fp32, accumulate, vec;
};
__global__ void __launch_bounds__(CSUM_TPB) column_sums(const __grid_constant__ ColumnSumArgs a, const __grid_constant__ DenseTab tab) {
  __shared__ float part[CSUM_ROWS][CSUM_COLS + 4];
  __shared__ float mine[CSUM_COLS];
  pdl_enter();
  const int slot = threadIdx.x >> 3, place = (threadIdx.x & 7) * 8;
  const int g = blockIdx.y, ranks = gridDim.z, me = blockIdx.z, col = blockIdx.x * CSUM_COLS + place, n = a.N - col;
  const int first = tab.row0[g], rows = tab.row1[g] - first;
  const int r0 = first + (int)((int64_t)rows * me / ranks), r1 = first + (int)((int64_t)rows * (me + 1) / ranks);
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  if (n > 0) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(a.dy) + (int64_t)(r0 + slot) * a.pitch + col;
    const int64_t step = (int64_t)CSUM_ROWS * a.pitch;
    int r = r0 + slot;
    if (a.vec && n >= 8) {
      constexpr int U = 8;
      auto take = [&](const uint4& w) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += widen((x[j >> 1] >> (16 * (j & 1))) & 0xFFFFu, a.bf16);
      };
      for (; r + (U - 1) * CSUM_ROWS < r1; r += U * CSUM_ROWS) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = *reinterpret_cast<const uint4*>(p + u * step);
        p += U * step;
#pragma unroll
        for (int u = 0; u < U; ++u) take(w[u]);
      }
      for (; r < r1; r += CSUM_ROWS, p += step) take(*reinterpret_cast<const uint4*>(p));
    } else {
      for (; r < r1; r += CSUM_ROWS, p += step) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) acc[j] += widen(p[j], a.bf16);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4*>(&part[slot][place + j]) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
  __syncthreads();
  if (threadIdx.x < CSUM_COLS) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < CSUM_ROWS; ++i) s += part[i][threadIdx.x];
    mine[threadIdx.x] = s;
  }
  cg::cluster_group cl = cg::this_cluster();
  cl.sync();
  const int c = blockIdx.x * CSUM_COLS + threadIdx.x;
  if (me == 0 && threadIdx.x < CSUM_COLS && c < a.N) {
    float s = 0.f;
    for (int k = 0; k < ranks; ++k) s += cl.map_shared_rank(mine, k)[threadIdx.x];
    const int64_t at = (int64_t)g * a.db_stride + c;
    if (a.db_fp32) {
      float* p = reinterpret_cast<float*>(a.db) + at;
      *p = a.accumulate ? *p + s : s;
    } else {
      uint16_t* p = reinterpret_cast<uint16_t*>(a.db) + at;
      if (a.accumulate) s += widen(*p, a.bf16);
      *p = (uint16_t)narrow2(s, 0.f, a.bf16);
    }
  }
  cl.sync();
}

// Matrices of 16-bit values to pitches that the tile copies can read: a warp per piece of LAY_WORDS words of a row, read in aligned words (a row that
// starts in the middle of one is shifted across the lanes) and written in words.  Up to three stacks in one launch, of a stack of weights those that
// are used.
constexpr int LAY_STEPS = 8, LAY_WORDS = 32 * LAY_STEPS;
struct LayStack {
  const uint16_t* src; uint16_t* dst;
  int64_t pitch, dst_pitch, stride, dst_stride, rows;      // of one matrix
  int32_t cols, pieces;                                    // pieces of a row
  int64_t first;                                           // units before this stack's
};
struct LayArgs { LayStack m[3]; int32_t n; int64_t units; };
__global__ void __launch_bounds__(256) lay_out_rows(const __grid_constant__ LayArgs a, const __grid_constant__ DenseTab tab) {
  pdl_enter();
  const int lane = threadIdx.x & 31;
  for (int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); unit < a.units; unit += (int64_t)gridDim.x * 8) {
    int k = 0;
    while (k + 1 < a.n && unit >= a.m[k + 1].first) ++k;
    const LayStack& m = a.m[k];
    const int64_t l = unit - m.first, row = l / m.pieces;
    const int piece = (int)(l - row * m.pieces);
    const int64_t which = row / m.rows, r = row - which * m.rows, w = m.stride ? tab.run_w[which] : 0;
    const uint16_t* src = m.src + w * m.stride + r * m.pitch;
    const uintptr_t at = (uintptr_t)src;
    const bool odd = (at & 2) != 0;
    const uint32_t* in = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3);
    uint32_t* out = reinterpret_cast<uint32_t*>(m.dst + w * m.dst_stride + r * m.dst_pitch);
    const int words = (m.cols + 1) / 2, last = (m.cols - 1 + (odd ? 1 : 0)) / 2;      // written; the last one that holds a value
    const int w0 = piece * LAY_WORDS;
    uint32_t v[LAY_STEPS + 1];
#pragma unroll
    for (int i = 0; i <= LAY_STEPS; ++i) {
      const int j = w0 + 32 * i + lane;
      v[i] = j <= last && (i < LAY_STEPS || (odd && lane == 0)) ? in[j] : 0u;
    }
#pragma unroll
    for (int i = 0; i < LAY_STEPS; ++i) {
      const uint32_t beside = __shfl_down_sync(0xffffffffu, v[i], 1), next = __shfl_sync(0xffffffffu, v[i + 1], 0);
      const int j = w0 + 32 * i + lane;
      if (j < words) out[j] = odd ? __funnelshift_r(v[i], lane == 31 ? next : beside, 16) : v[i];
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
constexpr int32_t MAX_FEATURES = 1 << 20;
constexpr int MAX_DEVICES = 64;
constexpr int64_t MAX_ROWS = (1ll << 31) - (1 << 20);

bool tma_ok(const void* p, int64_t pitch) { return ((uintptr_t)p & 15) == 0 && pitch % 8 == 0; }
// May `bytes` bytes be moved at once, from every multiple of that in a row on?  (No matrix: yes.)
bool moves(const void* p, int64_t pitch, int64_t stride, int size, int bytes) {
  return !p || (((uintptr_t)p % bytes) == 0 && (pitch * size) % bytes == 0 && (stride * size) % bytes == 0);
}
struct EpiMatrix { const void* p; int64_t pitch, stride; int size; };
void set_moves(DenseEpi& e, int columns, std::initializer_list<EpiMatrix> list) {
  e.pairs = columns % 2 == 0;
  e.quads = columns % 4 == 0;
  e.rows = e.wide = 1;
  for (const EpiMatrix& m : list) {
    e.pairs = e.pairs && moves(m.p, m.pitch, m.stride, m.size, 2 * m.size);
    e.quads = e.quads && moves(m.p, m.pitch, m.stride, m.size, 4 * m.size);
    e.rows = e.rows && moves(m.p, m.pitch, m.stride, m.size, 16);
    e.wide = e.wide && moves(m.p, m.pitch, m.stride, m.size, 32);
  }
}

// A 16-bit matrix, or a stack of them.
struct Operand {
  const void* p;
  int64_t rows, cols, pitch, count, stride;
};
bool operand_ok(const Operand& o) { return tma_ok(o.p, o.pitch) && (o.count == 1 || o.stride % 8 == 0); }
uint64_t laid_out_bytes(const Operand& o) {
  return operand_ok(o) ? 0 : (uint64_t)(o.rows * o.count * ((o.cols + 7) / 8 * 8)) * 2 + 256;
}

bool operand_map(CUtensorMap* m, const Operand& o, uint32_t box_rows) {
  const uint64_t dims[3] = {(uint64_t)o.cols, (uint64_t)o.rows, (uint64_t)o.count};
  const uint64_t bytes[2] = {(uint64_t)o.pitch * 2, (uint64_t)(o.count == 1 ? o.rows * o.pitch : o.stride) * 2};
  const uint32_t box[3] = {BK, box_rows, 1};
  return encode_tensor_map_bf16(m, reinterpret_cast<const uint16_t*>(o.p), 3, dims, bytes, box, 128);
}

template <class S> cudaError_t allow() { return allow_smem((const void*)dense_gemm<S>, S::SMEM); }

int32_t setup() {      // once per device
  static std::mutex mutex;
  static bool done[MAX_DEVICES] = {false};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return fail(PS_ERR_CUDA, "no current device");
  std::lock_guard<std::mutex> lock(mutex);
  if (done[dev]) return PS_OK;
  bool ok = configure_tc5_kernels() == 0;
  const cudaError_t e[] = {allow<Pair<D_FWD, false>>(), allow<Pair<D_FWD, true>>(), allow<Pair<D_DX, false>>(), allow<Pair<D_DX, true>>(), allow<Pair<D_DW, false>>(), allow<Pair<D_DW, true>>(),
                           allow<Single<D_FWD, false>>(), allow<Single<D_FWD, true>>(), allow<Single<D_DX, false>>(), allow<Single<D_DX, true>>(), allow<Single<D_DW, false>>(), allow<Single<D_DW, true>>(),
                           allow<Thin<D_FWD>>(), allow<Thin<D_DW>>(), allow<Split<D_FWD>>(), allow<Split<D_DX>>(), allow<Split<D_DW>>(),
                           allow<Few<D_FWD, 16>>(), allow<Few<D_FWD, 32>>(), allow<Few<D_FWD, 64>>(), allow<Few<D_DX, 16>>(), allow<Few<D_DX, 32>>(), allow<Few<D_DX, 64>>()};
  for (cudaError_t x : e) ok = ok && x == cudaSuccess;
  if (!ok) return fail(PS_ERR_CUDA, "kernel configuration failed: %s", cudaGetErrorString(cudaGetLastError()));
  done[dev] = true;
  return PS_OK;
}

int drain_blocks(const DenseEpi& e) { return e.out0_fp32 ? DRAIN_FP32 : (e.bf16 ? DRAIN_BF16 : DRAIN_FP16); }

struct Problem {
  DenseTab tab;          // merged groups (forward, input gradient) or workers (weight gradient)
  DenseArgs args;
  DenseEpi epi;
  Operand a, b;          // left and right operand of the plain orientation
  int64_t limit = WAIT_LIMIT_CYCLES;
  cudaStream_t st;
};

template <class S>
int32_t launch(const Problem& p, int split) {
  DenseMaps maps;
  const Operand &l = S::FEW ? p.b : p.a, &r = S::FEW ? p.a : p.b;
  if (!operand_map(&maps.a, l, S::A_MN ? 64 : BM) || !operand_map(&maps.b, r, S::B_MN ? 64 : S::B_ROWS)) return fail(PS_ERR_CUDA, "tensor map");
  DenseArgs a = p.args;
  a.limit = p.limit;
  a.idesc = (1u << 4) | (p.epi.bf16 ? (1u << 7) | (1u << 10) : 0u) | (S::A_MN ? 1u << 15 : 0u) | (S::B_MN ? 1u << 16 : 0u) | ((uint32_t)(S::BN >> 3) << 17) |
            ((uint32_t)(S::TM >> 4) << 24);
  a.chunk = S::DRAIN ? drain_blocks(p.epi) : 1 << 30;
  cudaLaunchConfig_t cfg = {};
  const int walkers = g_sm_count * S::PER_SM / S::CTAS;
  cfg.gridDim = S::SPLIT ? dim3(a.n_tiles, 1, split) : dim3(S::CTAS * std::min(a.n_tiles, walkers));
  cfg.blockDim = dim3(S::THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = p.st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = S::CTAS;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = S::SPLIT ? split : 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, dense_gemm<S>, maps, a, p.epi, p.tab);
  return e == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "dense layer launch: %s", cudaGetErrorString(e));
}

// Cuts the groups into blocks of `tm` rows and fills the prefix sums.  Returns the number of pairs of blocks (of the same run), or of blocks; per_block
// > 0: of tiles, that many to a block.
int64_t cut_rows(DenseTab& tab, int tm, bool pairs, int per_block = 0) {
  int64_t blocks = 0, units = 0;
  tab.runs = 0;
  for (int g = 0; g < tab.groups; ++g) {
    if (g == 0 || tab.w[g] != tab.w[g - 1]) {
      if (tab.runs) units += pairs ? (blocks - tab.run_blk0[tab.runs - 1] + 1) / 2 : (blocks - tab.run_blk0[tab.runs - 1]) * per_block;
      tab.run_blk0[tab.runs] = (int32_t)blocks;
      tab.run_pair0[tab.runs] = (int32_t)std::min<int64_t>(units, 1 << 30);
      tab.run_w[tab.runs++] = tab.w[g];
    }
    tab.blk0[g] = (int32_t)blocks;
    blocks += (tab.row1[g] - tab.row0[g] + tm - 1) / tm;
  }
  units += pairs ? (blocks - tab.run_blk0[tab.runs - 1] + 1) / 2 : (blocks - tab.run_blk0[tab.runs - 1]) * per_block;
  tab.blk0[tab.groups] = tab.run_blk0[tab.runs] = (int32_t)blocks;
  tab.run_pair0[tab.runs] = (int32_t)std::min<int64_t>(units, 1 << 30);
  return pairs || per_block ? units : blocks;
}
int div_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// CTAs that share a tile's blocks of k: as many as the chip has room for, at least two blocks each.
// us of captured calls, cold, with 1, 2, 4 and 8 CTAs (*: what the rule takes): 1 row 1568 -> 512 18, 14, 12*, 14; 4096 -> 4096 31, 23, 18, 20*; 4 workers of 40
// rows 4096 -> 4096 47, 41*, 49, 64; 16 of 3 rows 107*, 115, 133, 178; 512 rows 4096 -> 1024 33, 25, 20*, 43; 1,024 33, 25*, 35, 68; weight gradient 512 x 512 of
// 4,000 rows twice 33, 25, 20*, 43; of 2,000 rows once 23, 18, 16, 27*.
int split_for(int64_t tiles, int blocks, int room) {
  int split = 1;
  while (split < 8 && tiles * split * 2 <= room && blocks >= split * 4) split *= 2;
  return split;
}

// The tiles of a product, in numbers that tests ask for as well (dense_plan).
enum { PLAN_TOO_MANY = -1, PLAN_PAIR = 0, PLAN_SINGLE = 1, PLAN_THIN = 2, PLAN_SPLIT = 3, PLAN_FEW16 = 4, PLAN_FEW32 = 5, PLAN_FEW64 = 6 };
struct Plan { int tiles, split; bool drain; };

// Forward and input gradient: rows of groups x `features` columns, reduction over `red`.  Fills in the tiles' numbers and the groups' prefix sums.
Plan plan_rows(int op, DenseTab& tab, DenseArgs& a, const DenseEpi& epi, int features, int red, int sms) {
  int most = 0;
  int64_t rows = 0;
  for (int g = 0; g < tab.groups; ++g) {
    most = std::max(most, tab.row1[g] - tab.row0[g]);
    rows += tab.row1[g] - tab.row0[g];
  }
  const int blocks = div_up(red, BK);
  a.n_side = features;
  a.red = red;
  a.rows = (int32_t)rows;
  const bool drain = blocks > drain_blocks(epi);      // a shorter sum takes one accumulator either way
  // Few tiles for few rows a worker.  us of captured calls, cold, each worker on weights of its own, Few -> the other shape that there is: 4 workers
  // 4096 -> 4096, 48 rows each 41 -> 45 (Split), 64 41 -> 45, 96 49 -> 45; 16 workers 1568 -> 512, 48 rows 20.5 -> 20.5 (Split), 96 22.5 -> 20.5.  Where Single has
  // tiles enough for the chip it reads weights as fast: 16 workers 4096 -> 4096, 16 rows 108 -> 106, 48 115 -> 111, 96 143 -> 111; 64 workers 1024 -> 1024, 16
  // rows 47 -> 41, 96 70 -> 43.  The mean alone is asked for: a worker with 2,000 rows beside 63 with one, 2048 -> 2048, takes 143 (Single 117).
  if (rows <= 48ll * tab.groups) {
    const int bn = most <= 16 ? 16 : (most <= 32 ? 32 : 64);
    a.n_tiles_n = div_up(features, BM);
    const int64_t t = cut_rows(tab, bn, false, a.n_tiles_n);
    if (t >= 1 << 30) return {PLAN_TOO_MANY, 1, false};
    a.n_tiles = (int)t;
    return {bn == 16 ? PLAN_FEW16 : (bn == 32 ? PLAN_FEW32 : PLAN_FEW64), split_for(t, blocks, 2 * sms), drain};
  }
  // Thin tiles lack the registers to turn pieces of 16 bytes: such rows go to the others (us, 8,192 x 200 -> 5000 with pre: Thin 124, Pair 81; with everything
  // 142, 114); rows that go by columns stay (8,192 x 200 -> 4999 with everything: Thin 118, Pair 163).
  if (op == D_FWD) {
    a.n_tiles_n = div_up(features, 128);
    const int64_t row_blocks = cut_rows(tab, BM, false), t = row_blocks * a.n_tiles_n;
    if (red <= THIN_RED_FWD && (epi.wide || !epi.rows) && t > sms && t < 1 << 30) {
      a.m_tiles = (int)row_blocks;
      a.n_tiles = (int)t;
      return {PLAN_THIN, 1, false};
    }
  }
  a.n_tiles_n = div_up(features, 256);
  const int64_t row_blocks = cut_rows(tab, BM, false), pairs = cut_rows(tab, BM, true), singles = row_blocks * a.n_tiles_n;
  if (singles >= 1 << 30) return {PLAN_TOO_MANY, 1, false};
  // Pair -> Single, us as above, 16 workers 2048 -> 2048 with so many blocks of rows each: one 45 -> 41, two 47 -> 51, three (two pairs) 65 -> 63, four 68 -> 74, five
  // (three pairs) 86 -> 84, seven 100 -> 104.  Of one group's tiles, 4096 -> 2048: 64 pairs 37 -> 37, 80 55 -> 59.
  if (pairs * a.n_tiles_n * 2 >= sms && pairs * 10 <= row_blocks * 6) {
    a.m_tiles = (int)pairs;
    a.n_tiles = (int)pairs * a.n_tiles_n;
    return {PLAN_PAIR, 1, drain};
  }
  // Single -> Split, 4096 -> N, single tiles: 32 33 -> 25, 48 35 -> 35, 64 35 -> 35, 80 (its 128 x 128 tiles are more than the SMs) 37 -> 59.
  a.m_tiles = (int)row_blocks;
  if (singles * 3 >= sms * 2 || row_blocks * div_up(features, 128) > sms) {
    a.n_tiles = (int)singles;
    return {PLAN_SINGLE, 1, drain};
  }
  a.n_tiles_n = div_up(features, 128);
  a.n_tiles = (int)row_blocks * a.n_tiles_n;
  return {PLAN_SPLIT, split_for(a.n_tiles, blocks, sms), drain};
}

// Weight gradient: N x K for every worker, reduction over its rows.
Plan plan_weights(DenseTab& tab, DenseArgs& a, const DenseEpi& epi, int N, int K, int sms) {
  int most = 0;
  int64_t rows = 0;
  for (int g = 0; g < tab.groups; ++g) {
    most = std::max(most, tab.row1[g] - tab.row0[g]);
    rows += tab.row1[g] - tab.row0[g];
  }
  const bool few = most <= THIN_RED_DW || (most <= THIN_MOST_DW && rows <= (int64_t)THIN_MEAN_DW * tab.groups);
  const bool drain = div_up(most, BK) > drain_blocks(epi);
  a.m_side = N; a.n_side = K; a.red = 0;
  auto tiles = [&](int tm) { a.m_tiles = div_up(N, tm); return (int64_t)tab.groups * a.m_tiles * a.n_tiles_n; };
  a.n_tiles_n = div_up(K, 128);
  if (few && tiles(128) > sms && tiles(128) < 1 << 30) {
    a.n_tiles = (int)tiles(128);
    return {PLAN_THIN, 1, false};
  }
  a.n_tiles_n = div_up(K, 256);
  const int64_t pairs = tiles(256), singles = tiles(128);
  if (singles >= 1 << 30) return {PLAN_TOO_MANY, 1, false};
  // Pair -> Single, us of captured calls, cold, 16 workers of 1,000 rows, K = 2048, FP32 and BF16: N = 384 47 -> 41, 43 -> 37; 512 49 -> 49, 45 -> 43; 640 63 -> 57, 55 -> 49; 896
  // 74 -> 74, 63 -> 61.  Single -> Split, 2,000 rows, 1024 x 1024: one worker 22 -> 18, two 25 -> 25, four 27 -> 41.
  if (pairs * 2 >= sms && pairs * 2 <= singles + singles / 5) {
    a.n_tiles = (int)tiles(256);
    return {PLAN_PAIR, 1, drain};
  }
  if (singles * 3 >= sms * 2 || singles / a.n_tiles_n * div_up(K, 128) > sms) {
    a.n_tiles = (int)tiles(128);
    return {PLAN_SINGLE, 1, drain};
  }
  a.n_tiles_n = div_up(K, 128);
  a.n_tiles = (int)tiles(128);
  return {PLAN_SPLIT, split_for(a.n_tiles, div_up(most, BK), sms), drain};
}

template <int OP>
int32_t run(Problem& p, const Plan& plan) {
  if (plan.tiles == PLAN_TOO_MANY) return fail(PS_ERR_BAD_ARG, "too many tiles");
  if (plan.tiles == PLAN_PAIR) return plan.drain ? launch<Pair<OP, true>>(p, 1) : launch<Pair<OP, false>>(p, 1);
  if (plan.tiles == PLAN_SINGLE) return plan.drain ? launch<Single<OP, true>>(p, 1) : launch<Single<OP, false>>(p, 1);
  if constexpr (OP != D_DX)
    if (plan.tiles == PLAN_THIN) return launch<Thin<OP>>(p, 1);
  if constexpr (OP != D_DW) {
    if (plan.tiles == PLAN_FEW16) return launch<Few<OP, 16>>(p, plan.split);
    if (plan.tiles == PLAN_FEW32) return launch<Few<OP, 32>>(p, plan.split);
    if (plan.tiles == PLAN_FEW64) return launch<Few<OP, 64>>(p, plan.split);
  }
  return launch<Split<OP>>(p, plan.split);
}

// The groups that have rows, by their weights; those that follow one another, in that order and in memory, are one.
void sort_groups(const int32_t* rows, const int32_t* weight_of, int groups, DenseTab& tab) {
  struct Group { int32_t w, row0, row1; } list[PS_MAX_WORKERS];
  int n = 0, at = 0;
  bool sorted = true;
  for (int g = 0; g < groups; ++g) {
    if (rows[g] == 0) continue;
    const int32_t w = weight_of ? weight_of[g] : g;
    if (n && list[n - 1].w == w) list[n - 1].row1 = at + rows[g];
    else {
      sorted = sorted && (n == 0 || list[n - 1].w < w);
      list[n++] = Group{w, at, at + rows[g]};
    }
    at += rows[g];
  }
  if (!sorted) std::stable_sort(list, list + n, [](const Group& a, const Group& b) { return a.w < b.w; });
  tab.groups = n;
  for (int g = 0; g < n; ++g) {
    tab.w[g] = (uint16_t)list[g].w;
    tab.row0[g] = list[g].row0;
    tab.row1[g] = list[g].row1;
  }
}

// All groups, each by itself (weight gradient, bias gradient).
void list_workers(const int32_t* rows, int groups, DenseTab& tab) {
  tab.groups = groups;
  for (int g = 0; g < groups; ++g) {
    tab.row0[g] = g ? tab.row1[g - 1] : 0;
    tab.row1[g] = tab.row0[g] + rows[g];
  }
}

int32_t check_layer(const ps_dense_layer* l, int64_t* rows_out) {
  if (!l) return fail(PS_ERR_BAD_ARG, "NULL argument");
  if (l->groups < 1 || l->groups > PS_MAX_WORKERS || !l->rows) return fail(PS_ERR_BAD_ARG, "groups must be 1..%d, with rows", PS_MAX_WORKERS);
  if (l->n_weights < 1 || l->n_weights > 65535) return fail(PS_ERR_BAD_ARG, "n_weights must be 1..65535");
  if (l->type != PS_TYPE_BF16 && l->type != PS_TYPE_FP16) return fail(PS_ERR_BAD_ARG, "type must be PS_TYPE_BF16 or PS_TYPE_FP16");
  if (l->in_features < 1 || l->in_features > MAX_FEATURES || l->out_features < 1 || l->out_features > MAX_FEATURES)
    return fail(PS_ERR_BAD_ARG, "in_features and out_features must be 1..%d", MAX_FEATURES);
  if (l->activation < PS_ACT_NONE || l->activation > PS_ACT_SILU) return fail(PS_ERR_BAD_ARG, "unknown activation %d", l->activation);
  int64_t rows = 0;
  for (int g = 0; g < l->groups; ++g) {
    if (l->rows[g] < 0) return fail(PS_ERR_BAD_ARG, "group %d has %d rows", g, l->rows[g]);
    const int32_t w = l->weight_of ? l->weight_of[g] : g;
    if (w < 0 || w >= l->n_weights) return fail(PS_ERR_BAD_ARG, "group %d holds weights %d of %d", g, w, l->n_weights);
    rows += l->rows[g];
  }
  if (rows > MAX_ROWS) return fail(PS_ERR_BAD_ARG, "%lld rows are too many", (long long)rows);
  if (!l->weight || l->weight_pitch < l->in_features || (l->n_weights > 1 && l->weight_stride < (int64_t)(l->out_features - 1) * l->weight_pitch + l->in_features))
    return fail(PS_ERR_BAD_ARG, "weight is NULL, or its pitch or stride is too small");
  if (rows > 0 && (!l->x || l->x_pitch < l->in_features)) return fail(PS_ERR_BAD_ARG, "x is NULL or its pitch is too small");
  if (((uintptr_t)l->weight | (uintptr_t)l->x) & 1) return fail(PS_ERR_BAD_ARG, "an operand is not aligned to its type");
  *rows_out = rows;
  return PS_OK;
}
// An optional matrix of `size`-byte elements.
int32_t check_matrix(const char* name, const void* p, int64_t pitch, int64_t cols, int size) {
  if (p && (pitch < cols || ((uintptr_t)p & (size - 1)))) return fail(PS_ERR_BAD_ARG, "%s: its pitch is too small, or it is not aligned to its type", name);
  return PS_OK;
}

Operand weight_operand(const ps_dense_layer* l) { return Operand{l->weight, l->out_features, l->in_features, l->weight_pitch, l->n_weights, l->weight_stride}; }
Operand row_operand(const void* p, int64_t rows, int64_t cols, int64_t pitch) {
  return Operand{p, rows, cols, rows == 1 ? (cols + 7) / 8 * 8 : pitch, 1, 0};      // one row: there is no pitch to obey
}

struct Layout {      // hands out the workspace
  uint8_t* at;
  uint64_t left;
  LayArgs args;
};
// Has the operand laid out, if the tile copies cannot read it as it is.  used: the weight matrices that are (0: this is no stack of weights).
int32_t lay_out(Operand& o, Layout& ws, int used) {
  if (operand_ok(o)) return PS_OK;
  const uint64_t need = laid_out_bytes(o);
  if (!ws.at || ws.left < need) return fail(PS_ERR_ARENA_TOO_SMALL, "an operand has to be laid out anew (its base is not on 16 bytes or its pitch no multiple of 8): %llu more bytes of workspace needed", (unsigned long long)need);
  uint16_t* d = reinterpret_cast<uint16_t*>(((uintptr_t)ws.at + 255) & ~(uintptr_t)255);
  const int64_t pitch = (o.cols + 7) / 8 * 8;
  LayStack& m = ws.args.m[ws.args.n++];
  m.src = reinterpret_cast<const uint16_t*>(o.p); m.dst = d;
  m.pitch = o.pitch; m.dst_pitch = pitch; m.rows = o.rows;
  m.stride = used && o.count > 1 ? o.stride : 0; m.dst_stride = o.rows * pitch;
  m.cols = (int32_t)o.cols; m.pieces = (int32_t)(((o.cols + 1) / 2 + LAY_WORDS - 1) / LAY_WORDS);
  m.first = ws.args.units;
  ws.args.units += (used ? std::min<int64_t>(used, o.count) : 1) * o.rows * m.pieces;
  ws.at += need;
  ws.left -= need;
  o = Operand{d, o.rows, o.cols, pitch, o.count, o.rows * pitch};
  return PS_OK;
}
int32_t run_layout(const Layout& ws, const DenseTab& tab, cudaStream_t st) {
  if (ws.args.n == 0) return PS_OK;
  launch_pdl(lay_out_rows, dim3((unsigned)std::min<int64_t>((ws.args.units + 7) / 8, 148 * 32)), 256, 0, st, ws.args, tab);
  return cudaGetLastError() == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "operand copy launch");
}
// The weight matrices in use, each once, into run_w (cut_rows makes the same list again).
int list_used(DenseTab& tab) {
  tab.runs = 0;
  for (int g = 0; g < tab.groups; ++g)
    if (g == 0 || tab.w[g] != tab.w[g - 1]) tab.run_w[tab.runs++] = tab.w[g];
  return tab.runs;
}

}  // namespace

// What a call on a device of `sms` SMs would take: the tiles (PLAN_*), + 16 where sums are drained, + 32 * log2 of the CTAs that share a tile.  wide: bytes that
// its results' rows are moved in (32, 16, or 0 for columns).
int dense_plan(int op, const int32_t* rows, const int32_t* weight_of, int groups, int N, int K, int fp32, int bf16, int wide, int sms) {
  DenseTab tab = {};
  DenseArgs a = {};
  DenseEpi e = {};
  e.out0_fp32 = fp32; e.bf16 = bf16; e.wide = wide == 32; e.rows = wide != 0;
  if (op == D_DW) list_workers(rows, groups, tab);
  else sort_groups(rows, weight_of, groups, tab);
  const Plan p = op == D_DW ? plan_weights(tab, a, e, N, K, sms) : plan_rows(op, tab, a, e, op == D_FWD ? N : K, op == D_FWD ? K : N, sms);
  int shared = 0;
  while (1 << shared < p.split) ++shared;
  return p.tiles + (p.drain ? 16 : 0) + 32 * shared;
}

}  // namespace psk

using namespace psk;

extern "C" {

int32_t workers_dense_workspace(const ps_dense_layer* l, const void* dy, int64_t dy_pitch, uint64_t* bytes) {
  int64_t rows = 0;
  int32_t rc = check_layer(l, &rows);
  if (rc != PS_OK) return rc;
  if (!bytes) return fail(PS_ERR_BAD_ARG, "NULL argument");
  *bytes = 0;
  if (rows == 0) return PS_OK;
  *bytes = laid_out_bytes(weight_operand(l)) + laid_out_bytes(row_operand(l->x, rows, l->in_features, l->x_pitch));
  if (dy) *bytes += laid_out_bytes(row_operand(dy, rows, l->out_features, dy_pitch));
  return PS_OK;
}

int32_t workers_dense_status(void* stream) {
  static thread_local uint32_t seen[MAX_DEVICES] = {0};
  uint32_t count = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= MAX_DEVICES)) return fail(PS_ERR_CUDA, "no current device");
  if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(&count, g_dense_failures, sizeof(count), 0, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return fail(PS_ERR_CUDA, "workers_dense_status: %s", cudaGetErrorString(e));
  if (count == seen[dev]) return PS_OK;
  seen[dev] = count;
  return fail(PS_ERR_DEVICE_STATUS, "a bounded wait in a dense-layer kernel gave up: results since the last call are not to be used");
}

int32_t workers_dense_selftest_wait_timeout(int64_t limit_cycles, void* stream) {
  if (limit_cycles < 1 || limit_cycles > WAIT_LIMIT_CYCLES) return fail(PS_ERR_BAD_ARG, "limit_cycles must be 1..2e9");
  dense_wait_probe<<<1, 32, 0, (cudaStream_t)stream>>>(limit_cycles);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "probe launch: %s", cudaGetErrorString(e));
}

int32_t workers_dense_forward(const ps_dense_layer* l, const ps_dense_output* o) {
  int64_t rows = 0;
  int32_t rc = check_layer(l, &rows);
  if (rc != PS_OK) return rc;
  if (!o) return fail(PS_ERR_BAD_ARG, "NULL argument");
  const int N = l->out_features, K = l->in_features;
  if (o->y_type != l->type && o->y_type != PS_TYPE_FP32) return fail(PS_ERR_BAD_ARG, "y_type must be the operands' type or PS_TYPE_FP32");
  const int ys = o->y_type == PS_TYPE_FP32 ? 4 : 2;
  if (rows > 0 && !o->y) return fail(PS_ERR_BAD_ARG, "y is NULL");
  if ((rc = check_matrix("y", o->y, o->y_pitch, N, ys)) != PS_OK || (rc = check_matrix("pre", o->pre, o->pre_pitch, N, 2)) != PS_OK ||
      (rc = check_matrix("residual", o->residual, o->residual_pitch, N, 2)) != PS_OK ||
      (rc = check_matrix("bias", o->bias, l->n_weights > 1 ? o->bias_stride : N, N, 2)) != PS_OK)
    return rc;
  if (rows == 0) return PS_OK;
  if ((rc = setup()) != PS_OK) return rc;
  Problem p = {};
  p.st = (cudaStream_t)l->stream;
  p.a = row_operand(l->x, rows, K, l->x_pitch);
  p.b = weight_operand(l);
  sort_groups(l->rows, l->weight_of, l->groups, p.tab);
  Layout ws = {(uint8_t*)l->workspace, l->workspace_bytes, {}};
  if ((rc = lay_out(p.a, ws, 0)) != PS_OK || (rc = lay_out(p.b, ws, list_used(p.tab))) != PS_OK || (rc = run_layout(ws, p.tab, p.st)) != PS_OK) return rc;
  DenseEpi& e = p.epi;
  e.in0 = o->bias; e.in0_stride = o->bias_stride;
  e.in1 = o->residual; e.in1_pitch = o->residual_pitch;
  e.out0 = o->y; e.out0_pitch = o->y_pitch; e.out0_fp32 = ys == 4;
  e.out1 = o->pre; e.out1_pitch = o->pre_pitch;
  e.act = l->activation; e.bf16 = l->type == PS_TYPE_BF16;
  set_moves(e, N, {{o->residual, o->residual_pitch, 0, 2}, {o->y, o->y_pitch, 0, ys}, {o->pre, o->pre_pitch, 0, 2}});
  return run<D_FWD>(p, plan_rows(D_FWD, p.tab, p.args, e, N, K, g_sm_count));
}

static int32_t backward(const ps_dense_layer* l, const ps_dense_gradients* o, int64_t limit) {
  int64_t rows = 0;
  int32_t rc = check_layer(l, &rows);
  if (rc != PS_OK) return rc;
  if (!o) return fail(PS_ERR_BAD_ARG, "NULL argument");
  const int N = l->out_features, K = l->in_features;
  if (o->dw_type != l->type && o->dw_type != PS_TYPE_FP32) return fail(PS_ERR_BAD_ARG, "dw_type must be the operands' type or PS_TYPE_FP32");
  if (o->accumulate != 0 && o->accumulate != 1) return fail(PS_ERR_BAD_ARG, "accumulate must be 0 or 1");
  const int ds = o->dw_type == PS_TYPE_FP32 ? 4 : 2;
  if (rows > 0 && !o->dy) return fail(PS_ERR_BAD_ARG, "dy is NULL");
  if (o->dx_pre && !o->x_pre && rows > 0) return fail(PS_ERR_BAD_ARG, "dx_pre needs x_pre");
  if ((rc = check_matrix("dy", o->dy, o->dy_pitch, N, 2)) != PS_OK || (rc = check_matrix("x_pre", o->x_pre, o->x_pre_pitch, K, 2)) != PS_OK ||
      (rc = check_matrix("dx_add", o->dx_add, o->dx_add_pitch, K, 2)) != PS_OK || (rc = check_matrix("dx", o->dx, o->dx_pitch, K, 2)) != PS_OK ||
      (rc = check_matrix("dx_pre", o->dx_pre, o->dx_pre_pitch, K, 2)) != PS_OK || (rc = check_matrix("dw", o->dw, o->dw_pitch, K, ds)) != PS_OK ||
      (rc = check_matrix("dw", o->dw, l->groups > 1 ? o->dw_stride : (int64_t)N * o->dw_pitch, (int64_t)(N - 1) * o->dw_pitch + K, ds)) != PS_OK ||
      (rc = check_matrix("db", o->db, l->groups > 1 ? o->db_stride : N, N, ds)) != PS_OK)
    return rc;
  if ((rc = setup()) != PS_OK) return rc;
  cudaStream_t st = (cudaStream_t)l->stream;
  Operand x = row_operand(l->x, rows, K, l->x_pitch), dy = row_operand(o->dy, rows, N, o->dy_pitch), w = weight_operand(l);
  DenseTab sorted = {};
  if (rows > 0) {
    sort_groups(l->rows, l->weight_of, l->groups, sorted);
    const bool want_x = o->dw != nullptr, want_w = o->dx || o->dx_pre;
    Layout ws = {(uint8_t*)l->workspace, l->workspace_bytes, {}};
    if ((want_x || want_w) && (rc = lay_out(dy, ws, 0)) != PS_OK) return rc;
    if (want_x && (rc = lay_out(x, ws, 0)) != PS_OK) return rc;
    if (want_w && (rc = lay_out(w, ws, list_used(sorted))) != PS_OK) return rc;
    if ((rc = run_layout(ws, sorted, st)) != PS_OK) return rc;
  } else {      // nobody has a row: the gradients are zero
    cudaError_t ce = cudaSuccess;
    for (int g = 0; g < l->groups && !o->accumulate && ce == cudaSuccess; ++g) {
      if (o->dw) ce = cudaMemset2DAsync((uint8_t*)o->dw + (int64_t)g * o->dw_stride * ds, (size_t)o->dw_pitch * ds, 0, (size_t)K * ds, (size_t)N, st);
      if (o->db && ce == cudaSuccess) ce = cudaMemsetAsync((uint8_t*)o->db + (int64_t)g * o->db_stride * ds, 0, (size_t)N * ds, st);
    }
    return ce == cudaSuccess ? PS_OK : fail(PS_ERR_CUDA, "clearing gradients: %s", cudaGetErrorString(ce));
  }
  DenseTab workers = {};
  list_workers(l->rows, l->groups, workers);
  if (o->db) {
    ColumnSumArgs c = {};
    c.dy = dy.p; c.db = o->db; c.pitch = dy.pitch; c.db_stride = o->db_stride;
    c.N = N; c.bf16 = l->type == PS_TYPE_BF16; c.db_fp32 = ds == 4; c.accumulate = o->accumulate;
    c.vec = operand_ok(dy);
    const int blocks = div_up(N, CSUM_COLS) * l->groups;
    int split = 1;
    while (split < 8 && blocks * split < 4 * g_sm_count && rows / l->groups >= CSUM_ROWS * split) split *= 2;
    launch_cluster(column_sums, dim3((unsigned)div_up(N, CSUM_COLS), (unsigned)l->groups, (unsigned)split), CSUM_TPB, 0, split, st, c, workers);
    if (cudaGetLastError() != cudaSuccess) return fail(PS_ERR_CUDA, "column sum launch");
  }
  if (o->dx || o->dx_pre) {
    Problem p = {};
    p.st = st;
    p.a = dy;
    p.b = w;
    p.tab = sorted;
    DenseEpi& e = p.epi;
    e.in1 = o->dx_add; e.in1_pitch = o->dx_add_pitch;
    e.in2 = o->x_pre; e.in2_pitch = o->x_pre_pitch;
    e.out0 = o->dx; e.out0_pitch = o->dx_pitch;
    e.out1 = o->dx_pre; e.out1_pitch = o->dx_pre_pitch;
    e.act = l->activation; e.bf16 = l->type == PS_TYPE_BF16;
    set_moves(e, K, {{o->dx_add, o->dx_add_pitch, 0, 2}, {o->dx_pre ? o->x_pre : nullptr, o->x_pre_pitch, 0, 2}, {o->dx, o->dx_pitch, 0, 2}, {o->dx_pre, o->dx_pre_pitch, 0, 2}});
    p.limit = limit;
    p.args.join = !o->db ? JOIN_FIRST : (o->dw ? JOIN_BETWEEN : JOIN_LAST);
    if ((rc = run<D_DX>(p, plan_rows(D_DX, p.tab, p.args, e, K, N, g_sm_count))) != PS_OK) return rc;
  }
  if (o->dw) {
    Problem p = {};
    p.st = st;
    p.a = dy;
    p.b = x;
    p.tab = workers;
    DenseEpi& e = p.epi;
    e.out0 = o->dw; e.out0_pitch = o->dw_pitch; e.out0_stride = o->dw_stride; e.out0_fp32 = ds == 4; e.accumulate = o->accumulate;
    e.bf16 = l->type == PS_TYPE_BF16;
    set_moves(e, K, {{o->dw, o->dw_pitch, l->groups > 1 ? o->dw_stride : 0, ds}});
    p.limit = limit;
    p.args.join = o->db || o->dx || o->dx_pre ? JOIN_LAST : JOIN_FIRST;
    if ((rc = run<D_DW>(p, plan_weights(p.tab, p.args, e, N, K, g_sm_count))) != PS_OK) return rc;
  }
  return PS_OK;
}

int32_t workers_dense_backward(const ps_dense_layer* l, const ps_dense_gradients* o) { return backward(l, o, WAIT_LIMIT_CYCLES); }

int32_t workers_dense_selftest_backward(const ps_dense_layer* l, const ps_dense_gradients* o, int64_t limit_cycles) {
  if (limit_cycles < 1 || limit_cycles > WAIT_LIMIT_CYCLES) return fail(PS_ERR_BAD_ARG, "limit_cycles must be 1..2e9");
  return backward(l, o, limit_cycles);
}

}  // extern "C"
