// Products of the matrix cores over rows of 16-bit elements: C[i][j] = sum_k A[i][k] B[j][k], both operands with k along
// their rows, sums in binary32.  Shared by the kernels that multiply; not part of the public interface.
#pragma once
#include "qa_rows.h"

#if defined(__HIPCC__)

namespace qa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kProductStep = 32;                   // elements of k that lie in LDS per step: 64 bytes of a row

// A number of more bits than an element has is two elements ("parts"), hi + lo; their products are hi hi, lo hi and hi lo
// (the fourth is below binary32's rounding), one after the other for each step of k.
struct ProductArgs {
  const uint16_t *a, *b;                           // 16-byte aligned, as are all strides
  int64_t lda, ldb;                                // elements between rows, < 2^22
  int64_t a_part, b_part;                          // elements from an operand's hi to its lo
  int64_t a_batch, b_batch;                        // elements between matrices (gridDim.z)
  int64_t m, n;                                    // rows of a and of b; past them the last one is read again
  int steps, split_steps;                          // steps of k, and those of one split (gridDim.y)
  unsigned tiles_m, tiles_n;
};

// WM x WN waves, FM x FN blocks of 32 x 32 each.
//
// Rows come straight from memory to LDS, 16 bytes per lane: a wave's instruction brings 64 bytes of sixteen rows.  In LDS
// a row's four octets stand at octet ^ (row / 4 % 4), which the lanes' addresses in memory see to, so that the sixteen
// rows that are read at a time lie in different banks.  Four buffers: while step s is multiplied, s + 1 is there and
// s + 2 and s + 3 are on their way, into the buffer that step s - 1 had.
template <bool BF16, int PASSES, int WM, int WN, int FM, int FN>
struct Product {
  static constexpr int kM = 32 * WM * FM, kN = 32 * WN * FN, kGroup = WM * WN * kWave;
  static constexpr int kBuffer = (kM + kN) * kProductStep, kBuffers = 4;
  static constexpr int kA = kM / 16 / (WM * WN), kB = kN / 16 / (WM * WN), kLoads = kA + kB;      // instructions per wave and step
  static_assert(kA * 16 * WM * WN == kM && kB * 16 * WM * WN == kN, "a wave brings rows of one operand at a time");

  f32x16 acc[FM][FN];
  u32x4 a[2][FM], b[2][FN];                        // operands of the two halves of a step
  const char *a_from, *b_from;                     // k = 0 of the tile's first row
  const char *a_at, *b_at;                         // what is loaded next
  int64_t a_part, b_part, k_at;                    // bytes
  int to_load, pass;
  uint32_t off[kLoads];
  int a_lane, b_lane, half[2], wave;

  __device__ __forceinline__ void next() {
    if (to_load > 1) {
      if constexpr (PASSES == 1) {
        a_at += 2 * kProductStep;
        b_at += 2 * kProductStep;
      } else {
        if (++pass == PASSES) pass = 0, k_at += 2 * kProductStep;
        a_at = a_from + k_at + (pass == 1 ? a_part : 0);
        b_at = b_from + k_at + (pass == 2 ? b_part : 0);
      }
    }
    --to_load;
  }
  __device__ __forceinline__ void load(uint16_t* lds) {
#pragma unroll
    for (int v = 0; v < kLoads; ++v)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)((v < kA ? a_at : b_at) + off[v]),
                                       (__attribute__((address_space(3))) void*)(lds + (v * WM * WN + wave) * 16 * kProductStep), 16, 0, 0);
    next();
  }
  __device__ __forceinline__ void read(const uint16_t* lds, int h) {
#pragma unroll
    for (int j = 0; j < FN; ++j) b[h][j] = *reinterpret_cast<const u32x4*>(lds + b_lane + half[h] + 32 * j * kProductStep);
#pragma unroll
    for (int i = 0; i < FM; ++i) a[h][i] = *reinterpret_cast<const u32x4*>(lds + a_lane + half[h] + 32 * i * kProductStep);
  }
  __device__ __forceinline__ void multiply(int h) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if constexpr (BF16)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[h][i]), __builtin_bit_cast(bf16x8, b[h][j]), acc[i][j], 0, 0, 0);
        else
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a[h][i]), __builtin_bit_cast(f16x8, b[h][j]), acc[i][j], 0, 0, 0);
      }
  }
  // Waits until at most LEFT of this wave's loads are on their way, then for the other waves.  Loads into LDS are the only
  // ones that the loop makes.
  template <int LEFT>
  static __device__ __forceinline__ void arrive() {
    static_assert(LEFT < 64, "the counter's bits");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
  }
  // The three buffers lie apart, as the compiler is told: it would wait for all loads before each read otherwise.
  static __device__ __forceinline__ void step(Product& p, const uint16_t* __restrict__ now, const uint16_t* __restrict__ then,
                                              uint16_t* __restrict__ last) {
    p.read(now, 1);
    p.multiply(0);
    arrive<kLoads>();                              // `then` is there, and nobody reads `last` any more
    p.load(last);
    p.read(then, 0);
    p.multiply(1);
  }
  // Sums of split blockIdx.y, 0 where it has no steps.
  __device__ __forceinline__ void run(const ProductArgs& A, int64_t m0, int64_t n0, uint16_t* lds) {
    const int lane = threadIdx.x % kWave;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x16{};
    const int first = (int)blockIdx.y * A.split_steps, steps = min(A.steps - first, A.split_steps) * PASSES;
    if (steps <= 0) return;
    a_from = (const char*)(A.a + (int64_t)blockIdx.z * A.a_batch + m0 * A.lda + (int64_t)first * kProductStep);
    b_from = (const char*)(A.b + (int64_t)blockIdx.z * A.b_batch + n0 * A.ldb + (int64_t)first * kProductStep);
    a_at = a_from;
    b_at = b_from;
    a_part = 2 * A.a_part;
    b_part = 2 * A.b_part;
    k_at = 0;
    to_load = steps;
    pass = 0;
    const uint32_t octet = (uint32_t)((lane & 3) ^ (lane >> 4 & 3)) * 16;
#pragma unroll
    for (int v = 0; v < kLoads; ++v) {
      const int row = (v < kA ? v : v - kA) * 16 * WM * WN + wave * 16 + lane / 4;
      const int64_t most = (v < kA ? A.m - m0 : A.n - n0) - 1;
      off[v] = (uint32_t)min((int64_t)row, most) * (uint32_t)(2 * (v < kA ? A.lda : A.ldb)) + octet;
    }
    a_lane = (wave % WM * 32 * FM + lane % 32) * kProductStep;
    b_lane = (kM + wave / WM * 32 * FN + lane % 32) * kProductStep;
    half[0] = ((lane / 32) ^ (lane >> 2 & 3)) * 8;
    half[1] = ((2 + lane / 32) ^ (lane >> 2 & 3)) * 8;

    int now = 0, then = kBuffer, later = 2 * kBuffer, last = 3 * kBuffer;
    load(lds + now);
    load(lds + then);
    load(lds + later);
    arrive<2 * kLoads>();
    read(lds + now, 0);
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      step(*this, lds + now, lds + then, lds + last);
      const int free = now;
      now = then;
      then = later;
      later = last;
      last = free;
    }
    arrive<0>();                                   // loads past the last step, before LDS is used for something else
  }
  __device__ __forceinline__ int64_t wave_m(int64_t m0) const { return m0 + wave % WM * 32 * FM; }
  __device__ __forceinline__ int64_t wave_n(int64_t n0) const { return n0 + wave / WM * 32 * FN; }
};

// The numbers that a lane has of block (i, j): rows 8 q + 4 (lane / 32) + e, e < 4, of column lane % 32.

// Consecutive work-groups go to the eight dies in turn.  Each die takes tiles that lie together, in bands eight tiles wide,
// so that its cache is asked for the same rows.  LOWER: tiles on and below the diagonal only.
template <bool LOWER>
__device__ __forceinline__ void tile_of(const ProductArgs& A, unsigned& tm, unsigned& tn) {
  const unsigned die = blockIdx.x % 8, each = gridDim.x / 8, more = gridDim.x % 8;
  const unsigned tile = die * each + min(die, more) + blockIdx.x / 8;
  if constexpr (LOWER) {
    unsigned r = (unsigned)((__builtin_sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= tile) ++r;
    while (r * (r + 1) / 2 > tile) --r;
    tm = r;
    tn = tile - r * (r + 1) / 2;
  } else {
    const unsigned band = tile / (8 * A.tiles_m), wide = min(8u, A.tiles_n - 8 * band), in_band = tile - band * 8 * A.tiles_m;
    tm = in_band / wide;
    tn = 8 * band + in_band % wide;
  }
}

template <bool BF16, int PASSES, int WM, int WN, int FM, int FN, bool LOWER, class Epilogue>
__global__ __launch_bounds__(WM* WN* kWave, 2) void product_kernel(ProductArgs A, Epilogue out) {
  typedef Product<BF16, PASSES, WM, WN, FM, FN> P;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[P::kBuffers * P::kBuffer];
  unsigned tm, tn;
  tile_of<LOWER>(A, tm, tn);
  const int64_t m0 = (int64_t)tm * P::kM, n0 = (int64_t)tn * P::kN;
  P p;
  p.run(A, m0, n0, lds);
  out(p, p.wave_m(m0), p.wave_n(n0));
}

// Launches tiles of the given form over all of A, splits and batches as they are set.
template <bool BF16, int PASSES, int WM, int WN, int FM, int FN, bool LOWER = false, class Epilogue>
int product_launch(ProductArgs A, const Epilogue& out, unsigned splits, unsigned batch, hipStream_t stream) {
  typedef Product<BF16, PASSES, WM, WN, FM, FN> P;
  A.tiles_m = (unsigned)ceil_div(A.m, P::kM);
  A.tiles_n = (unsigned)ceil_div(A.n, P::kN);
  A.split_steps = (int)ceil_div(A.steps, splits);
  const unsigned tiles = LOWER ? A.tiles_m * (A.tiles_m + 1) / 2 : A.tiles_m * A.tiles_n;
  product_kernel<BF16, PASSES, WM, WN, FM, FN, LOWER><<<dim3(tiles, splits, batch), P::kGroup, 0, stream>>>(A, out);
  return launch_status();
}

// v as hi + lo of binary16: 22 bits and a sign between them, as long as v is at least 2^-13; what is lost below is 2^-25 at most.
__device__ __forceinline__ void split_f16(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

}  // namespace qa

#endif  // __HIPCC__
