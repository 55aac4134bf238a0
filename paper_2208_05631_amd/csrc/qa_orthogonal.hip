// A matrix's update orthogonalised by products: with n the smaller and m the larger of its sides and X the n x m matrix
// G / |G| (or its transpose),
//     A = X X^T,  B = b A + c A A,  X <- a X + B X        once per step,
// which takes every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors: values in (0, 1] come near 1.
//
// Numbers are held as two binary16 parts, 2^10 hi + 2^10 lo: 22 bits and a sign, as many as binary32 has but for one, so
// that the matrix cores multiply them: three products (hi hi, lo hi, hi lo) at sixteen times the rate of binary32's.
// One part alone (11 bits) is not enough: rounding X adds the same noise in all directions, and a direction with a small
// singular value grows by a = 3.4 in each step, the noise in it too (256 x 512, eight large singular values over a floor of
// 1/100: 3.6 % off, 2 % of which a rounded bfloat16 result would hide).  a X is added to the sum behind the product, not to
// B's diagonal, where it would swallow the sums' last bits: half of the error.
//
// A and B are symmetric: tiles on and below the diagonal, written twice.  Large matrices are bound by the matrix cores (4096 x 4096, five steps: 3.6 to 3.8 ms, fifteen
// products of 208 to 340 us, 1.31 to 1.35 PFLOP/s), small ones by the launches that wait for each other (64 of 128 x 1024: 204 to 245 us in seventeen), but for those that fit LDS
// (96 x 96: 29 us, under 2 for a product).
#include <algorithm>

#include "qa_product.h"
#include "qa_product_plan.h"

namespace qa {
namespace {

constexpr float kUnit = 1024.0f;                   // a stored number is so many times the number it stands for
constexpr int kNormBlocks = 1024;                 // work-groups that add one matrix's squares

// ---- the matrix's norm, and its parts ---------------------------------------------------------------------------------

struct SourceArgs {
  qa_matrices M;
  const void* g;
  float* momentum;                                 // NULL: none
  double* partial;                                 // [matrix][norm_blocks]: sums of squares
  _Float16* x;                                     // X in parts
  int64_t ld, batch;
  float mu;
  int nesterov, norm_blocks, lanes;                // lanes: threads side by side along a row, a power of two
};

// Eight elements of what is orthogonalised: g itself, or the momentum with it.  UPDATE: the momentum is written.
template <int TYPE, bool UPDATE>
__device__ __forceinline__ void source8(const SourceArgs& A, int64_t at, int n, float (&v)[kVec]) {
  to_f32<TYPE>(load_raw<TYPE>((const ElemT<TYPE>*)A.g + at, n), v);
  if (!A.momentum) return;
  float m[kVec];
  to_f32<QA_F32>(load_raw<QA_F32>(A.momentum + at, n), m);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    if (UPDATE) m[i] = A.mu * m[i] + v[i];
    v[i] = A.nesterov ? v[i] + A.mu * m[i] : m[i];
  }
  if (UPDATE) store_raw<QA_F32>(A.momentum + at, from_f32<QA_F32>(m), n);
}

// What the numbers are multiplied by, from the sum of their squares.  A matrix of zeros stays one; one with an infinity or a NaN has
// no direction.
__device__ __forceinline__ double scale_for(double all) {
  return all == 0.0 ? 0.0 : __builtin_isfinite(all) ? (double)kUnit / __builtin_sqrt(all) : (double)__builtin_nanf("");
}

// Squares are added in binary64: those of any finite numbers are finite there, and none is lost.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void orthogonal_norm_kernel(SourceArgs A) {
  __shared__ double sums[kWaves];
  const int64_t base = (int64_t)blockIdx.y * A.M.matrix_stride;
  const int lane = threadIdx.x % A.lanes, row = threadIdx.x / A.lanes, rows = kThreads / A.lanes;
  double s = 0.0;
  for (int64_t r = (int64_t)blockIdx.x * rows + row; r < A.M.rows; r += (int64_t)gridDim.x * rows)
    for (int64_t c = lane * kVec; c < A.M.cols; c += A.lanes * kVec) {
      const int n = (int)min((int64_t)kVec, A.M.cols - c);
      float v[kVec];
      source8<TYPE, true>(A, base + r * A.M.stride + c, n, v);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s += i < n ? (double)v[i] * (double)v[i] : 0.0;
    }
  s = wave_sum_f64(s);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) A.partial[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// X = u / |u| in parts, the shorter side along its rows: tiles of 64 x 64, turned by way of LDS for a TALL matrix.  Rows and columns are
// filled with zeros up to a whole step.
template <int TYPE, bool TALL>
__global__ __launch_bounds__(kThreads) void orthogonal_parts_kernel(SourceArgs A) {
  constexpr int kSide = 64;
  __shared__ float tile[TALL ? kSide : 1][kSide + 1];
  __shared__ double sums[kWaves];
  const int64_t z = blockIdx.z, r0 = (int64_t)blockIdx.y * kSide, c0 = (int64_t)blockIdx.x * kSide, base = z * A.M.matrix_stride;
  double part = 0.0;
#pragma unroll
  for (int b = 0; b < kNormBlocks; b += kThreads)
    if (b + (int)threadIdx.x < A.norm_blocks) part += A.partial[z * A.norm_blocks + b + threadIdx.x];
  part = wave_sum_f64(part);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = part;
  __syncthreads();
  const double all = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  const double scale = scale_for(all);
  const int64_t x_rows = whole(TALL ? A.M.cols : A.M.rows, kPartsStep), x_cols = A.ld / 2;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = h * 32 + (int)threadIdx.x / 8, col = (int)threadIdx.x % 8 * kVec;
    const int64_t r = r0 + row, c = c0 + col;
    const int n = r < A.M.rows ? (int)max((int64_t)0, min((int64_t)kVec, A.M.cols - c)) : 0;
    float v[kVec] = {};
    if (n) source8<TYPE, false>(A, base + r * A.M.stride + c, n, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      v[i] = i < n ? (float)((double)v[i] * scale) : 0.0f;
      if (TALL) tile[row][col + i] = v[i];
    }
    if (!TALL && r < x_rows && c < x_cols) put_parts(A.x + z * A.batch + r * A.ld + 2 * c, v);
  }
  if constexpr (TALL) {
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = h * 32 + (int)threadIdx.x / 8, row = (int)threadIdx.x % 8 * kVec;
      const int64_t c = c0 + col, r = r0 + row;
      float v[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = tile[row + i][col];
      if (c < x_rows && r < x_cols) put_parts(A.x + z * A.batch + c * A.ld + 2 * r, v);
    }
  }
}

// ---- what becomes of a product's sums ------------------------------------------------------------------------------------

// A matrix in parts; rows of `ld` elements, two per number.
struct Parts {
  _Float16* p;
  int64_t ld, batch, rows, cols;
  __device__ __forceinline__ _Float16* at(int64_t matrix, int64_t row, int64_t col) const { return p + matrix * batch + row * ld + 2 * col; }
  // Eight numbers of a row; zeros behind its end.
  __device__ __forceinline__ void put(int64_t matrix, int64_t row, int64_t col, const float (&v)[kVec]) const {
    float w[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) w[e] = col + e < cols ? v[e] : 0.0f;
    put_parts(at(matrix, row, col), w);
  }
  __device__ __forceinline__ bool holds(int64_t row, int64_t col) const { return row < rows && 2 * col < ld; }
};

// A = X X^T or B = b A + c A A, tiles on and below the diagonal; the others are their transposes.
template <bool SQUARE>
struct SymmetricOut {
  Parts to, a;
  float cb, cc;
  // Eight numbers of a row.
  __device__ __forceinline__ void put(int64_t matrix, int64_t row, int64_t col, float (&v)[kVec]) const {
    if (!to.holds(row, col)) return;
    float x[kVec] = {};
    if (SQUARE) get_parts(a.at(matrix, row, col), x);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = SQUARE ? cb * x[e] + (cc / kUnit) * v[e] : v[e] * (1.0f / kUnit);
    to.put(matrix, row, col, v);
  }
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0, char* lds) const {
    const auto same = [](int, int, float (&)[kVec]) {};
    const auto run = [&](int64_t i, int64_t j, float (&v)[kVec]) { put(p.matrix, j, i, v); };
    const auto turned = [&](int64_t i, int64_t j, float (&v)[kVec]) { put(p.matrix, i, j, v); };
    if (m0 / P::kM == n0 / P::kN) p.template for_runs<false>(m0, n0, lds, same, run, turned);
    else p.template for_runs<true>(m0, n0, lds, same, run, turned);
  }
};
// X' = a X + B X, with rows of zeros up to a whole step.
struct NextOut {
  Parts x, to;
  float ca;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0, char* lds) const {
    p.for_runs(m0, n0, lds, [&](int64_t i, int64_t j, float (&v)[kVec]) {
      if (j >= whole(to.rows, kPartsStep) || 2 * i >= to.ld) return;
      float o[kVec] = {};
      if (j < to.rows) get_parts(x.at(p.matrix, j, i), o);
#pragma unroll
      for (int e = 0; e < kVec; ++e) o[e] = j < to.rows ? ca * o[e] + v[e] * (1.0f / kUnit) : 0.0f;
      to.put(p.matrix, j, i, o);
    });
  }
};
// The last X', rounded once, or the parameters stepped with it.
template <int TYPE, bool STEP>
__device__ __forceinline__ void put_last(ElemT<TYPE>* at, int n, const float (&o)[kVec], float eta, float shrink) {
  if constexpr (STEP) {
    float w[kVec];
    to_f32<TYPE>(load_raw<TYPE>(at, n), w);
#pragma unroll
    for (int e = 0; e < kVec; ++e) w[e] = shrink * w[e] - eta * o[e];
    store_raw<TYPE>(at, from_f32<TYPE>(w), n);
  } else {
    store_raw<TYPE>(at, from_f32<TYPE>(o), n);
  }
}
template <int TYPE, bool STEP, bool TALL>
struct LastOut {
  Parts x;
  ElemT<TYPE>* out;
  int64_t stride, matrix_stride;
  float ca, eta, shrink;
  __device__ __forceinline__ void put(int64_t matrix, int64_t row, int64_t col, int64_t cols, const float (&o)[kVec]) const {
    put_last<TYPE, STEP>(out + matrix * matrix_stride + row * stride + col, (int)min((int64_t)kVec, cols - col), o, eta, shrink);
  }
  // X' goes to LDS complete where its rows are the caller's columns, and straight to memory where they are rows.
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0, char* lds) const {
    const auto complete = [&](int64_t i, int64_t j, float (&v)[kVec]) {
      float o[kVec] = {};
      if (j < x.rows && i < x.cols) get_parts(x.at(p.matrix, j, i), o);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = (ca * o[e] + v[e] * (1.0f / kUnit)) * (1.0f / kUnit);
    };
    if constexpr (TALL) {
      p.template for_runs<true>(m0, n0, lds, [&](int i, int j, float (&v)[kVec]) { complete(m0 + i, n0 + j, v); }, [](int64_t, int64_t, float (&)[kVec]) {},
                                [&](int64_t i, int64_t j, float (&o)[kVec]) {
        if (i < x.cols && j < x.rows) put(p.matrix, i, j, x.rows, o);
      });
    } else {
      p.for_runs(m0, n0, lds, [&](int64_t i, int64_t j, float (&v)[kVec]) {
        if (j >= x.rows || i >= x.cols) return;
        complete(i, j, v);
        put(p.matrix, j, i, x.cols, v);
      });
    }
  }
};

// ---- small matrices ------------------------------------------------------------------------------------------------------------

// A matrix that fits LDS beside its A: one work-group takes all steps, without a launch between the products.  X and A lie there as
// rows of parts; B takes A's place.  Sides are whole blocks of 32, zeros behind the matrix, and a wave has a block of 32 x 32 of each product
// (kSmallBlocks of X').  What bounds it is LDS: a block reads 4 KiB for three matrix instructions.
//
// 16 bytes behind each row, so that sixteen rows that are read side by side lie in different banks.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / kWave, kSmallBlocks = 2, kSmallVecs = 4;
constexpr int64_t kSmallLds = 156 << 10;
constexpr int64_t small_row(int64_t cols) { return whole(cols, 32) * 4 + 16; }
inline int64_t small_bytes(int64_t n, int64_t m) { return whole(n, 32) * (small_row(m) + small_row(n)); }
inline bool is_small(int64_t n, int64_t m) {
  return n <= 128 && m <= 512 && small_bytes(n, m) <= kSmallLds && whole(n, 32) / 32 * (whole(m, 32) / 32) <= kSmallWaves * kSmallBlocks &&
         std::max(n * ceil_div(m, kVec), m * ceil_div(n, kVec)) <= kSmallThreads * kSmallVecs;
}

template <int TYPE>
struct SmallArgs {
  SourceArgs S;                                    // g, momentum
  ElemT<TYPE>* out;
  int n, m, steps;
  float eta, shrink;
  float coefficients[3 * QA_ORTHOGONAL_STEPS_MAX];
};

__device__ __forceinline__ char* small_at(char* p, int pitch, int row, int byte) { return p + row * pitch + byte; }
__device__ __forceinline__ void small_put(char* p, int pitch, int row, int col, const float (&v)[kVec]) {
  _Float16 hi[kVec], lo[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) split_f16(v[i], hi[i], lo[i]);
  __builtin_memcpy(__builtin_assume_aligned(small_at(p, pitch, row, 4 * col), 16), hi, sizeof hi);
  __builtin_memcpy(__builtin_assume_aligned(small_at(p, pitch, row, 4 * col + 16), 16), lo, sizeof lo);
}
__device__ __forceinline__ void small_put(char* p, int pitch, int row, int col, float v) {
  _Float16 hi, lo;
  split_f16(v, hi, lo);
  *(_Float16*)small_at(p, pitch, row, col / kVec * 32 + col % kVec * 2) = hi;
  *(_Float16*)small_at(p, pitch, row, col / kVec * 32 + col % kVec * 2 + 16) = lo;
}
__device__ __forceinline__ void small_get(char* p, int pitch, int row, int col, float (&v)[kVec]) {
  _Float16 hi[kVec], lo[kVec];
  __builtin_memcpy(hi, __builtin_assume_aligned(small_at(p, pitch, row, 4 * col), 16), sizeof hi);
  __builtin_memcpy(lo, __builtin_assume_aligned(small_at(p, pitch, row, 4 * col + 16), 16), sizeof lo);
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

// One block of sums over k, a multiple of 32: rows a0 ... of A and b0 ... of B, or (COLUMNS) columns a0 ... of A, whose rows k are.
template <bool COLUMNS>
__device__ __forceinline__ f32x16 small_block(char* a, int a_pitch, int a0, char* b, int b_pitch, int b0, int k) {
  const int lane = threadIdx.x % kWave, half = lane / 32;
  f32x16 acc = {}, more = {};                      // two, as a sum waits for the one before
  const char *a_at[2][2], *b_at[2][2];             // k = 0 and 16 of a row, or four k and the next four; hi and lo
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      b_at[h][p] = small_at(b, b_pitch, b0 + lane % 32, h * 64 + half * 32 + p * 16);
      a_at[h][p] = COLUMNS ? small_at(a, a_pitch, 8 * half + 4 * h + (lane % 16 >> 2), (a0 + (lane & 16) + 4 * (lane & 3)) / 8 * 32 + p * 16) + (lane & 1) * 8
                           : small_at(a, a_pitch, a0 + lane % 32, h * 64 + half * 32 + p * 16);
    }
#pragma unroll 1
  for (int s = 0; s < k / 32; ++s) {
    u32x4 x[2][2], y[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        y[h][p] = *reinterpret_cast<const u32x4*>(b_at[h][p] + s * 128);
        if constexpr (COLUMNS) {
          s16x4 part[2];
#pragma unroll
          for (int e = 0; e < 2; ++e)
            part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a_at[e][p] + (2 * s + h) * 16 * a_pitch));
          __builtin_memcpy(&x[h][p], part, sizeof part);
        } else {
          x[h][p] = *reinterpret_cast<const u32x4*>(a_at[h][p] + s * 128);
        }
      }
    const auto times = [&](const u32x4& i, const u32x4& j, f32x16& c) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, i), __builtin_bit_cast(f16x8, j), c, 0, 0, 0);
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      times(x[h][0], y[h][0], acc);
      times(x[h][0], y[h][1], more);
      times(x[h][1], y[h][0], more);
    }
  }
  return acc + more;
}
// each(quarter, first of eight i within the block, j, sums)
template <class Each>
__device__ __forceinline__ void small_eights(const f32x16& acc, const Each& each) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    float v[kVec];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto both = __builtin_amdgcn_permlane32_swap(as_u32(acc[8 * q + e]), as_u32(acc[8 * q + 4 + e]), false, false);
      v[e] = as_f32(both[0]);
      v[4 + e] = as_f32(both[1]);
    }
    each(q, 16 * q + 8 * ((int)threadIdx.x % kWave / 32), (int)threadIdx.x % 32, v);
  }
}

// BYTES: half of a compute unit's LDS, or all of it, by what the matrix takes.  Registers leave room for one work-group of 1024 threads either way, and
// both take as long (600 of 64 x 64: 55 us, of 96 x 96: 102.5, with either).
template <int TYPE, bool STEP, bool TALL, int BYTES>
__global__ __launch_bounds__(kSmallThreads) void orthogonal_small_kernel(SmallArgs<TYPE> A) {
  __shared__ __attribute__((aligned(16))) char lds[BYTES];
  __shared__ double sums[kSmallWaves];
  const int np = (A.n + 31) / 32 * 32, mp = (A.m + 31) / 32 * 32, x_pitch = mp * 4 + 16, a_pitch = np * 4 + 16;
  char* const x = lds;
  char* const a = lds + np * x_pitch;
  const int wave = threadIdx.x / kWave, across = (A.S.M.cols + kVec - 1) / kVec, vecs = (int)A.S.M.rows * across;
  const int64_t base = (int64_t)blockIdx.x * A.S.M.matrix_stride;
  float u[kSmallVecs][kVec];
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < kSmallVecs; ++k) {
    const int i = k * kSmallThreads + threadIdx.x, r = i / across, c = i % across * kVec;
    if (i >= vecs) continue;
    const int n = min(kVec, (int)A.S.M.cols - c);
    source8<TYPE, true>(A.S, base + r * A.S.M.stride + c, n, u[k]);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      u[k][e] = e < n ? u[k][e] : 0.0f;
      s += (double)u[k][e] * (double)u[k][e];
    }
  }
  s = wave_sum_f64(s);
  if (threadIdx.x % kWave == 0) sums[wave] = s;
  for (int i = threadIdx.x; i < np * x_pitch / 16; i += kSmallThreads) reinterpret_cast<u32x4*>(x)[i] = u32x4{};
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) all += sums[w];
  const double scale = scale_for(all);
#pragma unroll
  for (int k = 0; k < kSmallVecs; ++k) {
    const int i = k * kSmallThreads + threadIdx.x, r = i / across, c = i % across * kVec;
    if (i >= vecs) continue;
#pragma unroll
    for (int e = 0; e < kVec; ++e) u[k][e] = (float)((double)u[k][e] * scale);
    if constexpr (!TALL) {
      small_put(x, x_pitch, r, c, u[k]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (c + e < A.n) small_put(x, x_pitch, c + e, r, u[k][e]);
    }
  }
  __syncthreads();

  // All blocks of A are computed, those that mirror others too: there is a wave for each, and a mirrored write takes longer.
  const int nb = np / 32, mb = mp / 32, br = wave / nb, bc = wave % nb;
  const bool has = br < nb;
  const auto put_a = [&](int i, int j, const float (&v)[kVec]) { small_put(a, a_pitch, 32 * bc + j, 32 * br + i, v); };
  for (int step = 0; step < A.steps; ++step) {
    const float ca = A.coefficients[3 * step], cb = A.coefficients[3 * step + 1], cc = A.coefficients[3 * step + 2];
    if (has) {
      const f32x16 acc = small_block<false>(x, x_pitch, 32 * br, x, x_pitch, 32 * bc, mp);
      small_eights(acc, [&](int, int i, int j, float (&v)[kVec]) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = v[e] * (1.0f / kUnit);
        put_a(i, j, v);
      });
    }
    __syncthreads();
    f32x16 square = {};
    if (has) square = small_block<false>(a, a_pitch, 32 * br, a, a_pitch, 32 * bc, np);
    float b[2][kVec];
    if (has)
      small_eights(square, [&](int q, int i, int j, float (&v)[kVec]) {
        float w[kVec];
        small_get(a, a_pitch, 32 * bc + j, 32 * br + i, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) b[q][e] = cb * w[e] + (cc / kUnit) * v[e];
      });
    __syncthreads();
    if (has) {
#pragma unroll
      for (int q = 0; q < 2; ++q) put_a(16 * q + 8 * ((int)threadIdx.x % kWave / 32), (int)threadIdx.x % 32, b[q]);
    }
    __syncthreads();
    const bool last = step + 1 == A.steps;
    float next[kSmallBlocks][2][kVec];
#pragma unroll
    for (int k = 0; k < kSmallBlocks; ++k) {
      const int block = k * kSmallWaves + wave, bm = block / nb, bn = block % nb;
      if (block >= nb * mb) continue;
      const f32x16 acc = small_block<true>(x, x_pitch, 32 * bm, a, a_pitch, 32 * bn, np);
      small_eights(acc, [&](int q, int i, int j, float (&v)[kVec]) {
        float w[kVec];
        small_get(x, x_pitch, 32 * bn + j, 32 * bm + i, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) next[k][q][e] = ca * w[e] + v[e] * (1.0f / kUnit);
      });
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSmallBlocks; ++k) {
      const int block = k * kSmallWaves + wave, bm = block / nb, bn = block % nb;
      if (block >= nb * mb) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int i = 32 * bm + 16 * q + 8 * ((int)threadIdx.x % kWave / 32), j = 32 * bn + (int)threadIdx.x % 32;
        // Behind the last step X' is wanted as it is: binary32 in the place of the parts.
        if (last) {
          __builtin_memcpy(__builtin_assume_aligned(small_at(x, x_pitch, j, 4 * i), 16), next[k][q], 16);
          __builtin_memcpy(__builtin_assume_aligned(small_at(x, x_pitch, j, 4 * i + 16), 16), next[k][q] + 4, 16);
        } else {
          small_put(x, x_pitch, j, i, next[k][q]);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < kSmallVecs; ++k) {
    const int i = k * kSmallThreads + threadIdx.x, r = i / across, c = i % across * kVec;
    if (i >= vecs) continue;
    float o[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      o[e] = *reinterpret_cast<const float*>(TALL ? small_at(x, x_pitch, min(c + e, A.n - 1), r * 4) : small_at(x, x_pitch, r, (c + e) * 4)) * (1.0f / kUnit);
    put_last<TYPE, STEP>(A.out + base + r * A.S.M.stride + c, min(kVec, (int)A.S.M.cols - c), o, A.eta, A.shrink);
  }
}

// ---- the steps ---------------------------------------------------------------------------------------------------------------

struct Plan {
  int64_t n, m, np, mp;                            // sides, and with whole steps
  int lanes, norm_blocks;                          // of the squares' sums
  size_t x, a, norms, bytes;                       // of one buffer for all matrices, and of everything
};
Plan plan_of(const qa_matrices& M) {
  Plan P;
  P.n = std::min(M.rows, M.cols);
  P.m = std::max(M.rows, M.cols);
  P.np = whole(P.n, kPartsStep);
  P.mp = whole(P.m, kPartsStep);
  P.x = (size_t)whole(M.count * P.np * 2 * P.mp * 2, 256);
  P.a = (size_t)whole(M.count * P.n * 2 * P.np * 2, 256);
  P.lanes = 1;
  while (P.lanes < kThreads && P.lanes * kVec < M.cols) P.lanes *= 2;
  P.norm_blocks = (int)std::min<int64_t>(std::max<int64_t>(kNormBlocks / std::max<int64_t>(M.count, 1), 16), ceil_div(M.rows * P.lanes, kThreads));
  P.norms = (size_t)whole(M.count * P.norm_blocks * 8, 256);
  P.bytes = is_small(P.n, P.m) ? 0 : 2 * P.x + 2 * P.a + P.norms;
  return P;
}

template <Lies LA, Lies LB, bool LOWER, class Epilogue>
int multiply(const Parts& a, const Parts& b, int64_t k, int64_t count, const Epilogue& out, hipStream_t stream) {
  const Operand oa = {a.p, a.ld, a.batch, in_rows(LA) ? a.rows : a.cols}, ob = {b.p, b.ld, b.batch, in_rows(LB) ? b.rows : b.cols};
  // X' has many tiles, A and B have few.
  constexpr unsigned kAllowed = LOWER ? ~0u : tiles_bit(kTiles256) | tiles_bit(kTiles128) | tiles_bit(kTiles64Two);
  const unsigned batch = (unsigned)count;
  const Tiles tiles = product_plan(kAllowed, ProductShape{oa.n, ob.n, ceil_div(k, kPartsStep), count, LOWER, 1.0}, 1).tiles;
  switch (tiles) {
    case kTiles256: return product_launch<Product<false, LA, LB, 2, 2, 4, 4>, LOWER>(oa, ob, k, out, batch, stream);
    case kTiles128: return product_launch<Product<false, LA, LB, 2, 2, 2, 2>, LOWER>(oa, ob, k, out, batch, stream);
    case kTiles64Two: return product_launch<Product<false, LA, LB, 2, 2, 1, 1, 2>, LOWER>(oa, ob, k, out, batch, stream);
    default: break;
  }
  if constexpr (LOWER) {
    switch (tiles) {
      case kTiles192: return product_launch<Product<false, LA, LB, 2, 2, 3, 3>, LOWER>(oa, ob, k, out, batch, stream);
      case kTiles128Two: return product_launch<Product<false, LA, LB, 2, 2, 2, 2, 2>, LOWER>(oa, ob, k, out, batch, stream);
      default: return product_launch<Product<false, LA, LB, 1, 1, 2, 2, 4>, LOWER>(oa, ob, k, out, batch, stream);
    }
  }
  return QA_ERR_INVALID_ARG;                       // not reached: all that is allowed is above
}

template <int TYPE, bool STEP, bool TALL>
int orthogonal_launch(const qa_matrices& M, const void* g, float* momentum, void* out, float mu, int nesterov, int steps,
                      const float* coefficients, float eta, float shrink, char* ws, hipStream_t stream) {
  const Plan P = plan_of(M);
  constexpr float usual[3] = {3.4445f, -4.7750f, 2.0315f};
  if (is_small(P.n, P.m)) {
    SmallArgs<TYPE> A = {};
    A.S.M = M;
    A.S.g = g;
    A.S.momentum = momentum;
    A.S.mu = mu;
    A.S.nesterov = nesterov;
    A.out = (ElemT<TYPE>*)out;
    A.n = (int)P.n;
    A.m = (int)P.m;
    A.steps = steps;
    A.eta = eta;
    A.shrink = shrink;
    for (int i = 0; i < 3 * steps; ++i) A.coefficients[i] = coefficients ? coefficients[i] : usual[i % 3];
    const auto kernel = small_bytes(P.n, P.m) <= kSmallLds / 2 ? orthogonal_small_kernel<TYPE, STEP, TALL, kSmallLds / 2> : orthogonal_small_kernel<TYPE, STEP, TALL, kSmallLds>;
    kernel<<<(unsigned)M.count, kSmallThreads, 0, stream>>>(A);
    return launch_status();
  }
  Parts x[2], ab[2];
  for (int i = 0; i < 2; ++i) {
    x[i] = {(_Float16*)(ws + i * P.x), 2 * P.mp, P.np * 2 * P.mp, P.n, P.m};
    ab[i] = {(_Float16*)(ws + 2 * P.x + i * P.a), 2 * P.np, P.n * 2 * P.np, P.n, P.n};
  }
  const Parts &a = ab[0], &b = ab[1];

  SourceArgs S = {};
  S.M = M;
  S.g = g;
  S.momentum = momentum;
  S.partial = (double*)(ws + 2 * P.x + 2 * P.a);
  S.x = x[0].p;
  S.ld = x[0].ld;
  S.batch = x[0].batch;
  S.mu = mu;
  S.nesterov = nesterov;
  S.lanes = P.lanes;
  S.norm_blocks = P.norm_blocks;
  orthogonal_norm_kernel<TYPE><<<dim3(S.norm_blocks, (unsigned)M.count), kThreads, 0, stream>>>(S);
  orthogonal_parts_kernel<TYPE, TALL><<<dim3((unsigned)ceil_div(M.cols, 64), (unsigned)ceil_div(M.rows, 64), (unsigned)M.count), kThreads, 0, stream>>>(S);
  if (const int rc = launch_status()) return rc;

  for (int s = 0, now = 0; s < steps; ++s, now ^= 1) {
    const float* c = coefficients ? coefficients + 3 * s : usual;
    if (const int rc = multiply<kRowsOfParts, kRowsOfParts, true>(x[now], x[now], P.m, M.count, SymmetricOut<false>{a, a, 0.0f, 0.0f}, stream)) return rc;
    if (const int rc = multiply<kRowsOfParts, kRowsOfParts, true>(a, a, P.n, M.count, SymmetricOut<true>{b, a, c[1], c[2]}, stream)) return rc;
    int rc;
    if (s + 1 < steps)
      rc = multiply<kColumnsOfParts, kRowsOfParts, false>(x[now], b, P.n, M.count, NextOut{x[now], x[now ^ 1], c[0]}, stream);
    else
      rc = multiply<kColumnsOfParts, kRowsOfParts, false>(
          x[now], b, P.n, M.count, LastOut<TYPE, STEP, TALL>{x[now], (ElemT<TYPE>*)out, M.stride, M.matrix_stride, c[0], eta, shrink}, stream);
    if (rc) return rc;
  }
  return QA_OK;
}
template <int TYPE, bool STEP>
int orthogonal(const qa_matrices& M, const void* g, float* momentum, void* out, float mu, int nesterov, int steps, const float* coefficients,
               float eta, float shrink, void* ws, void* stream) {
  const auto launch = M.rows > M.cols ? orthogonal_launch<TYPE, STEP, true> : orthogonal_launch<TYPE, STEP, false>;
  const int64_t most = most_side_by_side(M.rows, M.cols);
  for (int64_t i = 0; i < M.count; i += most) {    // once, but for tens of thousands of long thin ones; each time the workspace's front
    qa_matrices here = M;
    here.count = std::min(most, M.count - i);
    const int64_t at = i * M.matrix_stride;
    const int rc = launch(here, (const ElemT<TYPE>*)g + at, momentum ? momentum + at : nullptr, (ElemT<TYPE>*)out + at, mu, nesterov, steps, coefficients, eta,
                          shrink, (char*)ws, (hipStream_t)stream);
    if (rc) return rc;
  }
  return QA_OK;
}

int check_matrices(const qa_matrices* M) {
  if (!M) return QA_ERR_INVALID_ARG;
  constexpr int64_t kMost = int64_t(1) << 20, kMany = 1 << 16;
  if (M->count < 0 || M->count >= kMany || M->rows < 1 || M->rows >= kMost || M->cols < 1 || M->cols >= kMost) return QA_ERR_INVALID_ARG;
  if (M->stride < M->cols || M->stride >= (int64_t(1) << 40)) return QA_ERR_INVALID_ARG;
  if (M->count > 1 && (M->matrix_stride < (M->rows - 1) * M->stride + M->cols || M->matrix_stride >= (int64_t(1) << 56))) return QA_ERR_INVALID_ARG;
  return QA_OK;
}
int check_steps(int steps, const float* coefficients) {
  if (steps < 1 || steps > QA_ORTHOGONAL_STEPS_MAX) return QA_ERR_INVALID_ARG;
  for (int i = 0; coefficients && i < 3 * steps; ++i)
    if (!(coefficients[i] > -64.0f && coefficients[i] < 64.0f)) return QA_ERR_INVALID_ARG;
  return QA_OK;
}
int check_workspace(const qa_matrices* M, const void* ws, size_t ws_bytes) {
  const size_t need = plan_of(*M).bytes;
  if (need == 0) return QA_OK;
  if (!ws || ws_bytes < need) return QA_ERR_WORKSPACE;
  return aligned(ws, 256) ? QA_OK : QA_ERR_ALIGNMENT;
}

}  // namespace
}  // namespace qa

using namespace qa;

extern "C" size_t qa_orthogonal_workspace_bytes(const qa_matrices* matrices, int type) {
  if (check_matrices(matrices) != QA_OK || !known_type(type) || matrices->count == 0) return 0;
  return plan_of(*matrices).bytes;
}

extern "C" int qa_orthogonalize(const qa_matrices* matrices, int type, const void* g, int steps, const float* coefficients,
                                void* out, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_matrices(matrices)) return rc;
  if (const int rc = check_steps(steps, coefficients)) return rc;
  if (!known_type(type)) return QA_ERR_INVALID_ARG;
  if (matrices->count == 0) return QA_OK;
  if (!g || !out) return QA_ERR_INVALID_ARG;
  if (!element_aligned(g, type) || !element_aligned(out, type)) return QA_ERR_ALIGNMENT;
  if (const int rc = check_workspace(matrices, ws, ws_bytes)) return rc;
  const auto launch = type == QA_F32 ? orthogonal<QA_F32, false> : type == QA_BF16 ? orthogonal<QA_BF16, false> : orthogonal<QA_F16, false>;
  return launch(*matrices, g, nullptr, out, 0.0f, 0, steps, coefficients, 0.0f, 0.0f, ws, stream);
}

extern "C" int qa_step_orthogonal(const qa_matrices* matrices, const float* g, float* momentum, float* x, float mu, int nesterov,
                                  int steps, const float* coefficients, float eta, float shrink, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_matrices(matrices)) return rc;
  if (const int rc = check_steps(steps, coefficients)) return rc;
  if (!(mu >= 0.0f && mu <= 1.0f) || (nesterov != 0 && nesterov != 1) || !(eta >= 0.0f && eta < 1e30f) || !(shrink >= 0.0f && shrink <= 1.0f))
    return QA_ERR_INVALID_ARG;
  if (matrices->count == 0) return QA_OK;
  if (!g || !x) return QA_ERR_INVALID_ARG;
  if (!aligned(g, 4) || !aligned(momentum, 4) || !aligned(x, 4)) return QA_ERR_ALIGNMENT;
  if (const int rc = check_workspace(matrices, ws, ws_bytes)) return rc;
  return orthogonal<QA_F32, true>(*matrices, g, momentum, x, mu, nesterov, steps, coefficients, eta, shrink, ws, stream);
}
