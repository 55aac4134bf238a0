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
#include <algorithm>

#include "qa_product.h"

namespace qa {
namespace {

constexpr float kUnit = 1024.0f;                   // a stored number is so many times the number it stands for
constexpr int kNormBlocks = 128;

// ---- the matrix's norm, and its parts ---------------------------------------------------------------------------------

struct SourceArgs {
  qa_matrices M;
  const void* g;
  float* momentum;                                 // NULL: none
  double* partial;                                 // [matrix][norm_blocks]: sums of squares
  _Float16 *rm, *tr;                               // hi of the matrix as it lies, and of its transpose
  int64_t rm_ld, tr_ld, rm_part, tr_part, rm_batch, tr_batch;
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

// Tiles of 64 x 64, as they lie and transposed by way of LDS; rows are filled with zeros up to a whole step of k.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void orthogonal_parts_kernel(SourceArgs A) {
  constexpr int kSide = 64;
  __shared__ uint32_t tile[kSide][kSide + 1];
  __shared__ double sums[kWaves];
  const int64_t z = blockIdx.z, r0 = (int64_t)blockIdx.y * kSide, c0 = (int64_t)blockIdx.x * kSide, base = z * A.M.matrix_stride;
  const double part = wave_sum_f64((int)threadIdx.x < A.norm_blocks ? A.partial[z * A.norm_blocks + threadIdx.x] : 0.0);
  if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = part;
  __syncthreads();
  const double all = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  // A matrix of zeros stays one; one with an infinity or a NaN has no direction.
  const double scale = all == 0.0 ? 0.0 : __builtin_isfinite(all) ? (double)kUnit / __builtin_sqrt(all) : (double)__builtin_nanf("");
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = h * 32 + (int)threadIdx.x / 8, col = (int)threadIdx.x % 8 * kVec;
    const int64_t r = r0 + row, c = c0 + col;
    const int n = r < A.M.rows ? (int)max((int64_t)0, min((int64_t)kVec, A.M.cols - c)) : 0;
    float v[kVec] = {};
    if (n) source8<TYPE, false>(A, base + r * A.M.stride + c, n, v);
    _Float16 hi[kVec], lo[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      split_f16(i < n ? (float)((double)v[i] * scale) : 0.0f, hi[i], lo[i]);
      tile[row][col + i] = (uint32_t)__builtin_bit_cast(uint16_t, hi[i]) | (uint32_t)__builtin_bit_cast(uint16_t, lo[i]) << 16;
    }
    if (r < A.M.rows && c < A.rm_ld) {
      _Float16* p = A.rm + z * A.rm_batch + r * A.rm_ld + c;
      __builtin_memcpy(__builtin_assume_aligned(p, 16), hi, sizeof hi);
      __builtin_memcpy(__builtin_assume_aligned(p + A.rm_part, 16), lo, sizeof lo);
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = h * 32 + (int)threadIdx.x / 8, row = (int)threadIdx.x % 8 * kVec;
    const int64_t c = c0 + col, r = r0 + row;
    if (c >= A.M.cols || r >= A.tr_ld) continue;
    u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = tile[row + 2 * i][col], v = tile[row + 2 * i + 1][col];
      hi[i] = __builtin_amdgcn_perm(v, u, 0x05040100u);
      lo[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
    }
    _Float16* p = A.tr + z * A.tr_batch + c * A.tr_ld + r;
    *reinterpret_cast<u32x4*>(p) = hi;
    *reinterpret_cast<u32x4*>(p + A.tr_part) = lo;
  }
}

// ---- what becomes of a product's sums ------------------------------------------------------------------------------------

// A matrix in parts: rows of `ld` elements, zeros behind `cols`.
struct Parts {
  _Float16* p;
  int64_t ld, part, batch, rows, cols;
  __device__ __forceinline__ _Float16* at(int64_t row, int64_t col) const { return p + (int64_t)blockIdx.z * batch + row * ld + col; }
  // Four numbers of a row.
  __device__ __forceinline__ void get4(int64_t row, int64_t col, float (&v)[4]) const {
    const f16x4 hi = *reinterpret_cast<const f16x4*>(at(row, col)), lo = *reinterpret_cast<const f16x4*>(at(row, col) + part);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)hi[e] + (float)lo[e];
  }
};

// Calls each(row, column, sums of four rows) for all that a lane holds.
template <class P, class Each>
__device__ __forceinline__ void for_all(P& p, int64_t m0, int64_t n0, const Each& each) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int i = 0; i < (int)(sizeof p.acc / sizeof p.acc[0]); ++i)
#pragma unroll
    for (int j = 0; j < (int)(sizeof p.acc[0] / sizeof p.acc[0][0]); ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = p.acc[i][j][4 * q + e];
        each(m0 + 32 * i + 8 * q + 4 * (lane / 32), n0 + 32 * j + lane % 32, v);
      }
}

// C and its transpose: t's row is C's column.  c.p NULL: the transpose alone.
__device__ __forceinline__ void put_parts(const Parts& c, const Parts& t, int64_t row, int64_t col, float (&v)[4], bool both) {
  if (col >= t.rows && col >= c.ld) return;
  f16x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    _Float16 h, l;
    split_f16(row + e < t.cols && col < t.rows ? v[e] : 0.0f, h, l);
    hi[e] = h;
    lo[e] = l;
  }
  if (col < t.rows && row < t.ld) {
    *reinterpret_cast<f16x4*>(t.at(col, row)) = hi;
    *reinterpret_cast<f16x4*>(t.at(col, row) + t.part) = lo;
  }
  if (both && col < c.ld) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (row + e < c.rows) {
        *c.at(row + e, col) = hi[e];
        c.at(row + e, col)[c.part] = lo[e];
      }
  }
}

// A = X X^T, tiles on and below the diagonal; the others are their transposes.
struct GramOut {
  Parts a;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0) const {
    const bool both = m0 / P::kM != n0 / P::kN;
    for_all(p, m0, n0, [&](int64_t row, int64_t col, float (&v)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * (1.0f / kUnit);
      put_parts(a, a, row, col, v, both);
    });
  }
};
// B = b A + c A A, the same way.
struct SquareOut {
  Parts a, b;
  float cb, cc;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0) const {
    const bool both = m0 / P::kM != n0 / P::kN;
    for_all(p, m0, n0, [&](int64_t row, int64_t col, float (&v)[4]) {
      float x[4] = {};
      if (col < a.rows && row < a.ld) a.get4(col, row, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = cb * x[e] + (cc / kUnit) * v[e];
      put_parts(b, b, row, col, v, both);
    });
  }
};
// X' = a X + B X and its transpose.
struct NextOut {
  Parts x_t, c, t;                                 // X^T; X' and X'^T
  float ca;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0) const {
    for_all(p, m0, n0, [&](int64_t row, int64_t col, float (&v)[4]) {
      float x[4] = {};
      if (col < x_t.rows && row < x_t.ld) x_t.get4(col, row, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = ca * x[e] + v[e] * (1.0f / kUnit);
      put_parts(c, t, row, col, v, true);
    });
  }
};
// The last X', rounded once, or the parameters stepped with it: rows are those of the caller's matrix.
template <int TYPE, bool STEP>
struct LastOut {
  Parts x_t;                                       // transpose of X in the caller's rows
  ElemT<TYPE>* out;
  int64_t stride, matrix_stride;
  float ca, eta, shrink;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0) const {
    for_all(p, m0, n0, [&](int64_t row, int64_t col, float (&v)[4]) {
      if (col >= x_t.rows || row >= x_t.cols) return;
      float x[4];
      x_t.get4(col, row, x);
      ElemT<TYPE>* at = out + (int64_t)blockIdx.z * matrix_stride + row * stride + col;
#pragma unroll
      for (int e = 0; e < 4; ++e, at += stride) {
        if (row + e >= x_t.cols) break;
        const float o = (ca * x[e] + v[e] * (1.0f / kUnit)) * (1.0f / kUnit);
        *at = STEP ? (ElemT<TYPE>)(shrink * (float)*at - eta * o) : (ElemT<TYPE>)o;
      }
    });
  }
};

// ---- the steps ---------------------------------------------------------------------------------------------------------------

struct Plan {
  int64_t n, m, np, mp;                            // sides, and their rows' lengths: whole steps of k
  bool tall;                                       // the caller's rows are the longer side
  size_t x, xt, a, norms, bytes;                   // of one buffer (both parts, all matrices), and of everything
};
Plan plan_of(const qa_matrices& M) {
  Plan P;
  P.tall = M.rows > M.cols;
  P.n = std::min(M.rows, M.cols);
  P.m = std::max(M.rows, M.cols);
  P.np = ceil_div(P.n, kProductStep) * kProductStep;
  P.mp = ceil_div(P.m, kProductStep) * kProductStep;
  const auto room = [&](int64_t elements) { return ((size_t)(M.count * elements) * 2 + 255) / 256 * 256; };
  P.x = room(2 * P.n * P.mp);
  P.xt = room(2 * P.m * P.np);
  P.a = room(2 * P.n * P.np);
  P.norms = ((size_t)M.count * kNormBlocks * 8 + 255) / 256 * 256;
  P.bytes = 2 * P.x + 2 * P.xt + 2 * P.a + P.norms;
  return P;
}

template <bool LOWER, class Epilogue>
int multiply(const Parts& a, const Parts& b, int64_t k, int64_t count, const Epilogue& out, hipStream_t stream) {
  ProductArgs A = {};
  A.a = (const uint16_t*)a.p;
  A.b = (const uint16_t*)b.p;
  A.lda = a.ld;
  A.ldb = b.ld;
  A.a_part = a.part;
  A.b_part = b.part;
  A.a_batch = a.batch;
  A.b_batch = b.batch;
  A.m = a.rows;
  A.n = b.rows;
  A.steps = (int)(k / kProductStep);
  const auto tiles = [&](int64_t side) {
    const int64_t tm = ceil_div(A.m, side), tn = ceil_div(A.n, side);
    return count * (LOWER ? tm * (tm + 1) / 2 : tm * tn);
  };
  if (tiles(256) >= 192) return product_launch<false, 3, 2, 4, 4, 2, LOWER>(A, out, 1, (unsigned)count, stream);
  if (tiles(128) >= 128) return product_launch<false, 3, 2, 2, 2, 2, LOWER>(A, out, 1, (unsigned)count, stream);
  return product_launch<false, 3, 2, 2, 1, 1, LOWER>(A, out, 1, (unsigned)count, stream);
}

template <int TYPE, bool STEP>
int orthogonal_launch(const qa_matrices& M, const void* g, float* momentum, void* out, float mu, int nesterov, int steps,
                      const float* coefficients, float eta, float shrink, char* ws, hipStream_t stream) {
  const Plan P = plan_of(M);
  const auto parts = [&](size_t at, int64_t rows, int64_t cols, int64_t ld) {
    return Parts{(_Float16*)(ws + at), ld, M.count * rows * ld, rows * ld, rows, cols};
  };
  Parts x[2], xt[2];
  for (int i = 0; i < 2; ++i) {
    x[i] = parts((size_t)i * P.x, P.n, P.m, P.mp);
    xt[i] = parts(2 * P.x + (size_t)i * P.xt, P.m, P.n, P.np);
  }
  const Parts a = parts(2 * (P.x + P.xt), P.n, P.n, P.np), b = parts(2 * (P.x + P.xt) + P.a, P.n, P.n, P.np);
  const Parts &rm = P.tall ? xt[0] : x[0], &tr = P.tall ? x[0] : xt[0];

  SourceArgs S = {};
  S.M = M;
  S.g = g;
  S.momentum = momentum;
  S.partial = (double*)(ws + 2 * (P.x + P.xt + P.a));
  S.rm = rm.p;
  S.tr = tr.p;
  S.rm_ld = rm.ld;
  S.tr_ld = tr.ld;
  S.rm_part = rm.part;
  S.tr_part = tr.part;
  S.rm_batch = rm.batch;
  S.tr_batch = tr.batch;
  S.mu = mu;
  S.nesterov = nesterov;
  S.lanes = 1;
  while (S.lanes < kThreads && S.lanes * kVec < M.cols) S.lanes *= 2;
  S.norm_blocks = (int)std::min<int64_t>(kNormBlocks, ceil_div(M.rows * S.lanes, kThreads));
  orthogonal_norm_kernel<TYPE><<<dim3(S.norm_blocks, (unsigned)M.count), kThreads, 0, stream>>>(S);
  orthogonal_parts_kernel<TYPE><<<dim3((unsigned)ceil_div(M.cols, 64), (unsigned)ceil_div(M.rows, 64), (unsigned)M.count), kThreads, 0, stream>>>(S);
  if (const int rc = launch_status()) return rc;

  constexpr float usual[3] = {3.4445f, -4.7750f, 2.0315f};
  for (int s = 0, now = 0; s < steps; ++s, now ^= 1) {
    const float* c = coefficients ? coefficients + 3 * s : usual;
    if (const int rc = multiply<true>(x[now], x[now], P.mp, M.count, GramOut{a}, stream)) return rc;
    if (const int rc = multiply<true>(a, a, P.np, M.count, SquareOut{a, b, c[1], c[2]}, stream)) return rc;
    int rc;
    if (s + 1 < steps) {
      rc = multiply<false>(b, xt[now], P.np, M.count, NextOut{xt[now], x[now ^ 1], xt[now ^ 1], c[0]}, stream);
    } else {
      const Parts& back = P.tall ? x[now] : xt[now];
      const LastOut<TYPE, STEP> last{back, (ElemT<TYPE>*)out, M.stride, M.matrix_stride, c[0], eta, shrink};
      rc = P.tall ? multiply<false>(xt[now], b, P.np, M.count, last, stream) : multiply<false>(b, xt[now], P.np, M.count, last, stream);
    }
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
  if (!ws || ws_bytes < plan_of(*M).bytes) return QA_ERR_WORKSPACE;
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
  const auto launch = type == QA_F32 ? orthogonal_launch<QA_F32, false> : type == QA_BF16 ? orthogonal_launch<QA_BF16, false> : orthogonal_launch<QA_F16, false>;
  return launch(*matrices, g, nullptr, out, 0.0f, 0, steps, coefficients, 0.0f, 0.0f, (char*)ws, (hipStream_t)stream);
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
  return orthogonal_launch<QA_F32, true>(*matrices, g, momentum, x, mu, nesterov, steps, coefficients, eta, shrink, (char*)ws, (hipStream_t)stream);
}
