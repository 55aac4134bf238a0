// Weight gradient of a linear layer from the 8-bit codes of its input: dW = dY^T X.
//
// A code times its power of two is exact in bfloat16, and so are dY's elements, or two (binary16) or three (binary32)
// bfloat16 parts of them, so every product of the matrix cores is exact and the sums are held in binary32.
#include <algorithm>

#include "qa_rows.h"

namespace qa {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct WeightGradArgs {
  qa_coded_rows R;
  const int8_t* codes;
  const uint8_t* scales;
  const void* dy;
  float* out;                                      // dW, or a split's sums [n][cols]
  int64_t dy_stride, out_stride, split_stride, n;
  int64_t piece;                                   // rows of one split
  int64_t tiles_n;                                 // tiles along n
  int accumulate;
};

constexpr int kTileN = 128, kTileK = 128, kTileT = 32;      // columns of dY, columns of X, rows of both
constexpr int kChunks = 16;                        // 16-byte chunks of a tile's row

// A tile lies in LDS as rows of 128 bfloat16, as in memory; matrix instructions want eight rows of one column per
// lane, which the transposing reads give: of 16 lanes each reads four columns of one of four rows and receives four rows
// of one column.  Chunks of 16 bytes are swapped by their row so that the four rows lie in different banks.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * kTileK + (chunk ^ ((row & 3) << 2)) * kVec; }

__device__ __forceinline__ bf16x8 eight_rows(const __bf16* tile, int row0, int col0) {
  const int lane = threadIdx.x % 16, chunk = (col0 >> 3) + (lane >> 1 & 1), half = (lane & 1) * 4;
  bf16x8 v;
  s16x4 part[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(tile + chunk_at(row0 + 4 * h + (lane >> 2), chunk) + half));
  __builtin_memcpy(&v, part, sizeof v);
  return v;
}

// v as `P` bfloat16 parts, each the leading eight bits of what is left: exact for 8 P bits.
template <int P>
__device__ __forceinline__ void split_parts(float (&v)[kVec], u32x4 (&part)[P]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) part[p][i] = __builtin_amdgcn_perm(as_u32(v[2 * i + 1]), as_u32(v[2 * i]), 0x07060302u);
    if (p + 1 < P) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = v[i] - as_f32(as_u32(v[i]) & 0xFFFF0000u);
    }
  }
}
template <int TYPE> constexpr int parts_of = TYPE == QA_F32 ? 3 : TYPE == QA_F16 ? 2 : 1;

template <int TYPE>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(WeightGradArgs A) {
  typedef ElemT<TYPE> T;
  constexpr int P = parts_of<TYPE>;
  __shared__ __bf16 lds_dy[P][kTileT * kTileN];
  __shared__ __bf16 lds_x[kTileT * kTileK];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t n0 = (int64_t)(blockIdx.x % A.tiles_n) * kTileN, k0 = (int64_t)(blockIdx.x / A.tiles_n) * kTileK;
  const int64_t t_begin = (int64_t)blockIdx.y * A.piece, t_end = min(A.R.rows, t_begin + A.piece);
  const int row = threadIdx.x / 8, col = (threadIdx.x % 8) * 16;       // this thread's 16 elements of each tile
  const int wn = (wave & 1) * 64, wk = (wave >> 1) * 64;               // this wave's quarter of the output tile
  f32x16 acc[2][2] = {};
  const int left_n = (int)max((int64_t)0, min((int64_t)16, A.n - n0 - col));
  const bool has_x = k0 + col < A.R.cols;
  for (int64_t t0 = t_begin; t0 < t_end; t0 += kTileT) {
    const int64_t t = t0 + row;
    const bool here = t < t_end;
    float v[2][kVec] = {};
    if (here) {
      const T* p = (const T*)A.dy + t * A.dy_stride + n0 + col;
      to_f32<TYPE>(load_raw<TYPE>(p, left_n), v[0]);
      to_f32<TYPE>(load_raw<TYPE>(p + kVec, left_n - kVec), v[1]);
    }
    u32x4 code = {0, 0, 0, 0};
    float scale = 0.0f;
    if (here && has_x) {
      code = *reinterpret_cast<const u32x4*>(A.codes + t * A.R.code_stride + k0 + col);
      scale = scale_of(A.scales[t * A.R.scale_stride + (k0 + col) / A.R.group]);
    }
    __syncthreads();                               // the tiles of the round before have been read
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 part[P];
      split_parts<P>(v[h], part);
#pragma unroll
      for (int p = 0; p < P; ++p) *reinterpret_cast<u32x4*>(lds_dy[p] + chunk_at(row, col / 8 + h)) = part[p];
      u32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = code[2 * h + i / 2] >> (16 * (i % 2));
        const float lo = (float)(int8_t)w * scale, hi = (float)(int8_t)(w >> 8) * scale;
        x[i] = __builtin_amdgcn_perm(as_u32(hi), as_u32(lo), 0x07060302u);
      }
      *reinterpret_cast<u32x4*>(lds_x + chunk_at(row, col / 8 + h)) = x;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int row0 = 16 * s + 8 * (lane / 32), col0 = lane & 16;
      bf16x8 x[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) x[j] = eight_rows(lds_x, row0, wk + 32 * j + col0);
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bf16x8 d = eight_rows(lds_dy[p], row0, wn + 32 * i + col0);
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d, x[j], acc[i][j], 0, 0, 0);
        }
    }
  }
  float* out = A.out + (int64_t)blockIdx.y * A.split_stride;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t n = n0 + wn + 32 * i + 8 * (e / 4) + 4 * (lane / 32) + e % 4, k = k0 + wk + 32 * j + lane % 32;
        if (n < A.n && k < A.R.cols) {
          float* p = out + n * A.out_stride + k;
          *p = A.accumulate ? *p + acc[i][j][e] : acc[i][j][e];
        }
      }
}

// dW from the splits' sums, in their order.
__global__ __launch_bounds__(kThreads) void weight_grad_join_kernel(const float* __restrict__ parts, int splits, int64_t n, int64_t cols,
                                                                    float* dw, int64_t dw_stride, int accumulate) {
  const int64_t all = n * cols;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kThreads) {
    float s = splits ? parts[i] : 0.0f;
    for (int k = 1; k < splits; ++k) s += parts[k * all + i];
    float* p = dw + i / cols * dw_stride + i % cols;
    *p = accumulate ? *p + s : s;
  }
}

// ---- which form ----------------------------------------------------------------------------------------------

// Few tiles leave compute units idle: the rows are split then, 256 at least to a split, towards four work-groups per
// compute unit.
int64_t splits_for(int64_t rows, int64_t cols, int64_t n) {
  const int64_t tiles = ceil_div(n, kTileN) * ceil_div(cols, kTileK);
  return std::max<int64_t>(1, std::min(ceil_div(1024, tiles), rows / 256));
}

template <int TYPE>
int weight_grad_launch(WeightGradArgs& A, int64_t splits, hipStream_t stream) {
  const dim3 grid((unsigned)(A.tiles_n * ceil_div(A.R.cols, kTileK)), (unsigned)splits);
  weight_grad_kernel<TYPE><<<grid, kThreads, 0, stream>>>(A);
  return launch_status();
}

}  // namespace

size_t weight_grad_workspace_bytes(const qa_coded_rows* R, int, int64_t n) {
  const int64_t splits = splits_for(R->rows, R->cols, n);
  return splits == 1 ? 0 : (size_t)splits * (size_t)n * (size_t)R->cols * sizeof(float);
}

}  // namespace qa

using namespace qa;

extern "C" int qa_rows_weight_grad(const qa_coded_rows* rows, const int8_t* codes, const uint8_t* scales, int type,
                                   const void* dy, int64_t dy_stride, int64_t n, float* dw, int64_t dw_stride,
                                   int accumulate, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || n < 1 || n >= (int64_t(1) << 24) || dy_stride < n || dw_stride < rows->cols ||
      (accumulate != 0 && accumulate != 1) || !dw)
    return QA_ERR_INVALID_ARG;
  if (!aligned(dw, 4)) return QA_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  const int64_t all = n * rows->cols;
  const dim3 join((unsigned)std::min<int64_t>(ceil_div(all, kThreads), 4096));
  if (rows->rows == 0) {
    if (accumulate) return QA_OK;
    weight_grad_join_kernel<<<join, kThreads, 0, s>>>(nullptr, 0, n, rows->cols, dw, dw_stride, 0);
    return launch_status();
  }
  if (!codes || !scales || !dy) return QA_ERR_INVALID_ARG;
  if (!element_aligned(dy, type) || !aligned(codes, 16)) return QA_ERR_ALIGNMENT;
  const int64_t splits = splits_for(rows->rows, rows->cols, n);
  WeightGradArgs A{*rows, codes, scales, dy, dw, dy_stride, dw_stride, 0, n, rows->rows, ceil_div(n, kTileN), accumulate};
  if (splits > 1) {
    if (!ws || ws_bytes < weight_grad_workspace_bytes(rows, type, n)) return QA_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return QA_ERR_ALIGNMENT;
    A.out = (float*)ws;
    A.out_stride = rows->cols;
    A.split_stride = all;
    A.accumulate = 0;
    A.piece = ceil_div(ceil_div(rows->rows, splits), kTileT) * kTileT;
  }
  int rc = type == QA_F32    ? weight_grad_launch<QA_F32>(A, splits, s)
           : type == QA_BF16 ? weight_grad_launch<QA_BF16>(A, splits, s)
                             : weight_grad_launch<QA_F16>(A, splits, s);
  if (rc || splits == 1) return rc;
  weight_grad_join_kernel<<<join, kThreads, 0, s>>>((const float*)ws, (int)splits, n, rows->cols, dw, dw_stride, accumulate);
  return launch_status();
}
