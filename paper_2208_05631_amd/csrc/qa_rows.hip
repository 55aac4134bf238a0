// Rows of activations in 8 bits: coding them, decoding them, and the sizes of the workspaces of what reads them.
#include <algorithm>

#include "qa_rows.h"

namespace qa {

size_t rms_norm_grad_workspace_bytes(const qa_coded_rows* R, int type);
size_t weight_grad_workspace_bytes(const qa_coded_rows* R, int type, int64_t n);

namespace {

// A lane holds eight columns of a row, a group four to sixteen neighbouring lanes.  `per_row` lanes, a multiple of
// 16, cover a row; narrow rows share a work-group, wide ones are split over blockIdx.y.
//
// Eight work-groups per compute unit go over the rows: 144 us for the two calls of 16384 x 8192 bfloat16, and 155 with a work-group
// for each 2048 columns of a row.  Calls beyond the caches whose rows one work-group covers have 32 (262144 x 512: 137 us, with
// eight 144, without an end 154; 137096 x 979 180, 201 and 174; 994205 x 135 334, 350 and 320), others lose by as many (16384 x 8192: 165,
// 211060 x 64 25.5 and 21.9).
struct RowGrid {
  int per_row;      // lanes of a row that one work-group covers
  int rows;         // rows of one work-group
  dim3 grid;
};
RowGrid row_grid(int64_t rows, int64_t cols, bool beyond) {
  RowGrid g;
  const int64_t lanes = ceil_div(ceil_div(cols, kVec), 16) * 16;
  g.per_row = (int)(lanes < kThreads ? lanes : kThreads);
  g.rows = kThreads / g.per_row;
  const int64_t across = ceil_div(lanes, g.per_row);
  const int64_t most = across == 1 && beyond ? 8192 : std::max<int64_t>(2048 / across, 1);
  g.grid = dim3((unsigned)std::min<int64_t>(ceil_div(rows, g.rows), most), (unsigned)across);
  return g;
}

// One read, the group's largest magnitude from its lanes, one write.  Bound by memory: codes of 16384 x 8192 bfloat16 and their
// values again 144 us for the two calls, 813 MB at 5.6 TB/s (155 with reads that go through the caches); 333 x 2051: 10 us, two
// launches.
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(kThreads) void rows_pack_kernel(qa_coded_rows R, int per_row, int rows_per_group,
                                                             const ElemT<TYPE>* __restrict__ x, int64_t x_stride,
                                                             int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int local = threadIdx.x / per_row;
  const int64_t col = ((int64_t)blockIdx.y * per_row + (int)threadIdx.x % per_row) * kVec;
  const int n = local < rows_per_group && col < R.cols ? (int)min((int64_t)kVec, R.cols - col) : 0;
  const int lanes = R.group / kVec;
  for (int64_t first = (int64_t)blockIdx.x * rows_per_group; first < R.rows; first += (int64_t)gridDim.x * rows_per_group) {
    const int64_t row = first + local;
    const bool here = n > 0 && row < R.rows;
    float v[kVec] = {}, value[kVec];
    if (here) to_f32<TYPE>(load_raw<TYPE, STREAM>(x + row * x_stride + col, n), v);
    const uint32_t b = scale_byte(lanes_max_u32(most_of(v), lanes));
    if (here) {
      store_codes<STREAM>(codes + row * R.code_stride + col, code8(v, b, value), n);
      if ((threadIdx.x % lanes) == 0) scales[row * R.scale_stride + col / R.group] = (uint8_t)b;
    }
  }
}

template <int TYPE, bool STREAM>
__global__ __launch_bounds__(kThreads) void rows_unpack_kernel(qa_coded_rows R, int per_row, int rows_per_group,
                                                               const int8_t* __restrict__ codes,
                                                               const uint8_t* __restrict__ scales,
                                                               ElemT<TYPE>* __restrict__ x, int64_t x_stride) {
  const int local = threadIdx.x / per_row;
  const int64_t col = ((int64_t)blockIdx.y * per_row + (int)threadIdx.x % per_row) * kVec;
  if (local >= rows_per_group || col >= R.cols) return;
  const int n = (int)min((int64_t)kVec, R.cols - col);
  for (int64_t row = (int64_t)blockIdx.x * rows_per_group + local; row < R.rows;
       row += (int64_t)gridDim.x * rows_per_group) {
    float v[kVec];
    const u32x2* code = reinterpret_cast<const u32x2*>(codes + row * R.code_stride + col);
    decode8(STREAM ? __builtin_nontemporal_load(code) : *code, scales[row * R.scale_stride + col / R.group], v);
    store_raw<TYPE, STREAM>(x + row * x_stride + col, from_f32<TYPE>(v), n);
  }
}

bool beyond_caches(const qa_coded_rows* R, int type) {
  return streams((double)R->rows * (double)R->cols * (double)(type_bytes(type) + 1));
}

template <int TYPE>
int pack_launch(const qa_coded_rows* R, const void* x, int64_t x_stride, int8_t* codes, uint8_t* scales,
                hipStream_t stream) {
  // Narrow rows of binary32 that begin inside 16 bytes are not read past the caches (497102 x 135: the two calls 168 us, and 195 if so).
  const bool beyond = beyond_caches(R, TYPE), past = beyond && !(TYPE == QA_F32 && R->cols <= 512 && x_stride % 4);
  const RowGrid g = row_grid(R->rows, R->cols, beyond);
  const auto kernel = past ? rows_pack_kernel<TYPE, true> : rows_pack_kernel<TYPE, false>;
  kernel<<<g.grid, kThreads, 0, stream>>>(*R, g.per_row, g.rows, (const ElemT<TYPE>*)x, x_stride, codes, scales);
  return launch_status();
}
template <int TYPE>
int unpack_launch(const qa_coded_rows* R, const int8_t* codes, const uint8_t* scales, void* x, int64_t x_stride,
                  hipStream_t stream) {
  const bool beyond = beyond_caches(R, TYPE);
  const RowGrid g = row_grid(R->rows, R->cols, beyond);
  const auto kernel = beyond ? rows_unpack_kernel<TYPE, true> : rows_unpack_kernel<TYPE, false>;
  kernel<<<g.grid, kThreads, 0, stream>>>(*R, g.per_row, g.rows, codes, scales, (ElemT<TYPE>*)x, x_stride);
  return launch_status();
}

}  // namespace
}  // namespace qa

using namespace qa;

extern "C" size_t qa_rows_workspace_bytes(const qa_coded_rows* rows, int op, int type, int64_t n) {
  if (check_rows(rows) != QA_OK || !known_type(type)) return 0;
  if (op == QA_OP_NORM_GRAD) return rms_norm_grad_workspace_bytes(rows, type);
  if (op == QA_OP_WEIGHT_GRAD && n >= 1 && n < (int64_t(1) << 24)) return weight_grad_workspace_bytes(rows, type, n);
  return 0;
}

extern "C" int qa_rows_pack(const qa_coded_rows* rows, int type, const void* x, int64_t x_stride, int8_t* codes,
                            uint8_t* scales, void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || x_stride < rows->cols) return QA_ERR_INVALID_ARG;
  if (rows->rows == 0) return QA_OK;
  if (!x || !codes || !scales) return QA_ERR_INVALID_ARG;
  if (!element_aligned(x, type) || !aligned(codes, 16)) return QA_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return pack_launch<QA_F32>(rows, x, x_stride, codes, scales, s);
  if (type == QA_BF16) return pack_launch<QA_BF16>(rows, x, x_stride, codes, scales, s);
  return pack_launch<QA_F16>(rows, x, x_stride, codes, scales, s);
}

extern "C" int qa_rows_unpack(const qa_coded_rows* rows, const int8_t* codes, const uint8_t* scales, int type,
                              void* x_out, int64_t x_stride, void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || x_stride < rows->cols) return QA_ERR_INVALID_ARG;
  if (rows->rows == 0) return QA_OK;
  if (!x_out || !codes || !scales) return QA_ERR_INVALID_ARG;
  if (!element_aligned(x_out, type) || !aligned(codes, 16)) return QA_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return unpack_launch<QA_F32>(rows, codes, scales, x_out, x_stride, s);
  if (type == QA_BF16) return unpack_launch<QA_BF16>(rows, codes, scales, x_out, x_stride, s);
  return unpack_launch<QA_F16>(rows, codes, scales, x_out, x_stride, s);
}
