// Root-mean-square norm of a residual stream with an output in 8 bits, and its backward pass.
//
// Both are bound by memory, hold a row in registers between its sum and its outputs, and read the next row meanwhile.  Forward, 8192 x
// 4096 bfloat16 with everything written: 303 MB in 52 us, 5.8 TB/s; one row of 8192: 1.5 us of device time in a call of 6.  Backward,
// 16384 x 4096 with the gradient that comes past the norm: 537 MB in 88 us, 6.1 TB/s.  Rows that end inside a vector cost more: 8192 x
// 4097 71 us and 76, 8192 x 4104 59 and 62.  That is neither where they begin (4097 columns in rows of 4104 elements take as long) nor the
// stores of their last elements (69 without these).
#include <algorithm>
#include <type_traits>

#include "qa_rows.h"

namespace qa {
namespace {

// A row is held in the registers of LANES lanes, NV vectors of eight columns each: one read of everything.  Rows of
// up to 1024 columns lie inside a wave and need no barrier; of up to 128, the norms of attention heads, four do, of up to 64 eight.
// (524288 rows of 128 bfloat16: 100 us, and 301 with a wave for each; of 64: 51, and 85 with sixteen lanes.)
constexpr int kHeldCols = 16384;                   // 16 waves, two vectors per lane; longer rows are read twice

// Sum over the LANES lanes of a row.  `lds` holds a float for each of their waves that no other call uses before the next
// barrier but one: the callers alternate between two.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  if constexpr (LANES < kWave) {
    v += as_f32(other_lane<1>(as_u32(v)));
    v += as_f32(other_lane<2>(as_u32(v)));
    v += as_f32(other_lane<4>(as_u32(v)));
    if constexpr (LANES >= 16) v += as_f32(other_lane<8>(as_u32(v)));
    if constexpr (LANES == 32) v += as_f32(other_lane<16>(as_u32(v)));
    return v;
  } else {
    v = wave_sum_f32(v);
    if constexpr (LANES == kWave) return v;
    constexpr int W = LANES / kWave;
    if ((threadIdx.x % kWave) == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) s += lds[w];
    return s;
  }
}

// The next row is read ahead where that leaves registers for five waves per SIMD forward and three backward.  (16384 columns backward,
// which would spill: 195 us -> 218.)
template <int TYPE, int LANES, int NV> constexpr bool kAhead = LANES < 1024 && !(TYPE == QA_F32 && NV == 2);
template <int LANES> constexpr int kLeast = LANES < 1024 ? 5 : 4;
template <int LANES> constexpr int kLeastGrad = LANES < 1024 ? 3 : 4;

// Eight columns of a row from `col`, of which it has n.  The end of a row is read from its last eight elements, and placed() moves
// them to where they belong: a branch around a load waits for it, and rows are read ahead.  (16384 x 2047 bfloat16, backward: 80 us ->
// 69 in all.)  Rows of fewer than eight columns, of the narrowest form, are read by elements, and
// those of sixteen waves, which have no registers for this.
template <typename I>
struct Place {
  I at;                                            // read from here
  int shift;
};
template <int LANES, typename I>
__device__ __forceinline__ Place<I> place_of(I col, int n, I cols) {
  if (LANES == 1024) return {col, 0};
  if (LANES == 8 && cols < kVec) return {0, 0};
  return {min(col, cols - kVec), max(0, min(kVec, kVec - n))};
}
template <int TYPE, bool STREAM, int LANES, typename I>
__device__ __forceinline__ Raw8<TYPE> load_place(const ElemT<TYPE>* row, Place<I> place, int n, int64_t cols) {
  if (LANES == 1024 || (LANES == 8 && cols < kVec)) return load_raw<TYPE, STREAM>(row + place.at, n);
  return load_raw<TYPE, STREAM>(row + place.at);
}
template <typename I>
__device__ __forceinline__ void placed(Place<I> place, float (&v)[kVec]) {
  if (place.shift == 0) return;
#pragma unroll
  for (int by = 1; by <= kVec; by *= 2)
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (place.shift & by) v[i] = i + by < kVec ? v[i + by] : 0.0f;
}

struct NormArgs {
  qa_coded_rows R;
  const void* x;
  const void* residual;
  const float* weight;
  void* h;
  int8_t* codes;
  uint8_t* scales;
  __bf16* y;
  float* rstd;
  int64_t x_stride, residual_stride, h_stride, y_stride;
  float eps;
  bool stream;
};

template <int LANES> constexpr int threads_of = LANES <= kWave ? kThreads : LANES;
template <int LANES> constexpr int rows_of = threads_of<LANES> / LANES;
template <int LANES> constexpr int waves_of = LANES <= kWave ? 1 : LANES / kWave;

// Codes and values of eight columns of y, which their lane and its neighbours of the same group hold.
template <int LANES, bool STREAM>
__device__ __forceinline__ void write_y(const NormArgs& A, int64_t row, int64_t col, int n, const float (&y)[kVec]) {
  const int lanes = LANES < 16 ? min(A.R.group / kVec, LANES) : A.R.group / kVec;  // of one row
  const uint32_t b = scale_byte(lanes_max_u32(most_of(y), lanes));
  if (n <= 0) return;
  float value[kVec];
  const u32x2 code = code8(y, b, value);
  if (A.codes) {
    store_codes<STREAM>(A.codes + row * A.R.code_stride + col, code, n);
    if ((threadIdx.x % lanes) == 0) A.scales[row * A.R.scale_stride + col / A.R.group] = (uint8_t)b;
  }
  if (A.y) store_raw<QA_BF16, STREAM>(A.y + row * A.y_stride + col, from_f32<QA_BF16>(value), n);
}

template <int TYPE, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(threads_of<LANES>) __attribute__((amdgpu_waves_per_eu(kLeast<LANES>))) void rms_norm_kernel(NormArgs A) {
  typedef ElemT<TYPE> T;
  __shared__ float sums[2][waves_of<LANES>];
  const int t = threadIdx.x % LANES;
  const int64_t step = (int64_t)gridDim.x * rows_of<LANES>;
  const int cols = (int)A.R.cols;
  int col[NV], n[NV];
  Place<int> place[NV];
  float w[NV][kVec];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    col[v] = (v * LANES + t) * kVec;
    n[v] = min(kVec, cols - col[v]);
    place[v] = place_of<LANES>(col[v], n[v], cols);
    to_f32<QA_F32>(load_raw<QA_F32>(A.weight + col[v], n[v]), w[v]);
  }
  Raw8<TYPE> x[NV], r[NV];
  auto read = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v] = load_place<TYPE, STREAM, LANES>((const T*)A.x + row * A.x_stride, place[v], n[v], cols);
    if (A.residual) {
#pragma unroll
      for (int v = 0; v < NV; ++v) r[v] = load_place<TYPE, STREAM, LANES>((const T*)A.residual + row * A.residual_stride, place[v], n[v], cols);
    }
  };
  int turn = 0;
  int64_t row = (int64_t)blockIdx.x * rows_of<LANES> + threadIdx.x / LANES;
  if (kAhead<TYPE, LANES, NV> && row < A.R.rows) read(row);
  for (; row < A.R.rows; row += step) {
    if (!kAhead<TYPE, LANES, NV>) read(row);
    float h[NV][kVec], s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      to_f32<TYPE>(x[v], h[v]);
      if (A.residual) {
        float more[kVec];
        to_f32<TYPE>(r[v], more);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[v][i] += more[i];
      }
      placed(place[v], h[v]);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s = __builtin_fmaf(h[v][i], h[v][i], s);
    }
    if (kAhead<TYPE, LANES, NV> && row + step < A.R.rows) read(row + step);
    const float rstd = 1.0f / sqrtf(row_sum<LANES>(s, sums[turn]) / (float)A.R.cols + A.eps);
    turn ^= 1;
    if (A.rstd && t == 0) A.rstd[row] = rstd;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (A.h && n[v] > 0) store_raw<TYPE, STREAM>((T*)A.h + row * A.h_stride + col[v], from_f32<TYPE>(h[v]), n[v]);
      float y[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) y[i] = (h[v][i] * rstd) * w[v][i];
      write_y<LANES, STREAM>(A, row, col[v], n[v], y);
    }
  }
}

// Rows that registers do not hold: 16 waves per row, x and residual read twice.  A lane writes h where it has itself
// read x and residual for the last time, so h may be either of them.
template <int TYPE>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(NormArgs A) {
  typedef ElemT<TYPE> T;
  __shared__ float sums[2][16];
  int turn = 0;
  const int64_t pieces = ceil_div(A.R.cols, (int64_t)1024 * kVec);
  for (int64_t row = blockIdx.x; row < A.R.rows; row += gridDim.x) {
    const T* x = (const T*)A.x + row * A.x_stride;
    const T* r = A.residual ? (const T*)A.residual + row * A.residual_stride : nullptr;
    auto stream = [&](int64_t col, int n, float (&h)[kVec]) {
      to_f32<TYPE>(load_raw<TYPE>(x + col, n), h);
      if (r) {
        float more[kVec];
        to_f32<TYPE>(load_raw<TYPE>(r + col, n), more);
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[i] += more[i];
      }
    };
    float s = 0.0f;
    for (int64_t p = 0; p < pieces; ++p) {
      const int64_t col = (p * 1024 + threadIdx.x) * kVec;
      float h[kVec];
      stream(col, (int)min((int64_t)kVec, A.R.cols - col), h);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s = __builtin_fmaf(h[i], h[i], s);
    }
    const float rstd = 1.0f / sqrtf(row_sum<1024>(s, sums[turn]) / (float)A.R.cols + A.eps);
    turn ^= 1;
    if (A.rstd && threadIdx.x == 0) A.rstd[row] = rstd;
    for (int64_t p = 0; p < pieces; ++p) {
      const int64_t col = (p * 1024 + threadIdx.x) * kVec;
      const int n = (int)min((int64_t)kVec, A.R.cols - col);
      float h[kVec], w[kVec], y[kVec];
      stream(col, n, h);
      to_f32<QA_F32>(load_raw<QA_F32>(A.weight + col, n), w);
      if (A.h && n > 0) store_raw<TYPE>((T*)A.h + row * A.h_stride + col, from_f32<TYPE>(h), n);
#pragma unroll
      for (int i = 0; i < kVec; ++i) y[i] = (h[i] * rstd) * w[i];
      write_y<1024, false>(A, row, col, n, y);
    }
  }
}

// ---- backward ----------------------------------------------------------------------------------------------

struct NormGradArgs {
  qa_coded_rows R;
  const void* dy;
  const void* h;
  const int8_t* codes;
  const uint8_t* scales;
  const float* weight;
  const float* rstd;
  const void* dh;
  void* dx;
  float* parts;                                    // sums over the rows of one work-group; NULL: not wanted
  int64_t dy_stride, h_stride, dh_stride, dx_stride;
  bool stream;
};

// Eight columns of the residual stream, of its own type or codes, as they are in memory.
template <int TYPE, bool CODED> struct RawH { Raw8<TYPE> h; };
template <int TYPE> struct RawH<TYPE, true> { u32x2 code; uint32_t scale; };
template <int TYPE, bool CODED, bool STREAM, int LANES, typename I>
__device__ __forceinline__ RawH<TYPE, CODED> load_h(const NormGradArgs& A, int64_t row, I col, Place<I> place, int n) {
  RawH<TYPE, CODED> raw;
  if constexpr (CODED) {                           // no branch: one would wait for the loads at its end
    if (n <= 0) col = 0;
    raw.code = *reinterpret_cast<const u32x2*>(A.codes + row * A.R.code_stride + col);
    raw.scale = A.scales[row * A.R.scale_stride + (col >> __builtin_ctz(A.R.group))];
  } else {
    raw.h = load_place<TYPE, STREAM, LANES>((const ElemT<TYPE>*)A.h + row * A.h_stride, place, n, A.R.cols);
  }
  return raw;
}
template <int TYPE, bool CODED, typename I>
__device__ __forceinline__ void values_of(const RawH<TYPE, CODED>& raw, Place<I> place, int n, float (&h)[kVec]) {
  if constexpr (CODED) {
    decode8(raw.code, raw.scale, h);
#pragma unroll
    for (int i = 0; i < kVec; ++i) h[i] = i < n ? h[i] : 0.0f;
  } else {
    to_f32<TYPE>(raw.h, h);
    placed(place, h);
  }
}

template <int TYPE, int LANES, int NV, bool CODED, bool STREAM>
__global__ __launch_bounds__(threads_of<LANES>) __attribute__((amdgpu_waves_per_eu(kLeastGrad<LANES>))) void rms_norm_grad_kernel(NormGradArgs A) {
  typedef ElemT<TYPE> T;
  __shared__ float sums[2][waves_of<LANES>];
  const int t = threadIdx.x % LANES;
  const int64_t first = (int64_t)blockIdx.x * rows_of<LANES> + threadIdx.x / LANES;
  const int cols = (int)A.R.cols;
  int col[NV], n[NV];
  Place<int> place[NV];
  float w[NV][kVec], dw[NV][kVec];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    col[v] = (v * LANES + t) * kVec;
    n[v] = min(kVec, cols - col[v]);
    place[v] = place_of<LANES>(col[v], n[v], cols);
    to_f32<QA_F32>(load_raw<QA_F32>(A.weight + col[v], n[v]), w[v]);
#pragma unroll
    for (int i = 0; i < kVec; ++i) dw[v][i] = 0.0f;
  }
  const int64_t step = (int64_t)gridDim.x * rows_of<LANES>;
  Raw8<TYPE> next_dy[NV], next_dh[NV];
  RawH<TYPE, CODED> next_h[NV];
  float next_rstd = 0.0f;
  auto read = [&](int64_t row) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      next_dy[v] = load_place<TYPE, STREAM, LANES>((const T*)A.dy + row * A.dy_stride, place[v], n[v], cols);
      next_h[v] = load_h<TYPE, CODED, STREAM, LANES>(A, row, col[v], place[v], n[v]);
    }
    next_rstd = A.rstd[row];
  };
  auto read_dh = [&](Raw8<TYPE> (&dh)[NV], int64_t row) {
    if (!A.dh) return;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      dh[v] = load_place<TYPE, STREAM, LANES>((const T*)A.dh + row * A.dh_stride, place[v], n[v], cols);
  };
  // Codes take the registers that reading dh ahead takes, and those of two vectors per lane inside a wave lose by any reading ahead
  // (42744 x 785 bfloat16: 54 us, and 71).
  constexpr bool AHEAD = kAhead<TYPE, LANES, NV> && !(CODED && LANES == kWave && NV == 2), DH_AHEAD = AHEAD && !CODED;
  int turn = 0;
  if (AHEAD && first < A.R.rows) read(first);
  if (DH_AHEAD && first < A.R.rows) read_dh(next_dh, first);
  for (int64_t row = first; row < A.R.rows; row += step) {
    if (!AHEAD) read(row);
    if (!DH_AHEAD) read_dh(next_dh, row);
    Raw8<TYPE> dy_raw[NV], dh_raw[NV];
    float h[NV][kVec];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      dy_raw[v] = next_dy[v];
      if (A.dh) dh_raw[v] = next_dh[v];
      values_of<TYPE, CODED>(next_h[v], place[v], n[v], h[v]);
    }
    const float rstd = next_rstd;
    if (AHEAD && row + step < A.R.rows) read(row + step);
    if (DH_AHEAD && row + step < A.R.rows) read_dh(next_dh, row + step);
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float dy[kVec];
      to_f32<TYPE>(dy_raw[v], dy);
      placed(place[v], dy);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        h[v][i] *= rstd;                           // n
        s = __builtin_fmaf(dy[i] * w[v][i], h[v][i], s);
        dw[v][i] = __builtin_fmaf(dy[i], h[v][i], dw[v][i]);
      }
    }
    const float c = row_sum<LANES>(s, sums[turn]) / (float)A.R.cols;
    turn ^= 1;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float dy[kVec], dx[kVec];
      if constexpr (TYPE != QA_F32) asm("" : "+v"(dy_raw[v].a));  // what is kept is the words, not what they were converted to
      to_f32<TYPE>(dy_raw[v], dy);
      placed(place[v], dy);
#pragma unroll
      for (int i = 0; i < kVec; ++i) dx[i] = rstd * (dy[i] * w[v][i] - h[v][i] * c);
      if (A.dh) {
        float dh[kVec];
        if constexpr (TYPE != QA_F32) asm("" : "+v"(dh_raw[v].a));
        to_f32<TYPE>(dh_raw[v], dh);
        placed(place[v], dh);
#pragma unroll
        for (int i = 0; i < kVec; ++i) dx[i] += dh[i];
      }
      if (n[v] > 0) store_raw<TYPE, STREAM>((T*)A.dx + row * A.dx_stride + col[v], from_f32<TYPE>(dx), n[v]);
    }
  }
  if (!A.parts) return;
  if constexpr (LANES <= kWave) {                  // the work-group's rows have the same columns
    __shared__ f32x4 others[kWaves - 1][2 * NV][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if constexpr (LANES <= 8) dw[v][i] += as_f32(other_lane<8>(as_u32(dw[v][i])));
        if constexpr (LANES <= 16) dw[v][i] += as_f32(other_lane<16>(as_u32(dw[v][i])));
        if constexpr (LANES <= 32) dw[v][i] += as_f32(other_lane<32>(as_u32(dw[v][i])));
      }
    if (wave > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Raw8<QA_F32> r = from_f32<QA_F32>(dw[v]);
        others[wave - 1][2 * v][lane] = r.a;
        others[wave - 1][2 * v + 1][lane] = r.b;
      }
    }
    __syncthreads();
    if (threadIdx.x >= LANES) return;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) dw[v][i] += others[w][2 * v + i / 4][lane][i % 4];
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (n[v] > 0) store_raw<QA_F32>(A.parts + (int64_t)blockIdx.x * A.R.cols + col[v], from_f32<QA_F32>(dw[v]), n[v]);
}

// Rows that registers do not hold: everything is read twice, and a work-group's sums lie in the workspace.
template <int TYPE, bool CODED>
__global__ __launch_bounds__(1024) void rms_norm_grad_long_kernel(NormGradArgs A) {
  typedef ElemT<TYPE> T;
  __shared__ float sums[2][16];
  int turn = 0;
  const int64_t pieces = ceil_div(A.R.cols, (int64_t)1024 * kVec);
  for (int64_t row = blockIdx.x; row < A.R.rows; row += gridDim.x) {
    const T* dy_row = (const T*)A.dy + row * A.dy_stride;
    const float rstd = A.rstd[row];
    float s = 0.0f;
    for (int64_t p = 0; p < pieces; ++p) {
      const int64_t col = (p * 1024 + threadIdx.x) * kVec;
      const int n = (int)min((int64_t)kVec, A.R.cols - col);
      float dy[kVec], h[kVec], w[kVec];
      to_f32<TYPE>(load_raw<TYPE>(dy_row + col, n), dy);
      const auto place = place_of<1024>(col, n, A.R.cols);
      values_of<TYPE, CODED>(load_h<TYPE, CODED, false, 1024>(A, row, col, place, n), place, n, h);
      to_f32<QA_F32>(load_raw<QA_F32>(A.weight + col, n), w);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s = __builtin_fmaf(dy[i] * w[i], h[i] * rstd, s);
    }
    const float c = row_sum<1024>(s, sums[turn]) / (float)A.R.cols;
    turn ^= 1;
    for (int64_t p = 0; p < pieces; ++p) {
      const int64_t col = (p * 1024 + threadIdx.x) * kVec;
      const int n = (int)min((int64_t)kVec, A.R.cols - col);
      if (n <= 0) continue;
      float dy[kVec], h[kVec], w[kVec], dw[kVec], dx[kVec];
      to_f32<TYPE>(load_raw<TYPE>(dy_row + col, n), dy);
      const auto place = place_of<1024>(col, n, A.R.cols);
      values_of<TYPE, CODED>(load_h<TYPE, CODED, false, 1024>(A, row, col, place, n), place, n, h);
      to_f32<QA_F32>(load_raw<QA_F32>(A.weight + col, n), w);
      float* part = A.parts ? A.parts + (int64_t)blockIdx.x * A.R.cols + col : nullptr;
      if (part && row != blockIdx.x) {
        to_f32<QA_F32>(load_raw<QA_F32>(part, n), dw);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) dw[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float v = h[i] * rstd;
        dw[i] = __builtin_fmaf(dy[i], v, dw[i]);
        dx[i] = rstd * (dy[i] * w[i] - v * c);
      }
      if (part) store_raw<QA_F32>(part, from_f32<QA_F32>(dw), n);
      if (A.dh) {
        float dh[kVec];
        to_f32<TYPE>(load_raw<TYPE>((const T*)A.dh + row * A.dh_stride + col, n), dh);
#pragma unroll
        for (int i = 0; i < kVec; ++i) dx[i] += dh[i];
      }
      store_raw<TYPE>((T*)A.dx + row * A.dx_stride + col, from_f32<TYPE>(dx), n);
    }
  }
}

// A work-group adds the weight's gradient over its rows in registers and leaves one sum per column: 4 bytes per column for every
// work-group, at most 1024 of them, where an atomic addition would make the result depend on their order.
//
// dweight from the sums of the work-groups, in their order: 64 columns per work-group, the parts split over its waves.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float* __restrict__ parts, int64_t n_parts, int64_t cols,
                                                           float* __restrict__ dweight, int accumulate) {
  __shared__ float sums[16][kWave];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t col = (int64_t)blockIdx.x * kWave + lane;
  float s = 0.0f;
  if (col < cols) {
    const int64_t i0 = n_parts * wave / 16, i1 = n_parts * (wave + 1) / 16;
#pragma unroll 16
    for (int64_t i = i0; i < i1; ++i) s += parts[i * cols + col];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < cols) {
    s = sums[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    dweight[col] = accumulate ? dweight[col] + s : s;
  }
}

// ---- which form -----------------------------------------------------------------------------------------------

// Lanes per row (0: the row is read twice) and vectors per lane.
struct Form { int lanes, vecs; };
Form form_of(int64_t cols) {
  if (cols <= 64) return {8, 1};
  if (cols <= 128) return {16, 1};
  if (cols <= 256) return {32, 1};
  if (cols <= 512) return {64, 1};
  if (cols <= 1024) return {64, 2};
  if (cols <= 2048) return {256, 1};
  if (cols <= 4096) return {256, 2};
  if (cols <= 8192) return {512, 2};
  if (cols <= kHeldCols) return {1024, 2};
  return {0, 0};
}
// Work-groups, from threads per compute unit.  Some 4096 columns at a time are to be on their way to each where rows are read ahead, and
// twice as many where they are codes; more are slower, by the rows that meet in memory and, backward, by the work-groups' sums
// (16384 x 4096 bfloat16, 256 threads, 512 and 1024: forward 101 us, 114 and 113, backward 87, 90 and 105).
int64_t groups_for(int64_t rows, Form f, int64_t threads_per_unit) {
  const int64_t threads = f.lanes == 0 ? 1024 : f.lanes <= kWave ? kThreads : f.lanes;
  return std::min<int64_t>(ceil_div(rows, f.lanes && f.lanes <= kWave ? kThreads / f.lanes : 1),
                           256 * std::max<int64_t>(threads_per_unit / threads, 1));
}
// Rows bring less where they leave lanes empty, where they come without a residual, and, measured, where a row of several waves ends inside
// a vector: twice the threads, and twice again for two of these with two vectors.  With one vector per lane (1024 threads and 512): 32263 x 1040 63 us and 91, 63550 x 272 33 and 41, but 20164 x 1664 56 and 55, 93206 x 360 68 and
// 62; without residual 16384 x 2048 45 and 46, 123361 x 272 58 and 81.  With two (512 and 256): 20000 x 2051 103 and 180, 10000 x 4095 84 and
// 109, but 10000 x 4000 69 and 65, 40000 x 1003, in one wave, 77 and 74; without residual 8192 x 4096 45 and 47, and (1024 and 512)
// 15307 x 2192 50 and 58, 8190 x 4097 54 and 60.  Calls that the caches hold are not slower with 512.
int64_t norm_groups(int64_t rows, int64_t cols, int type, bool residual, bool stream) {
  const Form f = form_of(cols);
  const int64_t full = f.lanes * f.vecs * kVec;
  const bool in_wave = f.lanes <= kWave;
  if (f.lanes == 0) return groups_for(rows, f, 1024);
  if (f.vecs == 1) return groups_for(rows, f, !residual || 8 * cols <= (in_wave ? 5 : 6) * full ? 1024 : 512);
  if (type == QA_F32) return groups_for(rows, f, 512);
  const bool filled = (cols % kVec == 0 || in_wave) && 4 * cols > 3 * full;
  if (residual) return groups_for(rows, f, filled && stream ? 256 : 512);
  return groups_for(rows, f, filled ? 512 : 1024);
}
// Backward the sums make small calls dearer: 30840 x 272 20.8 us with 512 threads, 19.4 with 1024, 10459 x 401 13.7 and 15.0, but 61680 x 272 37 and
// 32, 123361 x 272 73 and 62, 9847 x 1761 33 and 36; two vectors, 256 and 512: 16000 x 3000 85 and 72, 1913 x 2192 15.9 and 14.1, 10000 x 4095 81 and
// 77, but 2000 x 4095 21 and 23, 10000 x 4096 57 and 59.  Binary32 rows of one vector lose with 1024 (32263 x 1040: 105 and 111).
int64_t norm_grad_groups(int64_t rows, int64_t cols, int type, bool coded, bool stream) {
  const Form f = form_of(cols);
  const int64_t full = f.lanes * f.vecs * kVec;
  if (f.lanes == 0 || (type == QA_F32 && f.vecs == 2)) return groups_for(rows, f, 1024);
  if (coded) return groups_for(rows, f, f.vecs == 2 ? 512 : 1024);
  if (f.vecs == 1) return groups_for(rows, f, 6 * cols < 5 * full && type != QA_F32 && rows * cols >= 1 << 24 ? 1024 : 512);
  return groups_for(rows, f, 8 * cols < 7 * full || (stream && cols < full) ? 512 : 256);
}

// Calls `launch` with the lanes and vectors of a form as constants.
template <int LANES, int VECS, typename F>
bool launched(Form f, F launch) {
  if (f.lanes != LANES || f.vecs != VECS) return false;
  launch(std::integral_constant<int, LANES>{}, std::integral_constant<int, VECS>{});
  return true;
}
template <typename F>
bool with_form(Form f, F launch) {
  return launched<8, 1>(f, launch) || launched<16, 1>(f, launch) || launched<32, 1>(f, launch) || launched<64, 1>(f, launch) ||
         launched<64, 2>(f, launch) || launched<256, 1>(f, launch) || launched<256, 2>(f, launch) || launched<512, 2>(f, launch) ||
         launched<1024, 2>(f, launch);
}

template <int TYPE>
int norm_launch(const NormArgs& A, hipStream_t stream) {
  const Form f = form_of(A.R.cols);
  const dim3 grid((unsigned)norm_groups(A.R.rows, A.R.cols, TYPE, A.residual != nullptr, A.stream));
  auto held = [&](auto lanes, auto vecs) {
    constexpr bool STREAM = TYPE != QA_F32;
    if (STREAM && A.stream) rms_norm_kernel<TYPE, lanes, vecs, STREAM><<<grid, threads_of<lanes>, 0, stream>>>(A);
    else rms_norm_kernel<TYPE, lanes, vecs, false><<<grid, threads_of<lanes>, 0, stream>>>(A);
  };
  if (!with_form(f, held)) rms_norm_long_kernel<TYPE><<<grid, 1024, 0, stream>>>(A);
  return launch_status();
}

template <int TYPE, bool CODED>
int norm_grad_launch(const NormGradArgs& A, float* dweight, int accumulate, hipStream_t stream) {
  const Form f = form_of(A.R.cols);
  const dim3 grid((unsigned)norm_grad_groups(A.R.rows, A.R.cols, TYPE, CODED, A.stream));
  if (A.R.rows > 0) {
    auto held = [&](auto lanes, auto vecs) {
      constexpr bool STREAM = TYPE != QA_F32;
      if (STREAM && A.stream) rms_norm_grad_kernel<TYPE, lanes, vecs, CODED, STREAM><<<grid, threads_of<lanes>, 0, stream>>>(A);
      else rms_norm_grad_kernel<TYPE, lanes, vecs, CODED, false><<<grid, threads_of<lanes>, 0, stream>>>(A);
    };
    if (!with_form(f, held))
      rms_norm_grad_long_kernel<TYPE, CODED><<<grid, 1024, 0, stream>>>(A);
    if (const int rc = launch_status()) return rc;
  }
  if (!dweight) return QA_OK;
  norm_weight_kernel<<<dim3((unsigned)ceil_div(A.R.cols, kWave)), 1024, 0, stream>>>(
      A.parts, grid.x, A.R.cols, dweight, accumulate);
  return launch_status();
}
template <int TYPE>
int norm_grad_launch(const NormGradArgs& A, float* dweight, int accumulate, hipStream_t stream) {
  return A.codes ? norm_grad_launch<TYPE, true>(A, dweight, accumulate, stream)
                 : norm_grad_launch<TYPE, false>(A, dweight, accumulate, stream);
}

}  // namespace

size_t rms_norm_grad_workspace_bytes(const qa_coded_rows* R, int type) {
  return (size_t)norm_grad_groups(R->rows, R->cols, type, true, true) * (size_t)R->cols * sizeof(float);
}

}  // namespace qa

using namespace qa;

extern "C" int qa_rms_norm(const qa_coded_rows* rows, int type, const void* x, int64_t x_stride,
                           const void* residual, int64_t residual_stride, const float* weight, float eps,
                           void* h_out, int64_t h_stride, int8_t* codes, uint8_t* scales, void* y_out,
                           int64_t y_stride, float* rstd, void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || x_stride < rows->cols || (residual && residual_stride < rows->cols) ||
      (h_out && h_stride < rows->cols) || (y_out && y_stride < rows->cols) || !(eps >= 0.0f) || !(eps < 1e30f))
    return QA_ERR_INVALID_ARG;
  if (rows->rows == 0) return QA_OK;
  if (!x || !weight || !codes != !scales || (!codes && !y_out)) return QA_ERR_INVALID_ARG;
  if (!element_aligned(x, type) || !element_aligned(residual, type) || !element_aligned(h_out, type) ||
      !aligned(y_out, 2) || !aligned(weight, 4) || !aligned(rstd, 4) || !aligned(codes, 16))
    return QA_ERR_ALIGNMENT;
  const NormArgs A{*rows, x, residual, weight, h_out, codes, scales, (__bf16*)y_out, rstd,
                   x_stride, residual_stride, h_stride, y_stride, eps,
                   streams((double)rows->rows * (double)rows->cols *
                           (double)(type_bytes(type) * (1 + (residual != nullptr) + (h_out != nullptr)) + (codes != nullptr) + 2 * (y_out != nullptr)))};
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return norm_launch<QA_F32>(A, s);
  if (type == QA_BF16) return norm_launch<QA_BF16>(A, s);
  return norm_launch<QA_F16>(A, s);
}

extern "C" int qa_rms_norm_grad(const qa_coded_rows* rows, int type, const void* dy, int64_t dy_stride, const void* h,
                                int64_t h_stride, const int8_t* h_codes, const uint8_t* h_scales,
                                const float* weight, const float* rstd, const void* dh, int64_t dh_stride, void* dx,
                                int64_t dx_stride, float* dweight, int accumulate, void* ws, size_t ws_bytes,
                                void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || dy_stride < rows->cols || (h && h_stride < rows->cols) ||
      (dh && dh_stride < rows->cols) || dx_stride < rows->cols || (accumulate != 0 && accumulate != 1))
    return QA_ERR_INVALID_ARG;
  if (!aligned(dweight, 4)) return QA_ERR_ALIGNMENT;
  if (rows->rows > 0) {
    if (!dy || !weight || !rstd || !dx || !h == !h_codes || !h_codes != !h_scales) return QA_ERR_INVALID_ARG;
    if (!element_aligned(dy, type) || !element_aligned(h, type) || !element_aligned(dh, type) ||
        !element_aligned(dx, type) || !aligned(weight, 4) || !aligned(rstd, 4) || !aligned(h_codes, 16))
      return QA_ERR_ALIGNMENT;
    if (dweight && (!ws || ws_bytes < rms_norm_grad_workspace_bytes(rows, type))) return QA_ERR_WORKSPACE;
    if (dweight && !aligned(ws, 256)) return QA_ERR_ALIGNMENT;
  } else if (!dweight || accumulate) {
    return QA_OK;
  }
  const NormGradArgs A{*rows, dy, h, h_codes, h_scales, weight, rstd, dh, dx, dweight ? (float*)ws : nullptr,
                       dy_stride, h_stride, dh_stride, dx_stride,
                       streams((double)rows->rows * (double)rows->cols *
                               (double)(type_bytes(type) * (2 + (dh != nullptr)) + (h ? type_bytes(type) : 1)))};
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return norm_grad_launch<QA_F32>(A, dweight, accumulate, s);
  if (type == QA_BF16) return norm_grad_launch<QA_BF16>(A, dweight, accumulate, s);
  return norm_grad_launch<QA_F16>(A, dweight, accumulate, s);
}
