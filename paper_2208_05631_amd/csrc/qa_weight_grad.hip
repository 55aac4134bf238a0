// Weight gradient of a linear layer from the 8-bit codes of its input: dW = dY^T X.
//
// A code times its power of two is exact in bfloat16, and so are dY's elements, or two (binary16) or three (binary32)
// bfloat16 parts of them, so every product of the matrix cores is exact and the sums are held in binary32.
//
// 16384 rows, 8192 x 4096: 0.88-0.93 ms from card to card, 1.18-1.25 PFLOP/s; a bfloat16 product of the same shape by the library, from
// operands that are bfloat16 already, takes 1.06 ms, its largest square ones reach 1.35.  Bound by the card's power: it takes 1.57 million
// cycles, two thirds of which the matrix cores are busy, at 1.75 GHz of 2.4, and at 1.4 for some launches soon after a pause, which take 1.1 ms
// (four waves of 128 x 128 instead of eight of 128 x 64: half of the cycles at 2.0 GHz, 1.00 ms).  8192 rows, 4096 x 4096: bfloat16 0.23 ms,
// binary16 0.41, binary32 0.61.
#include <algorithm>

#include "qa_rows.h"
#include "qa_weight_plan.h"

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

constexpr int kStep = kWeightStep;                 // rows of both that lie in LDS at a time

// A tile's rows lie in LDS as bfloat16, as in memory; matrix instructions want eight rows of one column per lane, which
// the transposing reads give: of 16 lanes each reads four columns of one of four rows and receives four rows of one
// column.  A row is followed by 64 bytes of nothing, so that four rows lie in different banks.
constexpr int kGap = 32;                           // elements
template <int COLS>
__device__ __forceinline__ bf16x8 eight_rows(const __bf16* lane_at) {
  bf16x8 v;
  s16x4 part[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lane_at + 4 * h * (COLS + kGap)));
  __builtin_memcpy(&v, part, sizeof v);
  return v;
}

template <int TYPE> constexpr int parts_of = TYPE == QA_F32 ? 3 : TYPE == QA_F16 ? 2 : 1;

// The order of a phase's instructions: N times a matrix instruction and in its shadow READS reads of LDS, VECTOR vector instructions,
// WRITES writes to LDS and LOADS reads of memory.
template <int N, int READS, int VECTOR, int WRITES, int LOADS>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
    __builtin_amdgcn_sched_group_barrier(0x200, WRITES, 0);
    __builtin_amdgcn_sched_group_barrier(0x020, LOADS, 0);
  }
}

// WN x WK waves, FN x FK tiles of 32 x 32 each: a work-group has 32 WN FN columns of dY and 32 WK FK of X.  While one step's
// rows are multiplied the next ones' elements are on their way to registers, from where they go to LDS as bfloat16.  The codes
// are decoded there, once per tile: two and a half vector instructions per code, a third of the matrix instructions' time, and
// the 8 bits are all that is read of X.
template <int TYPE, int WN, int WK, int FN, int FK, bool EDGE>
struct Worker {
  typedef ElemT<TYPE> T;
  static constexpr int P = parts_of<TYPE>, kTile = 32 * WN * FN, kGroup = WN * WK * kWave;
  static_assert(WN * FN == WK * FK, "tiles are square");
  static constexpr int kDy = kStep * kTile / kVec / kGroup, kX = kStep * kTile / 16 / kGroup;       // vectors per thread
  static constexpr int kRow = kTile + kGap, kPart = kStep * kRow, kBuffer = (P + 1) * kPart;
  static constexpr int kBuffers = P == 1 ? 3 : 2;  // of 160 KiB
  static_assert(P == 1 || kDy + 2 <= 2 * P, "a step has a phase for each part of its work");
  // Steps whose elements are on their way (one in the large tile: 0.99 ms).  A step of a small tile takes a third of the time that a
  // read takes, unless dY has several parts: bfloat16, 4096 rows, 2048 x 2048: 53 us (with two 57), and binary16, 2048 rows: 45 (44).
  // Rows are taken kAhead steps at a time, so that one row costs 1.6 us more with four than with two.
  static constexpr int kAhead = FN * FK == 8 || P > 1 ? 2 : 4;

  const WeightGradArgs& A;
  int64_t n0, k0, t_end, t_load;
  const char* dy_from;                             // row t_load
  const int8_t* x_from;
  const uint8_t* scale_from;
  uint32_t dy_at[kDy], x_at[kX], scale_at[kX];     // bytes from there to this thread's vectors
  uint32_t dy_tail[kDy], x_tail[kX], scale_tail[kX];       // the same in the last step
  int left;                                        // columns of dY that this thread's vectors have
  int d_lane, x_lane;                              // where a lane reads in LDS
  struct Loaded { Raw8<TYPE> dy[kDy]; u32x4 code[kX]; uint32_t scale[kX]; };
  f32x16 acc[FN][FK];

  // Of dY eight elements, of X sixteen (eight, with writes to LDS side by side, take twice the reads: 2 % slower).
  static __device__ __forceinline__ int row_of(int v) { return (v * kGroup + (int)threadIdx.x) / (kTile / kVec); }
  static __device__ __forceinline__ int x_row(int v) { return (v * kGroup + (int)threadIdx.x) / (kTile / 16); }
  static __device__ __forceinline__ int x_chunk() { return threadIdx.x % (kTile / 16); }
  static __device__ __forceinline__ int chunk() { return threadIdx.x % (kTile / kVec); }

  __device__ __forceinline__ Worker(const WeightGradArgs& a, int64_t n, int64_t k, int64_t begin, int64_t end)
      : A(a), n0(n), k0(k), t_end(end), t_load(begin) {
    // A vector that the end cuts off, or that lies past it, is the last eight columns instead: write() knows.  With fewer
    // than eight columns (EDGE) elements are read one by one.
    const int64_t col = n0 + chunk() * kVec;
    left = (int)max((int64_t)0, min((int64_t)kVec, A.n - col));
    dy_from = (const char*)A.dy + begin * A.dy_stride * (int64_t)sizeof(T);
    x_from = A.codes + begin * A.R.code_stride;
    scale_from = A.scales + begin * A.R.scale_stride;
    const uint32_t dy_col = (uint32_t)(EDGE ? col : min(col, A.n - kVec)) * (uint32_t)sizeof(T);
    const uint32_t x_col = (uint32_t)min(k0 + x_chunk() * 16, (A.R.cols - 1) / 16 * 16);
    const uint32_t scale_col = x_col / (uint32_t)A.R.group;
    const int last = (int)((end - begin - 1) % kStep);
#pragma unroll
    for (int v = 0; v < kDy; ++v) {
      const uint32_t stride = (uint32_t)(A.dy_stride * (int64_t)sizeof(T));
      dy_at[v] = (uint32_t)row_of(v) * stride + dy_col;
      dy_tail[v] = (uint32_t)min(row_of(v), last) * stride + dy_col;
    }
#pragma unroll
    for (int v = 0; v < kX; ++v) {
      x_at[v] = (uint32_t)x_row(v) * (uint32_t)A.R.code_stride + x_col;
      x_tail[v] = (uint32_t)min(x_row(v), last) * (uint32_t)A.R.code_stride + x_col;
      scale_at[v] = (uint32_t)x_row(v) * (uint32_t)A.R.scale_stride + scale_col;
      scale_tail[v] = (uint32_t)min(x_row(v), last) * (uint32_t)A.R.scale_stride + scale_col;
    }
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int at = (8 * (lane / 32) + (lane % 16 >> 2)) * kRow + (lane & 16) + (lane & 3) * 4;
    d_lane = at + wave % WN * 32 * FN;
    x_lane = at + wave / WN * 32 * FK;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FK; ++j) acc[i][j] = f32x16{};
  }
  // The next step's elements.  Rows past the end are read from the last one, steps past the end from the last step.
  __device__ __forceinline__ void load(Loaded& to) {
    const bool tail = t_load + kStep >= t_end;
#pragma unroll
    for (int v = 0; v < kDy; ++v) {
      const T* p = (const T*)(dy_from + (tail ? dy_tail[v] : dy_at[v]));
      to.dy[v] = EDGE ? load_raw<TYPE>(p, left) : load_raw<TYPE>(p);
    }
#pragma unroll
    for (int v = 0; v < kX; ++v) {
      to.code[v] = *reinterpret_cast<const u32x4*>(x_from + (tail ? x_tail[v] : x_at[v]));
      to.scale[v] = scale_from[tail ? scale_tail[v] : scale_at[v]];
    }
    const int64_t go = tail ? 0 : -1;              // no branch: the matrix instructions around this are one block
    t_load += kStep & go;
    dy_from += (kStep * A.dy_stride * (int64_t)sizeof(T)) & go;
    x_from += (kStep * A.R.code_stride) & go;
    scale_from += (kStep * A.R.scale_stride) & go;
  }
  __device__ __forceinline__ void store_dy(Loaded& from, int v, __bf16* lds) {
    float f[kVec];
    u32x4 part[P];
    if constexpr (TYPE == QA_BF16) {
      part[0] = from.dy[v].a;
    } else {
      to_f32<TYPE>(from.dy[v], f);
      split_parts<P>(f, part);
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
      *reinterpret_cast<u32x4*>(lds + p * kPart + row_of(v) * kRow + chunk() * kVec) = part[p];
  }
  // X is 0 past the end.
  __device__ __forceinline__ void store_x(Loaded& from, __bf16* lds, int64_t t0) {
    // A signed byte times its scale: exact, and finite for every scale that a finite group has (a bias taken off behind the scaling
    // would be infinite from 2^121 on).  The zeros are not known to the compiler, which would take a code's bytes apart, and wait
    // for them, where they are loaded.
    uint32_t none;
    asm("s_mov_b32 %0, 0" : "=s"(none));
#pragma unroll
    for (int v = 0; v < kX; ++v) {
      const float s = t0 + x_row(v) < t_end ? scale_of(from.scale[v]) : 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w = from.code[v][2 * h + i / 2] ^ none;
          const float lo = (float)(int8_t)(w >> (16 * (i % 2))) * s, hi = (float)(int8_t)(w >> (16 * (i % 2) + 8)) * s;
          x[i] = __builtin_amdgcn_perm(as_u32(hi), as_u32(lo), 0x07060302u);
        }
        *reinterpret_cast<u32x4*>(lds + P * kPart + x_row(v) * kRow + x_chunk() * 16 + h * kVec) = x;
      }
    }
  }
  // A step has 2 P phases of FN x FK matrix instructions, each for 16 rows and one part of dY.  A phase's operands are read
  // while the one before it is multiplied, the first one's of the next step, too, where there are three buffers: the
  // one that is read next is complete then before the step begins.
  bf16x8 d[2][FN], x[2][FK];
  __device__ __forceinline__ void operands(const __bf16* lds, int phase) {
    const int s = phase / P, p = phase % P;
    if (p == 0) {
#pragma unroll
      for (int j = 0; j < FK; ++j) x[s & 1][j] = eight_rows<kTile>(lds + x_lane + (P * kPart + 16 * s * kRow + 32 * j));
    }
#pragma unroll
    for (int i = 0; i < FN; ++i) d[phase & 1][i] = eight_rows<kTile>(lds + d_lane + (p * kPart + 16 * s * kRow + 32 * i));
  }
  __device__ __forceinline__ void multiply(int phase) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FK; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(d[phase & 1][i], x[phase / P & 1][j], acc[i][j], 0, 0, 0);
  }
  // One step: the buffer `now` is multiplied, what was loaded for the step that is kBuffers - 1 ahead goes to `last`.  What is to be
  // done beside the matrix instructions is laid out over as many phases as there are, and inside a phase it stands in their
  // shadow: left to the compiler the reads of LDS and the decoding stand together in front of them (large bfloat16 tiles: 1.04 ms
  // instead of 0.94).  It is told that the three lie apart.  With two buffers the next one is the one that is written: it is
  // read behind the step only, and `now` stands in its place here.
  template <int PHASE>
  static __device__ __forceinline__ void phases(Worker& w, Loaded& loaded, int64_t t, const __bf16* __restrict__ now,
                                                const __bf16* __restrict__ next, __bf16* __restrict__ last) {
    constexpr int kAll = FN * FK, kXPhase = P == 1 ? 0 : kDy, kLoadPhase = kXPhase + 1;
    if constexpr (PHASE + 1 < 2 * P) w.operands(now, PHASE + 1);
    else if constexpr (kBuffers == 3) w.operands(next, 0);
#pragma unroll
    for (int v = 0; v < kDy; ++v)
      if (PHASE == (P == 1 ? 0 : v)) w.store_dy(loaded, v, last);
    if constexpr (PHASE == kXPhase) w.store_x(loaded, last, t + (kBuffers - 1) * kStep);
    if constexpr (PHASE == kLoadPhase) w.load(loaded);
    w.multiply(PHASE);
    if constexpr (P == 1 && kAll == 8 && PHASE == 0) {
      interleave<4, 3, 4, 0, 0>();
      interleave<4, 0, 10, 1, 0>();
    } else if constexpr (P == 1 && kAll == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        interleave<1, 2, 2, 0, 0>();
        interleave<1, 2, 2, 0, 1>();
      }
    } else if constexpr (P > 1 && PHASE < kDy) {
      interleave<kAll, 8 / kAll, (P == 3 ? 64 : 36) / kAll, 1, 0>();
    } else if constexpr (P > 1 && PHASE == kXPhase) {
      interleave<kAll, 8 / kAll, 48 * kX / kAll, 1, 0>();
    } else if constexpr (P > 1) {
      interleave<kAll, 8 / kAll, 16 / kAll, 0, 8 / kAll>();
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PHASE + 1 < 2 * P) phases<PHASE + 1>(w, loaded, t, now, next, last);
  }
  static __device__ __forceinline__ void step(Worker& w, Loaded& loaded, int64_t t, const __bf16* __restrict__ now,
                                              const __bf16* __restrict__ next, __bf16* __restrict__ last) {
    phases<0>(w, loaded, t, now, next, last);
    __syncthreads();
  }
  __device__ __forceinline__ void run(int64_t t_begin, __bf16* lds) {
    Loaded loaded[kAhead];                         // step i's in i % kAhead
#pragma unroll
    for (int a = 0; a < kAhead; ++a) load(loaded[a]);
#pragma unroll
    for (int b = 0; b + 1 < kBuffers; ++b) {
#pragma unroll
      for (int v = 0; v < kDy; ++v) store_dy(loaded[b % kAhead], v, lds + b * kBuffer);
      store_x(loaded[b % kAhead], lds + b * kBuffer, t_begin + b * kStep);
      load(loaded[b % kAhead]);
    }
    __syncthreads();
    int now = 0, next = kBuffer, last = (kBuffers - 1) * kBuffer;          // read, read next, written
    operands(lds, 0);
    for (int64_t t = t_begin; t < t_end;) {        // X is 0 in a step past the end
#pragma unroll
      for (int a = 0; a < kAhead; ++a, t += kStep) {
        step(*this, loaded[(a + kBuffers - 1) % kAhead], t, lds + now, lds + (kBuffers == 2 ? now : next), lds + last);
        if (kBuffers == 2) operands(lds + last, 0);
        const int free = now;
        now = next;
        next = kBuffers == 2 ? free : last;
        last = free;
      }
    }
  }
  // INSIDE: the whole tile is.
  template <bool INSIDE, bool ADD>
  __device__ __forceinline__ void write(float* out) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t n1 = n0 + wave % WN * 32 * FN, k1 = k0 + wave / WN * 32 * FK + lane % 32;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t first = n1 + 32 * i + 8 * q;
        const int64_t n = (INSIDE || EDGE ? first : min(first, A.n - kVec)) + 4 * (lane / 32);
        float* p = out + n * A.out_stride + k1;
#pragma unroll
        for (int e = 0; e < 4; ++e, p += A.out_stride)
#pragma unroll
          for (int j = 0; j < FK; ++j) {
            if (!INSIDE && (n + e < first || n + e >= A.n || k1 + 32 * j >= A.R.cols)) continue;
            const float v = acc[i][j][4 * q + e];
            p[32 * j] = ADD ? p[32 * j] + v : v;
          }
        if (ADD) __builtin_amdgcn_sched_barrier(0);          // or all that is added to is held in registers at once
      }
  }
  __device__ __forceinline__ void write(float* out) {
    if (A.accumulate) write<false, true>(out);
    else if (n0 + kTile <= A.n && k0 + kTile <= A.R.cols) write<true, false>(out);
    else write<false, false>(out);
  }
};

template <int TYPE, int WN, int WK, int FN, int FK, bool EDGE>
__global__ __launch_bounds__(WN * WK * kWave) void weight_grad_kernel(WeightGradArgs A) {
  typedef Worker<TYPE, WN, WK, FN, FK, EDGE> W;
  __shared__ __bf16 lds[W::kBuffers * W::kBuffer];
  constexpr int kTile = W::kTile;
  // Consecutive work-groups go to the eight dies in turn.  Each die takes tiles that lie together, eight of X beside each
  // other, so that its cache is asked for the same rows.
  const unsigned die = blockIdx.x % 8, each = gridDim.x / 8, more = gridDim.x % 8;
  const unsigned tile = die * each + min(die, more) + blockIdx.x / 8;
  const unsigned tiles_n = (unsigned)A.tiles_n, tiles_k = gridDim.x / tiles_n;
  const unsigned band = tile / (8 * tiles_n), wide = min(8u, tiles_k - 8 * band), in_band = tile - band * 8 * tiles_n;
  const int64_t n0 = (int64_t)(in_band / wide) * kTile, k0 = (int64_t)(8 * band + in_band % wide) * kTile;
  const int64_t t_begin = (int64_t)blockIdx.y * A.piece, t_end = min(A.R.rows, t_begin + A.piece);
  float* out = A.out + (int64_t)blockIdx.y * A.split_stride;
  W w(A, n0, k0, t_begin, t_end);
  if (t_begin < t_end) w.run(t_begin, lds);
  w.write(out);
}

// dW from the splits' sums, in their order: a thread has four neighbouring elements, or, where there are few of them,
// SHARE threads do, each with every SHARE-th split.
template <int SHARE>
__global__ __launch_bounds__(kThreads) void weight_grad_join_kernel(const float* __restrict__ parts, int splits, int64_t n, int64_t cols,
                                                                    float* dw, int64_t dw_stride, int accumulate) {
  __shared__ f32x4 sums[SHARE][kThreads / SHARE];
  const int64_t all = n * cols;
  const int share = threadIdx.x / (kThreads / SHARE), lane = threadIdx.x % (kThreads / SHARE);
  for (int64_t first = (int64_t)blockIdx.x * (kThreads / SHARE) * 4; first < all; first += (int64_t)gridDim.x * (kThreads / SHARE) * 4) {
    const int64_t i = first + 4 * lane;
    const int here = (int)max((int64_t)0, min((int64_t)4, all - i));
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (here == 4) {
#pragma unroll 4
      for (int k = share; k < splits; k += SHARE) s += *reinterpret_cast<const f32x4_at4*>(parts + k * all + i);
    } else {
      for (int k = share; k < splits; k += SHARE)
        for (int e = 0; e < here; ++e) s[e] += parts[k * all + i + e];
    }
    if constexpr (SHARE > 1) {
      __syncthreads();
      sums[share][lane] = s;
      __syncthreads();
      if (share) continue;
#pragma unroll
      for (int k = 1; k < SHARE; ++k) s += sums[k][lane];
    }
    int64_t row = i / cols, col = i % cols;
    for (int e = 0; e < here; ++e) {
      float* p = dw + row * dw_stride + col;
      *p = accumulate ? *p + s[e] : s[e];
      if (++col == cols) col = 0, ++row;
    }
  }
}
int join_launch(const float* parts, int64_t splits, int64_t n, int64_t cols, float* dw, int64_t dw_stride, int accumulate,
                hipStream_t stream) {
  constexpr int kShare = 16;
  if (splits >= kShare && n * cols <= (int64_t)kThreads * 4 * 256) {
    const dim3 grid((unsigned)ceil_div(n * cols, kThreads / kShare * 4));
    weight_grad_join_kernel<kShare><<<grid, kThreads, 0, stream>>>(parts, (int)splits, n, cols, dw, dw_stride, accumulate);
  } else {
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n * cols, kThreads * 4), 4096));
    weight_grad_join_kernel<1><<<grid, kThreads, 0, stream>>>(parts, (int)splits, n, cols, dw, dw_stride, accumulate);
  }
  return launch_status();
}

// ---- which form ----------------------------------------------------------------------------------------------

int parts_for(int type) { return type == QA_F32 ? 3 : type == QA_F16 ? 2 : 1; }

template <int TYPE>
int weight_grad_launch(WeightGradArgs& A, const WeightPlan& plan, hipStream_t stream) {
  const dim3 grid((unsigned)plan.tiles, (unsigned)plan.splits);
  if (A.n < kVec) weight_grad_kernel<TYPE, 2, 2, 2, 2, true><<<grid, 256, 0, stream>>>(A);
  else if (plan.tile == 256) weight_grad_kernel<TYPE, 2, 4, 4, 2, false><<<grid, 512, 0, stream>>>(A);
  else weight_grad_kernel<TYPE, 2, 2, 2, 2, false><<<grid, 256, 0, stream>>>(A);
  return launch_status();
}

}  // namespace

size_t weight_grad_workspace_bytes(const qa_coded_rows* R, int type, int64_t n) {
  const int64_t splits = weight_plan(R->rows, R->cols, n, parts_for(type)).splits;
  return splits == 1 ? 0 : (size_t)splits * (size_t)n * (size_t)R->cols * sizeof(float);
}

}  // namespace qa

using namespace qa;

extern "C" int qa_rows_weight_grad(const qa_coded_rows* rows, const int8_t* codes, const uint8_t* scales, int type,
                                   const void* dy, int64_t dy_stride, int64_t n, float* dw, int64_t dw_stride,
                                   int accumulate, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_rows(rows)) return rc;
  if (!known_type(type) || n < 1 || n >= (int64_t(1) << 24) || dy_stride < n || dy_stride >= (int64_t(1) << 25) ||
      rows->code_stride >= (int64_t(1) << 25) || rows->scale_stride >= (int64_t(1) << 25) || dw_stride < rows->cols ||
      (accumulate != 0 && accumulate != 1) || !dw)
    return QA_ERR_INVALID_ARG;
  if (!aligned(dw, 4)) return QA_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  const int64_t all = n * rows->cols;
  if (rows->rows == 0) {
    if (accumulate) return QA_OK;
    return join_launch(nullptr, 0, n, rows->cols, dw, dw_stride, 0, s);
  }
  if (!codes || !scales || !dy) return QA_ERR_INVALID_ARG;
  if (!element_aligned(dy, type) || !aligned(codes, 16)) return QA_ERR_ALIGNMENT;
  const WeightPlan plan = weight_plan(rows->rows, rows->cols, n, parts_for(type));
  const int64_t splits = plan.splits;
  WeightGradArgs A{*rows, codes, scales, dy, dw, dy_stride, dw_stride, 0, n, rows->rows, plan.tiles_n, accumulate};
  if (splits > 1) {
    if (!ws || ws_bytes < weight_grad_workspace_bytes(rows, type, n)) return QA_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return QA_ERR_ALIGNMENT;
    A.out = (float*)ws;
    A.out_stride = rows->cols;
    A.split_stride = all;
    A.accumulate = 0;
    A.piece = ceil_div(ceil_div(rows->rows, splits), 2 * kStep) * 2 * kStep;
  }
  int rc = type == QA_F32    ? weight_grad_launch<QA_F32>(A, plan, s)
           : type == QA_BF16 ? weight_grad_launch<QA_BF16>(A, plan, s)
                             : weight_grad_launch<QA_F16>(A, plan, s);
  if (rc || splits == 1) return rc;
  return join_launch((const float*)ws, splits, n, rows->cols, dw, dw_stride, accumulate, s);
}
