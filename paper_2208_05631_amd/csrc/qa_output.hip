// Log probabilities of targets under an output layer, and their gradient, without the logits in memory.
//
// Logits are products of the matrix cores with rows of w along the tile's height and rows of x along its width, so that a lane holds
// many logits of one row: a tile's maximum and sums are formed in registers, and a row's numbers are joined from one triple per
// chunk of the vocabulary.  The backward pass multiplies the logits again, a piece of the vocabulary at a time, turns them into
// c, the gradient of the logits, which is written once, as rows of binary16 parts, and multiplies that from both sides: dx = c w, dw = c^T x.
//
// What bounds it: the matrix cores (8192 rows, 32768 x 4096 bfloat16: 1.75 to 1.8 ms scored, of which the softmax is a tenth, and 7.4 to 7.7 ms the gradient, four
// times the product's operations, as c goes to dw in two parts), and for few rows w's way from memory (one row, 128000 x 4096: 183 us, 5.7 TB/s).
#include <algorithm>
#include <type_traits>

#include "qa_product.h"
#include "qa_product_plan.h"
#include "qa_softmax.h"

namespace qa {
namespace {

struct LayerArgs {
  int64_t rows, vocab;
  const int *x_exp, *w_exp;                        // scored binary32: operands are x 2^x_exp[row], w 2^w_exp[row]
  const int32_t* target;
};

// ---- operands as the matrix cores take them ------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t finite_most(const float (&v)[kVec]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const uint32_t a = as_u32(v[i]) & 0x7FFFFFFFu;
    m = a >= 0x7F800000u ? m : max(m, a);
  }
  return m;
}
// The power of two that takes a magnitude to [2^14, 2^15), as an exponent: binary16 ends at 2^16.
__device__ __forceinline__ int exponent_for(uint32_t most) {
  return most == 0 ? 0 : min(126, max(-126, 14 - ((int)(max(most, 0x00800000u) >> 23) - 127)));
}

struct RowArgs {
  const int32_t* target;
  const float *stats, *entropy, *g_logprob, *g_entropy;
  int64_t vocab;
};
struct Row { float m, log_sum, h, a, e; int64_t at; };
__device__ __forceinline__ Row row_of(const RowArgs& A, int64_t t) {
  Row r;
  r.m = fmaxf(A.stats[2 * t], -FLT_MAX);
  r.log_sum = A.stats[2 * t + 1];
  const int64_t y = A.target ? A.target[t] : -1;
  r.at = y < 0 || y >= A.vocab ? -1 : y;
  r.a = A.g_logprob && r.at >= 0 ? A.g_logprob[t] : 0.0f;
  r.e = A.g_entropy ? A.g_entropy[t] : 0.0f;
  r.h = A.g_entropy ? A.entropy[t] : 0.0f;
  return r;
}
__device__ __forceinline__ bool counts(const Row& r) { return r.a != 0.0f || r.e != 0.0f; }

// The gradient's operands are scaled by powers of two, so that binary16 holds them to 2^-39 of a largest magnitude: c of its row's bound,
// r 2^c_exp, and x for the logits of its row's largest element.  A row's dx is as exact as if it were alone, then, whatever the others weigh.  dw is a sum
// over rows, whose c are so scaled: x is multiplied there by 2^(x_exp - c_exp) of its row, with one x_exp by which the largest |c| |x| is
// 2^29.  w has one scale for dx, where it is summed over, and for the logits too, unless those are large.
//
// Work-groups leave their largest magnitudes side by side, the next kernel's find the largest of them, and its first one leaves
// the exponents for the kernels behind it: no atomics, nothing to clear.  (One word for the maximum: 100 us for 8192 atomics.)
enum { kOfRows, kOfX, kOfW };
enum { kBesideC, kInX, kInW };                     // key_of() rows' c and x; bits of what is largest in x, and in w
constexpr int kMostBlocks = 1024;
struct Scales {
  int x_exp, w_exp;
  int wide;                                        // w's rows have scales of their own for the logits
  int rows;                                        // that count
  uint32_t found[3][kMostBlocks];
  int counted[kMostBlocks];                        // of each share of the rows
};
// The largest |c| that a row can have: p <= 1, p |log p| <= 1 / e, and an entropy of at most log 2^24 < 17.  (The bound itself may leave binary32.)
__device__ __forceinline__ int exponent_of_c(const Row& r) {
  const uint32_t most = as_u32(fabsf(r.a) + 18.0f * fabsf(r.e));
  return exponent_for(most) - (most >= 0x7F800000u ? 5 : 0);
}
// Of a row's largest |c| |x|: an exponent as a number that is not 0, larger for larger ones; and what x_exp follows from the largest.
constexpr int kKeyOfOne = 1024 + 127;
__device__ __forceinline__ uint32_t key_of(uint32_t most_x, int c_exp) { return most_x == 0 ? 0 : 1024 + max(most_x >> 23, 1u) - c_exp; }
__device__ __forceinline__ int x_exp_for(uint32_t key) { return key == 0 ? 0 : 14 - ((int)key - kKeyOfOne); }
// With one scale an element of w is off by 2^-39 of the largest, and a logit by at most features max|x| max|w| 2^-38.  That is below 2^-16
// unless it could be 2^22 (a row of w that is 2^30 times as large as the others, or so is x).  Then a second copy of w for the logits is worth its time.
__device__ __forceinline__ bool wide_for(uint32_t most_x, uint32_t most_w, int64_t features) {
  return (int)(most_x >> 23) - 127 + (int)(most_w >> 23) - 127 + (64 - __builtin_clzll((uint64_t)features)) > 21;
}
__device__ __forceinline__ uint32_t most_in_wave(uint32_t most) {
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s, kWave));
  return most;
}
template <int N>
__device__ __forceinline__ void most_in_block(uint32_t (&most)[N]) {
  __shared__ uint32_t waves[N][kWaves];
#pragma unroll
  for (int i = 0; i < N; ++i) most[i] = most_in_wave(most[i]);
  __syncthreads();
  if (threadIdx.x % kWave == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) waves[i][threadIdx.x / kWave] = most[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) most[i] = max(max(waves[i][0], waves[i][1]), max(waves[i][2], waves[i][3]));
}

struct MostArgs {
  RowArgs R;
  int64_t rows, vocab, features;
  const void *x, *w;
  int64_t x_stride, w_stride;
  Scales* scales;
  int* place;                                      // of a row among those of its share that count; -1: it does not
  int64_t share;                                   // of the rows, a work-group
  int blocks[3];                                   // work-groups for which rows count, for x and for w; 0: not wanted
};
template <int TYPE>
__device__ __forceinline__ uint32_t most_of_row(const ElemT<TYPE>* p, int64_t cols) {
  constexpr int kAtOnce = 4;                       // reads that are on their way
  const int lane = threadIdx.x % kWave;
  uint32_t most = 0;
  int64_t c = lane * kVec;
  for (; c + (kAtOnce - 1) * kWave * kVec + kVec <= cols; c += kAtOnce * kWave * kVec) {
    Raw8<TYPE> raw[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) raw[k] = load_raw<TYPE>(p + c + k * kWave * kVec);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      float v[kVec];
      to_f32<TYPE>(raw[k], v);
      most = max(most, finite_most(v));
    }
  }
  for (; c < cols; c += kWave * kVec) {
    float v[kVec];
    to_f32<TYPE>(load_raw<TYPE>(p + c, (int)min((int64_t)kVec, cols - c)), v);
    most = max(most, finite_most(v));
  }
  return most;
}
// The largest finite magnitudes of rows of x that count, and of w.  And which rows count: the others take no part in the products.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void output_most_kernel(MostArgs A) {
  int block = blockIdx.x, which = 0;
  while (block >= A.blocks[which]) block -= A.blocks[which++];
  uint32_t most = 0, key = 0;
  if (which == kOfRows) {
    __shared__ int waves[kWaves];
    const int64_t first = block * A.share, end = min(A.rows, first + A.share);
    int counted = 0;
    for (int64_t t0 = first; t0 < end; t0 += kThreads) {
      const int64_t t = t0 + threadIdx.x;
      bool here = false;
      if (t < end) {
        here = counts(row_of(A.R, t));
      }
      const uint64_t all = __ballot(here);
      if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = __popcll(all);
      __syncthreads();
      int before = counted + __popcll(all & ((uint64_t(1) << threadIdx.x % kWave) - 1));
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        before += w < (int)threadIdx.x / kWave ? waves[w] : 0;
        counted += waves[w];
      }
      if (t < end) A.place[t] = here ? before : -1;
      __syncthreads();
    }
    if (threadIdx.x == 0) A.scales->counted[block] = counted;
  } else {
    const int64_t first = (int64_t)block * kWaves + threadIdx.x / kWave, next = (int64_t)A.blocks[which] * kWaves;
    if (which == kOfW) {
      for (int64_t row = first; row < A.vocab; row += next) most = max(most, most_of_row<TYPE>((const ElemT<TYPE>*)A.w + row * A.w_stride, A.features));
    } else {
      for (int64_t row = first; row < A.rows; row += next) {
        const Row r = row_of(A.R, row);
        if (!counts(r)) continue;
        const uint32_t here = most_in_wave(most_of_row<TYPE>((const ElemT<TYPE>*)A.x + row * A.x_stride, A.features));
        most = max(most, here);
        key = max(key, key_of(here, exponent_of_c(r)));
      }
    }
  }
  if (which == kOfRows) return;
  uint32_t both[2] = {most, key};
  most_in_block(both);
  if (threadIdx.x != 0) return;
  A.scales->found[which == kOfX ? kInX : kInW][block] = both[0];
  if (which == kOfX) A.scales->found[kBesideC][block] = both[1];
}

// Rows copied, a wave per row: 16-bit elements as they are, or binary16 (binary32 elements: in two parts) times a power of two: of the row's largest
// magnitude, one for all of w, or of x beside c.
enum Copies { kAsTheyAre, kOwnScale, kScaleOfW, kScaleBesideC };
struct Copy {
  int how;
  const void* from;
  int64_t stride, rows, cols;
  void* to;
  int64_t ld, to_rows;                             // zeros up to ld / parts columns, and in rows from `rows` on
  int* exps;                                       // kOwnScale, and rows in wide_to: written
  void* wide_to;                                   // NULL, or where rows go a second time, by scales of their own, if logits are large
  bool gather;                                     // the rows that count, one behind the other, and zeros up to a whole step of the products
  bool unless_all;                                 // count
  int blocks;
};
constexpr int kCopies = 4;
struct CopyArgs {
  Copy copy[kCopies];
  Scales* scales;
  bool first;                                      // the largest magnitudes are found, and their exponents left
  int found[3];                                    // how many work-groups left them: for which rows count, for x, for w
  int64_t features;
  RowArgs R;
  const int* place;                                // of rows that are gathered, in shares; the first copy gathers, and writes which there are
  int64_t share;
  int *list, *c_exp;                               // c_exp: of the rows in the list
  void* zero;                                      // NULL, or zeros go to its rows that do not count
  int64_t zero_stride;
};
// GRAD: a gradient's; the others find nothing and gather nothing, and have registers for more waves.
template <int TYPE, bool GRAD>
__global__ __launch_bounds__(kThreads) void output_copy_kernel(CopyArgs A) {
  constexpr int kParts = TYPE == QA_F32 ? 2 : 1;
  int x_exp = 0, w_exp = 0;
  bool wide = false;
  if (GRAD && A.first) {
    uint32_t most[3] = {};
    for (int b = threadIdx.x; b < A.found[kOfX]; b += kThreads) {
      most[kBesideC] = max(most[kBesideC], A.scales->found[kBesideC][b]);
      most[kInX] = max(most[kInX], A.scales->found[kInX][b]);
    }
    for (int b = threadIdx.x; b < A.found[kOfW]; b += kThreads) most[kInW] = max(most[kInW], A.scales->found[kInW][b]);
    most_in_block(most);
    x_exp = x_exp_for(most[kBesideC]);
    w_exp = exponent_for(most[kInW]);
    wide = wide_for(most[kInX], most[kInW], A.features);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      A.scales->x_exp = x_exp;
      A.scales->w_exp = w_exp;
      A.scales->wide = wide;
    }
  } else if (GRAD && TYPE != QA_F16) {
    w_exp = A.scales->w_exp;
    wide = A.scales->wide;
  }
  int block = blockIdx.x, at = 0;
  while (at < kCopies && block >= A.copy[at].blocks) block -= A.copy[at++].blocks;
  if (at == kCopies) return;
  const Copy& C = A.copy[at];
  const int lane = threadIdx.x % kWave;
  const auto copy = [&](int how, void* whereto, int64_t from, int64_t to, int64_t cols) {
    const ElemT<TYPE>* p = (const ElemT<TYPE>*)C.from + from * C.stride;
    _Float16* q = (_Float16*)whereto + to * C.ld;
    int exp = w_exp;
    if (TYPE != QA_F16 && how == kOwnScale) {
      exp = exponent_for(most_in_wave(cols ? most_of_row<TYPE>(p, cols) : 0));
      if (lane == 0) C.exps[to] = exp;
    }
    if (GRAD && how == kScaleBesideC && cols) exp = x_exp - exponent_of_c(row_of(A.R, from));
    for (int64_t c = lane * kVec; c < C.ld / kParts; c += kWave * kVec) {
      const int n = (int)max((int64_t)0, min((int64_t)kVec, cols - c));
      bool copied = false;
      if constexpr (TYPE != QA_F32) {
        copied = how == kAsTheyAre || (TYPE == QA_F16 && how != kScaleBesideC);
        if (copied) *reinterpret_cast<u32x4*>(q + c) = n ? load_raw<TYPE>(p + c, n).a : u32x4{};
      }
      if (!copied) {
        float v[kVec] = {};
        if (n) to_f32<TYPE>(load_raw<TYPE>(p + c, n), v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = ldexpf(v[i], exp);
        if constexpr (kParts == 2) put_parts(q + 2 * c, v);
        else *reinterpret_cast<u32x4*>(q + c) = from_f32<QA_F16>(v).a;
      }
    }
  };
  const int64_t first = (int64_t)block * kWaves + threadIdx.x / kWave, next = (int64_t)C.blocks * kWaves;
  if (!GRAD || !C.gather) {
    for (int64_t row = first; row < C.to_rows; row += next) copy(C.how, C.to, row, row, row < C.rows ? C.cols : 0);
    if (GRAD && TYPE != QA_F16 && C.wide_to && wide)
      for (int64_t row = first; row < C.to_rows; row += next) copy(kOwnScale, C.wide_to, row, row, row < C.rows ? C.cols : 0);
    return;
  }
  __shared__ int before[kMostBlocks], waves[kWaves];           // rows that count before each share
  constexpr int kEach = kMostBlocks / kThreads;
  int mine[kEach], sum = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int b = threadIdx.x * kEach + e;
    mine[e] = sum;
    sum += b < A.found[kOfRows] ? A.scales->counted[b] : 0;
  }
  int upto = sum;
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) {
    const int other = __shfl_up(upto, s, kWave);
    upto += lane >= s ? other : 0;
  }
  if (lane == kWave - 1) waves[threadIdx.x / kWave] = upto;
  __syncthreads();
  int rows = 0, ahead = upto - sum;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    ahead += w < (int)threadIdx.x / kWave ? waves[w] : 0;
    rows += waves[w];
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) before[threadIdx.x * kEach + e] = ahead + mine[e];
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) A.scales->rows = rows;
  for (int64_t row = first; row < C.rows; row += next) {
    const int place = A.place[row];
    if (place >= 0) {
      const int64_t to = before[row / A.share] + place;
      if (!(C.unless_all && rows == C.rows)) copy(C.how, C.to, row, to, C.cols);
      if (at == 0 && lane == 0) {
        A.list[to] = (int)row;
        A.c_exp[to] = exponent_of_c(row_of(A.R, row));
      }
    } else if (at == 0 && A.zero) {
      constexpr float zeros[kVec] = {};
      for (int64_t c = lane * kVec; c < C.cols; c += kWave * kVec)
        store_raw<TYPE>((ElemT<TYPE>*)A.zero + row * A.zero_stride + c, from_f32<TYPE>(zeros), (int)min((int64_t)kVec, C.cols - c));
    }
  }
  if (block == 0)
    for (int64_t to = rows + threadIdx.x / kWave; to < whole(max(1, rows), kPartsStep); to += kWaves) copy(C.how, C.to, 0, to, 0);
}

// ---- scoring ------------------------------------------------------------------------------------------------------------------
//
// w's rows along the tile's height: sixteen logits of a matrix instruction in a lane are of one row of x, so that maximum and sums need one exchange
// between the halves of a wave, and a chunk (a wave's logits of a row) leaves three numbers, 12 bytes for 64 or 128 logits.

// A lane's logits of block column j, four at a time: each(the first one's place behind v0, block row, quarter, logits).
template <bool SCALED, class P, class Each>
__device__ __forceinline__ void for_logits(P& p, const LayerArgs& L, int64_t v0, int j, int x_exp, const Each& each) {
  const int first = 4 * ((int)threadIdx.x % kWave / 32), last = (int)min((int64_t)(1 << 24), L.vocab - 1 - v0);
  const int* const w_exp = L.w_exp + v0;
#pragma unroll
  for (int i = 0; i < (int)(sizeof p.acc / sizeof p.acc[0]); ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int v = 32 * i + 8 * q + first;
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[e] = p.acc[i][j][4 * q + e];
        if (SCALED) z[e] = ldexpf(z[e], -(x_exp + w_exp[min(v + e, last)]));
      }
      each(v, i, q, z);
      __builtin_amdgcn_sched_barrier(0);           // or all exponents and addresses are held in registers at once
    }
}

struct ScoreArgs {
  float *m, *s, *w;                                // [chunk][rows]: a wave's part of a tile
  float* given;                                    // the targets' logits
  int64_t first, first_chunk;                      // of this launch's vocabulary
};

template <bool SCALED>
struct ScoreOut {
  LayerArgs L;                                     // vocab: of this launch
  ScoreArgs A;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t v0, int64_t t0, char*) const {
    constexpr int kChunk = 32 * (int)(sizeof p.acc / sizeof p.acc[0]);
    const int left = (int)max((int64_t)0, min((int64_t)kChunk, L.vocab - v0));       // of this wave's logits there are
#pragma unroll
    for (int j = 0; j < (int)(sizeof p.acc[0] / sizeof p.acc[0][0]); ++j) {
      const int64_t t = t0 + 32 * j + threadIdx.x % 32;
      const int x_exp = SCALED ? L.x_exp[min(t, L.rows - 1)] : 0;
      const int64_t at = L.target && t < L.rows ? (int64_t)L.target[t] - A.first - v0 : -1;
      const int here = at >= 0 && at < left ? (int)at : -1;
      Sums a = no_sums();
      float given = 0.0f;
      for_logits<SCALED>(p, L, v0, j, x_exp, [&](int v, int i, int q, float (&z)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          given = v + e == here ? z[e] : given;
          z[e] = v + e < left ? z[e] : -__builtin_inff();
          p.acc[i][j][4 * q + e] = z[e];
          a.m = fmaxf(a.m, z[e]);
        }
      });
      if (here >= 0 && here / 4 % 2 == (int)threadIdx.x % kWave / 32) A.given[t] = given;
      a.m = fmaxf(a.m, as_f32(other_lane<32>(as_u32(a.m))));
#pragma unroll
      for (int i = 0; i < kChunk / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float y = (p.acc[i][j][r] - a.m) * kLog2e, e = __builtin_amdgcn_exp2f(y);
          a.s += e;
          a.w = __builtin_fmaf(e, fmaxf(y, kFar), a.w);
        }
      a.s += as_f32(other_lane<32>(as_u32(a.s)));
      a.w += as_f32(other_lane<32>(as_u32(a.w)));
      if (threadIdx.x % kWave < 32 && t < L.rows) {
        const int64_t to = (A.first_chunk + v0 / kChunk) * L.rows + t;
        A.m[to] = a.m;
        A.s[to] = a.s;
        A.w[to] = a.w;
      }
    }
  }
};

// ---- scoring of few rows --------------------------------------------------------------------------------------------------------
//
// Up to 64 rows: reading w is what takes time.  It goes from memory to registers, from any place and in any type, and each of its elements
// is multiplied at once with all rows of x, which lie in LDS, a piece of k at a time: binary32 in three bfloat16 parts (six products, what is
// left out is below 2^-24).  A wave has sixteen rows of w twice, eight waves go over the work-group's share of the vocabulary, and a lane keeps
// the maximum and the sums of its logits all along.  Those 256 rows are read whatever the share: where it is smaller, or ends among them, the
// neighbours' rows are multiplied too and left out (4 times w's rows at a vocabulary of 32768, 2.7 at 47236, 1.2 at 100003: 48 rows, 32768 x 1024 binary32: 109 us,
// 22 for w once; 48 rows, 100003 x 2049 binary16: 227 us, 67).

typedef float f32x4m __attribute__((ext_vector_type(4)));
constexpr int kStreamGroup = 512, kStreamWaves = kStreamGroup / kWave, kStreamRows = 2 * 16 * kStreamWaves;
template <int TYPE> constexpr int stream_parts = TYPE == QA_F32 ? 3 : 1;
// Columns of k of x in LDS, in steps of 32: 64 KiB.
template <int TYPE, int NB> constexpr int stream_k = 2048 / NB / stream_parts<TYPE> / 128 * 128;

struct StreamArgs {
  LayerArgs L;                                     // without exponents
  ScoreArgs A;
  const void *x, *w;
  int64_t x_stride, w_stride;
  int features;
  int64_t each;                                    // of the vocabulary per work-group, a multiple of 16
};

template <int TYPE, int NB>
__global__ __launch_bounds__(kStreamGroup, 4) void output_stream_kernel(StreamArgs S) {
  typedef ElemT<TYPE> T;
  constexpr int P = stream_parts<TYPE>, KC = stream_k<TYPE, NB>, kPitch = KC + 8, kPlane = 16 * NB * kPitch;
  constexpr int U = TYPE == QA_F32 ? 1 : NB == 1 ? 4 : 2;      // steps of w that are on their way, twice: what registers hold
  static_assert(KC % (64 * U) == 0, "whole blocks, two by two");
  __shared__ __attribute__((aligned(16))) uint16_t lds[P * kPlane];
  __shared__ Sums joined[kStreamWaves][16 * NB];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, K = S.features;
  const int64_t r0 = (int64_t)blockIdx.x * S.each, r1 = min(S.L.vocab, r0 + S.each);
  Sums sums[NB];
  int64_t at[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    sums[n] = no_sums();
    const int64_t t = 16 * n + lane % 16;
    at[n] = S.L.target && t < S.L.rows ? S.L.target[t] : -1;
  }

  for (int64_t base = r0; base < r1; base += kStreamRows) {
    const T* from[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) from[g] = (const T*)S.w + min(base + (2 * wave + g) * 16 + lane % 16, S.L.vocab - 1) * S.w_stride;
    f32x4m acc[2][NB] = {};
    Raw8<TYPE> raw[2][2][U];
    const auto load = [&](Raw8<TYPE> (&to)[2][U], int k) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int g = 0; g < 2; ++g)
          // No branch, which would wait for what is on its way: past the end the last eight, and nobody uses them.
          to[g][u] = load_raw<TYPE>(from[g] + min(k + 32 * u + 8 * (lane / 16), K - kVec));
    };
    const auto multiply = [&](const auto& of, int k, auto steps) {
#pragma unroll
      for (int u = 0; u < decltype(steps)::value; ++u) {
        u32x4 a[2][P];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if constexpr (TYPE == QA_F32) {
            float v[kVec];
            to_f32<TYPE>(of[g][u], v);
            split_parts<P>(v, a[g]);
          } else {
            a[g][0] = of[g][u].a;
          }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int q = 0; q < P; ++q) {
            const u32x4 b = *reinterpret_cast<const u32x4*>(lds + q * kPlane + (16 * n + lane % 16) * kPitch + k + 32 * u + 8 * (lane / 16));
#pragma unroll
            for (int p = 0; p + q < P; ++p)
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                if constexpr (TYPE == QA_F16)
                  acc[g][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a[g][p]), __builtin_bit_cast(f16x8, b), acc[g][n], 0, 0, 0);
                else
                  acc[g][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[g][p]), __builtin_bit_cast(bf16x8, b), acc[g][n], 0, 0, 0);
              }
          }
      }
    };
    load(raw[0], 0);
    for (int k0 = 0; k0 < K; k0 += KC) {
      if (K > KC || base == r0) {                  // or all of x lies there already
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * NB * (KC / kVec); i += kStreamGroup) {
          const int row = i / (KC / kVec), col = i % (KC / kVec) * kVec;
          const int n = row < S.L.rows ? max(0, min(kVec, K - k0 - col)) : 0;
          float v[kVec] = {};
          u32x4 part[P] = {};
          if constexpr (TYPE == QA_F32) {
            if (n) to_f32<TYPE>(load_raw<TYPE>((const T*)S.x + row * S.x_stride + k0 + col, n), v);
            split_parts<P>(v, part);
          } else if (n) {
            part[0] = load_raw<TYPE>((const T*)S.x + row * S.x_stride + k0 + col, n).a;
          }
#pragma unroll
          for (int p = 0; p < P; ++p) *reinterpret_cast<u32x4*>(lds + p * kPlane + row * kPitch + col) = part[p];
        }
        __syncthreads();
      }
      typedef std::integral_constant<int, U> All;
      const int end = min(KC, K - k0), blocks = end / (64 * U) * (64 * U);
#pragma unroll 1
      for (int k = 0; k < blocks; k += 64 * U) {
        load(raw[1], k0 + k + 32 * U);
        multiply(raw[0], k, All());
        load(raw[0], k0 + k + 64 * U);
        multiply(raw[1], k + 32 * U, All());
      }
#pragma unroll 1
      for (int k = blocks; k < end; k += 32) {     // the end of the rows
        Raw8<TYPE> one[2][1];
#pragma unroll
        for (int g = 0; g < 2; ++g) one[g][0] = load_raw<TYPE>(from[g] + k0 + k + 8 * (lane / 16), K - (k0 + k + 8 * (lane / 16)));
        multiply(one, k, std::integral_constant<int, 1>());
      }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float most = sums[n].m;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t v = base + (2 * wave + g) * 16 + 4 * (lane / 16) + e;
          if (v == at[n] && v < r1) S.A.given[16 * n + lane % 16] = acc[g][n][e];
          acc[g][n][e] = v < r1 ? acc[g][n][e] : -__builtin_inff();
          most = fmaxf(most, acc[g][n][e]);
        }
      raise(sums[n], most);
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = (acc[g][n][e] - most) * kLog2e, q = __builtin_amdgcn_exp2f(y);
          sums[n].s += q;
          sums[n].w = __builtin_fmaf(q, fmaxf(y, kFar), sums[n].w);
        }
    }
  }
  const auto join = [](Sums& a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    a.s += b.s;
    a.w += b.w;
  };
#pragma unroll
  for (int n = 0; n < NB; ++n) {
#pragma unroll
    for (int s = 16; s < kWave; s *= 2) join(sums[n], Sums{__shfl_xor(sums[n].m, s, kWave), __shfl_xor(sums[n].s, s, kWave), __shfl_xor(sums[n].w, s, kWave)});
    if (lane < 16) joined[wave][16 * n + lane] = sums[n];
  }
  __syncthreads();
  if ((int)threadIdx.x < S.L.rows) {
    Sums a = joined[0][threadIdx.x];
#pragma unroll 1
    for (int i = 1; i < kStreamWaves; ++i) join(a, joined[i][threadIdx.x]);
    const int64_t to = (int64_t)blockIdx.x * S.L.rows + threadIdx.x;
    S.A.m[to] = a.m;
    S.A.s[to] = a.s;
    S.A.w[to] = a.w;
  }
}

// ---- a row's numbers -------------------------------------------------------------------------------------------------------------

// A row's numbers from its chunks': ROWS rows per work-group, the other threads along the chunks.
template <int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void output_join_kernel(ScoreArgs A, int64_t rows, int64_t chunks, int64_t vocab, const int32_t* target,
                                                               float* logprob, float* entropy, float* stats) {
  constexpr int kShare = THREADS / ROWS;
  __shared__ Sums part[kShare][ROWS];
  const int r = threadIdx.x % ROWS, share = threadIdx.x / ROWS;
  const int64_t t = (int64_t)blockIdx.x * ROWS + r;
  Sums a = no_sums();
  if (t < rows) {
    for (int64_t c = share; c < chunks; c += kShare) {
      const int64_t at = c * rows + t;
      Sums b = {A.m[at], A.s[at], A.w[at]};
      const float m = fmaxf(a.m, b.m);
      raise(a, m);
      raise(b, m);
      a.s += b.s;
      a.w += b.w;
    }
  }
  part[share][r] = a;
  __syncthreads();
#pragma unroll
  for (int half = kShare / 2; half >= 1; half /= 2) {
    if (share < half) {
      Sums b = part[share + half][r];
      const float m = fmaxf(a.m, b.m);
      raise(a, m);
      raise(b, m);
      a.s += b.s;
      a.w += b.w;
      part[share][r] = a;
    }
    __syncthreads();
  }
  if (share || t >= rows) return;
  const bool empty = a.s == 0.0f;
  const float m = empty ? -__builtin_inff() : a.m, log_sum = empty ? 0.0f : kLn2 * __builtin_amdgcn_logf(a.s);
  if (stats) {
    stats[2 * t] = m;
    stats[2 * t + 1] = log_sum;
  }
  if (entropy) entropy[t] = empty ? 0.0f : log_sum - kLn2 * (a.w / a.s);
  if (logprob) {
    const int32_t y = target[t];
    logprob[t] = y < 0 || y >= vocab ? 0.0f : empty ? m : (A.given[t] - m) - log_sum;
  }
}

// ---- the gradient of the logits -------------------------------------------------------------------------------------------
//
// Rows that do not count are left out before anything is multiplied: the device finds which they are, x's others are gathered, and
// the products, launched for all rows, end early or have more splits where fewer are left (4096 rows of which half count, 50021 x 1024 binary16: 1.36 ms, 2.11
// with all of them multiplied).

// c of a piece of the vocabulary, scaled, in rows of parts, for the rows that count: zeros behind the piece, and in rows up to a whole step.
// SCALED: of operands scaled by a power of two per row of x, and one of w or, if logits are large, of each of its rows.
// log p is never above 0, though statistics and logits of 10^8, multiplied in another order, are tens apart: c stays within its bound, and
// binary16 with it (NaN stays NaN).
template <bool SCALED, bool ENTROPY>
struct LogitsGradOut {
  int64_t vocab;                                   // of this piece
  RowArgs R;
  const int *list, *x_exp, *w_exps;                // rows that count; SCALED: of each of them, and of the piece's rows of w
  int64_t first;                                   // of the piece
  const Scales* scales;
  _Float16* c;
  int64_t ld;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t v0, int64_t t0, char* lds) const {
    const int lane = threadIdx.x % kWave;
    const bool own_w = SCALED && scales->wide;
    const int w_exp = SCALED && !own_w ? scales->w_exp : 0;
    constexpr int FN = (int)(sizeof p.acc[0] / sizeof p.acc[0][0]);
    float m[FN], log_sum[FN], a[FN], e[FN], h[FN];
    int here[FN], z_exp[FN];
    bool none[FN];
    const int64_t rows = scales->rows, to_rows = whole(max((int64_t)1, rows), kPartsStep);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t t = t0 + 32 * j + lane % 32;
      const int64_t at_most = max((int64_t)0, min(t, rows - 1));
      const Row r = row_of(R, rows ? list[at_most] : 0);
      const int exp = exponent_of_c(r);
      z_exp[j] = SCALED ? -(x_exp[at_most] + w_exp) : 0;
      m[j] = r.m;
      log_sum[j] = r.log_sum * kLog2e;
      a[j] = ldexpf(r.a, exp);
      e[j] = ldexpf(r.e, exp) * kLn2;
      h[j] = r.h * kLog2e;
      none[j] = t >= rows;
      const int64_t at = r.at - first - v0;
      here[j] = at >= 0 && at < P::kM ? (int)at : -kVec;
    }
    const int left = (int)max((int64_t)0, min((int64_t)P::kM, vocab - v0)), wide = (int)max((int64_t)0, min((int64_t)P::kM, ld / 2 - v0));
    p.template for_runs<false>(0, 0, lds, [&](int v, int col, float (&z)[kVec]) {
      const int j = col / 32;
      float g[kVec];
      if (own_w) {
        int own[kVec];                             // (what stands there behind the vocabulary's end serves nobody)
        __builtin_memcpy(own, __builtin_assume_aligned(w_exps + v0 + v, 16), sizeof own);
#pragma unroll
        for (int k = 0; k < kVec; ++k) z[k] = ldexpf(z[k], -own[k]);
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        if (SCALED) z[k] = ldexpf(z[k], z_exp[j]);
        const float lp = __builtin_elementwise_minimum(__builtin_fmaf(z[k] - m[j], kLog2e, -log_sum[j]), 0.0f), q = __builtin_amdgcn_exp2f(lp);  // in powers of two
        g[k] = ENTROPY ? -q * (a[j] + e[j] * (fmaxf(lp, kFar) + h[j])) : -q * a[j];
      }
      if (__any((unsigned)(here[j] - v) < kVec)) {           // few eights have a target
#pragma unroll
        for (int k = 0; k < kVec; ++k)
          if (v + k == here[j]) g[k] += a[j];
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) z[k] = none[j] || v + k >= left ? 0.0f : g[k];
      __builtin_amdgcn_sched_barrier(0);           // or all exponents and addresses are held in registers at once
    }, [&](int64_t v, int64_t col, float (&g)[kVec]) {
      if (t0 + col < to_rows && v < wide) put_parts(c + (t0 + col) * ld + 2 * (v0 + v), g);
    }, 0);
  }
};

// Sums of a product, unscaled, rounded to the type or added in binary32; the product's columns are the rows that are written.
// LISTED: dx, whose rows are those that count; else dw.
template <int TYPE, bool LISTED>
struct GradOut {
  ElemT<TYPE>* out;
  float* sums;                                     // [split][rows][cols]; NULL: none before this piece, and this is the last
  const Scales* scales;
  int64_t stride, rows, cols;
  bool add, last;                                  // to what is in sums (or, of binary32, in out); the last piece writes out
  const int *list, *c_exp;                         // LISTED: where the rows go, and their c's exponents
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0, char* lds) const {
    const int of_all = -(LISTED ? scales->w_exp : scales->x_exp);
    const int64_t all = LISTED ? scales->rows : rows;
    float* const its_sums = sums + p.split * all * cols;
    const bool writes = last || !sums;
    p.for_runs(m0, n0, lds, [&](int64_t col, int64_t row, float (&v)[kVec]) {
      if (row >= all || col >= cols) return;
      const int n = (int)min((int64_t)kVec, cols - col);
      const int exp = LISTED ? of_all - c_exp[row] : of_all;
      ElemT<TYPE>* const at = out + (LISTED && writes ? list[row] : row) * stride + col;
      float* const s = its_sums + row * cols + col;
      float before[kVec] = {};
      if (add) {
        if (sums) to_f32<QA_F32>(load_raw<QA_F32>(s, n), before);
        else to_f32<TYPE>(load_raw<TYPE>(at, n), before);
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = before[e] + (p.empty ? 0.0f : ldexpf(v[e], exp));
      if (last) store_raw<TYPE>(at, from_f32<TYPE>(v), n);
      else store_raw<QA_F32>(s, from_f32<QA_F32>(v), n);
    });
  }
};
// A gradient from the splits' sums, in their order.
struct Splits {
  int splits, most;                                // as planned, and where few rows count
  unsigned side;                                   // of the product's tiles, along the rows
};
template <int TYPE>
__global__ __launch_bounds__(kThreads) void output_sum_kernel(const float* sums, Splits of, int64_t rows, int64_t cols, ElemT<TYPE>* out, int64_t stride,
                                                              int accumulate, const int* list, const Scales* scales) {
  const int splits = list ? splits_of_fewer(of.splits, of.most, of.side, (unsigned)rows, max(1, scales->rows)) : of.splits;
  if (list) rows = scales->rows;
  const int64_t across = ceil_div(cols, kVec), all = rows * across;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / across, col = i % across * kVec;
    const int n = (int)min((int64_t)kVec, cols - col);
    float v[kVec] = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      float w[kVec];
      to_f32<QA_F32>(load_raw<QA_F32>(sums + (s * rows + row) * cols + col, n), w);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] += w[e];
    }
    ElemT<TYPE>* const at = out + (list ? list[row] : row) * stride + col;
    if (accumulate) {
      float w[kVec];
      to_f32<TYPE>(load_raw<TYPE>(at, n), w);
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] += w[e];
    }
    store_raw<TYPE>(at, from_f32<TYPE>(v), n);
  }
}
__global__ __launch_bounds__(kThreads) void output_zero_kernel(float* p, int64_t stride, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) p[r * stride + c] = 0.0f;
}

// ---- what a call does ------------------------------------------------------------------------------------------------------------

// Bytes of a piece's c, of its copy of w and of sums that are joined (of one split at least): about what the last-level cache holds.  (Gradient of 8192 rows, 32768 x 4096: 7.74 ms, 8.03
// with half of it, 7.66 with twice and four times as much; 4096 rows, 50021 x 1024: 2.29, 2.28, 2.41, 2.20.)
constexpr int64_t kPieceBytes = int64_t(256) << 20;

struct Room {
  size_t bytes = 0;
  size_t take(int64_t n) {
    const size_t at = bytes;
    bytes += (size_t)whole(n, 256);
    return at;
  }
};

constexpr int64_t kFewRows = 64;

// Time of a step of k beside one of three products of 16: 32 k and one product bring as much for two thirds of the matrix instructions.
constexpr double kOneProduct = 0.75, kTwoProducts = 0.65, kThreeProducts = 1.0;

// Which tiles multiply the logits, in vocabulary by rows: 256 x 64 for few rows, or one of those of the other products.  Those of 256 x 256
// have no registers to hold a binary32 product's small parts apart (1681 rows of 5248: log probabilities 1e-6 off, and 5e-7).
enum Tall { kTall256, kTall128, kTall128Two, kTall64, kFlat };
Tall logits_tiles(int64_t rows, int64_t vocab, int64_t features, int type) {
  // Few rows: reading w is what takes time, and tiles of 256 bring the least of x beside it, unless they leave most compute units without any (48 rows,
  // 8000 x 2048: 29 us, 16 with tiles of 64; 25000 x 2048: 42 and 39; 33024 x 4096: 78 and 86).
  if (rows <= kFewRows) return vocab <= 64 * 384 ? kTall64 : kFlat;
  const ProductShape S = {vocab, rows, ceil_div(features, type == QA_F32 ? kPartsStep : kWholeStep), 1, false, type == QA_F32 ? kThreeProducts : kOneProduct};
  const unsigned small = tiles_bit(kTiles128) | tiles_bit(kTiles128Two) | tiles_bit(kTiles64Four);
  switch (product_plan(type == QA_F32 ? small : small | tiles_bit(kTiles256), S, 1).tiles) {
    case kTiles256: return kTall256;
    case kTiles128: return kTall128;
    case kTiles128Two: return kTall128Two;
    default: return kTall64;
  }
}
constexpr int64_t height_of(Tall t) { return t == kTall64 ? 64 : t == kTall128 || t == kTall128Two ? 128 : 256; }
constexpr int64_t chunks_of(Tall t) { return t == kFlat ? 4 : t == kTall64 ? 1 : 2; }         // of a tile

// Equal pieces of n, whole tiles each, of at most `most`.
int64_t piece_of(int64_t n, int64_t most) { return std::min(whole(n, kWholeStep), whole(ceil_div(n, ceil_div(n, most)), 256)); }
// Pieces of the vocabulary whose tiles of 256 x 256 leave the fewest compute units without one at the end of each piece.
int64_t even_piece_of(int64_t n, int64_t most, int64_t rows) {
  int64_t best = piece_of(n, most), least = 0;
  for (int64_t piece = whole(std::min(n, most), 256); piece >= 256 && 2 * piece >= std::min(n, most); piece -= 256) {
    int64_t rounds = 0;
    for (int64_t first = 0; first < n; first += piece) rounds += ceil_div(ceil_div(std::min(piece, n - first), 256) * ceil_div(rows, 256), 256);
    if (least == 0 || rounds < least) {
      least = rounds;
      best = piece;
    }
  }
  return std::min(whole(n, kWholeStep), best);
}
int64_t power_of_two_within(int64_t n, int64_t least) {
  while (2 * least <= n) least *= 2;
  return least;
}

struct Plan {
  bool copy_x, copy_w;                             // for the logits
  int64_t parts, hp, piece, pieces;                // a copied row's columns; vocabulary of a launch
  int64_t rows;                                    // of a launch
  bool copies;                                     // gradient: both
  bool streams;                                    // w, for few rows that would have to be copied
  Tall tiles;
  size_t x, w, x_exp, w_exp;                       // copies and exponents
  size_t m, s, sw, given;                          // scoring
  int64_t chunks, each;                            // each: of the vocabulary per work-group, where w is streamed
  size_t scales, place, list, c_exp, xr, xc, wc, wr, c, sums;   // gradient: rows of x and (if they are large) of w for the logits; x and w as the products with c take them
  size_t dw_sums;
  int64_t hc, tp, vp;
  ProductPlan dx;
  size_t bytes;
};
ProductPlan grad_plan(const ProductShape& S, int64_t most) { return product_plan(tiles_bit(kTiles256) | tiles_bit(kTiles128) | tiles_bit(kTiles128Two), S, most); }

// Of a piece's dw: its tiles are few where both sides are small.
ProductPlan dw_plan(const qa_output_layer& L, int type, int64_t vocab) {
  return grad_plan({L.features, vocab, ceil_div(L.rows, kPartsStep), 1, false, type == QA_F32 ? kThreeProducts : kTwoProducts},
                   std::min(std::max<int64_t>(1, kPieceBytes / (4 * vocab * L.features)), int64_t(64)));
}

bool in_place(const void* p, int64_t stride) { return stride % 8 == 0 && stride < (int64_t(1) << 22) && aligned(p, 16); }

// x and w NULL: at places of any alignment.
Plan plan_of(const qa_output_layer& L, int op, int type, const void* x, const void* w) {
  Plan P = {};
  Room room;
  P.parts = type == QA_F32 ? 2 : 1;
  const bool rows_as_they_are = type != QA_F32 && L.features % kWholeStep == 0;
  P.copy_x = !x || !rows_as_they_are || !in_place(x, L.x_stride);
  P.copy_w = !w || !rows_as_they_are || !in_place(w, L.w_stride);
  P.hp = whole(L.features, kWholeStep);
  P.rows = L.rows;
  // Copying w takes longer than the products of few rows with it (48 rows, 100003 x 2049 binary16: 294 us, 220 from where it lies; one row,
  // 47236 x 515 binary32: 76, 57), but where it can be brought straight to LDS, that is faster (100003 x 2048: 107, 123).
  P.streams = op == QA_OP_LOGPROB && L.rows <= kFewRows && L.features >= kVec && (P.copy_x || P.copy_w);
  if (P.streams) {
    P.copy_x = P.copy_w = false;
    P.each = whole(ceil_div(L.vocab, 512), 16);
    P.chunks = ceil_div(L.vocab, P.each);
  } else if (op == QA_OP_LOGPROB) {
    P.tiles = logits_tiles(L.rows, L.vocab, L.features, type);
    P.piece = P.copy_w ? piece_of(L.vocab, power_of_two_within(kPieceBytes / (P.hp * 2 * P.parts), 16384)) : L.vocab;
    P.pieces = ceil_div(L.vocab, P.piece);
    P.chunks = chunks_of(P.tiles) * ((P.pieces - 1) * ceil_div(P.piece, height_of(P.tiles)) + ceil_div(L.vocab - (P.pieces - 1) * P.piece, height_of(P.tiles)));
    // So that the chunks' numbers stay within bounds, and the tiles within a grid's.
    P.rows = std::min(L.rows, std::max<int64_t>(256, 4 * kPieceBytes / (12 * P.chunks) / 256 * 256));
  } else {
    P.tp = whole(L.rows, kPartsStep);
    // Where x or w have to be copied for the logits, w as dx takes it serves for both.
    P.copies = P.copy_x || P.copy_w;
    P.copy_x = P.copy_w = false;
    P.hc = whole(L.features, P.copies ? kWholeStep : 8);
    P.piece = even_piece_of(L.vocab, std::min(power_of_two_within(kPieceBytes / (4 * P.tp), 1024), power_of_two_within(kPieceBytes / (P.hp * 2 * P.parts), 1024)), L.rows);
    P.pieces = ceil_div(L.vocab, P.piece);
    P.vp = whole(P.piece, kWholeStep);
    P.scales = room.take(sizeof(Scales));
    P.place = room.take(4 * L.rows);
    P.list = room.take(4 * L.rows);
    P.c_exp = room.take(4 * P.tp);
    P.x_exp = room.take(P.copies && type != QA_F16 ? 4 * P.tp : 0);
    P.xr = room.take(2 * P.parts * P.tp * P.hc);
    P.xc = room.take(2 * P.parts * P.tp * P.hc);
    P.wc = room.take(2 * P.parts * P.vp * P.hc);
    P.wr = room.take(P.copies && type != QA_F16 ? 2 * P.parts * P.vp * P.hc : 0);
    P.w_exp = room.take(P.copies && type != QA_F16 ? 4 * whole(P.vp, 256) : 0);
    P.c = room.take(2 * 2 * P.tp * P.vp);
    // dx has few tiles and sums over the vocabulary.
    const bool one = type == QA_BF16;
    const int64_t vocab = std::min(P.piece, L.vocab), fit = std::max<int64_t>(1, kPieceBytes / (4 * L.rows * L.features));
    P.dx = grad_plan({L.features, L.rows, ceil_div(vocab, one ? kWholeStep : kPartsStep), 1, false, one ? kOneProduct : type == QA_F32 ? kThreeProducts : kTwoProducts}, std::min<int64_t>(64, fit));
    P.sums = room.take(P.pieces > 1 || P.dx.splits > 1 ? 4 * P.dx.splits * L.rows * L.features : 0);
    int64_t dw_sums = 0;
    for (const int64_t of : {vocab, L.vocab - (P.pieces - 1) * P.piece})
      if (const int64_t splits = dw_plan(L, type, of).splits; splits > 1) dw_sums = std::max(dw_sums, 4 * splits * of * L.features);
    P.dw_sums = room.take(dw_sums);
  }
  if (op == QA_OP_LOGPROB) {
    P.m = room.take(4 * P.chunks * P.rows);
    P.s = room.take(4 * P.chunks * P.rows);
    P.sw = room.take(4 * P.chunks * P.rows);
    P.given = room.take(4 * P.rows);
  }
  if (op == QA_OP_LOGPROB) {
    P.x_exp = room.take(P.copy_x && type == QA_F32 ? 4 * P.rows : 0);
    P.w_exp = room.take(P.copy_w && type == QA_F32 ? 4 * P.piece : 0);
  }
  P.x = room.take(P.copy_x ? 2 * P.parts * P.rows * P.hp : 0);
  P.w = room.take(P.copy_w ? 2 * P.parts * P.piece * P.hp : 0);
  P.bytes = room.bytes;
  return P;
}
// Rows of a gradient's launches: so many that a piece of c can be 1024 wide, or the whole vocabulary.
int64_t grad_rows_of(const qa_output_layer& L) { return piece_of(L.rows, kPieceBytes / (4 * whole(std::min<int64_t>(L.vocab, 1024), kWholeStep)) / 256 * 256); }
// At most, whatever the alignment of x and w.
size_t bytes_of(const qa_output_layer& L, int op, int type) {
  if (const int64_t piece = grad_rows_of(L); op == QA_OP_LOGPROB_GRAD && piece < L.rows) {
    qa_output_layer full = L, last = L;
    full.rows = piece;
    last.rows = (L.rows - 1) % piece + 1;
    return std::max(bytes_of(full, op, type), bytes_of(last, op, type));
  }
  alignas(16) static const char aligned_place[16] = {};
  size_t most = 0;
  for (const void* x : {(const void*)nullptr, (const void*)aligned_place})
    for (const void* w : {(const void*)nullptr, (const void*)aligned_place}) most = std::max(most, plan_of(L, op, type, x, w).bytes);
  return most;
}

// Copies that one kernel makes.
struct CopyList {
  CopyArgs A = {};
  int n = 0, blocks = 0;
  void add(int how, const void* from, int64_t stride, int64_t rows, int64_t cols, void* to, int64_t ld, int64_t to_rows, int* exps, bool gather, bool unless_all = false, void* wide_to = nullptr) {
    Copy& C = A.copy[n++];
    // A gradient's first copies begin with finding the largest magnitudes: few work-groups, several rows each (333 rows, 32771 x 257 binary32: 145 us
    // with 1024, 147.5 with 4096, 151.5 with 8368).
    const int64_t most = A.first ? 1024 : 1 << 14;
    C = {how, from, stride, rows, cols, to, ld, to_rows, exps, wide_to, gather, unless_all, (int)std::min<int64_t>(ceil_div(to_rows, kWaves), most)};
    blocks += C.blocks;
  }
  template <int TYPE> int launch(hipStream_t stream) {
    if (!A.first && n == 0) return QA_OK;
    const auto kernel = A.scales ? output_copy_kernel<TYPE, true> : output_copy_kernel<TYPE, false>;
    kernel<<<(unsigned)std::max(blocks, 1), kThreads, 0, stream>>>(A);
    *this = CopyList{{.scales = A.scales}};
    return launch_status();
  }
};
// Rows for the logits: where they lie, or copied.
Operand logits_operand(CopyList& copies, int type, const void* from, int64_t stride, int64_t rows, const qa_output_layer& L, const Plan& P, bool copy, char* to,
                       int* exps) {
  if (!copy) return {from, stride, 0, rows};
  copies.add(type == QA_F32 ? kOwnScale : kAsTheyAre, from, stride, rows, L.features, to, P.parts * P.hp, rows, exps, false);
  return {to, P.parts * P.hp, 0, rows};
}
// Logits of a piece of the vocabulary: w's rows by x's.
template <bool BF16, Lies LIE, HowMany MANY, class Epilogue>
int logits_launch(const Operand& w, const Operand& x, int64_t features, Tall tiles, const Epilogue& out, hipStream_t stream, const Fewer& fewer = {}) {
  constexpr bool kApart = LIE == kRowsOfParts;
  switch (tiles) {
    case kTall128: return product_launch<Product<BF16, LIE, LIE, 2, 2, 2, 2, 1, kApart>, false, MANY>(w, x, features, out, 1, stream, 1, fewer);
    case kTall128Two: return product_launch<Product<BF16, LIE, LIE, 2, 2, 2, 2, 2, kApart>, false, MANY>(w, x, features, out, 1, stream, 1, fewer);
    case kTall64: return product_launch<Product<BF16, LIE, LIE, 1, 1, 2, 2, 4, kApart>, false, MANY>(w, x, features, out, 1, stream, 1, fewer);
    case kFlat: return product_launch<Product<BF16, LIE, LIE, 4, 1, 2, 2, 1, kApart>, false, MANY>(w, x, features, out, 1, stream, 1, fewer);
    default: break;
  }
  if constexpr (!kApart) return product_launch<Product256<BF16, LIE, LIE>, false, MANY>(w, x, features, out, 1, stream, 1, fewer);
  return QA_ERR_INVALID_ARG;                       // not reached: no such tiles with parts
}

int join_launch(const ScoreArgs& A, const qa_output_layer& L, int64_t chunks, const int32_t* target, float* logprob, float* entropy, float* stats, hipStream_t stream) {
  const auto launch = [&](auto kernel, int rows, int threads) {
    kernel<<<(unsigned)ceil_div(L.rows, rows), threads, 0, stream>>>(A, L.rows, chunks, L.vocab, target, logprob, entropy, stats);
    return launch_status();
  };
  if (L.rows <= kFewRows) return launch(output_join_kernel<1, 1024>, 1, 1024);
  if (L.rows <= 2048) return launch(output_join_kernel<4, kThreads>, 4, kThreads);
  return launch(output_join_kernel<16, kThreads>, 16, kThreads);
}
template <int TYPE>
int score_launch(const qa_output_layer& L, const void* x, const void* w, const int32_t* target, float* logprob, float* entropy, float* stats,
                 char* ws, hipStream_t stream) {
  const Plan P = plan_of(L, QA_OP_LOGPROB, TYPE, x, w);
  int* const x_exp = (int*)(ws + P.x_exp);
  int* const w_exp = (int*)(ws + P.w_exp);
  ScoreArgs A = {(float*)(ws + P.m), (float*)(ws + P.s), (float*)(ws + P.sw), (float*)(ws + P.given), 0, 0};
  if (P.streams) {
    const StreamArgs S = {LayerArgs{L.rows, L.vocab, nullptr, nullptr, target}, A, x, w, L.x_stride, L.w_stride, (int)L.features, P.each};
    const auto kernel = L.rows <= 16 ? output_stream_kernel<TYPE, 1> : L.rows <= 32 ? output_stream_kernel<TYPE, 2> : output_stream_kernel<TYPE, 4>;
    kernel<<<(unsigned)P.chunks, kStreamGroup, 0, stream>>>(S);
    return join_launch(A, L, P.chunks, target, logprob, entropy, stats, stream);
  }
  const auto from = [](auto* p, int64_t n) { return p ? p + n : p; };
  for (int64_t t = 0; t < L.rows; t += P.rows) {
    qa_output_layer here = L;
    here.rows = std::min(P.rows, L.rows - t);
    const int32_t* const its_target = from(target, t);
    CopyList copies;
    const Operand xo = logits_operand(copies, TYPE, (const ElemT<TYPE>*)x + t * L.x_stride, L.x_stride, here.rows, here, P, P.copy_x, ws + P.x, x_exp);
    for (int64_t first = 0; first < L.vocab; first += P.piece) {
      const int64_t vocab = std::min(P.piece, L.vocab - first);
      const Operand wo = logits_operand(copies, TYPE, (const ElemT<TYPE>*)w + first * L.w_stride, L.w_stride, vocab, here, P, P.copy_w, ws + P.w, w_exp);
      if (const int rc = copies.launch<TYPE>(stream)) return rc;
      A.first = first;
      A.first_chunk = first / P.piece * chunks_of(P.tiles) * ceil_div(P.piece, height_of(P.tiles));
      const ScoreOut<TYPE == QA_F32> out{LayerArgs{here.rows, vocab, x_exp, w_exp, its_target}, A};
      if (const int rc = logits_launch<TYPE == QA_BF16, TYPE == QA_F32 ? kRowsOfParts : kRows, kAll>(wo, xo, L.features, P.tiles, out, stream)) return rc;
    }
    if (const int rc = join_launch(A, here, P.chunks, its_target, from(logprob, t), from(entropy, t), from(stats, 2 * t), stream)) return rc;
  }
  return QA_OK;
}

template <int TYPE>
int sum_launch(const float* sums, const Splits& splits, int64_t rows, int64_t cols, ElemT<TYPE>* out, int64_t stride, int accumulate, hipStream_t stream,
               const int* list = nullptr, const Scales* scales = nullptr) {
  const int64_t vecs = rows * ceil_div(cols, kVec);
  output_sum_kernel<TYPE><<<(unsigned)std::min<int64_t>(ceil_div(vecs, kThreads), 4096), kThreads, 0, stream>>>(sums, splits, rows, cols, out, stride, accumulate, list, scales);
  return launch_status();
}
template <Lies LA, Lies LB, HowMany MANY, class Epilogue>
int grad_product(const Operand& a, const Operand& b, int64_t k, const Epilogue& out, const ProductPlan& plan, const Fewer& fewer, hipStream_t stream) {
  if (plan.tiles == kTiles256) return product_launch<Product256<false, LA, LB>, false, MANY>(a, b, k, out, 1, stream, plan.splits, fewer);
  if (plan.tiles == kTiles128) return product_launch<Product128<false, LA, LB>, false, MANY>(a, b, k, out, 1, stream, plan.splits, fewer);
  return product_launch<Product<false, LA, LB, 2, 2, 2, 2, 2>, false, MANY>(a, b, k, out, 1, stream, plan.splits, fewer);
}

struct GradCall {
  const void *x, *w;
  RowArgs rows;
  void* dx;
  int64_t dx_stride;
  float* dw;
  int64_t dw_stride;
  int accumulate;
};

template <int TYPE>
int grad_rows_launch(const qa_output_layer& L, const GradCall& G, char* ws, hipStream_t stream) {
  const Plan P = plan_of(L, QA_OP_LOGPROB_GRAD, TYPE, G.x, G.w);
  Scales* const scales = (Scales*)(ws + P.scales);
  const auto blocks = [](bool wanted, int64_t n, int64_t each) { return wanted ? (int)std::min<int64_t>(kMostBlocks, ceil_div(n, each)) : 0; };
  const int64_t share = whole(ceil_div(L.rows, kMostBlocks), kThreads);
  int* const place = (int*)(ws + P.place);
  int* const list = (int*)(ws + P.list);
  int* const c_exp = (int*)(ws + P.c_exp);
  int* const x_exp = (int*)(ws + P.x_exp);
  int* const w_exp = (int*)(ws + P.w_exp);
  const bool can_be_wide = P.copies && TYPE != QA_F16;
  const Fewer rows = {.n = &scales->rows};
  const MostArgs most = {G.rows, L.rows, L.vocab, L.features, G.x, G.w, L.x_stride, L.w_stride, scales, place, share,
                         {(int)ceil_div(L.rows, share), blocks(G.dw || P.copies, L.rows, kWaves), blocks(TYPE != QA_F16 && (G.dx || P.copies), L.vocab, kWaves)}};
  output_most_kernel<TYPE><<<(unsigned)(most.blocks[0] + most.blocks[1] + most.blocks[2]), kThreads, 0, stream>>>(most);
  if (const int rc = launch_status()) return rc;

  const int64_t copied = P.parts * P.hc;
  CopyList copies;
  copies.A.scales = scales;
  copies.A.first = true;
  for (int i = 0; i < 3; ++i) copies.A.found[i] = most.blocks[i];
  copies.A.features = L.features;
  copies.A.R = G.rows;
  copies.A.place = place;
  copies.A.share = share;
  copies.A.list = list;
  copies.A.c_exp = c_exp;
  copies.A.zero = G.dx;
  copies.A.zero_stride = G.dx_stride;
  // For the logits, and beside c.
  copies.add(TYPE == QA_F16 || !P.copies ? kAsTheyAre : kOwnScale, G.x, L.x_stride, L.rows, L.features, ws + P.xr, copied, L.rows, x_exp, true, !P.copies);
  if (G.dw) copies.add(kScaleBesideC, G.x, L.x_stride, L.rows, L.features, ws + P.xc, copied, L.rows, nullptr, true);
  // Where few rows count, dx has more splits instead of tiles, in the same room.
  Fewer dx_rows = rows;
  const int64_t dx_side = P.dx.tiles == kTiles256 ? 256 : 128;
  const Splits dx_splits = {(int)P.dx.splits, (int)std::max(P.dx.splits, std::min<int64_t>(64, std::min(P.piece, L.vocab) / (8 * kWholeStep))),
                            (unsigned)dx_side};
  if (P.dx.splits > 1) dx_rows.most_splits = dx_splits.most;
  constexpr Lies kColumnsOf = TYPE == QA_F32 ? kColumnsOfParts : kColumns;
  for (int64_t first = 0; first < L.vocab; first += P.piece) {
    const int64_t vocab = std::min(P.piece, L.vocab - first);
    const void* const from = (const ElemT<TYPE>*)G.w + first * L.w_stride;
    Operand wc = {from, L.w_stride, 0, L.features};
    if (P.copies || (G.dx && (TYPE != QA_F16 || vocab % kWholeStep))) {
      wc = {ws + P.wc, copied, 0, L.features};
      copies.add(kScaleOfW, from, L.w_stride, vocab, L.features, ws + P.wc, copied, whole(vocab, kWholeStep), w_exp, false, false, can_be_wide ? ws + P.wr : nullptr);
    }
    if (const int rc = copies.launch<TYPE>(stream)) return rc;
    _Float16* const c = (_Float16*)(ws + P.c);
    const Tall tiles = logits_tiles(L.rows, vocab, L.features, TYPE);
    const auto logits = [&](auto entropy) {
      constexpr bool kEntropy = decltype(entropy)::value;
      if (P.copies) {
        const LogitsGradOut<TYPE != QA_F16, kEntropy> grad{vocab, G.rows, list, x_exp, w_exp, first, scales, c, 2 * P.vp};
        Fewer or_wide = rows;
        if (can_be_wide) {
          or_wide.wide = &scales->wide;
          or_wide.wide_a = ws + P.wr;
        }
        return logits_launch<false, TYPE == QA_F32 ? kRowsOfParts : kRows, kFewerOfB>(Operand{wc.p, wc.ld, 0, vocab}, Operand{ws + P.xr, copied, 0, L.rows}, L.features, tiles, grad, stream, or_wide);
      }
      if constexpr (TYPE != QA_F32) {              // copied always
        const LogitsGradOut<false, kEntropy> grad{vocab, G.rows, list, nullptr, nullptr, first, scales, c, 2 * P.vp};
        Fewer or_all = rows;
        or_all.all = G.x;
        or_all.all_ld = L.x_stride;
        return logits_launch<TYPE == QA_BF16, kRows, kFewerOfB>(Operand{from, L.w_stride, 0, vocab}, Operand{ws + P.xr, copied, 0, L.rows}, L.features, tiles, grad, stream, or_all);
      }
      return (int)QA_ERR_INVALID_ARG;              // not reached
    };
    if (const int rc = G.rows.g_entropy ? logits(std::true_type()) : logits(std::false_type())) return rc;
    if (G.dx) {
      const bool last = first + P.piece >= L.vocab;
      const GradOut<TYPE, true> out{(ElemT<TYPE>*)G.dx, P.pieces > 1 || P.dx.splits > 1 ? (float*)(ws + P.sums) : nullptr, scales, G.dx_stride, L.rows, L.features,
                              first > 0, last && P.dx.splits == 1, list, c_exp};
      // One part of c has 11 bits, which is little beside bfloat16's 8, but as much as binary16's own.
      constexpr Lies kC = TYPE == QA_BF16 ? kHiOfRows : kRowsOfParts;
      if (const int rc = grad_product<kColumnsOf, kC, kFewerOfB>(wc, Operand{c, 2 * P.vp, 0, L.rows}, vocab, out, P.dx, dx_rows, stream)) return rc;
      if (last && P.dx.splits > 1)
        if (const int rc = sum_launch<TYPE>((const float*)(ws + P.sums), dx_splits, L.rows, L.features, (ElemT<TYPE>*)G.dx, G.dx_stride, 0, stream, list, scales)) return rc;
    }
    if (G.dw) {
      float* const dw = G.dw + first * G.dw_stride;
      const ProductPlan plan = dw_plan(L, TYPE, vocab);
      float* const sums = plan.splits > 1 ? (float*)(ws + P.dw_sums) : nullptr;
      const GradOut<QA_F32, false> out{dw, sums, scales, G.dw_stride, vocab, L.features, !sums && G.accumulate, !sums, nullptr, nullptr};
      if (const int rc = grad_product<kColumnsOf, kColumnsOfParts, kFewerOfK>(Operand{ws + P.xc, copied, 0, L.features}, Operand{c, 2 * P.vp, 0, vocab}, L.rows, out, plan, rows, stream)) return rc;
      if (sums)
        if (const int rc = sum_launch<QA_F32>(sums, Splits{(int)plan.splits}, vocab, L.features, dw, G.dw_stride, G.accumulate, stream)) return rc;
    }
  }
  return QA_OK;
}

template <int TYPE>
int grad_launch(const qa_output_layer& L, const GradCall& G, char* ws, hipStream_t stream) {
  const auto from = [](auto* p, int64_t n) { return p ? p + n : p; };
  const int64_t piece = grad_rows_of(L);
  for (int64_t t = 0; t < L.rows; t += piece) {
    qa_output_layer here = L;
    here.rows = std::min(piece, L.rows - t);
    GradCall its = G;
    its.x = (const ElemT<TYPE>*)G.x + t * L.x_stride;
    its.rows.target = from(G.rows.target, t);
    its.rows.stats = G.rows.stats + 2 * t;
    its.rows.entropy = from(G.rows.entropy, t);
    its.rows.g_logprob = from(G.rows.g_logprob, t);
    its.rows.g_entropy = from(G.rows.g_entropy, t);
    its.dx = from((ElemT<TYPE>*)G.dx, t * G.dx_stride);
    its.accumulate = t > 0 || G.accumulate;
    if (const int rc = grad_rows_launch<TYPE>(here, its, ws, stream)) return rc;
  }
  return QA_OK;
}

int check_layer(const qa_output_layer* L, int type) {
  if (!L || !known_type(type)) return QA_ERR_INVALID_ARG;
  constexpr int64_t kMost = int64_t(1) << 24, kStride = int64_t(1) << 40;
  if (L->rows < 0 || L->rows >= kMost || L->vocab < 1 || L->vocab >= kMost || L->features < 1 || L->features >= (int64_t(1) << 20)) return QA_ERR_INVALID_ARG;
  if (L->x_stride < L->features || L->x_stride >= kStride || L->w_stride < L->features || L->w_stride >= kStride) return QA_ERR_INVALID_ARG;
  return QA_OK;
}

}  // namespace
}  // namespace qa

using namespace qa;

extern "C" size_t qa_output_workspace_bytes(const qa_output_layer* layer, int op, int type) {
  if (check_layer(layer, type) != QA_OK || layer->rows == 0 || (op != QA_OP_LOGPROB && op != QA_OP_LOGPROB_GRAD)) return 0;
  return bytes_of(*layer, op, type);
}

extern "C" int qa_output_logprob(const qa_output_layer* layer, int type, const void* x, const void* w, const int32_t* target, float* logprob,
                                 float* entropy, float* stats, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_layer(layer, type)) return rc;
  if (layer->rows == 0) return QA_OK;
  if (!x || !w || !target != !logprob) return QA_ERR_INVALID_ARG;
  if (!element_aligned(x, type) || !element_aligned(w, type) || !aligned(target, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(stats, 4))
    return QA_ERR_ALIGNMENT;
  if (!ws || ws_bytes < bytes_of(*layer, QA_OP_LOGPROB, type)) return QA_ERR_WORKSPACE;
  if (!aligned(ws, 256)) return QA_ERR_ALIGNMENT;
  const auto launch = type == QA_F32 ? score_launch<QA_F32> : type == QA_BF16 ? score_launch<QA_BF16> : score_launch<QA_F16>;
  return launch(*layer, x, w, target, logprob, entropy, stats, (char*)ws, (hipStream_t)stream);
}

extern "C" int qa_output_logprob_grad(const qa_output_layer* layer, int type, const void* x, const void* w, const int32_t* target, const float* stats,
                                      const float* entropy, const float* g_logprob, const float* g_entropy, void* dx, int64_t dx_stride, float* dw,
                                      int64_t dw_stride, int accumulate, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_layer(layer, type)) return rc;
  if ((!dx && !dw) || (dx && dx_stride < layer->features) || (dw && dw_stride < layer->features) || (accumulate != 0 && accumulate != 1)) return QA_ERR_INVALID_ARG;
  if (!aligned(dw, 4) || (dx && !element_aligned(dx, type))) return QA_ERR_ALIGNMENT;
  const hipStream_t s = (hipStream_t)stream;
  if (layer->rows == 0) {
    if (!dw || accumulate) return QA_OK;
    output_zero_kernel<<<(unsigned)std::min<int64_t>(layer->vocab, 4096), kThreads, 0, s>>>(dw, dw_stride, layer->vocab, layer->features);
    return launch_status();
  }
  if (!x || !w || !stats || !entropy != !g_entropy || (g_logprob && !target)) return QA_ERR_INVALID_ARG;
  if (!element_aligned(x, type) || !element_aligned(w, type) || !aligned(target, 4) || !aligned(stats, 4) || !aligned(entropy, 4) || !aligned(g_logprob, 4) ||
      !aligned(g_entropy, 4))
    return QA_ERR_ALIGNMENT;
  if (!ws || ws_bytes < bytes_of(*layer, QA_OP_LOGPROB_GRAD, type)) return QA_ERR_WORKSPACE;
  if (!aligned(ws, 256)) return QA_ERR_ALIGNMENT;
  const GradCall G = {x, w, RowArgs{target, stats, entropy, g_logprob, g_entropy, layer->vocab}, dx, dx_stride, dw, dw_stride, accumulate};
  const auto launch = type == QA_F32 ? grad_launch<QA_F32> : type == QA_BF16 ? grad_launch<QA_BF16> : grad_launch<QA_F16>;
  return launch(*layer, G, (char*)ws, s);
}
