// Log probabilities of targets under an output layer, and their gradient, without the logits in memory.
//
// Logits are products of the matrix cores with rows of w along the tile's height and rows of x along its width, so that a lane holds
// many logits of one row: a tile's maximum and sums are formed in registers, and a row's numbers are joined from one triple per
// chunk of the vocabulary.  The backward pass multiplies the logits again, a piece of the vocabulary at a time, turns them into
// c, the gradient of the logits, which is written in binary16 parts along the vocabulary (for dx = c w) and along the rows
// (for dw = c^T x), and multiplies those with transposes of w's piece and of x.
#include <algorithm>

#include "qa_product.h"
#include "qa_softmax.h"

namespace qa {
namespace {

struct LayerArgs {
  int64_t rows, vocab;
  const int *x_exp, *w_exp;                        // binary32: operands are x 2^x_exp[row], w 2^w_exp[row]
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

// Rows copied to whole steps of k: 16-bit elements as they are, binary32 ones in two parts times a power of two per row.  A wave per row.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void output_rows_kernel(const void* from, int64_t stride, int64_t rows, int64_t cols, uint16_t* to,
                                                               int64_t ld, int64_t part, int* exps) {
  const int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
  const int lane = threadIdx.x % kWave;
  if (row >= rows) return;
  const ElemT<TYPE>* p = (const ElemT<TYPE>*)from + row * stride;
  uint16_t* q = to + row * ld;
  if constexpr (TYPE != QA_F32) {
    for (int64_t c = lane * kVec; c < ld; c += kWave * kVec) {
      const int n = (int)max((int64_t)0, min((int64_t)kVec, cols - c));
      *reinterpret_cast<u32x4*>(q + c) = n ? load_raw<TYPE>(p + c, n).a : u32x4{};
    }
  } else {
    uint32_t most = 0;
    for (int64_t c = lane * kVec; c < cols; c += kWave * kVec) {
      float v[kVec];
      to_f32<TYPE>(load_raw<TYPE>(p + c, (int)min((int64_t)kVec, cols - c)), v);
      most = max(most, finite_most(v));
    }
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s, kWave));
    const int exp = exponent_for(most);
    if (lane == 0) exps[row] = exp;
    for (int64_t c = lane * kVec; c < ld; c += kWave * kVec) {
      const int n = (int)max((int64_t)0, min((int64_t)kVec, cols - c));
      float v[kVec] = {};
      if (n) to_f32<TYPE>(load_raw<TYPE>(p + c, n), v);
      _Float16 hi[kVec], lo[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) split_f16(i < n ? ldexpf(v[i], exp) : 0.0f, hi[i], lo[i]);
      __builtin_memcpy(__builtin_assume_aligned(q + c, 16), hi, sizeof hi);
      __builtin_memcpy(__builtin_assume_aligned(q + part + c, 16), lo, sizeof lo);
    }
  }
}

// ---- scoring ------------------------------------------------------------------------------------------------------------------

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
  float *m, *s, *w;                                // [chunk][rows]
  float* given;                                    // the targets' logits
  int64_t first, first_chunk;                      // of this launch's vocabulary
};

template <bool SCALED>
struct ScoreOut {
  LayerArgs L;                                     // vocab: of this launch
  ScoreArgs A;
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t v0, int64_t t0) const {
    constexpr int kChunk = 32 * (int)(sizeof p.acc / sizeof p.acc[0]);
    if (v0 >= L.vocab) return;
#pragma unroll
    for (int j = 0; j < (int)(sizeof p.acc[0] / sizeof p.acc[0][0]); ++j) {
      const int64_t t = t0 + 32 * j + threadIdx.x % 32;
      const int x_exp = SCALED ? L.x_exp[min(t, L.rows - 1)] : 0;
      const int64_t at = L.target && t < L.rows ? (int64_t)L.target[t] - A.first - v0 : -1;
      const int here = at >= 0 && at < kChunk ? (int)at : -1, left = (int)min((int64_t)kChunk, L.vocab - v0);
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
      if (here >= 0 && here < left && here / 4 % 2 == (int)threadIdx.x % kWave / 32) A.given[t] = given;
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

// A row's numbers from its chunks': ROWS rows per work-group, the other threads along the chunks.
template <int ROWS>
__global__ __launch_bounds__(kThreads) void output_join_kernel(ScoreArgs A, int64_t rows, int64_t chunks, int64_t vocab, const int32_t* target,
                                                               float* logprob, float* entropy, float* stats) {
  constexpr int kShare = kThreads / ROWS;
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

// Exponents of the powers of two that the gradient's operands are scaled by, and largest magnitudes (bits) before them.
struct Scales { uint32_t most[4]; };
enum { kOfC, kOfX, kOfW };

__global__ void output_clear_kernel(Scales* s) { s->most[threadIdx.x] = 0; }

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

// The largest |c| that a row can have: p <= 1, p |log p| <= 1 / e, and an entropy of at most log 2^24 < 17.
__global__ __launch_bounds__(kThreads) void output_weights_kernel(RowArgs A, int64_t rows, Scales* scales) {
  uint32_t most = 0;
  for (int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x; t < rows; t += (int64_t)gridDim.x * kThreads) {
    const Row r = row_of(A, t);
    const uint32_t c = as_u32(fabsf(r.a) + 18.0f * fabsf(r.e));
    if (c < 0x7F800000u) most = max(most, c);
  }
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s, kWave));
  if (threadIdx.x % kWave == 0) atomicMax(&scales->most[kOfC], most);
}

// The largest finite magnitude of rows that count.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void output_most_kernel(const void* from, int64_t stride, int64_t rows, int64_t cols, RowArgs A, bool masked,
                                                               Scales* scales, int which) {
  uint32_t most = 0;
  const int lane = threadIdx.x % kWave;
  for (int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; row < rows; row += (int64_t)gridDim.x * kWaves) {
    if (masked && !counts(row_of(A, row))) continue;
    const ElemT<TYPE>* p = (const ElemT<TYPE>*)from + row * stride;
    for (int64_t c = lane * kVec; c < cols; c += kWave * kVec) {
      float v[kVec];
      to_f32<TYPE>(load_raw<TYPE>(p + c, (int)min((int64_t)kVec, cols - c)), v);
      most = max(most, finite_most(v));
    }
  }
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s, kWave));
  if (lane == 0) atomicMax(&scales->most[which], most);
}

// Transpose of rows [0, rows) in one or two binary16 parts, scaled, with zeros up to a whole step of k and in rows that do not count.
template <int TYPE, int PARTS>
__global__ __launch_bounds__(kThreads) void output_transpose_kernel(const void* from, int64_t stride, int64_t rows, int64_t cols, RowArgs A, bool masked,
                                                                    const Scales* scales, int which, _Float16* to, int64_t ld, int64_t part) {
  constexpr int kSide = 64;
  __shared__ uint32_t tile[kSide][kSide + 1];
  const int64_t r0 = (int64_t)blockIdx.x * kSide, c0 = (int64_t)blockIdx.y * kSide;
  const int exp = TYPE == QA_F16 ? 0 : exponent_for(scales->most[which]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = h * 32 + (int)threadIdx.x / 8, col = (int)threadIdx.x % 8 * kVec;
    const int64_t r = r0 + row, c = c0 + col;
    int n = r < rows ? (int)max((int64_t)0, min((int64_t)kVec, cols - c)) : 0;
    if (n && masked && !counts(row_of(A, r))) n = 0;
    float v[kVec] = {};
    if (n) to_f32<TYPE>(load_raw<TYPE>((const ElemT<TYPE>*)from + r * stride + c, n), v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      _Float16 hi, lo;
      split_f16(i < n ? ldexpf(v[i], exp) : 0.0f, hi, lo);
      tile[row][col + i] = (uint32_t)__builtin_bit_cast(uint16_t, hi) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = h * 32 + (int)threadIdx.x / 8, row = (int)threadIdx.x % 8 * kVec;
    const int64_t c = c0 + col, r = r0 + row;
    if (c >= cols || r >= ld) continue;
    u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = tile[row + 2 * i][col], v = tile[row + 2 * i + 1][col];
      hi[i] = __builtin_amdgcn_perm(v, u, 0x05040100u);
      lo[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
    }
    _Float16* p = to + c * ld + r;
    *reinterpret_cast<u32x4*>(p) = hi;
    if (PARTS == 2) *reinterpret_cast<u32x4*>(p + part) = lo;
  }
}

// c of a piece of the vocabulary, scaled: along the vocabulary (C_PARTS parts, none: not wanted) and along the rows (two parts).
template <bool SCALED, int C_PARTS, bool DW>
struct LogitsGradOut {
  LayerArgs L;                                     // vocab: of this piece
  RowArgs R;
  int64_t first;                                   // of the piece
  const Scales* scales;
  _Float16 *c, *ct;
  int64_t c_ld, c_part, ct_ld, ct_part;            // whole steps of k: zeros behind the piece and behind the rows
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t v0, int64_t t0) const {
    const int exp = exponent_for(scales->most[kOfC]);
#pragma unroll
    for (int j = 0; j < (int)(sizeof p.acc[0] / sizeof p.acc[0][0]); ++j) {
      const int64_t t = t0 + 32 * j + threadIdx.x % 32;
      const int x_exp = SCALED ? L.x_exp[min(t, L.rows - 1)] : 0;
      const Row r = row_of(R, min(t, L.rows - 1));
      const bool none = t >= L.rows || !counts(r);
      const int64_t at = r.at - first - v0;
      const int here = at >= 0 && at < P::kM ? (int)at : -1, left = (int)max((int64_t)0, min((int64_t)P::kM, L.vocab - v0));
      const int wide = (int)max((int64_t)0, min((int64_t)P::kM, c_ld - v0));
      _Float16 *const c_row = c + t * c_ld + v0, *const ct_row = ct + v0 * ct_ld + t;
      for_logits<SCALED>(p, L, v0, j, x_exp, [&](int v, int, int, float (&z)[4]) {
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lp = (z[e] - r.m) - r.log_sum, q = __builtin_amdgcn_exp2f(lp * kLog2e);
          float g = -q * (r.a + r.e * (fmaxf(lp, kFar) + r.h));
          if (v + e == here) g += r.a;
          _Float16 a, b;
          split_f16(none || v + e >= left ? 0.0f : ldexpf(g, exp), a, b);
          hi[e] = a;
          lo[e] = b;
        }
        if (C_PARTS && t < L.rows && v < wide) {
          *reinterpret_cast<f16x4*>(c_row + v) = hi;
          if (C_PARTS == 2) *reinterpret_cast<f16x4*>(c_row + c_part + v) = lo;
        }
        if (DW && t < ct_ld) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < left) {
              ct_row[(v + e) * ct_ld] = hi[e];
              ct_row[(v + e) * ct_ld + ct_part] = lo[e];
            }
        }
      });
    }
  }
};

// Sums of a product, unscaled, rounded to the type or added in binary32.
template <int TYPE>
struct GradOut {
  ElemT<TYPE>* out;
  float* sums;                                     // NULL: none before this piece, and this is the last
  const Scales* scales;
  int64_t stride, rows, cols;
  int which;
  bool add, last;                                  // to what is in sums (or, of binary32, in out); the last piece writes out
  template <class P> __device__ __forceinline__ void operator()(P& p, int64_t m0, int64_t n0) const {
    const int lane = threadIdx.x % kWave, x = which == kOfX || which == kOfW ? (int)scales->most[which] : 0;
    const int exp = -(exponent_for(scales->most[kOfC]) + exponent_for((uint32_t)x));
#pragma unroll
    for (int i = 0; i < (int)(sizeof p.acc / sizeof p.acc[0]); ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t row = m0 + 32 * i + 8 * q + 4 * (lane / 32) + e;
          if (row >= rows) continue;
#pragma unroll
          for (int j = 0; j < (int)(sizeof p.acc[0] / sizeof p.acc[0][0]); ++j) {
            const int64_t col = n0 + 32 * j + lane % 32;
            if (col >= cols) continue;
            float v = ldexpf(p.acc[i][j][4 * q + e], exp);
            if (sums) {
              float* s = sums + row * cols + col;
              if (add) v += *s;
              if (!last) *s = v;
            } else if (add) {
              v += (float)out[row * stride + col];
            }
            if (last) out[row * stride + col] = (ElemT<TYPE>)v;
          }
        }
  }
};
__global__ __launch_bounds__(kThreads) void output_zero_kernel(float* p, int64_t stride, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) p[r * stride + c] = 0.0f;
}

// ---- what a call does ------------------------------------------------------------------------------------------------------------

constexpr int64_t kPieceBytes = int64_t(256) << 20;

int64_t whole_steps(int64_t k) { return ceil_div(k, kProductStep) * kProductStep; }
int parts_for(int type) { return type == QA_F32 ? 2 : 1; }

struct Room {
  size_t bytes = 0;
  size_t take(int64_t n) {
    const size_t at = bytes;
    bytes += ((size_t)n + 255) / 256 * 256;
    return at;
  }
};

// Which tiles multiply the logits: heights (vocabulary) of chunks, and widths (rows).
enum { kTiles256, kTiles128, kTiles64 };
int logits_tiles(int64_t rows, int64_t vocab) {
  if (rows <= 64) return kTiles64;
  return ceil_div(rows, 256) * ceil_div(vocab, 256) >= 192 ? kTiles256 : kTiles128;
}
constexpr int64_t chunk_of(int tiles) { return tiles == kTiles256 ? 128 : 64; }

struct Plan {
  bool copy_x, copy_w;
  int64_t hp, piece, pieces;                       // copied rows' length; vocabulary of a launch
  int tiles;
  size_t xs, ws, x_exp, w_exp;                     // copies and exponents
  size_t m, s, w, given;                           // scoring
  int64_t chunks;
  size_t scales, xt, wt, c, ct, sums;              // gradient
  int64_t tp, vp;
  size_t bytes;
};

bool in_place(int type, const void* p, int64_t stride, int64_t features) {
  return type != QA_F32 && features % kProductStep == 0 && stride % 8 == 0 && stride < (int64_t(1) << 22) && aligned(p, 16);
}
// p NULL: a place of any alignment.
Plan plan_of(const qa_output_layer& L, int op, int type, const void* x, const void* w) {
  Plan P = {};
  Room room;
  const int parts = parts_for(type);
  P.copy_x = !x || !in_place(type, x, L.x_stride, L.features);
  P.copy_w = !w || !in_place(type, w, L.w_stride, L.features);
  P.hp = whole_steps(L.features);
  if (op == QA_OP_LOGPROB) {
    P.tiles = logits_tiles(L.rows, L.vocab);
    const int64_t most = std::max<int64_t>(16384, kPieceBytes / (P.hp * 2 * parts) / 256 * 256);
    P.piece = P.copy_w ? std::min(L.vocab, most) : L.vocab;
    P.pieces = ceil_div(L.vocab, P.piece);
    P.chunks = ceil_div(L.vocab, chunk_of(P.tiles));
    P.m = room.take(4 * P.chunks * L.rows);
    P.s = room.take(4 * P.chunks * L.rows);
    P.w = room.take(4 * P.chunks * L.rows);
    P.given = room.take(4 * L.rows);
  } else {
    const int64_t each = L.rows * 2 * (parts + 2) + L.features * 2 * parts;
    P.piece = std::min(whole_steps(L.vocab), std::max<int64_t>(1024, 2 * kPieceBytes / each / 256 * 256));
    P.pieces = ceil_div(L.vocab, P.piece);
    P.tiles = logits_tiles(L.rows, P.piece);
    P.tp = whole_steps(L.rows);
    P.vp = P.piece;
    P.scales = room.take(sizeof(Scales));
    P.xt = room.take(2 * parts * L.features * P.tp);
    P.wt = room.take(2 * parts * L.features * P.vp);
    P.c = room.take(2 * parts * L.rows * P.vp);
    P.ct = room.take(2 * 2 * P.piece * P.tp);
    P.sums = room.take(P.pieces > 1 ? 4 * L.rows * L.features : 0);
  }
  P.x_exp = room.take(type == QA_F32 ? 4 * L.rows : 0);
  P.w_exp = room.take(type == QA_F32 ? 4 * P.piece : 0);
  P.xs = room.take(P.copy_x ? 2 * parts * L.rows * P.hp : 0);
  P.ws = room.take(P.copy_w ? 2 * parts * P.piece * P.hp : 0);
  P.bytes = room.bytes;
  return P;
}
// Any alignment of x and w: the most that a call may take.
size_t bytes_of(const qa_output_layer& L, int op, int type) { return plan_of(L, op, type, nullptr, nullptr).bytes; }

struct Operand { const uint16_t* p; int64_t ld, part; };

template <int TYPE>
int copy_rows(const void* from, int64_t stride, int64_t rows, int64_t cols, uint16_t* to, int64_t ld, int* exps, hipStream_t stream) {
  output_rows_kernel<TYPE><<<(unsigned)ceil_div(rows, kWaves), kThreads, 0, stream>>>(from, stride, rows, cols, to, ld, rows * ld, exps);
  return launch_status();
}

// Logits of a piece of the vocabulary: w's rows by x's.
template <int TYPE, class Epilogue>
int logits_launch(const Operand& w, const Operand& x, int64_t vocab, int64_t rows, int64_t hp, int tiles, const Epilogue& out, hipStream_t stream) {
  ProductArgs A = {};
  A.a = w.p;
  A.b = x.p;
  A.lda = w.ld;
  A.ldb = x.ld;
  A.a_part = w.part;
  A.b_part = x.part;
  A.m = vocab;
  A.n = rows;
  A.steps = (int)(hp / kProductStep);
  constexpr bool kBf16 = TYPE == QA_BF16;
  constexpr int kPasses = TYPE == QA_F32 ? 3 : 1;
  if (tiles == kTiles256) return product_launch<kBf16, kPasses, 2, 4, 4, 2>(A, out, 1, 1, stream);
  if (tiles == kTiles128) return product_launch<kBf16, kPasses, 2, 2, 2, 2>(A, out, 1, 1, stream);
  return product_launch<kBf16, kPasses, 4, 1, 2, 2>(A, out, 1, 1, stream);
}

template <int TYPE>
int score_launch(const qa_output_layer& L, const void* x, const void* w, const int32_t* target, float* logprob, float* entropy, float* stats,
                 char* ws, hipStream_t stream) {
  const Plan P = plan_of(L, QA_OP_LOGPROB, TYPE, x, w);
  int* const x_exp = (int*)(ws + P.x_exp);
  int* const w_exp = (int*)(ws + P.w_exp);
  Operand xo = {(const uint16_t*)x, L.x_stride, 0};
  if (P.copy_x) {
    xo = {(const uint16_t*)(ws + P.xs), P.hp, L.rows * P.hp};
    if (const int rc = copy_rows<TYPE>(x, L.x_stride, L.rows, L.features, (uint16_t*)(ws + P.xs), P.hp, x_exp, stream)) return rc;
  }
  ScoreArgs A = {(float*)(ws + P.m), (float*)(ws + P.s), (float*)(ws + P.w), (float*)(ws + P.given), 0, 0};
  for (int64_t first = 0; first < L.vocab; first += P.piece) {
    const int64_t vocab = std::min(P.piece, L.vocab - first);
    const void* const from = (const ElemT<TYPE>*)w + first * L.w_stride;
    Operand wo = {(const uint16_t*)from, L.w_stride, 0};
    if (P.copy_w) {
      wo = {(const uint16_t*)(ws + P.ws), P.hp, vocab * P.hp};
      if (const int rc = copy_rows<TYPE>(from, L.w_stride, vocab, L.features, (uint16_t*)(ws + P.ws), P.hp, w_exp, stream)) return rc;
    }
    A.first = first;
    A.first_chunk = first / chunk_of(P.tiles);
    const ScoreOut<TYPE == QA_F32> out{LayerArgs{L.rows, vocab, x_exp, w_exp, target}, A};
    if (const int rc = logits_launch<TYPE>(wo, xo, vocab, L.rows, P.hp, P.tiles, out, stream)) return rc;
  }
  if (L.rows < 256)
    output_join_kernel<1><<<(unsigned)L.rows, kThreads, 0, stream>>>(A, L.rows, P.chunks, L.vocab, target, logprob, entropy, stats);
  else
    output_join_kernel<16><<<(unsigned)ceil_div(L.rows, 16), kThreads, 0, stream>>>(A, L.rows, P.chunks, L.vocab, target, logprob, entropy, stats);
  return launch_status();
}

template <int PASSES, class Epilogue>
int grad_product(const Operand& a, const Operand& b, int64_t m, int64_t n, int64_t k, const Epilogue& out, hipStream_t stream) {
  ProductArgs A = {};
  A.a = a.p;
  A.b = b.p;
  A.lda = a.ld;
  A.ldb = b.ld;
  A.a_part = a.part;
  A.b_part = b.part;
  A.m = m;
  A.n = n;
  A.steps = (int)(k / kProductStep);
  if (ceil_div(m, 256) * ceil_div(n, 256) >= 192) return product_launch<false, PASSES, 2, 4, 4, 2>(A, out, 1, 1, stream);
  return product_launch<false, PASSES, 2, 2, 2, 2>(A, out, 1, 1, stream);
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
template <int TYPE, int C_PARTS, bool DW>
int logits_grad(const Operand& w, const Operand& x, const LayerArgs& L, const RowArgs& R, int64_t hp, int64_t first, const Scales* scales, const Operand& c,
                const Operand& ct, int tiles, hipStream_t stream) {
  const LogitsGradOut<TYPE == QA_F32, C_PARTS, DW> out{L, R, first, scales, (_Float16*)c.p, (_Float16*)ct.p, c.ld, c.part, ct.ld, ct.part};
  return logits_launch<TYPE>(w, x, L.vocab, L.rows, hp, tiles, out, stream);
}

template <int TYPE>
int grad_launch(const qa_output_layer& L, const GradCall& G, char* ws, hipStream_t stream) {
  const Plan P = plan_of(L, QA_OP_LOGPROB_GRAD, TYPE, G.x, G.w);
  constexpr int kParts = TYPE == QA_F32 ? 2 : 1;
  int* const x_exp = (int*)(ws + P.x_exp);
  int* const w_exp = (int*)(ws + P.w_exp);
  Scales* const scales = (Scales*)(ws + P.scales);
  const auto most_blocks = [](int64_t rows) { return (unsigned)std::min<int64_t>(2048, ceil_div(rows, kWaves)); };
  output_clear_kernel<<<1, 4, 0, stream>>>(scales);
  output_weights_kernel<<<(unsigned)std::min<int64_t>(256, ceil_div(L.rows, kThreads)), kThreads, 0, stream>>>(G.rows, L.rows, scales);
  if (TYPE != QA_F16 && G.dw) output_most_kernel<TYPE><<<most_blocks(L.rows), kThreads, 0, stream>>>(G.x, L.x_stride, L.rows, L.features, G.rows, true, scales, kOfX);
  if (TYPE != QA_F16 && G.dx) output_most_kernel<TYPE><<<most_blocks(L.vocab), kThreads, 0, stream>>>(G.w, L.w_stride, L.vocab, L.features, G.rows, false, scales, kOfW);
  const Operand xt = {(const uint16_t*)(ws + P.xt), P.tp, L.features * P.tp}, wt = {(const uint16_t*)(ws + P.wt), P.vp, L.features * P.vp};
  if (G.dw)
    output_transpose_kernel<TYPE, kParts><<<dim3((unsigned)ceil_div(P.tp, 64), (unsigned)ceil_div(L.features, 64)), kThreads, 0, stream>>>(
        G.x, L.x_stride, L.rows, L.features, G.rows, true, scales, kOfX, (_Float16*)xt.p, xt.ld, xt.part);
  if (const int rc = launch_status()) return rc;
  Operand xo = {(const uint16_t*)G.x, L.x_stride, 0};
  if (P.copy_x) {
    xo = {(const uint16_t*)(ws + P.xs), P.hp, L.rows * P.hp};
    if (const int rc = copy_rows<TYPE>(G.x, L.x_stride, L.rows, L.features, (uint16_t*)(ws + P.xs), P.hp, x_exp, stream)) return rc;
  }
  const Operand c = {(const uint16_t*)(ws + P.c), P.vp, L.rows * P.vp}, ct = {(const uint16_t*)(ws + P.ct), P.tp, P.piece * P.tp};
  for (int64_t first = 0; first < L.vocab; first += P.piece) {
    const int64_t vocab = std::min(P.piece, L.vocab - first), vp = whole_steps(vocab);
    const void* const from = (const ElemT<TYPE>*)G.w + first * L.w_stride;
    Operand wo = {(const uint16_t*)from, L.w_stride, 0};
    if (P.copy_w) {
      wo = {(const uint16_t*)(ws + P.ws), P.hp, vocab * P.hp};
      if (const int rc = copy_rows<TYPE>(from, L.w_stride, vocab, L.features, (uint16_t*)(ws + P.ws), P.hp, w_exp, stream)) return rc;
    }
    const LayerArgs piece = {L.rows, vocab, x_exp, w_exp, nullptr};
    const auto form = G.dx && G.dw ? logits_grad<TYPE, kParts, true> : G.dx ? logits_grad<TYPE, kParts, false> : logits_grad<TYPE, 0, true>;
    if (const int rc = form(wo, xo, piece, G.rows, P.hp, first, scales, c, ct, P.tiles, stream)) return rc;
    if (G.dx) {
      output_transpose_kernel<TYPE, kParts><<<dim3((unsigned)ceil_div(vp, 64), (unsigned)ceil_div(L.features, 64)), kThreads, 0, stream>>>(
          from, L.w_stride, vocab, L.features, G.rows, false, scales, kOfW, (_Float16*)wt.p, wt.ld, wt.part);
      if (const int rc = launch_status()) return rc;
      const bool last = first + P.piece >= L.vocab;
      const GradOut<TYPE> out{(ElemT<TYPE>*)G.dx, P.pieces > 1 ? (float*)(ws + P.sums) : nullptr, scales, G.dx_stride, L.rows, L.features,
                              TYPE == QA_F16 ? -1 : kOfW, first > 0, last};
      if (const int rc = grad_product<TYPE == QA_F32 ? 3 : 1>(c, wt, L.rows, L.features, vp, out, stream)) return rc;
    }
    if (G.dw) {
      const GradOut<QA_F32> out{G.dw + first * G.dw_stride, nullptr, scales, G.dw_stride, vocab, L.features, TYPE == QA_F16 ? -1 : kOfX,
                                G.accumulate != 0, true};
      if (const int rc = grad_product<TYPE == QA_F32 ? 3 : 2>(ct, xt, vocab, L.features, P.tp, out, stream)) return rc;
    }
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
