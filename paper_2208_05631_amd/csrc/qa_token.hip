// Log probabilities of given tokens, entropy and the most likely alternatives, and the logits' gradient.
//
// Scoring reads every logit once.  4096 x 100003 bfloat16: without alternatives 133 us, 6.2 TB/s, bound by memory; with 8 alternatives
// 157, with 64 some 221, bound by instructions: some nine per logit, one of them an exponential that takes four times as long,
// and a few thousand per row for the alternatives.  One row of 128000 with 20 alternatives: 12 us, two launches of some 4 us each and
// a chain of dependent reads.
#include <algorithm>
#include <cfloat>

#include "qa_rows.h"

namespace qa {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFar = -1e4f;                      // 2^kFar is 0
constexpr int kTop = QA_TOP_MAX;                   // a lane for each alternative
static_assert(kTop == kWave, "the alternatives of a row are held one per lane");

__device__ __forceinline__ float wave_max_f32(float v) {
  v = fmaxf(v, as_f32((uint32_t)dpp_i32<kDppQuadXor1>((int)as_u32(v))));
  v = fmaxf(v, as_f32((uint32_t)dpp_i32<kDppQuadXor2>((int)as_u32(v))));
  v = fmaxf(v, as_f32((uint32_t)dpp_i32<kDppRowHalfMirror>((int)as_u32(v))));
  v = fmaxf(v, as_f32((uint32_t)dpp_i32<kDppRowMirror>((int)as_u32(v))));
  const int i = (int)as_u32(v);
  return fmaxf(fmaxf(as_f32((uint32_t)__builtin_amdgcn_readlane(i, 0)), as_f32((uint32_t)__builtin_amdgcn_readlane(i, 16))),
               fmaxf(as_f32((uint32_t)__builtin_amdgcn_readlane(i, 32)), as_f32((uint32_t)__builtin_amdgcn_readlane(i, 48))));
}

// ---- sums of a softmax -----------------------------------------------------------------------------------------
//
// With m the largest logit so far: s = sum of 2^t and w = sum of 2^t t, t = (x - m) log2 e.  Then log p = (x - m) -
// log s and entropy = log s - ln2 w / s; both terms of the entropy are >= 0, nothing cancels.
// m is -FLT_MAX at least, so that -infinity has t = -infinity and adds nothing; in the product t is kFar at least.
struct Sums { float m, s, w; };
__device__ __forceinline__ Sums no_sums() { return {-FLT_MAX, 0.0f, 0.0f}; }

// The same sums against another maximum.
__device__ __forceinline__ void raise(Sums& a, float m) {
  const float t = fmaxf((a.m - m) * kLog2e, kFar), f = __builtin_amdgcn_exp2f(t);
  a.w = (a.w + a.s * t) * f;
  a.s *= f;
  a.m = m;
}
// Sums over the lanes of a wave, each with a maximum of its own.
__device__ __forceinline__ Sums over_lanes(Sums a) {
  raise(a, wave_max_f32(a.m));
  a.s = wave_sum_f32(a.s);
  a.w = wave_sum_f32(a.w);
  return a;
}

// ---- alternatives ------------------------------------------------------------------------------------------------
//
// A logit and its place are one whole number: the logit's bits in an order that whole numbers have, above the place's
// complement, so that the larger number is the better alternative and no two are equal.  A NaN counts as -infinity.
__device__ __forceinline__ uint32_t ordered(float x) {
  if (x != x) return 0x007FFFFFu;
  const uint32_t u = as_u32(x + 0.0f);             // -0 to +0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return as_f32(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t index) { return (uint64_t)order << 32 | (uint32_t)~index; }

template <int SIZE, int STRIDE, typename U>
__device__ __forceinline__ U merge_steps(U v) {
  const int lane = threadIdx.x % kWave;
  const U o = other_lane<STRIDE>(v);
  const bool larger = ((lane & STRIDE) == 0) == ((lane & SIZE) == 0);
  v = (v > o) == larger ? v : o;
  if constexpr (STRIDE > 1) v = merge_steps<SIZE, STRIDE / 2>(v);
  return v;
}
// The wave's 64 values, the largest in lane 0.
template <typename U, int SIZE = 2>
__device__ __forceinline__ U sort_lanes(U v) {
  v = merge_steps<SIZE, SIZE / 2>(v);
  if constexpr (SIZE < kWave) v = sort_lanes<U, 2 * SIZE>(v);
  return v;
}
// The 64 largest of two sorted sequences, sorted; `reversed` holds the second one's value 63 - lane.
template <typename U>
__device__ __forceinline__ U merge_lanes(U v, U reversed) {
  return merge_steps<kWave, kWave / 2>(v > reversed ? v : reversed);
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// A wave's alternatives: sorted, and those that wait in LDS to be sorted in.
struct Best {
  uint64_t sorted = 0, last = 0;                   // last: the `top`-th, 0 while there are fewer
  int waiting = 0;
};
constexpr int kWaiting = 2 * kWave;

__device__ __forceinline__ void sort_in(Best& b, uint64_t* wait, int top) {
  const int lane = threadIdx.x % kWave;
  const uint64_t v = sort_lanes(lane < b.waiting ? wait[lane] : (uint64_t)0);
  b.sorted = merge_lanes(b.sorted, __shfl(v, kWave - 1 - lane, kWave));
  b.last = lane_u64(b.sorted, top - 1);
  const int more = b.waiting - kWave;
  if (more > 0) {
    const uint64_t u = wait[kWave + lane];
    __builtin_amdgcn_wave_barrier();
    wait[lane] = u;
    __builtin_amdgcn_wave_barrier();
  }
  b.waiting = more > 0 ? more : 0;
}

struct TokenArgs {
  const void* x;
  const int32_t* target;
  float *logprob, *entropy, *stats, *top_logprob;
  int32_t* top_index;
  float* part_sums;                                // [row][split][4]: m, s, w
  uint64_t* part_best;                             // [row][split][top]
  int64_t rows, vocab, stride;
  int64_t piece;                                   // logits of one split
  int splits, top;
  bool stream;
};

// What a row's sums and alternatives become.  `best` is lane i's alternative i; one wave writes.  Log probabilities are
// (x - m) - log s: the difference of two logits first, which no rounding of m + log s comes into.
// `given`: the target's logit, which is read before the row, as two reads in a row take as long as 16 KiB of logits.
struct Given { float x; bool is; };
template <int TYPE>
__device__ __forceinline__ Given given_of(const TokenArgs& A, int64_t row) {
  Given g{0.0f, false};
  if (A.logprob) {
    const int32_t y = A.target[row];
    g.is = y >= 0 && y < A.vocab;
    if (g.is) g.x = (float)((const ElemT<TYPE>*)A.x)[row * A.stride + y];
  }
  return g;
}
template <bool TOP>
__device__ __forceinline__ void write_row(const TokenArgs& A, int64_t row, const Given& given, const Sums& a, uint64_t best) {
  const int lane = threadIdx.x % kWave;
  const bool empty = a.s == 0.0f;
  const float log_sum = empty ? 0.0f : kLn2 * __builtin_amdgcn_logf(a.s);
  if (lane == 0) {
    if (A.stats) {
      A.stats[2 * row] = empty ? -INFINITY : a.m;
      A.stats[2 * row + 1] = log_sum;
    }
    if (A.entropy) A.entropy[row] = empty ? 0.0f : log_sum - kLn2 * (a.w / a.s);
    if (A.logprob) A.logprob[row] = !given.is ? 0.0f : empty ? -INFINITY : (given.x - a.m) - log_sum;
  }
  if constexpr (TOP) {
    if (lane < A.top) {
      A.top_logprob[row * A.top + lane] = empty ? -INFINITY : (from_ordered((uint32_t)(best >> 32)) - a.m) - log_sum;
      A.top_index[row * A.top + lane] = (int32_t)~(uint32_t)best;
    }
  }
}

// ---- a row, or a split of one, read by WAVES waves --------------------------------------------------------------------
//
// The waves take chunks of NV vectors per lane in turn.  Each lane has sums against a maximum of its own.  For the
// alternatives it only notes a chunk's largest logit: at the row's end the `top`-th largest of the lanes' largest is a
// bound that `top` logits reach, and the few chunks that reach it are read again.  (A sorted list that each wave keeps while it
// reads: 278 us for 4096 x 100003 with 8 alternatives; eight waves per row instead of four, sorts through LDS: 221.)
constexpr int kTokenWaves = 4, kTokenThreads = kTokenWaves * kWave;
constexpr int kTokenVecs = 2;
constexpr int64_t kTokenChunk = (int64_t)kTokenVecs * kTokenThreads * kVec;
constexpr int kNoted = 48;                         // chunks per lane: longer rows are split
constexpr int kFound = 256;                        // alternatives of all waves; what is more goes to the waves' own

template <int WAVES, int CHUNKS, bool TOP>
struct RowShared {
  uint16_t most[TOP ? CHUNKS + 1 : 1][WAVES * kWave];      // a row that begins inside 16 bytes has one more
  uint32_t largest[WAVES][kWave];
  uint64_t found[TOP ? kFound : 1];
  uint64_t wait[TOP ? WAVES : 1][kWaiting];
  uint64_t lists[TOP ? WAVES : 1][kWave];
  Sums sums[WAVES];
  uint32_t count, bound;
};
template <int WAVES>
__device__ __forceinline__ void row_barrier() {
  if constexpr (WAVES > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The waves' sorted values merged into wave 0's.
template <int WAVES>
__device__ __forceinline__ uint64_t merge_waves(uint64_t v, uint64_t (*lists)[kWave]) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
  for (int w = 1; w < WAVES; w *= 2) {
    if ((wave & (2 * w - 1)) == w) lists[wave][kWave - 1 - lane] = v;
    row_barrier<WAVES>();
    if ((wave & (2 * w - 1)) == 0) v = merge_lanes(v, lists[wave + w][lane]);
  }
  return v;
}

// x[at ..) of a chunk; what lies outside [begin, end) is -infinity.
template <int TYPE, int NV, bool STREAM>
__device__ __forceinline__ void load_chunk(Raw8<TYPE> (&raw)[NV], const ElemT<TYPE>* x, int64_t at, int64_t begin, int64_t end) {
  const int lane = threadIdx.x % kWave;
  const ElemT<TYPE>* p = x + at + lane * kVec;
  if (at >= begin && at + NV * kWave * kVec <= end) {
#pragma unroll
    for (int k = 0; k < NV; ++k) raw[k] = load_raw<TYPE, STREAM>(p + k * kWave * kVec);
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t i = at + (k * kWave + lane) * kVec;
      if (i >= begin) {
        raw[k] = load_raw<TYPE>(p + k * kWave * kVec, (int)max((int64_t)0, min((int64_t)kVec, end - i)), -INFINITY);
      } else {
        ElemT<TYPE> v[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = i + e >= begin && i + e < end ? x[i + e] : (ElemT<TYPE>)-INFINITY;
        __builtin_memcpy(&raw[k], v, sizeof raw[k]);
      }
    }
  }
}
// The compiler's own maximum takes each operand through one more instruction, for the sake of signaling NaN.  Here such a one can hide
// what is beside it; read_row() knows then from the sum of exponentials.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
__device__ __forceinline__ float most_of_eight(const float (&v)[kVec]) {
  return max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[7]));
}

// The largest number of 16 leading bits that `top` of the wave's values reach.
template <int N>
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&values)[N], int top) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t higher = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int w = 0; w < N; ++w) n += __popcll(__ballot(values[w] >= higher));
    bound = n >= top ? higher : bound;
  }
  return bound;
}
// The wave's good keys join those found, or, once there is no room, its own.
template <typename S>
__device__ __forceinline__ void offer(S& shared, int wave, Best& b, uint64_t key, bool good, int top) {
  const int lane = threadIdx.x % kWave;
  const uint64_t mask = __ballot(good);
  if (!mask) return;
  const int n = __popcll(mask);
  const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  uint32_t place = 0;
  if (lane == 0) place = atomicAdd(&shared.count, (uint32_t)n);
  place = (uint32_t)__builtin_amdgcn_readfirstlane((int)place);
  if (place + n <= kFound) {
    if (good) shared.found[place + rank] = key;
  } else {
    if (place + lane < kFound) shared.found[place + lane] = 0;
    if (good) shared.wait[wave][b.waiting + rank] = key;
    b.waiting += n;
    __builtin_amdgcn_wave_barrier();
    if (b.waiting >= kWave) sort_in(b, shared.wait[wave], top);
  }
}
// The 64 best of what was offered, for wave 0.  Begins and ends with a barrier.
template <int WAVES, typename S>
__device__ __forceinline__ uint64_t settle(S& shared, int wave, Best& b, int top) {
  const int lane = threadIdx.x % kWave;
  uint64_t best = 0;
  if (b.waiting > 0) sort_in(b, shared.wait[wave], top);
  row_barrier<WAVES>();
  const int count = (int)shared.count;
  if (count <= kWave) {
    if (wave == 0) {                               // each goes to the place that as many better ones leave it
      const uint64_t key = lane < count ? shared.found[lane] : 0;
      int better = 0;
      for (int i = 0; i < count; ++i) better += lane_u64(key, i) > key;
      if (lane < count) shared.lists[0][better] = key;
      row_barrier<1>();
      best = lane < count ? shared.lists[0][lane] : 0;
    }
  } else {
    for (int i = wave * kWave; i < kFound && i < count; i += WAVES * kWave)
      b.sorted = merge_lanes(b.sorted, __shfl(sort_lanes(i + lane < count ? shared.found[i + lane] : (uint64_t)0), kWave - 1 - lane, kWave));
    best = merge_waves<WAVES>(b.sorted, shared.lists);
  }
  row_barrier<WAVES>();
  return best;
}

// The sums and alternatives of x[begin .. end); wave 0 receives them.  Ends with a barrier.
template <int TYPE, int WAVES, int NV, int CHUNKS, bool TOP, bool STREAM>
__device__ __forceinline__ void read_row(const ElemT<TYPE>* x, int64_t begin, int64_t end, int top,
                                         RowShared<WAVES, CHUNKS, TOP>& shared, Sums& a, uint64_t& best) {
  const int wave = WAVES > 1 ? threadIdx.x / kWave : 0, lane = threadIdx.x % kWave, me = wave * kWave + lane;
  constexpr int64_t kChunk = NV * kWave * kVec, kStride = WAVES * kChunk;
  if (TOP && lane == 0 && wave == 0) shared.count = 0;
  a = no_sums();
  float largest = -INFINITY;
  // Chunks begin on 16 bytes, wherever the row does (4096 rows of 100003 bfloat16 logits without alternatives: 171 -> 146 us).
  const int64_t mine = begin - (int64_t)((uintptr_t)(x + begin) % 16 / sizeof(ElemT<TYPE>)) + wave * kChunk;
  Raw8<TYPE> raw[NV];
  if (mine < end) load_chunk<TYPE, NV, STREAM>(raw, x, mine, begin, end);
  int chunks = 0;
  for (int64_t at = mine; at < end; at += kStride, ++chunks) {
    float v[NV][kVec], most[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      to_f32<TYPE>(raw[k], v[k]);
      most[k] = most_of_eight(v[k]);
    }
    if (at + kStride < end) load_chunk<TYPE, NV, STREAM>(raw, x, at + kStride, begin, end);
    float m = most[0];
#pragma unroll
    for (int k = 1; k < NV; ++k) m = fmaxf(m, most[k]);
    if constexpr (TOP) {
      shared.most[chunks][me] = (uint16_t)(as_u32(m) >> 16);
      largest = fmaxf(largest, m);
    }
    raise(a, fmaxf(a.m, m));
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float t = (v[k][i] - a.m) * kLog2e, e = __builtin_amdgcn_exp2f(t);
        a.s += e;
        a.w = __builtin_fmaf(e, fmaxf(t, kFar), a.w);
      }
  }
  a = over_lanes(a);
  if (WAVES > 1 && lane == 0) shared.sums[wave] = a;
  if (TOP && WAVES > 1) shared.largest[wave][lane] = ordered(largest);
  row_barrier<WAVES>();
  bool all = !(a.s == a.s);
  if constexpr (WAVES > 1) {
    Sums each = no_sums();
    if (lane < WAVES) each = shared.sums[lane];
    all = __any(!(each.s == each.s));
    if (wave == 0) a = over_lanes(each);
  }
  if constexpr (TOP) {
    // `top` lanes have a logit of at least this bound, to 16 bits.  A NaN can have hidden what came before it:
    // everything is looked at then.
    uint32_t bound = 0;
    if (wave == 0) {
      uint32_t values[WAVES];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) values[w] = WAVES > 1 ? shared.largest[w][lane] : ordered(largest);
      bound = bound_of(values, top);
      if (WAVES > 1 && lane == 0) shared.bound = bound;
    }
    if constexpr (WAVES > 1) {
      row_barrier<WAVES>();
      bound = (uint32_t)__builtin_amdgcn_readfirstlane((int)shared.bound);
    }
    if (all || bound <= 0x007FFFFFu) bound = 0;
    const float least = bound ? from_ordered(bound) : -INFINITY;
    uint64_t chosen = 0;                           // chunks with a lane that reaches it
    for (int c = 0; c < chunks; ++c)               // 16 bits of a bound of 16 bits: the comparison is that of the whole numbers
      chosen |= (uint64_t)(__any(all || !(as_f32((uint32_t)shared.most[c][me] << 16) < least)) != 0) << c;
    Best b;
    if (chosen) load_chunk<TYPE, NV, false>(raw, x, mine + __builtin_ctzll(chosen) * kStride, begin, end);
    while (chosen) {
      const int64_t at = mine + __builtin_ctzll(chosen) * kStride;
      chosen &= chosen - 1;
      float v[NV][kVec];
#pragma unroll
      for (int k = 0; k < NV; ++k) to_f32<TYPE>(raw[k], v[k]);
      if (chosen) load_chunk<TYPE, NV, false>(raw, x, mine + __builtin_ctzll(chosen) * kStride, begin, end);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (!__any(!(v[k][i] < least))) continue;
          const int64_t index = at + (k * kWave + lane) * kVec + i;
          const uint64_t key = key_of(ordered(v[k][i]), (uint32_t)index);
          const bool good = !(v[k][i] < least) && key > b.last && index >= begin && index < end;
          offer(shared, wave, b, key, good, top);
        }
    }
    best = settle<WAVES>(shared, wave, b, top);
  } else {
    row_barrier<WAVES>();                          // the next row's sums come to the same place
  }
}

// A wave per row, four rows per work-group.
template <int TYPE, int NV, int CHUNKS, bool TOP>
__global__ __launch_bounds__(kThreads) void token_narrow_kernel(TokenArgs A) {
  __shared__ RowShared<1, CHUNKS, TOP> shared[kWaves];
  const int wave = threadIdx.x / kWave;
  for (int64_t row = (int64_t)blockIdx.x * kWaves + wave; row < A.rows; row += (int64_t)gridDim.x * kWaves) {
    const Given given = given_of<TYPE>(A, row);
    Sums a;
    uint64_t best = 0;
    read_row<TYPE, 1, NV, CHUNKS, TOP, false>((const ElemT<TYPE>*)A.x + row * A.stride, 0, A.vocab, A.top, shared[wave], a, best);
    write_row<TOP>(A, row, given, a, best);
  }
}

// A work-group per row, or per split of a row.
template <int TYPE, int NV, bool TOP, bool STREAM>
__global__ __launch_bounds__(kTokenThreads, 4) void token_wide_kernel(TokenArgs A) {
  __shared__ RowShared<kTokenWaves, kNoted, TOP> shared;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t begin = (int64_t)blockIdx.y * A.piece, end = min(A.vocab, begin + A.piece);
  for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
    Given given{0.0f, false};
    if (A.splits == 1 && wave == 0) given = given_of<TYPE>(A, row);
    Sums a;
    uint64_t best = 0;
    read_row<TYPE, kTokenWaves, NV, kNoted, TOP, STREAM>((const ElemT<TYPE>*)A.x + row * A.stride, begin, end, A.top, shared, a, best);
    if (wave == 0) {
      if (A.splits == 1) {
        write_row<TOP>(A, row, given, a, best);
      } else {
        const int64_t part = row * A.splits + blockIdx.y;
        if (lane == 0) *reinterpret_cast<f32x4*>(A.part_sums + 4 * part) = f32x4{a.m, a.s, a.w, 0.0f};
        if (TOP && lane < A.top) A.part_best[part * A.top + lane] = best;
      }
    }
  }
}

// A row's splits put together: as a row is from its chunks, with the splits' best alternatives for the lanes' largest.
constexpr int kMostSplits = 512, kKeysAhead = 6;
template <int TYPE, bool TOP>
__global__ __launch_bounds__(kTokenThreads) void token_join_kernel(TokenArgs A) {
  __shared__ RowShared<kTokenWaves, 0, TOP> shared;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t row = blockIdx.x;
  const uint64_t* keys = TOP ? A.part_best + row * A.splits * A.top : nullptr;
  Given given{0.0f, false};
  if (wave == 0) given = given_of<TYPE>(A, row);
  if (TOP && threadIdx.x == 0) shared.count = 0;
  const int all = TOP ? A.splits * A.top : 0;
  uint64_t key[kKeysAhead];                        // the first keys are on their way while the bound is sought
#pragma unroll
  for (int k = 0; k < kKeysAhead; ++k) {
    const int i = k * kTokenThreads + (int)threadIdx.x;
    key[k] = i < all ? keys[i] : 0;
  }
  if (TOP && wave == 0) {
    uint32_t values[kMostSplits / kWave], bound;
#pragma unroll
    for (int i = 0; i < kMostSplits / kWave; ++i) {
      const int split = i * kWave + lane;
      values[i] = split < A.splits ? (uint32_t)(keys[(int64_t)split * A.top] >> 32) : 0;
    }
    if (A.splits <= kWave) {
      const uint32_t few[1] = {values[0]};
      bound = bound_of(few, A.top);
    } else {
      bound = bound_of(values, A.top);
    }
    if (lane == 0) shared.bound = bound;
  }
  Sums a = no_sums();
  for (int i = threadIdx.x; i < A.splits; i += kTokenThreads) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(A.part_sums + 4 * (row * A.splits + i));
    Sums b{v[0], v[1], v[2]};
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    a.s += b.s;
    a.w += b.w;
  }
  a = over_lanes(a);
  if (lane == 0) shared.sums[wave] = a;
  __syncthreads();
  uint64_t best = 0;
  if constexpr (TOP) {
    const uint64_t least = (uint64_t)shared.bound << 32;
    Best b;
#pragma unroll
    for (int k = 0; k < kKeysAhead; ++k) offer(shared, wave, b, key[k], key[k] >= least && key[k] > b.last, A.top);
    for (int first = kKeysAhead * kTokenThreads; first < all; first += kTokenThreads) {
      const int i = first + (int)threadIdx.x;
      const uint64_t more = i < all ? keys[i] : 0;
      offer(shared, wave, b, more, more >= least && more > b.last, A.top);
    }
    best = settle<kTokenWaves>(shared, wave, b, A.top);
  }
  if (wave == 0) {
    Sums each = no_sums();
    if (lane < kTokenWaves) each = shared.sums[lane];
    write_row<TOP>(A, row, given, over_lanes(each), best);
  }
}

// ---- gradient ----------------------------------------------------------------------------------------------------

struct TokenGradArgs {
  const void* x;
  const int32_t* target;
  const float *stats, *entropy, *g_logprob, *g_entropy;
  void* dx;
  int64_t rows, vocab, x_stride, dx_stride;
  bool stream;
};

struct GradRow {
  float a, c, e2, m, log_sum;
  int32_t y;
};
__device__ __forceinline__ GradRow grad_row(const TokenGradArgs& A, int64_t row) {
  GradRow r;
  r.y = A.target ? A.target[row] : -1;
  if (r.y >= A.vocab) r.y = -1;
  r.a = r.y >= 0 && A.g_logprob ? A.g_logprob[row] : 0.0f;
  const float e = A.g_entropy ? A.g_entropy[row] : 0.0f;
  r.c = r.a + (A.g_entropy ? e * A.entropy[row] : 0.0f);
  r.e2 = e * kLn2;
  r.m = fmaxf(A.stats[2 * row], -FLT_MAX);
  r.log_sum = A.stats[2 * row + 1];
  return r;
}
// dx_j = -p_j (a + e (log p_j + H)), and a more at the target.  Bound by memory: 8192 x 32768 bfloat16 178 us, 6.0 TB/s; 509 x 47236
// binary32 44 us, 4.4 TB/s, whether rows begin on 16 bytes or not (as much in rows of one piece 38, of six whole ones 42, copied by torch 37).
template <int TYPE>
__device__ __forceinline__ Raw8<TYPE> grad_of(const GradRow& r, const Raw8<TYPE>& raw, int64_t i) {
  float v[kVec], d[kVec];
  to_f32<TYPE>(raw, v);
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const float t = ((v[j] - r.m) - r.log_sum) * kLog2e, p = __builtin_amdgcn_exp2f(t);
    d[j] = -p * __builtin_fmaf(r.e2, fmaxf(t, kFar), r.c);
  }
  if (r.y >= i && r.y < i + kVec) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) d[j] += r.y - i == j ? r.a : 0.0f;
  }
  return from_f32<TYPE>(d);
}

constexpr int64_t kGradPiece = (int64_t)kThreads * kVec;       // logits that a work-group has in one vector per lane
// Pieces inside a row have no branch; a row's last piece has one around each load, which costs rows of a part of one piece most (8192 x
// 2049: 22 us, 8192 x 2048 in the form below: 15).  Past the caches pieces begin on 16 bytes of dx, wherever the row does, where there are
// more than two: 4096 x 100003 bfloat16 395 us -> 337.
template <int TYPE, int NV, bool STREAM>
__global__ __launch_bounds__(kThreads) void token_grad_kernel(TokenGradArgs A) {
  typedef ElemT<TYPE> T;
  constexpr int64_t kPiece = NV * kGradPiece;
  for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
    const T* x = (const T*)A.x + row * A.x_stride;
    T* dx = (T*)A.dx + row * A.dx_stride;
    const GradRow r = grad_row(A, row);
    const int64_t lead = STREAM && A.vocab > 2 * kPiece ? (int64_t)((uintptr_t)dx % 16 / sizeof(T)) : 0;
    for (int64_t first = (int64_t)blockIdx.y * kPiece - lead; first < A.vocab; first += (int64_t)gridDim.y * kPiece) {
      const int64_t lane0 = first + threadIdx.x * kVec;
      Raw8<TYPE> raw[NV];
      if (first >= 0 && first + kPiece <= A.vocab) {
#pragma unroll
        for (int k = 0; k < NV; ++k) raw[k] = load_raw<TYPE, STREAM>(x + lane0 + k * kGradPiece);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int64_t i = lane0 + k * kGradPiece;
          store_raw<TYPE, STREAM>(dx + i, grad_of<TYPE>(r, raw[k], i), kVec);
        }
      } else {
        auto elements = [&](int64_t i, auto each) {
#pragma unroll
          for (int j = 0; j < kVec; ++j)
            if (i + j >= 0 && i + j < A.vocab) each(i + j, j);
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int64_t i = lane0 + k * kGradPiece;
          const int n = (int)max((int64_t)0, min((int64_t)kVec, A.vocab - i));
          if (STREAM && i < 0) {
            T v[kVec] = {};
            elements(i, [&](int64_t at, int j) { v[j] = x[at]; });
            __builtin_memcpy(&raw[k], v, sizeof raw[k]);
          } else {
            raw[k] = load_raw<TYPE, STREAM>(x + i, n);
          }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int64_t i = lane0 + k * kGradPiece;
          const int n = (int)max((int64_t)0, min((int64_t)kVec, A.vocab - i));
          if (n == 0) continue;
          const Raw8<TYPE> d = grad_of<TYPE>(r, raw[k], i);
          if (STREAM && i < 0) {
            T v[kVec];
            __builtin_memcpy(v, &d, sizeof d);
            elements(i, [&](int64_t at, int j) { dx[at] = v[j]; });
          } else {
            store_raw<TYPE, STREAM>(dx + i, d, n);
          }
        }
      }
    }
  }
}
// Rows of up to 2048 logits: `per_row` lanes, a power of two, have one vector each (a work-group for each row: 16384 x 8 logits 61 us
// instead of 6, 8192 x 2000 36 instead of 14).
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(kThreads) void token_grad_narrow_kernel(TokenGradArgs A, int per_row) {
  typedef ElemT<TYPE> T;
  const int rows = kThreads / per_row, local = threadIdx.x / per_row, i = (int)threadIdx.x % per_row * kVec;
  const int n = (int)min((int64_t)kVec, A.vocab - i);
  if (n <= 0) return;
  for (int64_t row = (int64_t)blockIdx.x * rows + local; row < A.rows; row += (int64_t)gridDim.x * rows) {
    const Raw8<TYPE> raw = load_raw<TYPE, STREAM>((const T*)A.x + row * A.x_stride + i, n);
    store_raw<TYPE, STREAM>((T*)A.dx + row * A.dx_stride + i, grad_of<TYPE>(grad_row(A, row), raw, i), n);
  }
}

// ---- which form ----------------------------------------------------------------------------------------------------

constexpr int64_t kNarrow = 4096;                  // logits of a row that one wave reads
constexpr int64_t kSplitLogits = kTokenThreads * kVec;       // one vector per lane

// Rows longer than this are split where there are few: a second launch takes as long as it saves (one row, 20 alternatives: 16000
// logits 10.4 us in one piece and 12.3 split, 32000 13.4 and 13.1, 64000 17.6 and 12.2; 400 rows of 64000: 23.7 and 27.7).
constexpr int64_t kUnsplit = 16 * kSplitLogits;
int64_t splits_for(int64_t rows, int64_t vocab) {
  if (vocab <= kUnsplit) return 1;
  const int64_t least = ceil_div(vocab, kNoted * kTokenChunk);
  if (rows >= 256) return least;
  return std::max(least, std::min<int64_t>(std::min<int64_t>(ceil_div(vocab, kSplitLogits), kMostSplits), 1024 / rows));
}

// Whether a row is read past the caches.  With alternatives parts of it are read again, which pays for long rows only (8 of them, bfloat16:
// 40000 x 4100 344 us, and 365 past the caches, 16000 x 16384 166 and 177, 6000 x 50021 146 both, 4000 x 65536 114 and 108; without:
// 136 and 133, 92 and 90, 95 and 84); in binary32 without alternatives it pays in rows that begin on 16 bytes (8000 x 16384 89 and 85,
// but 1500 x 100003 104 and 112, 20000 x 4100 66 and 72), with 8 it does not (4000 x 32768 105 and 110).
bool token_streams(int type, int64_t rows, int64_t vocab, const void* logits, int64_t stride, int32_t top) {
  if (!streams((double)rows * (double)vocab * (double)type_bytes(type))) return false;
  if (top) return type != QA_F32 && vocab >= 1 << 16;
  return type != QA_F32 || (vocab >= 1 << 14 && aligned(logits, 16) && stride % 4 == 0);
}
// Whether the logits' gradient goes past the caches: not where a row is a part of one piece (bfloat16, 40000 x 2049: 109 us, and 126 if it did,
// 32768 x 4096: 100 and 118, 20000 x 6144: 87 and 88, 16000 x 8191: 110 and 105; 100000 x 1001, several rows to a work-group: 100 and 95), and
// in binary32 only for rows of a quarter of a work-group or an aligned half (180000 x 217: 66 and 63, 80000 x 512: 67 and 63, but 80000 x 511:
// 69 and 77, 4000 x 32768: 204 and 218).
constexpr int kGradVecs = 4;
bool token_grad_streams(int type, int64_t rows, int64_t vocab, int64_t x_stride, int64_t dx_stride) {
  if (!streams((double)rows * (double)vocab * (double)(2 * type_bytes(type)))) return false;
  if (type == QA_F32) return vocab <= 256 || (vocab <= 512 && x_stride % 4 == 0 && dx_stride % 4 == 0);
  return vocab <= kGradPiece || 4 * vocab > 3 * kGradVecs * kGradPiece;
}

template <int TYPE, bool TOP>
int token_launch(TokenArgs& A, hipStream_t stream) {
  constexpr bool STREAM = !(TOP && TYPE == QA_F32);
  const dim3 narrow((unsigned)std::min<int64_t>(ceil_div(A.rows, kWaves), 1 << 16));
  if (A.vocab <= 512) {
    token_narrow_kernel<TYPE, 1, 1, TOP><<<narrow, kThreads, 0, stream>>>(A);
  } else if (A.vocab <= kNarrow) {
    token_narrow_kernel<TYPE, kTokenVecs, 4, TOP><<<narrow, kThreads, 0, stream>>>(A);
  } else {
    const dim3 grid((unsigned)std::min<int64_t>(A.rows, 1 << 16), (unsigned)A.splits);
    A.piece = ceil_div(ceil_div(A.vocab, A.splits), kSplitLogits) * kSplitLogits;
    if (A.piece <= 2 * kSplitLogits) token_wide_kernel<TYPE, 1, TOP, false><<<grid, kTokenThreads, 0, stream>>>(A);
    else if (STREAM && A.stream) token_wide_kernel<TYPE, kTokenVecs, TOP, STREAM><<<grid, kTokenThreads, 0, stream>>>(A);
    else token_wide_kernel<TYPE, kTokenVecs, TOP, false><<<grid, kTokenThreads, 0, stream>>>(A);
    if (A.splits == 1) return launch_status();
    if (const int rc = launch_status()) return rc;
    token_join_kernel<TYPE, TOP><<<dim3((unsigned)A.rows), kTokenThreads, 0, stream>>>(A);
  }
  return launch_status();
}
template <int TYPE>
int token_launch(TokenArgs& A, hipStream_t stream) {
  return A.top ? token_launch<TYPE, true>(A, stream) : token_launch<TYPE, false>(A, stream);
}
template <int TYPE>
int token_grad_launch(const TokenGradArgs& A, hipStream_t stream) {
  if (A.vocab <= kGradPiece) {
    int per_row = 1;
    while (per_row * kVec < A.vocab) per_row *= 2;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(A.rows, kThreads / per_row), 1 << 22));
    const auto kernel = A.stream ? token_grad_narrow_kernel<TYPE, true> : token_grad_narrow_kernel<TYPE, false>;
    kernel<<<grid, kThreads, 0, stream>>>(A, per_row);
  } else {
    const dim3 grid((unsigned)std::min<int64_t>(A.rows, 1 << 22),
                    (unsigned)std::min<int64_t>(ceil_div(A.vocab, kGradVecs * kGradPiece), 1 << 14));
    constexpr bool STREAM = TYPE != QA_F32;
    const auto kernel = A.stream ? token_grad_kernel<TYPE, kGradVecs, STREAM> : token_grad_kernel<TYPE, kGradVecs, false>;
    kernel<<<grid, kThreads, 0, stream>>>(A);
  }
  return launch_status();
}

int check_logits(int type, int64_t rows, int64_t vocab, int64_t stride) {
  if (!known_type(type) || rows < 0 || rows >= (int64_t(1) << 31) || vocab < 1 || vocab >= (int64_t(1) << 31) ||
      stride < vocab)
    return QA_ERR_INVALID_ARG;
  return QA_OK;
}

}  // namespace
}  // namespace qa

using namespace qa;

extern "C" size_t qa_token_workspace_bytes(int64_t rows, int64_t vocab, int32_t top) {
  if (check_logits(QA_F32, rows, vocab, vocab) != QA_OK || top < 0 || top > QA_TOP_MAX || top > vocab || rows == 0)
    return 0;
  const int64_t splits = splits_for(rows, vocab);
  return splits == 1 ? 0 : (size_t)(rows * splits) * (16 + 8 * (size_t)top);
}

extern "C" int qa_token_logprob(int type, int64_t rows, int64_t vocab, const void* logits, int64_t stride,
                                const int32_t* target, int32_t top, float* logprob, float* entropy, float* stats,
                                float* top_logprob, int32_t* top_index, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_logits(type, rows, vocab, stride)) return rc;
  if (top < 0 || top > QA_TOP_MAX || top > vocab) return QA_ERR_INVALID_ARG;
  if (rows == 0) return QA_OK;
  if (!logits || !target != !logprob || (top && (!top_logprob || !top_index))) return QA_ERR_INVALID_ARG;
  if (!element_aligned(logits, type) || !aligned(target, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
      !aligned(stats, 4) || (top && (!aligned(top_logprob, 4) || !aligned(top_index, 4))))
    return QA_ERR_ALIGNMENT;
  TokenArgs A{logits, target, logprob, entropy, stats, top_logprob, top_index, nullptr, nullptr,
              rows, vocab, stride, vocab, (int)splits_for(rows, vocab), top, token_streams(type, rows, vocab, logits, stride, top)};
  if (A.splits > 1) {
    if (!ws || ws_bytes < qa_token_workspace_bytes(rows, vocab, top)) return QA_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return QA_ERR_ALIGNMENT;
    A.part_sums = (float*)ws;
    A.part_best = (uint64_t*)((char*)ws + (size_t)(rows * A.splits) * 16);
  }
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return token_launch<QA_F32>(A, s);
  if (type == QA_BF16) return token_launch<QA_BF16>(A, s);
  return token_launch<QA_F16>(A, s);
}

extern "C" int qa_token_logprob_grad(int type, int64_t rows, int64_t vocab, const void* logits, int64_t stride,
                                     const int32_t* target, const float* stats, const float* entropy,
                                     const float* g_logprob, const float* g_entropy, void* dlogits,
                                     int64_t dlogits_stride, void* stream) {
  if (const int rc = check_logits(type, rows, vocab, stride)) return rc;
  if (dlogits_stride < vocab) return QA_ERR_INVALID_ARG;
  if (rows == 0) return QA_OK;
  if (!logits || !stats || !dlogits || !entropy != !g_entropy) return QA_ERR_INVALID_ARG;
  if (!element_aligned(logits, type) || !element_aligned(dlogits, type) || !aligned(target, 4) || !aligned(stats, 4) ||
      !aligned(entropy, 4) || !aligned(g_logprob, 4) || !aligned(g_entropy, 4))
    return QA_ERR_ALIGNMENT;
  const TokenGradArgs A{logits, target, stats, entropy, g_logprob, g_entropy, dlogits, rows, vocab, stride, dlogits_stride,
                        token_grad_streams(type, rows, vocab, stride, dlogits_stride)};
  const hipStream_t s = (hipStream_t)stream;
  if (type == QA_F32) return token_grad_launch<QA_F32>(A, s);
  if (type == QA_BF16) return token_grad_launch<QA_BF16>(A, s);
  return token_grad_launch<QA_F16>(A, s);
}
