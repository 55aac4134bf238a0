// Products of the matrix cores over matrices of 16-bit elements: C[i][j] = sum_k A(i, k) B(j, k), sums in binary32.  Shared by
// the kernels that multiply; not part of the public interface.
#pragma once
#include "qa_rows.h"

namespace qa {

// A number of more bits than an element has is two elements ("parts"), hi + lo.  A row of parts is eight hi, the eight lo
// that belong to them, and so on: 16 bytes each.  Products are hi hi, hi lo and lo hi; the fourth is below binary32's rounding.
constexpr int64_t kPartsStep = 16, kWholeStep = 32;        // elements of k per step, of products with parts and without
constexpr int64_t whole(int64_t n, int64_t step) { return (n + step - 1) / step * step; }

#if defined(__HIPCC__)

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// How an operand lies in memory.
enum Lies {
  kRows,                                           // k along its rows
  kRowsOfParts,
  kHiOfRows,                                       // the hi of rows of parts
  kColumns,                                        // i along its rows: row k holds all i
  kColumnsOfParts
};
constexpr int parts_in(Lies l) { return l == kRowsOfParts || l == kColumnsOfParts ? 2 : 1; }
constexpr bool in_rows(Lies l) { return l <= kHiOfRows; }

struct Operand {
  const void* p;                                   // 16-byte aligned
  int64_t ld;                                      // elements between rows, a multiple of 8, < 2^22
  int64_t batch;                                   // elements between matrices
  int64_t n;                                       // how many i there are
};
// A product of which the device knows how many there are of B's, or of k; 0 counts as 1.
enum HowMany { kAll, kFewerOfB, kFewerOfK };
struct Fewer {
  const int* n;
  int most_splits;                                 // of B's fewer: more splits, up to so many, in their place; 0: as planned
  const void* all;                                 // NULL, or where B is if there are all of them
  int64_t all_ld;
  const int* wide;                                 // of B's fewer: NULL, or whether A is elsewhere
  const void* wide_a;
};
// Splits of a product in tiles of `side` along B, of whose `all` n are left: as many tiles and no more sums than with all of them.
__host__ __device__ constexpr unsigned splits_of_fewer(unsigned splits, unsigned most, unsigned side, unsigned all, unsigned n) {
  const unsigned tiles = splits * ((all + side - 1) / side) / ((n + side - 1) / side), sums = splits * all / n, more = tiles < sums ? tiles : sums;
  return more < most ? more : most;
}
struct ProductArgs {
  Operand a, b;
  int steps, split_steps;                          // of k, and of one split of them
  unsigned splits, tiles_m, tiles_n, tiles;        // tiles: of one matrix
  unsigned batch;
  Fewer fewer;
};

// Brings SIDE values of i and STEP of k to LDS, straight from memory, 16 bytes per lane.
//
// k along the rows: 64 bytes of each row, which are four octets of k, or the two octets' hi and then their lo.  An octet stands at
// octet ^ (row / 4 % 4), so that the sixteen rows that are read at a time lie in different banks.
// i along the rows: row k is SIDE elements (and then their lo); the eight elements c of it stand at c ^ 4 (k % 4), so that
// the four rows that a transposing read takes lie in different banks.
// The lanes' addresses in memory see to that: in LDS a wave's 64 lanes lie side by side.
template <Lies LIES, int SIDE, int STEP, int WAVES>
struct Bringer {
  static constexpr int kParts = parts_in(LIES);
  static constexpr int kBytes = in_rows(LIES) ? SIDE * 64 : STEP * SIDE * 2 * kParts;
  static constexpr int kLoads = kBytes / 1024 / WAVES;
  static constexpr int kPitch = in_rows(LIES) ? 64 : SIDE * 2 * kParts;        // bytes between rows in LDS
  static_assert(kLoads * 1024 * WAVES == kBytes && (in_rows(LIES) || SIDE >= 128 || kParts == 2), "whole instructions, 16 chunks a row");
  const char* at;
  int64_t advance;
  uint32_t off[kLoads];

  // Values of i from i0 up to `end`; past them the last ones are read again.
  __device__ __forceinline__ void begin(const Operand& O, int64_t matrix, int64_t i0, int64_t end, int first_step, int wave) {
    const int lane = threadIdx.x % kWave;
    const char* p = (const char*)O.p + matrix * O.batch * 2;
    if constexpr (in_rows(LIES)) {
      advance = LIES == kHiOfRows ? 128 : 64;
      at = p + i0 * O.ld * 2 + first_step * advance;
      const int slot = (lane & 3) ^ (lane >> 4 & 3);
      const uint32_t octet = (uint32_t)(LIES == kRows ? slot : LIES == kHiOfRows ? 2 * slot : 2 * (slot & 1) + (slot >> 1)) * 16;
#pragma unroll
      for (int v = 0; v < kLoads; ++v)
        off[v] = (uint32_t)min((int64_t)((v * WAVES + wave) * 16 + lane / 4), end - 1 - i0) * (uint32_t)(2 * O.ld) + octet;
    } else {
      advance = STEP * O.ld * 2;
      at = p + i0 * 2 * kParts + first_step * advance;
      const int last = (int)min((int64_t)SIDE, (end - i0 + 7) / 8 * 8) / 8 - 1;
#pragma unroll
      for (int v = 0; v < kLoads; ++v) {
        const int chunk = (v * WAVES + wave) * 64 + lane, k = chunk / (kPitch / 16), slot = (chunk % (kPitch / 16)) ^ 4 * (k & 3);
        const int part = slot / (SIDE / 8), c = slot % (SIDE / 8);
        off[v] = (uint32_t)k * (uint32_t)(2 * O.ld) + (uint32_t)((min(c, last) * kParts + part) * 16);
      }
    }
  }
  // Instructions [FROM, TO) of them.
  template <int FROM, int TO>
  __device__ __forceinline__ void bring(char* lds, int wave) const {
#pragma unroll
    for (int v = FROM < 0 ? 0 : FROM; v < (TO < kLoads ? TO : kLoads); ++v)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at + off[v]),
                                       (__attribute__((address_space(3))) void*)(lds + (v * WAVES + wave) * 1024), 16, 0, 0);
  }
};

// What a lane of a matrix instruction reads of it: i = lane % 32 of block f, k = 8 (lane / 32) ... + 7 of half h (or of part h).
// Of 16 lanes that read transposed each addresses four i of one of four k, and receives four k of one i.
template <Lies LIES, int SIDE, int STEP, int BLOCKS>
struct Reader {
  static constexpr int kPitch = Bringer<LIES, SIDE, STEP, 1>::kPitch;
  static constexpr bool kMixed = !in_rows(LIES) && SIDE / 8 % 16 != 0;       // lo lies among hi in groups of 16 chunks
  int lane_at[in_rows(LIES) || kMixed ? 2 * BLOCKS : BLOCKS];
  __device__ __forceinline__ void begin(int block0) {
    const int lane = threadIdx.x % kWave;
    if constexpr (in_rows(LIES)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) lane_at[h] = (32 * block0 + lane % 32) * 64 + ((2 * h + lane / 32) ^ (lane >> 2 & 3)) * 16;
    } else {
      const int k = 8 * (lane / 32) + (lane % 16 >> 2);
#pragma unroll
      for (int f = 0; f < BLOCKS; ++f) {
        const int i = 32 * (block0 + f) + (lane & 16) + 4 * (lane & 3);
        lane_at[f] = k * kPitch + ((i / 8) ^ 4 * (k & 3)) * 16 + (lane & 1) * 8;
        if constexpr (kMixed) lane_at[BLOCKS + f] = k * kPitch + ((SIDE / 8 + i / 8) ^ 4 * (k & 3)) * 16 + (lane & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ void read(const char* lds, int h, u32x4 (&v)[BLOCKS]) const {
#pragma unroll
    for (int f = 0; f < BLOCKS; ++f) {
      if constexpr (in_rows(LIES)) {
        v[f] = *reinterpret_cast<const u32x4*>(lds + lane_at[h] + f * 32 * 64);
      } else {
        const char* p = lds + (kMixed ? lane_at[h * BLOCKS + f] : lane_at[f] + h * (parts_in(LIES) == 2 ? 2 * SIDE : 16 * kPitch));
        s16x4 half[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          half[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 4 * e * kPitch));
        __builtin_memcpy(&v[f], half, sizeof half);
      }
    }
  }
};

// WM x WN waves, FM x FN blocks of 32 x 32 each.  SHARE > 1: so many times the waves, each lot with every SHARE-th step and buffers of its own;
// the first lot gets all sums.  APART: products with a lo have sums of their own, so that a sum is rounded a third as often.  Four buffers: while step s
// is multiplied, s + 1 is there, s + 2 on its way, and s + 3 sets out for the buffer that step s - 1 had.
//
// Four waves of 128 x 128 each on a tile of 256 x 256 read the least of LDS for a matrix instruction; eight of 128 x 64 read half as much again and are slower.
// Large products run at 1.1 to 1.2 PFLOP/s (bfloat16, 8192 x 4096 x 32768) and, in parts, three matrix instructions for what two bring, at 1.31 to
// 1.35 (8192 x 8192 x 2048): the card's power bounds both, at 1.4 to 1.8 GHz with the matrix cores busy in 54 to 72 % of the cycles.  Small ones are
// bound by a tile's first loads and its results, beside 0.07 to 0.4 us per step.
template <bool BF16, Lies LA, Lies LB, int WM, int WN, int FM, int FN, int SHARE = 1, bool APART = false>
struct Product {
  static constexpr int kM = 32 * WM * FM, kN = 32 * WN * FN, kWavesHere = WM * WN, kGroup = SHARE * kWavesHere * kWave;
  static constexpr int kWavesPerSimd = FM * FN == 16 ? 1 : SHARE > 1 ? SHARE : 2;        // of registers
  static constexpr int kPA = parts_in(LA), kPB = parts_in(LB);
  static constexpr int kStep = kPA * kPB == 1 ? kWholeStep : kPartsStep;
  static_assert(kPA <= kPB && !(kStep == kPartsStep && (LA == kRows || LA == kHiOfRows || LB == kRows || LB == kHiOfRows)), "forms that there are");
  typedef Bringer<LA, kM, kStep, kWavesHere> BringA;
  typedef Bringer<LB, kN, kStep, kWavesHere> BringB;
  static constexpr int kBuffer = BringA::kBytes + BringB::kBytes, kBuffers = 4, kLoads = BringA::kLoads + BringB::kLoads;
  static constexpr int kLate = (kLoads + 1) / (kPA + 1);       // a step's loads behind the barrier; the others follow in the next step

  // The other lots' sums stand behind the first lot's buffers, which its epilogue uses.
  static constexpr int kLotBytes = kWavesHere * kWave * FM * FN * 64, kShared = kBuffers * kBuffer + (SHARE - 1) * kLotBytes;
  static constexpr int kLds = SHARE * kBuffers * kBuffer > kShared ? SHARE * kBuffers * kBuffer : kShared;

  f32x16 acc[FM][FN], more[APART ? FM : 1][APART ? FN : 1];
  u32x4 a[2][FM], b[2][FN];
  BringA bring_a;
  BringB bring_b;
  Reader<LA, kM, kStep, FM> read_a;
  Reader<LB, kN, kStep, FN> read_b;
  int to_load, wave;
  int64_t matrix, split;                           // which of the batch, and of the splits of k
  bool owns;                                       // whether this wave has the sums
  bool empty;                                      // nothing is in this split, and what the sums hold is not meant

  // Instructions [FROM, TO) of a step's; behind the last one go on, past the last step to itself.
  template <int FROM, int TO>
  __device__ __forceinline__ void load(char* lds) {
    bring_a.template bring<FROM, TO>(lds, wave);
    bring_b.template bring<FROM - BringA::kLoads, TO - BringA::kLoads>(lds + BringA::kBytes, wave);
    if constexpr (TO == kLoads) {
      const int64_t go = --to_load > 0 ? -1 : 0;   // no branch: the matrix instructions around this are one block
      bring_a.at += bring_a.advance & go;
      bring_b.at += bring_b.advance & go;
    }
  }
  template <bool MORE = false>
  __device__ __forceinline__ void multiply(const u32x4 (&x)[FM], const u32x4 (&y)[FN]) {
    auto& to = [&]() -> auto& {
      if constexpr (MORE && APART) return more;
      else return acc;
    }();
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if constexpr (BF16)
          to[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[i]), __builtin_bit_cast(bf16x8, y[j]), to[i][j], 0, 0, 0);
        else
          to[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x[i]), __builtin_bit_cast(f16x8, y[j]), to[i][j], 0, 0, 0);
      }
  }
  // Waits until at most LEFT of this wave's loads are on their way, then for the other waves.  Loads into LDS are the only
  // ones that the loop makes.
  template <int LEFT>
  static __device__ __forceinline__ void arrive() {
    static_assert(LEFT < 64, "the counter's bits");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LEFT) : "memory");
  }
  // The order of a phase's instructions: MULTIPLIES matrix instructions, with READS reads of LDS in the shadow of the first ones, two each,
  // as they have to be there when the next phase begins, and LOADS reads of memory spread over all.
  template <int MULTIPLIES, int READS, int LOADS, int I = 0>
  static __device__ __forceinline__ void interleave() {
    if constexpr (I < MULTIPLIES) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      constexpr int kReads = 2 * I >= READS ? 0 : READS - 2 * I < 2 ? 1 : 2, kHere = (I + 1) * LOADS / MULTIPLIES - I * LOADS / MULTIPLIES;
      if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
      if constexpr (kHere > 0) __builtin_amdgcn_sched_group_barrier(0x020, kHere, 0);
      interleave<MULTIPLIES, READS, LOADS, I + 1>();
    } else {
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The first operands of a step are read beside the last products of the one before.  Half of the loads stand in front of the
  // barrier, half behind it: all at once, they wait for each other, and the products for them.  The buffers lie apart, as the
  // compiler is told: it would wait for all loads before each read otherwise.
  static __device__ __forceinline__ void step(Product& p, const char* __restrict__ now, const char* __restrict__ then, char* __restrict__ late,
                                              char* __restrict__ last) {
    constexpr int kAll = FM * FN, kReadA = FM * (in_rows(LA) ? 1 : 2), kReadB = FN * (in_rows(LB) ? 1 : 2);
    if constexpr (kPA == kPB) p.read_a.read(now, 1, p.a[1]);
    p.read_b.read(now + BringA::kBytes, 1, p.b[1]);
    p.template load<kLate, kLoads>(late);
    p.multiply(p.a[0], p.b[0]);
    if constexpr (kPA == 2) p.template multiply<true>(p.a[0], p.b[1]);
    interleave<kPA == 2 ? 2 * kAll : kAll, (kPA == kPB ? kReadA : 0) + kReadB, kLoads - kLate>();
    arrive<kLoads>();                              // `then` is there, and nobody reads `last` any more
    u32x4 a_next[FM], b_next[FN];
    p.read_a.read(then, 0, a_next);
    p.read_b.read(then + BringA::kBytes, 0, b_next);
    p.template load<0, kLate>(last);
    if constexpr (kPA == 2) p.template multiply<true>(p.a[1], p.b[0]);
    else if constexpr (kPB == 2) p.multiply(p.a[0], p.b[1]);
    else p.multiply(p.a[1], p.b[1]);
    interleave<kAll, kReadA + kReadB, kLate>();
#pragma unroll
    for (int i = 0; i < FM; ++i) p.a[0][i] = a_next[i];
#pragma unroll
    for (int j = 0; j < FN; ++j) p.b[0][j] = b_next[j];
  }
  // All steps of a tile's split, one at least.
  __device__ __forceinline__ void run(const ProductArgs& A, int64_t matrix_, int64_t split_, int64_t m0, int64_t n0, char* all_lds) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int share = SHARE == 1 ? 0 : wave / kWavesHere;
    wave -= share * kWavesHere;
    owns = share == 0;
    matrix = matrix_;
    split = split_;
    empty = (int)split * A.split_steps >= A.steps;
    const int begin = empty ? 0 : (int)split * A.split_steps, in_split = min(A.split_steps, A.steps - begin);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        acc[i][j] = f32x16{};
        if constexpr (APART) more[i][j] = f32x16{};
      }
    bring_a.begin(A.a, matrix, m0, A.a.n, begin + min(share, in_split - 1), wave);
    bring_b.begin(A.b, matrix, n0, A.b.n, begin + min(share, in_split - 1), wave);
    bring_a.advance *= SHARE;
    bring_b.advance *= SHARE;
    char* const lds = all_lds + share * kBuffers * kBuffer;
    const int steps = (in_split - share + SHARE - 1) / SHARE, all_steps = (in_split + SHARE - 1) / SHARE;       // this lot's, and the first one's
    read_a.begin(wave % WM * FM);
    read_b.begin(wave / WM * FN);
    to_load = steps;                               // a lot without any brings the last one and leaves it
    int now = 0, then = kBuffer, late = 2 * kBuffer, last = 3 * kBuffer;
    load<0, kLoads>(lds + now);
    load<0, kLoads>(lds + then);
    load<0, kLate>(lds + late);
    arrive<kLoads + kLate>();
    read_a.read(lds, 0, a[0]);
    read_b.read(lds + BringA::kBytes, 0, b[0]);
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      step(*this, lds + now, lds + then, lds + late, lds + last);
      const int free = now;
      now = then;
      then = late;
      late = last;
      last = free;
    }
    if constexpr (SHARE > 1)
      for (int s = max(steps, 0); s < all_steps; ++s) arrive<0>();
    arrive<0>();                                   // loads past the last step, before LDS is used for something else
    if constexpr (APART) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] += more[i][j];
    }
    if constexpr (SHARE > 1) {
      constexpr int kPieces = (int)(sizeof acc / sizeof(f32x4));
      f32x4 v[kPieces];
      __builtin_memcpy(v, &acc, sizeof v);
      f32x4* const at = (f32x4*)(all_lds + kBuffers * kBuffer) + threadIdx.x % (kWavesHere * kWave);
      constexpr int kLot = kLotBytes / 16;
      if (!owns) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) at[(share - 1) * kLot + i * kWavesHere * kWave] = v[i];
      }
      __syncthreads();
      if (owns) {
#pragma unroll 1
        for (int g = 1; g < SHARE; ++g)
#pragma unroll
          for (int i = 0; i < kPieces; ++i) v[i] += at[(g - 1) * kLot + i * kWavesHere * kWave];
        __builtin_memcpy(&acc, v, sizeof v);
      }
    }
  }
  __device__ __forceinline__ int64_t wave_m(int64_t m0) const { return m0 + wave % WM * 32 * FM; }
  __device__ __forceinline__ int64_t wave_n(int64_t n0) const { return n0 + wave / WM * 32 * FN; }

  // A lane holds of block (i, j) rows 8 q + 4 (lane / 32) + e, e < 4, of column lane % 32.  With its counterpart of the other half it changes
  // four rows for four, so that it has eight that follow each other, which it may change: change(i, j, eight sums), i and j
  // from the wave's first on.  By way of LDS they come to lanes that lie side by side along i, as they do in memory where C's columns are
  // rows: run(i, j, eight numbers), i .. i + 7 and j within C.  TURN: then side by side along j: turned(i, j, eight numbers), j .. j + 7.
  // (Eight at a time from where they are, every lane to a row of its own, took 25 us beside the 30 of 32 steps.)
  static constexpr int kRunPitch = FM == 1 ? 128 : FM == 2 ? 256 : 512;
  static_assert(32 * kRunPitch <= kBuffers * kBuffer / kWavesHere, "32 columns of a wave fit its share of the buffers");
  // Sixteen rows at one place, and one row, lie in different banks.
  static __device__ __forceinline__ int run_at(int row, int chunk) { return row * kRunPitch + (chunk ^ (FM == 1 ? row >> 1 & 7 : row & 15)) * 16; }
  template <bool TURN, class Change, class Run, class Turned>
  __device__ __forceinline__ void for_runs(int64_t m0, int64_t n0, char* lds, const Change& change, const Run& run, const Turned& turned) {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float v[kVec];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const auto both = __builtin_amdgcn_permlane32_swap(as_u32(acc[i][j][8 * q + e]), as_u32(acc[i][j][8 * q + 4 + e]), false, false);
            v[e] = as_f32(both[0]);
            v[4 + e] = as_f32(both[1]);
          }
          change(32 * i + 16 * q + 8 * (lane / 32), 32 * j + lane % 32, v);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            __builtin_memcpy(__builtin_assume_aligned(lds + run_at(lane % 32, 8 * i + 4 * q + 2 * (lane / 32) + h), 16), v + 4 * h, 16);
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll 2
      for (int r = lane; r < 32 * 4 * FM; r += kWave) {
        const int row = r / (4 * FM), at = r % (4 * FM);
        float v[kVec];
#pragma unroll
        for (int h = 0; h < 2; ++h) __builtin_memcpy(v + 4 * h, __builtin_assume_aligned(lds + run_at(row, 2 * at + h), 16), 16);
        run(m0 + 8 * at, n0 + 32 * j + row, v);
      }
      if constexpr (TURN) {
#pragma unroll 2
        for (int r = lane; r < 32 * 4 * FM; r += kWave) {
          const int i = r / 4, at = r % 4 * kVec;
          float v[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) __builtin_memcpy(v + e, lds + run_at(at + e, i / 4) + i % 4 * 4, 4);
          turned(m0 + i, n0 + 32 * j + at, v);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  template <class Run>
  __device__ __forceinline__ void for_runs(int64_t m0, int64_t n0, char* lds, const Run& run) {
    for_runs<false>(m0, n0, lds, [](int, int, float (&)[kVec]) {}, run, 0);
  }
};

// Consecutive work-groups go to the eight dies in turn.  Each die takes tiles that lie together, in bands eight tiles wide,
// so that its cache is asked for the same rows.
__device__ __forceinline__ unsigned on_its_die(unsigned all) {
  const unsigned die = blockIdx.x % 8, each = all / 8, more = all % 8;
  return die * each + min(die, more) + blockIdx.x / 8;
}
// LOWER: tiles on and below the diagonal only.
template <bool LOWER>
__device__ __forceinline__ void tile_of(const ProductArgs& A, unsigned tile, unsigned& tm, unsigned& tn) {
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

// A work-group per tile and split.
template <class P, bool LOWER, HowMany MANY, class Epilogue>
__global__ __launch_bounds__(P::kGroup, P::kWavesPerSimd) void product_kernel(ProductArgs A, Epilogue out) {
  __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
  if constexpr (MANY != kAll) {
    const int n = max(1, *A.fewer.n);
    if constexpr (MANY == kFewerOfK) {
      A.steps = (n + P::kStep - 1) / P::kStep;
    } else {
      const bool all = A.fewer.all && n == A.b.n;
      A.b.p = all ? A.fewer.all : A.b.p;
      A.b.ld = all ? A.fewer.all_ld : A.b.ld;
      if (A.fewer.wide) A.a.p = *A.fewer.wide ? A.fewer.wide_a : A.a.p;
      A.splits = A.fewer.most_splits ? splits_of_fewer(A.splits, A.fewer.most_splits, P::kN, (unsigned)A.b.n, n) : A.splits;
      A.b.n = n;
      A.tiles_n = (unsigned)(n + P::kN - 1) / P::kN;
      A.tiles = A.tiles_m * A.tiles_n;
    }
    A.split_steps = (A.steps + (int)A.splits - 1) / (int)A.splits;
    if (blockIdx.x >= A.tiles * A.batch * A.splits) return;
  }
  const unsigned tile = on_its_die(A.tiles * A.batch * A.splits), which = tile / A.tiles, matrix = which / A.splits;
  unsigned tm, tn;
  tile_of<LOWER>(A, tile - which * A.tiles, tm, tn);
  const int64_t m0 = (int64_t)tm * P::kM, n0 = (int64_t)tn * P::kN;
  P p;
  p.run(A, matrix, which - matrix * A.splits, m0, n0, lds);
  if (p.owns) out(p, p.wave_m(m0), p.wave_n(n0), lds + p.wave * (P::kBuffers * P::kBuffer / P::kWavesHere));
}

// Launches tiles of the given form over all of A and B; k: how many there are, zeros up to a whole step.
template <class P, bool LOWER = false, HowMany MANY = kAll, class Epilogue>
int product_launch(const Operand& a, const Operand& b, int64_t k, const Epilogue& out, unsigned batch, hipStream_t stream, int64_t splits = 1,
                   const Fewer& fewer = {}) {
  ProductArgs A = {a, b, (int)ceil_div(k, P::kStep), 0, 0, (unsigned)ceil_div(a.n, P::kM), (unsigned)ceil_div(b.n, P::kN), 0, batch, fewer};
  A.split_steps = (int)ceil_div(A.steps, splits);
  A.splits = (unsigned)ceil_div(A.steps, A.split_steps);       // none is empty
  A.tiles = LOWER ? A.tiles_m * (A.tiles_m + 1) / 2 : A.tiles_m * A.tiles_n;
  product_kernel<P, LOWER, MANY><<<A.tiles * batch * A.splits, P::kGroup, 0, stream>>>(A, out);
  return launch_status();
}
template <bool BF16, Lies LA, Lies LB> using Product256 = Product<BF16, LA, LB, 2, 2, 4, 4>;
template <bool BF16, Lies LA, Lies LB> using Product128 = Product<BF16, LA, LB, 2, 2, 2, 2>;
// v as hi + lo of binary16: 22 bits and a sign between them, as long as v is at least 2^-13; what is lost below is 2^-25 at most.
__device__ __forceinline__ void split_f16(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}
// Eight numbers to their place in a row of parts, and back.
__device__ __forceinline__ void put_parts(_Float16* p, const float (&v)[kVec]) {
  _Float16 hi[kVec], lo[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) split_f16(v[i], hi[i], lo[i]);
  __builtin_memcpy(__builtin_assume_aligned(p, 16), hi, sizeof hi);
  __builtin_memcpy(__builtin_assume_aligned(p + kVec, 16), lo, sizeof lo);
}
__device__ __forceinline__ void get_parts(const _Float16* p, float (&v)[kVec]) {
  _Float16 hi[kVec], lo[kVec];
  __builtin_memcpy(hi, __builtin_assume_aligned(p, 16), sizeof hi);
  __builtin_memcpy(lo, __builtin_assume_aligned(p + kVec, 16), sizeof lo);
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

#endif  // __HIPCC__

}  // namespace qa
