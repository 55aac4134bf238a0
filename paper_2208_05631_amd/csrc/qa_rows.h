// Rows of activations: loads and stores of eight elements of any type at any alignment, and the 8-bit code of a
// group of columns.  Shared by the kernels on activations; not part of the public interface.
#pragma once
#include "qa_common.h"

namespace qa {

inline bool known_type(int type) { return type == QA_F32 || type == QA_BF16 || type == QA_F16; }
inline int64_t type_bytes(int type) { return type == QA_F32 ? 4 : 2; }
inline bool element_aligned(const void* p, int type) { return aligned(p, (size_t)type_bytes(type)); }
inline int64_t groups_of(const qa_coded_rows* R) { return (R->cols + R->group - 1) / R->group; }
constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_rows(const qa_coded_rows* R) {
  if (!R) return QA_ERR_INVALID_ARG;
  if (R->rows < 0 || R->rows >= (int64_t(1) << 31)) return QA_ERR_INVALID_ARG;
  if (R->cols < 1 || R->cols >= (int64_t(1) << 24)) return QA_ERR_INVALID_ARG;
  if (R->group != 32 && R->group != 64 && R->group != 128) return QA_ERR_INVALID_ARG;
  if (R->code_stride < R->cols || R->code_stride % 16) return QA_ERR_INVALID_ARG;
  if (R->scale_stride < groups_of(R)) return QA_ERR_INVALID_ARG;
  return QA_OK;
}

// Whether a call reads and writes more than the last-level cache holds.  Its outputs, or what it reads once, go past the
// caches then, where its kernel has such a form and gains by it: the norm of 8192 x 4096 bfloat16 59 -> 52 us, its backward pass over
// 16384 x 4096 95 -> 88, codes of 16384 x 8192 and their values again 158 -> 144, log probabilities of 4096 x 100003 with 8 alternatives
// 169 -> 161, the logits' gradient of 8192 x 32768 198 -> 178.  Smaller calls lose by it if the caches hold what they read and
// write (norm of 4096 x 4096 23 -> 27, backward 24 -> 27) and gain if they do not (30 -> 28, 29 -> 28): their inputs are what the step
// before has just written.  The norm and log probabilities in binary32, rows that registers do not hold and weight gradients keep to the
// caches: a lane's eight binary32 elements are two words with another lane's between them, and a line is asked for twice
// (binary32, norm of 16384 x 4096: 181 us, and 194 past the caches, 30000 x 2047: 170 and 196; backward 206 both).
inline bool streams(double bytes) { return bytes > (double)(256 << 20); }

#if defined(__HIPCC__)

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
// The same at an element's alignment: rows of odd strides are read and written 16 bytes at a time all the same,
// which the memory pipeline does at any byte address.
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));

constexpr int kVec = 8;                            // elements that a lane holds side by side

template <int TYPE> struct Elem;
template <> struct Elem<QA_F32> { typedef float T; };
template <> struct Elem<QA_BF16> { typedef __bf16 T; };
template <> struct Elem<QA_F16> { typedef _Float16 T; };
template <int TYPE> using ElemT = typename Elem<TYPE>::T;

__device__ __forceinline__ float as_f32(uint32_t u) { return __uint_as_float(u); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __float_as_uint(f); }

// Eight elements as they lie in memory: registers of a load that is still on its way.
template <int TYPE> struct Raw8 { u32x4 a; };
template <> struct Raw8<QA_F32> { f32x4 a, b; };

// STREAM: past the caches, for calls that they do not hold (streams() above).
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ Raw8<TYPE> load_raw(const ElemT<TYPE>* p) {
  Raw8<TYPE> r;
  if constexpr (TYPE == QA_F32) {
    const f32x4_at4* q = reinterpret_cast<const f32x4_at4*>(p);
    r.a = STREAM ? __builtin_nontemporal_load(q) : q[0];
    r.b = STREAM ? __builtin_nontemporal_load(q + 1) : q[1];
  } else {
    const u32x4_at2* q = reinterpret_cast<const u32x4_at2*>(p);
    r.a = STREAM ? __builtin_nontemporal_load(q) : q[0];
  }
  return r;
}
// The first n of eight elements, the others `rest`.
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ Raw8<TYPE> load_raw(const ElemT<TYPE>* p, int n, float rest = 0.0f) {
  if (n >= kVec) return load_raw<TYPE, STREAM>(p);
  ElemT<TYPE> v[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = i < n ? p[i] : (ElemT<TYPE>)rest;
  Raw8<TYPE> r;
  __builtin_memcpy(&r, v, sizeof r);
  return r;
}
template <int TYPE>
__device__ __forceinline__ void to_f32(const Raw8<TYPE>& r, float (&v)[kVec]) {
  if constexpr (TYPE == QA_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
  } else if constexpr (TYPE == QA_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = as_f32(r.a[i] << 16); v[2 * i + 1] = as_f32(r.a[i] & 0xFFFF0000u); }
  } else {
    _Float16 h[kVec];
    __builtin_memcpy(h, &r, sizeof h);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)h[i];
  }
}
// Rounded once, to nearest and ties to even.
template <int TYPE>
__device__ __forceinline__ Raw8<TYPE> from_f32(const float (&v)[kVec]) {
  Raw8<TYPE> r;
  if constexpr (TYPE == QA_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.a[i] = v[i]; r.b[i] = v[4 + i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 two = {v[2 * i], v[2 * i + 1]};
      if constexpr (TYPE == QA_BF16)
        r.a[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
      else
        r.a[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, f16x2));
    }
  }
  return r;
}
template <int TYPE, bool STREAM = false>
__device__ __forceinline__ void store_raw(ElemT<TYPE>* p, const Raw8<TYPE>& r, int n = kVec) {
  if (n >= kVec) {
    if constexpr (TYPE == QA_F32) {
      f32x4_at4* q = reinterpret_cast<f32x4_at4*>(p);
      if constexpr (STREAM) {
        __builtin_nontemporal_store(r.a, q);
        __builtin_nontemporal_store(r.b, q + 1);
      } else {
        q[0] = r.a;
        q[1] = r.b;
      }
    } else {
      u32x4_at2* q = reinterpret_cast<u32x4_at2*>(p);
      if constexpr (STREAM) __builtin_nontemporal_store(r.a, q);
      else q[0] = r.a;
    }
    return;
  }
  ElemT<TYPE> v[kVec];
  __builtin_memcpy(v, &r, sizeof v);
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (i < n) p[i] = v[i];
}

// v as `P` bfloat16 parts, each the leading eight bits of what is left: exact for 8 P bits, but for what lies below 2^-133,
// bfloat16's last bit (matrix instructions take numbers under 2^-126 as they are).
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

// ---- between lanes ---------------------------------------------------------------------------------------

__device__ __forceinline__ float wave_sum_f32(float v) {
  v += as_f32((uint32_t)dpp_i32<kDppQuadXor1>((int)as_u32(v)));
  v += as_f32((uint32_t)dpp_i32<kDppQuadXor2>((int)as_u32(v)));
  v += as_f32((uint32_t)dpp_i32<kDppRowHalfMirror>((int)as_u32(v)));
  v += as_f32((uint32_t)dpp_i32<kDppRowMirror>((int)as_u32(v)));
  const int i = (int)as_u32(v);
  return (as_f32((uint32_t)__builtin_amdgcn_readlane(i, 0)) + as_f32((uint32_t)__builtin_amdgcn_readlane(i, 16))) +
         (as_f32((uint32_t)__builtin_amdgcn_readlane(i, 32)) + as_f32((uint32_t)__builtin_amdgcn_readlane(i, 48)));
}
constexpr int kDppQuadReverse = 0x1B;               // quad_perm:[3,2,1,0]
// The value of the lane whose number differs in `STRIDE` alone.  Up to 8 two moves between neighbours do it, a tenth of
// the time that a way through LDS takes; rows of 16 lanes are swapped with their neighbours.
template <int STRIDE>
__device__ __forceinline__ uint32_t other_lane(uint32_t v) {
  const int i = (int)v;
  if constexpr (STRIDE == 1) return (uint32_t)dpp_i32<kDppQuadXor1>(i);
  if constexpr (STRIDE == 2) return (uint32_t)dpp_i32<kDppQuadXor2>(i);
  if constexpr (STRIDE == 4) return (uint32_t)dpp_i32<kDppQuadReverse>(dpp_i32<kDppRowHalfMirror>(i));
  if constexpr (STRIDE == 8) return (uint32_t)dpp_i32<kDppRowHalfMirror>(dpp_i32<kDppRowMirror>(i));
  if constexpr (STRIDE == 16) {
    const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? both[0] : both[1];
  }
  if constexpr (STRIDE == 32) {
    const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? both[0] : both[1];
  }
}
template <int STRIDE>
__device__ __forceinline__ uint64_t other_lane(uint64_t v) {
  return (uint64_t)other_lane<STRIDE>((uint32_t)(v >> 32)) << 32 | other_lane<STRIDE>((uint32_t)v);
}

// ---- the 8-bit code of a group of columns -----------------------------------------------------------------
//
// A group has one byte b, its scale is 2^(b - 127): the smallest power of two by which the group's largest magnitude
// is at most 127, and 2^-126 at least.  A code is the nearest whole multiple, ties to even.  The scale is a power of
// two because a code times one has at most seven significant bits: it is exact in bfloat16, and matrix instructions
// that read the codes multiply exactly what the forward pass used.  It costs up to one of the eight bits.  A group
// with an infinity or a NaN has b = 255 and codes 0, and every value of it is read back as NaN.  At the largest scale
// that a finite magnitude needs, 2^122, codes end at 63: 64 would be 2^128.

constexpr uint32_t kNoScale = 255, kLargestScale = 249;

// b from the bits of the largest magnitude (1.984375 = 127 / 64 is the largest mantissa that still fits 127).
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  if (most >= 0x7F800000u) return kNoScale;
  const int b = (int)((most + 0x1FFFFu) >> 23) - 6;
  return (uint32_t)(b > 1 ? b : 1);
}
// Infinity for a group without values: 0 times it is the NaN that they are read back as.
__device__ __forceinline__ float scale_of(uint32_t b) { return as_f32(b << 23); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
  const uint32_t o = (uint32_t)dpp_i32<CTRL>((int)v);
  return v > o ? v : o;
}
// The largest of `lanes` (4, 8 or 16) aligned neighbours' values.
__device__ __forceinline__ uint32_t lanes_max_u32(uint32_t v, int lanes) {
  v = dpp_max_u32<kDppQuadXor1>(v);
  v = dpp_max_u32<kDppQuadXor2>(v);
  if (lanes > 4) v = dpp_max_u32<kDppRowHalfMirror>(v);
  if (lanes > 8) v = dpp_max_u32<kDppRowMirror>(v);
  return v;
}
__device__ __forceinline__ uint32_t most_of(const float (&v)[kVec]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const uint32_t a = as_u32(v[i]) & 0x7FFFFFFFu;
    m = m > a ? m : a;
  }
  return m;
}

// Codes of eight values as bytes of two words, and the values that they stand for.  1.5 * 2^23 added to a value
// below 2^22 leaves its nearest whole number, ties to even, in the low bits; the product in front is exact.
__device__ __forceinline__ u32x2 code8(const float (&v)[kVec], uint32_t b, float (&value)[kVec]) {
  constexpr float kWhole = 12582912.0f;
  const float inverse = as_f32((254u - b) << 23), scale = scale_of(b);
  uint32_t w[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const float r = __builtin_fmaf(v[i], inverse, kWhole);
    w[i] = as_u32(r);
    value[i] = (r - kWhole) * scale;
  }
  u32x2 code;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t lo = __builtin_amdgcn_perm(w[4 * k + 1], w[4 * k], 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(w[4 * k + 3], w[4 * k + 2], 0x04000C0Cu);
    code[k] = lo | hi;
  }
  if (b >= kLargestScale) {                        // rare
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int whole = b == kNoScale ? 0 : max(-63, min(63, (int)(int8_t)w[i]));
      code[i / 4] = (code[i / 4] & ~(0xFFu << (8 * (i % 4)))) | (uint32_t)(uint8_t)whole << (8 * (i % 4));
      value[i] = b == kNoScale ? __builtin_nanf("") : (float)whole * scale;
    }
  }
  return code;
}
__device__ __forceinline__ void decode8(u32x2 code, uint32_t b, float (&v)[kVec]) {
  const float scale = scale_of(b);
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = (float)(int8_t)(code[i / 4] >> (8 * (i % 4))) * scale;
}
// The first n of eight codes; rows begin on 16 bytes, so that eight always have their place.
template <bool STREAM>
__device__ __forceinline__ void store_codes(int8_t* p, u32x2 code, int n) {
  if (n >= kVec) {
    u32x2* q = reinterpret_cast<u32x2*>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(code, q);
    else *q = code;
    return;
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (i < n) p[i] = (int8_t)(code[i / 4] >> (8 * (i % 4)));
}

#endif  // __HIPCC__

}  // namespace qa
