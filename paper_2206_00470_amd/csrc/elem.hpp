// Elements of the token-table operators in memory: fp32, bf16 or fp16 words,
// VW consecutive ones at a time, as fp32 in registers.  Widening is exact,
// narrowing rounds to the nearest value, ties to the even one.
#pragma once

#include "common.hpp"

namespace adapm {

typedef _Float16 f16_t;

template <class T, int VW> struct Raw;   // the words of VW elements
template <> struct Raw<float, 1> { using type = uint32_t; };
template <> struct Raw<float, 4> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Raw<float, 8> { typedef uint32_t type __attribute__((ext_vector_type(8))); };
template <> struct Raw<bf16_t, 1> { using type = uint16_t; };
template <> struct Raw<bf16_t, 4> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Raw<bf16_t, 8> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct Raw<f16_t, 1> { using type = uint16_t; };
template <> struct Raw<f16_t, 4> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Raw<f16_t, 8> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

typedef uint32_t words4 __attribute__((ext_vector_type(4)));

template <class T, int VW>
using raw_t = typename Raw<T, VW>::type;

// Loads and stores at addresses aligned to the vector.
template <class T, int VW>
__device__ __forceinline__ raw_t<T, VW> load_raw(const T* p) {
  return *reinterpret_cast<const raw_t<T, VW>*>(p);
}

// Element e of the words.
template <class T, int VW>
__device__ __forceinline__ float raw_get(const raw_t<T, VW>& r, int e) {
  if constexpr (std::is_same_v<T, float>) {
    if constexpr (VW == 1) return __builtin_bit_cast(float, r);
    else return __builtin_bit_cast(float, (uint32_t)r[e]);
  } else {
    uint32_t w;
    if constexpr (VW == 1) w = r;
    else w = e & 1 ? r[e >> 1] >> 16 : r[e >> 1] & 0xffffu;
    if constexpr (std::is_same_v<T, bf16_t>) return __builtin_bit_cast(float, w << 16);
    else return (float)__builtin_bit_cast(f16_t, (uint16_t)w);
  }
}

__device__ __forceinline__ uint32_t narrow_word(bf16_t, float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ uint32_t narrow_word(f16_t, float f) {
  asm("" : "+v"(f));   // an fp32 word first: a product narrowed in one mixed instruction would be rounded once, not twice
  return __builtin_bit_cast(uint16_t, (f16_t)f);
}

// Two values in a word, the first in the low half.
typedef float float_pair __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t narrow_pair(bf16_t, float a, float b) {   // one instruction
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float_pair{a, b}), bf16_pair));
}
__device__ __forceinline__ uint32_t narrow_pair(f16_t, float a, float b) {
  return narrow_word(f16_t{}, a) | narrow_word(f16_t{}, b) << 16;
}

template <class T, int VW>
__device__ __forceinline__ raw_t<T, VW> raw_make(const float* x) {
  if constexpr (std::is_same_v<T, float>) {
    if constexpr (VW == 1) {
      return __builtin_bit_cast(uint32_t, x[0]);
    } else {
      raw_t<T, VW> r;
#pragma unroll
      for (int e = 0; e < VW; ++e) r[e] = __builtin_bit_cast(uint32_t, x[e]);
      return r;
    }
  } else if constexpr (VW == 1) {
    return (uint16_t)narrow_word(T{}, x[0]);
  } else {
    raw_t<T, VW> r;
#pragma unroll
    for (int e = 0; e < VW; e += 2) r[e / 2] = narrow_pair(T{}, x[e], x[e + 1]);
    return r;
  }
}

template <class T, int VW, bool NT = false>
__device__ __forceinline__ void store_raw(T* p, const raw_t<T, VW>& r) {
  if constexpr (NT) __builtin_nontemporal_store(r, reinterpret_cast<raw_t<T, VW>*>(p));
  else *reinterpret_cast<raw_t<T, VW>*>(p) = r;
}

// The same in global memory at addresses that are aligned to their elements
// only: global memory takes vectors of up to 16 bytes at any address.
typedef uint32_t words4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words2_any __attribute__((ext_vector_type(2), aligned(2)));

template <class T, int VW>
__device__ __forceinline__ raw_t<T, VW> load_any(const T* p) {
  constexpr int bytes = sizeof(T) * VW;
  if constexpr (bytes == 32) {
    const words4_any *q = reinterpret_cast<const words4_any*>(p);
    const words4 a = q[0], b = q[1];
    return raw_t<T, VW>{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  } else if constexpr (bytes == 16) {
    return *reinterpret_cast<const words4_any*>(p);
  } else if constexpr (bytes == 8) {
    return *reinterpret_cast<const words2_any*>(p);
  } else {
    return load_raw<T, VW>(p);
  }
}

template <class V, bool NT>
__device__ __forceinline__ void store_words(void* p, V v) {
  if constexpr (NT) __builtin_nontemporal_store(v, static_cast<V*>(p));
  else *static_cast<V*>(p) = v;
}

template <class T, int VW, bool NT = false>
__device__ __forceinline__ void store_any(T* p, const raw_t<T, VW>& r) {
  constexpr int bytes = sizeof(T) * VW;
  if constexpr (bytes == 32) {
    store_words<words4_any, NT>(p, words4{r[0], r[1], r[2], r[3]});
    store_words<words4_any, NT>(reinterpret_cast<char*>(p) + 16, words4{r[4], r[5], r[6], r[7]});
  } else if constexpr (bytes == 16) {
    store_words<words4_any, NT>(p, r);
  } else if constexpr (bytes == 8) {
    store_words<words2_any, NT>(p, r);
  } else {
    store_raw<T, VW, NT>(p, r);
  }
}

// f(T{}) for the element type that a type code of the C ABI names; the
// caller has checked the code.
template <class F>
auto with_type(int32_t type, F&& f) {
  if (type == 1) return f(bf16_t{});
  if (type == 2) return f(f16_t{});
  return f(0.0f);
}

inline int type_bytes(int32_t type) { return type == 0 ? 4 : 2; }

// Quotients by a divisor d < 2^15 of numbers below 2^16: x * (2^32 / d + 1) is
// off by less than x, so its high word is exact while x * d < 2^32.
struct SmallDiv {
  uint32_t d, magic;
};
inline SmallDiv small_div(uint32_t d) { return SmallDiv{d, d > 1 ? (uint32_t)((uint64_t(1) << 32) / d) + 1u : 0u}; }
__device__ __forceinline__ uint32_t quotient(uint32_t x, const SmallDiv& s) {
  return s.d > 1 ? __umulhi(x, s.magic) : x;
}

}  // namespace adapm
