// Vectors of elements of a caller's type, held as binary32 in registers.  A caller's rows may
// start at any element, so vectors are read and written at the element's alignment: gfx950
// takes 16-byte global accesses at any address, and the types below say so to the compiler.
#pragma once

#include "device.h"

namespace fp4r {

struct bf16_t { uint16_t bits; };
struct f16_t { uint16_t bits; };

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a1 __attribute__((aligned(1)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

FP4R_DEV float to_f32(float v) { return v; }
FP4R_DEV float to_f32(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
FP4R_DEV float to_f32(f16_t v) { return (float)__builtin_bit_cast(_Float16, v.bits); }

// Two elements of a 16-bit type, from and to one word.
FP4R_DEV void unpack2(bf16_t, uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xFFFF0000u);
}
FP4R_DEV void unpack2(f16_t, uint32_t w, float& a, float& b) {
  a = to_f32(f16_t{(uint16_t)w});
  b = to_f32(f16_t{(uint16_t)(w >> 16)});
}
// The binary32 value first: folded into the product before it (v_fma_mixlo_f16), the rounding
// to binary32 would be left out.
FP4R_DEV uint32_t f16_bits(float v) {
  asm("" : "+v"(v));
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}
// Round to nearest, ties to even, infinities past the largest; a NaN stays one.
FP4R_DEV uint32_t pack2(bf16_t, float a, float b) { return bf16_pair(a, b); }
FP4R_DEV uint32_t pack2(f16_t, float a, float b) { return f16_bits(a) | f16_bits(b) << 16; }

// A vector of N elements as it lies in memory (8 or 16 bytes), and its values.  NT: past the
// caches, which keep what they hold.
template <bool NT, class V, class P>
FP4R_DEV V load_as(const P* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool NT, class V, class P>
FP4R_DEV void store_as(P* p, V v) {
  if constexpr (NT) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <class T, int N, bool NT = false>
FP4R_DEV auto load_raw(const T* p) {
  static_assert(N * sizeof(T) == 16 || (N * sizeof(T) == 8 && sizeof(T) == 2), "one vector");
  if constexpr (sizeof(T) == 4) return load_as<NT, u32x4>(reinterpret_cast<const u32x4_a4*>(p));
  else if constexpr (N == 8) return load_as<NT, u32x4>(reinterpret_cast<const u32x4_a2*>(p));
  else return load_as<NT, u32x2>(reinterpret_cast<const u32x2_a2*>(p));
}
template <class T, int N, class V>
FP4R_DEV void unpack_raw(const V& w, float (&x)[N]) {
#pragma unroll
  for (int k = 0; k < (int)(N * sizeof(T) / 4); ++k) {
    if constexpr (sizeof(T) == 4) x[k] = __uint_as_float(w[k]);
    else unpack2(T{}, w[k], x[2 * k], x[2 * k + 1]);
  }
}
// N values as 16-byte vectors (4 of a 16-bit type: one of 8 bytes), past the caches: what is
// written once and not read by the same kernel displaces nothing (clipping 354 M BF16 elements
// into FP32 551 -> 501 us, twelve parameters of 2.0 M elements 12.6 -> 12.1).
template <class T, int N>
FP4R_DEV void store_full(T* p, const float (&x)[N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = __float_as_uint(x[4 * q + k]);
      store_as<true>(reinterpret_cast<u32x4_a4*>(p + 4 * q), w);
    }
  } else if constexpr (N == 4) {
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) w[k] = pack2(T{}, x[2 * k], x[2 * k + 1]);
    store_as<true>(reinterpret_cast<u32x2_a2*>(p), w);
  } else {
#pragma unroll
    for (int q = 0; q < N / 8; ++q) {
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = pack2(T{}, x[8 * q + 2 * k], x[8 * q + 2 * k + 1]);
      store_as<true>(reinterpret_cast<u32x4_a2*>(p + 8 * q), w);
    }
  }
}

// The first n of N elements; the others are 0, and nothing past them is touched.
template <class T, int N>
FP4R_DEV void load_vec(const T* p, int n, float (&x)[N]) {
  if (n >= N) {
    unpack_raw<T, N>(load_raw<T, N>(p), x);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = k < n ? to_f32(p[k]) : 0.0f;
  }
}
FP4R_DEV void put(float* p, float v) { *p = v; }
FP4R_DEV void put(bf16_t* p, float v) { p->bits = (uint16_t)pack2(bf16_t{}, v, 0.0f); }
FP4R_DEV void put(f16_t* p, float v) { p->bits = (uint16_t)f16_bits(v); }
template <class T, int N>
FP4R_DEV void store_vec(T* p, int n, const float (&x)[N]) {
  if (n >= N) {
    store_full<T, N>(p, x);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < n) put(p + k, x[k]);
  }
}

// Eight elements as they lie in memory: a kernel that keeps a row in registers holds 16-bit
// types packed and unpacks them where it uses them.
template <class T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
};
template <class T, bool NT = false>
FP4R_DEV Raw8<T> load_raw8(const T* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
      u32x4 v;
      if constexpr (sizeof(T) == 4) v = load_as<NT, u32x4>(reinterpret_cast<const u32x4_a4*>(p + 4 * q));
      else v = load_as<NT, u32x4>(reinterpret_cast<const u32x4_a2*>(p));
#pragma unroll
      for (int k = 0; k < 4; ++k) r.w[4 * q + k] = v[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k) {
      if constexpr (sizeof(T) == 4) {
        r.w[k] = k < n ? __float_as_uint(p[k]) : 0u;
      } else {
        const uint32_t lo = 2 * k < n ? p[2 * k].bits : 0u, hi = 2 * k + 1 < n ? p[2 * k + 1].bits : 0u;
        r.w[k] = lo | hi << 16;
      }
    }
  }
  return r;
}
template <class T, bool NT = false>
FP4R_DEV void store_raw8(T* p, int n, const Raw8<T>& r) {
  if (n >= 8) {
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
      u32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = r.w[4 * q + k];
      if constexpr (sizeof(T) == 4) store_as<NT>(reinterpret_cast<u32x4_a4*>(p + 4 * q), v);
      else store_as<NT>(reinterpret_cast<u32x4_a2*>(p), v);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= n) continue;
      if constexpr (sizeof(T) == 4) p[k] = __uint_as_float(r.w[k]);
      else p[k].bits = (uint16_t)(r.w[k / 2] >> (16 * (k & 1)));
    }
  }
}
template <class T>
FP4R_DEV void unpack8(const Raw8<T>& r, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r.w[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack2(T{}, r.w[k], x[2 * k], x[2 * k + 1]);
  }
}
template <class T>
FP4R_DEV Raw8<T> pack8(const float (&x)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k) r.w[k] = __float_as_uint(x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) r.w[k] = pack2(T{}, x[2 * k], x[2 * k + 1]);
  }
  return r;
}

}  // namespace fp4r
