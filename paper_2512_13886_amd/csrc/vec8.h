// Eight consecutive values of a row as one wide access, for kernels that take
// rows of any pitch: the 16-byte loads and stores need only the alignment of an
// element (gfx950 serves unaligned global accesses).
#pragma once

#include "common.h"

namespace optima {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_2 __attribute__((aligned(2)));
typedef u32x4 u32x4_4 __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_1 __attribute__((aligned(1)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct bf16_t {
  uint16_t bits;
};

// Two values rounded to bf16 (nearest even; NaN stays NaN), a in the low half.
__device__ inline uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, bf16x2));
}
__device__ inline float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight values as they are stored.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
  u32x4 w;
};
template <>
struct Raw8<float> {
  u32x4 w[2];
};

__device__ inline void load8(Raw8<bf16_t>& r, const bf16_t* p) {
  r.w = *reinterpret_cast<const u32x4_2*>(p);
}
__device__ inline void load8(Raw8<float>& r, const float* p) {
  r.w[0] = *reinterpret_cast<const u32x4_4*>(p);
  r.w[1] = *reinterpret_cast<const u32x4_4*>(p + 4);
}
__device__ inline void values8(const Raw8<bf16_t>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_low(r.w[i]);
    v[2 * i + 1] = bf16_high(r.w[i]);
  }
}
__device__ inline void values8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i >> 2][i & 3]);
}

// The first n (0 .. 8) of eight values; zeros for the rest.
__device__ inline void load_some(Raw8<bf16_t>& r, const bf16_t* p, int n) {
  r.w = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) r.w[i >> 1] |= uint32_t(p[i].bits) << (16 * (i & 1));
}
__device__ inline void load_some(Raw8<float>& r, const float* p, int n) {
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = i < n ? __float_as_uint(p[i]) : 0u;
}

// Eight values moved down by s (0 .. 7) places, zeros from above.
__device__ inline void shift_down(Raw8<bf16_t>& r, int s) {
  if (s & 4) r.w = u32x4{r.w[2], r.w[3], 0, 0};
  if (s & 2) r.w = u32x4{r.w[1], r.w[2], r.w[3], 0};
  if (s & 1)
    r.w = u32x4{__builtin_amdgcn_alignbit(r.w[1], r.w[0], 16),
                __builtin_amdgcn_alignbit(r.w[2], r.w[1], 16),
                __builtin_amdgcn_alignbit(r.w[3], r.w[2], 16), r.w[3] >> 16};
}
__device__ inline void shift_down(Raw8<float>& r, int s) {
  if (s & 4) r.w[0] = r.w[1], r.w[1] = u32x4{0, 0, 0, 0};
  if (s & 2) {
    r.w[0] = u32x4{r.w[0][2], r.w[0][3], r.w[1][0], r.w[1][1]};
    r.w[1] = u32x4{r.w[1][2], r.w[1][3], 0, 0};
  }
  if (s & 1) {
    r.w[0] = u32x4{r.w[0][1], r.w[0][2], r.w[0][3], r.w[1][0]};
    r.w[1] = u32x4{r.w[1][1], r.w[1][2], r.w[1][3], 0};
  }
}
// Values at .. at + 7 of a row of d; zeros past its end. A row's last piece is loaded
// from eight values before its end, and moved: one wide load like the others (value by
// value, each load waits for the one before: 8.4 us in place of 6.3 for the preparation of
// the gated gradient at 192 tokens, 64 -> 335).
template <typename T>
__device__ inline void load_piece(Raw8<T>& r, const T* row, int at, int d) {
  if (at + 8 <= d) {
    load8(r, row + at);
    return;
  }
  r = Raw8<T>{};
  if (at >= d) return;
  if (d < 8) {
    load_some(r, row + at, d - at);
  } else {
    load8(r, row + d - 8);
    shift_down(r, at + 8 - d);
  }
}

__device__ inline void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4_2*>(p) =
      u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
            pack_bf16(v[6], v[7])};
}
__device__ inline void store8(float* p, const float (&v)[8]) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __float_as_uint(v[i]);
    b[i] = __float_as_uint(v[4 + i]);
  }
  *reinterpret_cast<u32x4_4*>(p) = a;
  *reinterpret_cast<u32x4_4*>(p + 4) = b;
}
typedef u32x2 u32x2_2 __attribute__((aligned(2)));
// The first n (0 .. 4) of four values.
__device__ inline void store1(bf16_t* p, float v) { p->bits = uint16_t(pack_bf16(v, v)); }
__device__ inline void store1(float* p, float v) { *p = v; }
__device__ inline void store_upto4(bf16_t* p, const float (&v)[4], int n) {
  if (n >= 4) {
    *reinterpret_cast<u32x2_2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) store1(p + i, v[i]);
}
__device__ inline void store_upto4(float* p, const float (&v)[4], int n) {
  if (n >= 4) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]);
    *reinterpret_cast<u32x4_4*>(p) = a;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) store1(p + i, v[i]);
}
// Whole numbers within +-2^22: the low bytes of their bit patterns once 1.5 2^23 is added.
__device__ inline uint32_t int_bits(float v) { return __float_as_uint(v + 12582912.f); }
__device__ inline void store8(int8_t* p, const float (&v)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(int_bits(v[4 * h + 1]), int_bits(v[4 * h]), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(int_bits(v[4 * h + 3]), int_bits(v[4 * h + 2]), 0x04000C0Cu);
    w[h] = lo | hi;
  }
  *reinterpret_cast<u32x2_1*>(p) = u32x2{w[0], w[1]};
}
__device__ inline void store1(int8_t* p, float v) { *p = int8_t(int(v)); }
// The first n (0 .. 8) of eight values.
template <typename T>
__device__ inline void store_upto8(T* p, const float (&v)[8], int n) {
  if (n >= 8) {
    store8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) store1(p + i, v[i]);
}

}  // namespace optima
