// What the kernels that go over trajectories in chunks share (device code): the arrays as they lie in memory, eight columns of a row
// at a time, and the arithmetic of each element type on the matrix cores.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sf_memory.h"
#include "sf_split.h"

namespace sf {

// n / d for 0 <= n < 2^31, without a division on the device
struct Divisor {
  unsigned mul, shift;
  __device__ unsigned of(unsigned n) const { return (__umulhi(mul, n) + n) >> shift; }
};
inline Divisor divisor(unsigned d) {
  unsigned shift = 0;
  while ((1u << shift) < d) ++shift;
  return Divisor{(unsigned)(((1ull << 32) * ((1ull << shift) - d)) / d + 1), shift};
}

struct Strided {
  const void* p;
  int64_t st, sn, sh;  // step, row, head (elements)
  int shared;          // by the heads of a group
  int d;               // columns
  int vec;             // rows are read in 16-byte pieces
};

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

__device__ inline unsigned pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ inline float lo_of(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float hi_of(unsigned w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// two terms of two numbers
__device__ inline void split2(float a, float b, unsigned& t0, unsigned& t1) {
  t0 = pack_bf16(a, b);
  t1 = pack_bf16(a - lo_of(t0), b - hi_of(t0));
}

__device__ inline float pow2(float x) { return __builtin_amdgcn_exp2f(x); }  // (x <= 0 here; below 2^-126: 0)

// The arithmetic of one element type.  An operand is eight K-slots per lane.
template <int DTYPE>
struct Num;

template <>
struct Num<SF_DTYPE_BF16> {
  static constexpr int kBytes = 2, kPieceWords = 4;
  typedef u32x4 Raw;                                   // exact values
  struct Out { u32x4 t[2]; };                          // for the output: two terms
  struct Sum { u32x4 t[3]; };                          // for the state: three terms
  __device__ static Raw row(const unsigned char* p) { return *(const u32x4*)p; }  // eight neighbours of a row
  // four K-slots down column col(lane % 16) of rows at .. at + 3: `p` is this lane's share (its row, its four columns)
  __device__ static u32x2 column4(const unsigned char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
  }
  __device__ static void values(const Raw& r, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = lo_of(r[i]);
      x[2 * i + 1] = hi_of(r[i]);
    }
  }
  __device__ static Out out_terms(const float* x) {
    Out o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned a, b;
      split2(x[2 * i], x[2 * i + 1], a, b);
      o.t[0][i] = a;
      o.t[1][i] = b;
    }
    return o;
  }
  __device__ static Sum sum_terms(const float* x) {
    Sum o;
    float left = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned a, b, c;
      split_pair(x[2 * i], x[2 * i + 1], a, b, c, left);
      o.t[0][i] = a;
      o.t[1][i] = b;
      o.t[2][i] = c;
    }
    return o;
  }
  __device__ static f32x4 mma1(const u32x4& a, const u32x4& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  __device__ static f32x4 mma(const Raw& a, const Raw& b, f32x4 c) { return mma1(a, b, c); }
  __device__ static f32x4 mma(const Raw& a, const Out& b, f32x4 c) { return mma1(a, b.t[0], mma1(a, b.t[1], c)); }
  __device__ static f32x4 mma(const Out& a, const Raw& b, f32x4 c) { return mma1(a.t[0], b, mma1(a.t[1], b, c)); }
  __device__ static f32x4 mma(const Sum& a, const Raw& b, f32x4 c) { return mma1(a.t[0], b, mma1(a.t[1], b, mma1(a.t[2], b, c))); }
  __device__ static f32x4 mma(const Raw& a, const Sum& b, f32x4 c) { return mma1(a, b.t[0], mma1(a, b.t[1], mma1(a, b.t[2], c))); }
  // P in LDS: the terms of four slots of half `h`
  __device__ static void put4(unsigned char* frag, int term_pitch, int lane, int h, f32x4 x) {
    unsigned a0, a1, b0, b1;
    split2(x[0], x[1], a0, a1);
    split2(x[2], x[3], b0, b1);
    *(u32x2*)(frag + lane * 16 + h * 8) = u32x2{a0, b0};
    *(u32x2*)(frag + term_pitch + lane * 16 + h * 8) = u32x2{a1, b1};
  }
  __device__ static Out get(const unsigned char* frag, int term_pitch, int lane) {
    Out o;
    o.t[0] = *(const u32x4*)(frag + lane * 16);
    o.t[1] = *(const u32x4*)(frag + term_pitch + lane * 16);
    return o;
  }
  __device__ static float element(const unsigned char* p) { return __builtin_bit_cast(float, (unsigned)*(const uint16_t*)p << 16); }
  __device__ static void store(void* p, float x) { *(uint16_t*)p = (uint16_t)pack_bf16(x, 0.0f); }
};

template <>
struct Num<SF_DTYPE_FP32> {
  static constexpr int kBytes = 4, kPieceWords = 8;
  struct Raw { float x[8]; };
  typedef Raw Out;
  typedef Raw Sum;
  __device__ static Raw row(const unsigned char* p) {
    Raw r;
    *(f32x4*)&r.x[0] = *(const f32x4*)p;
    *(f32x4*)&r.x[4] = *(const f32x4*)(p + 16);
    return r;
  }
  __device__ static void values(const Raw& r, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r.x[i];
  }
  __device__ static Raw out_terms(const float* x) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.x[i] = x[i];
    return r;
  }
  __device__ static Raw sum_terms(const float* x) { return out_terms(x); }
  __device__ static f32x4 mma(const Raw& a, const Raw& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i], b.x[i], c, 0, 0, 0);
    return c;
  }
  __device__ static void put4(unsigned char* frag, int term_pitch, int lane, int h, f32x4 x) {
    *(f32x4*)(frag + h * term_pitch + lane * 16) = x;
  }
  __device__ static Raw get(const unsigned char* frag, int term_pitch, int lane) {
    Raw r;
    *(f32x4*)&r.x[0] = *(const f32x4*)(frag + lane * 16);
    *(f32x4*)&r.x[4] = *(const f32x4*)(frag + term_pitch + lane * 16);
    return r;
  }
  __device__ static float element(const unsigned char* p) { return *(const float*)p; }
  __device__ static void store(void* p, float x) { *(float*)p = x; }
};

// Eight numbers moved down by `n` places (0 .. 7), zeros behind them.
template <int DTYPE>
__device__ inline void move_down(unsigned* w, int n) {
  if constexpr (DTYPE == SF_DTYPE_BF16) {
    uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
    if (n & 4) {
      lo = hi;
      hi = 0;
    }
    const int bits = 16 * (n & 3);
    lo = lo >> bits | (hi << 1) << (63 - bits);
    hi >>= bits;
    w[0] = (unsigned)lo;
    w[1] = (unsigned)(lo >> 32);
    w[2] = (unsigned)hi;
    w[3] = (unsigned)(hi >> 32);
  } else {
#pragma unroll
    for (int by = 4; by; by >>= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = n & by ? (i + by < 8 ? w[i + by] : 0u) : w[i];
  }
}

// Eight columns of a row, zero past the array's end (col may lie past it altogether).
template <int DTYPE>
__device__ inline void load_piece(unsigned* w, const Strided& a, const unsigned char* row, int col, bool live) {
  typedef Num<DTYPE> M;
  constexpr int W = M::kPieceWords;
  if (live && a.vec && col < a.d) {  // (d is a multiple of 8 then)
#pragma unroll
    for (int i = 0; i < W; i += 4) *(u32x4*)(w + i) = *(const u32x4*)(row + (size_t)col * M::kBytes + 4 * i);
    return;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = 0;
  if (!live || a.vec || col >= a.d) return;
  if (a.d >= 8) {
    // any alignment; a piece that ends past the row is the row's last eight numbers, moved down
    const int back = max(col + 8 - a.d, 0);
    __builtin_memcpy(w, row + (int64_t)(col - back) * M::kBytes, 8 * M::kBytes);
    move_down<DTYPE>(w, back);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (col + i >= a.d) continue;
    if constexpr (DTYPE == SF_DTYPE_BF16)
      w[i / 2] |= (unsigned)*(const uint16_t*)(row + (size_t)(col + i) * 2) << (16 * (i & 1));
    else
      w[i] = *(const unsigned*)(row + (size_t)(col + i) * 4);
  }
}

// NaN if any of the numbers is NaN or infinite
template <int DTYPE>
__device__ inline float finite_test(const unsigned* w, float acc) {
#pragma unroll
  for (int i = 0; i < Num<DTYPE>::kPieceWords; ++i) {
    if constexpr (DTYPE == SF_DTYPE_BF16) {
      acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), __builtin_bit_cast(bf16x2, 0u), acc, false);
    } else {
      acc = fmaf(__builtin_bit_cast(float, w[i]), 0.0f, acc);
    }
  }
  return acc;
}

}  // namespace

}  // namespace sf
