// What the kernels of the gated delta rule share: their arguments, and what the steps of a chunk make of each other (device code; the
// mathematics is in k_delta.hip).
#pragma once

#include <type_traits>

#include "sf_chunk.h"
#include "sf_memory.h"

namespace sf {

struct DeltaArgs {
  Strided q, k, v, d_o;
  const float *log_decay, *beta;  // [T][N][H]
  const uint8_t* done;            // or null
  void* o;
  const float* s_in;              // state0 (backwards: dstate), or null
  float* s_out;                   // state (backwards: dstate0), or null
  float* kept;                    // [N * H][chunks] the states that enter each chunk (backwards: the R's), or null
  // gradients
  const float* kept_s;            // chunk c of (row, head) bh: state bh * chunks + c; null: state0, or none
  const float* kept_r;
  void *dq, *dk, *dv;
  float *dlog_decay, *dbeta;
  float* dstate0;                 // of one chunk, or null
  int f32;                        // dq and dk are fp32 whatever the arrays are (partial sums of shared heads)
  float* made;                    // [N * H][chunks] what the chunks' steps make of each other (made_words() each), or null
  // pieces of T, of whole chunks
  int n_seg, seg_len, piece;      // piece: the pieces' own states are what is made
  float* seg_state;               // [N * H][n_seg][dk * dv] first the pieces' own states, then what enters them
  float* seg_through;             // [N * H][n_seg] what a piece makes of the state that enters it, dk x dk by tiles (backwards: and its transpose)
  int* seg_begin;                 // [N * H][n_seg] an episode begins in the piece
  int T, N, H, chunks, back;
  int blocks_v, blocks;           // workgroups of a (row, head): for v's columns; and for the identity's besides
  float scale;
  Divisor heads, share, rows, round;  // H; heads that share one of q and k; N * H; 8 blocks
};

// All chunks' gradients, from the states and matrices that are made (k_delta_grad.hip).
hipError_t delta_gradients(const sf_deltarule_config* c, const DeltaArgs& g, hipStream_t st);

namespace {

constexpr int C = 32;    // steps of a chunk
constexpr int kMostHeads = 1 << 21;  // (row, head)s of a call
constexpr int DV = 64;   // columns of v of a workgroup that goes over the chunks: 16 a wave
constexpr int kMat = 36; // a row of a matrix of the chunk's steps, in fp32: 32 and 4, so that 16 rows' pieces lie in different banks
// A decay that is zero in 32 bits begins the memory anew, as done does.
constexpr double kLeastLog2 = -126.0;

typedef Num<SF_DTYPE_FP32> F32;

// Memory is read and written through buffers that begin at a uniform address: what differs from lane to lane is an offset, what is not
// there has an offset past the end (it is read as zero, not written).  A branch around a load would wait for the loads before it.
constexpr unsigned kOutside = 0x80000000u, kWholeBuffer = 0x7FFFFFFFu;
__device__ inline __amdgpu_buffer_rsrc_t buffer(const void* p, unsigned bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000); }
template <int WORDS>
__device__ inline void load_words(unsigned* w, __amdgpu_buffer_rsrc_t from, unsigned at) {
#pragma unroll
  for (int i = 0; i < WORDS; i += 4) *(u32x4*)(w + i) = __builtin_amdgcn_raw_buffer_load_b128(from, at + 4 * i, 0, 0);
}
__device__ inline float load_float(__amdgpu_buffer_rsrc_t from, unsigned at, int more) {
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, at, more, 0));
}

// Eight fp32 numbers as three bf16 terms, which are the numbers: each the leading 16 bits of what the ones before leave, or, where the first two are
// used by themselves (NEAREST; Num's out_terms alike), the nearest bf16 number to that.  Two such leave 2^-17 of the number, and the product
// of two second terms, which mma_oo leaves out, is 2^-16 of the whole one at most; of leading bits that would be 2^-15 and 2^-14, always towards zero.
// (Leading bits throughout: 512 steps of 64 rows, 8 heads of 128, 146 us, so 148; nearest numbers throughout: 16384 steps of one row 220 us, so
// 213, gradients of 1024 steps of 8 rows 338 and 331.)
__device__ inline unsigned high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
}
__device__ inline float behind(float a) { return a - __builtin_bit_cast(float, __builtin_bit_cast(unsigned, a) & 0xFFFF0000u); }
template <int DTYPE, bool NEAREST = false>
__device__ inline typename Num<DTYPE>::Sum three_terms(const float* x) {
  if constexpr (DTYPE == SF_DTYPE_BF16) {
    const auto term = [](float a, float b) { return NEAREST ? pack_bf16(a, b) : high_halves(a, b); };
    typename Num<DTYPE>::Sum o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = x[2 * i], b = x[2 * i + 1];
      o.t[0][i] = term(a, b);
      if constexpr (NEAREST) {
        a -= lo_of(o.t[0][i]);
        b -= hi_of(o.t[0][i]);
      } else {
        a = behind(a);
        b = behind(b);
      }
      o.t[1][i] = term(a, b);
      if constexpr (NEAREST) {
        a -= lo_of(o.t[1][i]);
        b -= hi_of(o.t[1][i]);
      } else {
        a = behind(a);
        b = behind(b);
      }
      o.t[2][i] = high_halves(a, b);  // (at most 8 bits are left)
    }
    return o;
  } else {
    return Num<DTYPE>::sum_terms(x);
  }
}

// Four K-slots of two fp32 operands.
__device__ inline f32x4 mm4(const f32x4 a, const f32x4 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}
template <int DTYPE>
__device__ inline f32x4 mma_oo(const typename Num<DTYPE>::Out& a, const typename Num<DTYPE>::Out& b, f32x4 c) {
  typedef Num<DTYPE> M;
  if constexpr (DTYPE == SF_DTYPE_BF16) return M::mma1(a.t[0], b.t[0], M::mma1(a.t[0], b.t[1], M::mma1(a.t[1], b.t[0], c)));
  else return M::mma(a, b, c);
}
template <int DTYPE>
__device__ inline typename Num<DTYPE>::Out leading(const typename Num<DTYPE>::Sum& s) {
  if constexpr (DTYPE == SF_DTYPE_BF16) return typename Num<DTYPE>::Out{{s.t[0], s.t[1]}};
  else return s;
}

// A lane's number from the lane N behind it in its row of 16 (0 where there is none).
template <int N>
__device__ inline float row_left(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x100 + N, 0xF, 0xF, true));
}
// Sum over the 16 lanes of a row (each lane gets it).
__device__ inline float row_sum(float x) {
#define SF_ROR(n) x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + (n), 0xF, 0xF, true))
  SF_ROR(8);
  SF_ROR(4);
  SF_ROR(2);
  SF_ROR(1);
#undef SF_ROR
  return x;
}
__device__ inline float wave_sum(float x) {
  x = row_sum(x);
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// What the chunk's steps have of their own.
struct Steps {
  float gh[C], gl[C];  // G in binary logarithms, as two numbers
  float enter[C];      // E
  float leave[C];      // W
  float beta[C];
  int ep[C];           // episode of the step, counted in the chunk; steps that are not there have their own, which is nobody else's
};
constexpr int kStepWords = sizeof(Steps) / 4;
// A chunk's matrices [32][32] and Steps, where a launch leaves them for others: T, P (backwards P^T and A^T), Steps.
constexpr int kDense = C * C;
__host__ __device__ constexpr int made_words(bool back) { return (back ? 3 : 2) * kDense + kStepWords; }

struct StepIn {
  float ld, beta;
  bool done;
};
// Lane i < 32 reads step t0 + i.
__device__ inline StepIn read_step(const DeltaArgs& g, int n, int h, int t0, int valid, int lane) {
  static_assert((int64_t)(C - 1) * kMostHeads * 4 < kWholeBuffer, "a chunk's steps are in reach of one buffer");
  const int64_t row = (int64_t)t0 * g.N + n;
  const unsigned at = (unsigned)(lane * g.N);
  const auto ld = buffer(g.log_decay + row * g.H + h, kWholeBuffer), be = buffer(g.beta + row * g.H + h, kWholeBuffer);
  const auto dn = buffer(g.done + (g.done ? row : 0), g.done ? kWholeBuffer : 0);
  StepIn s;
  s.ld = load_float(ld, lane < valid ? at * g.H * 4 : kOutside, 0);
  s.beta = load_float(be, lane < valid ? at * g.H * 4 : kOutside, 0);
  s.done = __builtin_amdgcn_raw_buffer_load_b8(dn, lane < valid ? at : kOutside, 0, 0) != 0;
  return s;
}
__device__ inline bool begins(const StepIn& s) { return s.done || s.ld * 1.44269504f < (float)kLeastLog2; }

// A lane's number from the lane n before it in its row of 16 (0 where there is none).
template <int N>
__device__ inline double row_shift(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, 0x110 + N, 0xF, 0xF, true), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), 0x110 + N, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)(unsigned)hi << 32 | (unsigned)lo);
}

// One wave: the arrays of Steps from the lanes' steps (all lanes call it; those from 32 on do as those before).
__device__ inline void put_steps(Steps& s, const StepIn& in, unsigned marks, int valid, int lane) {
  const int i = lane & (C - 1);
  const unsigned upto = (2u << i) - 1;
  const int e = __popc(marks & upto);
  // the sum since the episode's begin in the chunk: a lane adds what the one d before it has, if no episode begins behind that one
  double G = lane >= C || begins(in) || i >= valid ? 0.0 : (double)in.ld * 1.4426950408889634;
  const int reach = i - (31 - __clz((int)((marks & upto) | 1u)));  // steps since the last begin, or the chunk's
  double b = row_shift<1>(G);
  G += reach >= 1 ? b : 0.0;
  b = row_shift<2>(G);
  G += reach >= 2 ? b : 0.0;
  b = row_shift<4>(G);
  G += reach >= 4 ? b : 0.0;
  b = row_shift<8>(G);
  G += reach >= 8 ? b : 0.0;
  b = __shfl(G, 15);
  G += i >= 16 && reach >= i - 15 ? b : 0.0;
  const double last = __shfl(G, valid - 1);
  const int e_last = __popc(marks);
  if (lane < C) {
    const float hi = (float)G;
    s.gh[i] = hi;
    s.gl[i] = (float)(G - (double)hi);
    s.enter[i] = i < valid && e == 0 ? pow2((float)G) : 0.0f;
    s.leave[i] = i < valid && e == e_last ? pow2((float)(last - G)) : 0.0f;
    s.beta[i] = in.beta;
    s.ep[i] = i < valid ? e : C + i;
  }
}
// D of steps i >= j of one episode
__device__ inline float decay_of(float ghi, float gli, float ghj, float glj) { return pow2((ghi - ghj) + (gli - glj)); }

// Eight K-slots of a row of a step matrix: steps 4 lg .. and 16 + 4 lg ..
struct Slots {
  f32x4 a, b;
};
__device__ inline Slots slots_of(const float* m, int row, int lg) {
  return Slots{*(const f32x4*)(m + row * kMat + 4 * lg), *(const f32x4*)(m + row * kMat + 16 + 4 * lg)};
}
// The same of a column.
__device__ inline Slots slots_down(const float* m, int column, int lg) {
  Slots s;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    s.a[r] = m[(4 * lg + r) * kMat + column];
    s.b[r] = m[(16 + 4 * lg + r) * kMat + column];
  }
  return s;
}
// Between what lanes of a wave write to LDS and what others of it read.
__device__ inline void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wave: T = (1 + A beta)^-1 [i][j] from A^T [j][i].  The block above the diagonal is not written.
// A row of 16 lanes has a block of 16, a lane one column of A (times its beta) and one of T; what all lanes need of A comes from its
// lane by a broadcast within the row, so that nothing is read in between.
__device__ inline void invert(const float* at, const float* beta, float* T, int lane) {
  const int li = lane & 15, lg = lane >> 4, b0 = lane & 16;  // (rows 2 and 3 of the wave do as 0 and 1)
  float a[16], t[16];
  {
    const float b = -beta[b0 + li];
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const f32x4 x = *(const f32x4*)(at + (b0 + li) * kMat + b0 + i);
#pragma unroll
      for (int r = 0; r < 4; ++r) a[i + r] = b * x[r];
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) t[i] = i == li ? 1.0f : 0.0f;
  auto step = [&](auto at_l) {
    constexpr int l = decltype(at_l)::value;
#pragma unroll
    for (int i = l + 1; i < 16; ++i)
      t[i] = fmaf(__builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a[i]), 0x150 + l, 0xF, 0xF, true)), t[l], t[i]);
#pragma unroll
    for (int i = l + 1; i < 16; ++i) asm volatile("" : "+v"(a[i]), "+v"(t[i]));  // (else the broadcasts of all steps come first, in 120 registers)
  };
#define SF_STEP(l) step(std::integral_constant<int, l>())
  SF_STEP(0); SF_STEP(1); SF_STEP(2); SF_STEP(3); SF_STEP(4); SF_STEP(5); SF_STEP(6); SF_STEP(7);
  SF_STEP(8); SF_STEP(9); SF_STEP(10); SF_STEP(11); SF_STEP(12); SF_STEP(13); SF_STEP(14);
#undef SF_STEP
  if (lane < 32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) T[(b0 + i) * kMat + b0 + li] = t[i];
  }
  wave_order();
  // the lower left block: -T22 A21 beta T11
  f32x4 a21, bt, zero = {0.0f, 0.0f, 0.0f, 0.0f};
  const f32x4 be = *(const f32x4*)(beta + 4 * lg);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    a21[r] = at[(4 * lg + r) * kMat + 16 + li];
    bt[r] = be[r] * T[(4 * lg + r) * kMat + li];
  }
  const f32x4 z = mm4(a21, bt, zero);
  const f32x4 t21 = mm4(*(const f32x4*)(T + (16 + li) * kMat + 16 + 4 * lg), z, zero);
#pragma unroll
  for (int r = 0; r < 4; ++r) T[(16 + 4 * lg + r) * kMat + li] = -t21[r];
}

// A tile of products of steps with D and the mask: its rows are steps 16 rows + 4 lg + r, its columns 16 columns + li; rows_later: a row is
// the later step of the two; strict: not the step with itself.
__device__ inline f32x4 decayed(const Steps& steps, f32x4 x, int rows, int columns, bool rows_later, bool strict, float scale, int li, int lg) {
  const int c = 16 * columns + li, ec = steps.ep[c];
  const float hc = steps.gh[c], lc = steps.gl[c];
  const f32x4 h4 = *(const f32x4*)(steps.gh + 16 * rows + 4 * lg), l4 = *(const f32x4*)(steps.gl + 16 * rows + 4 * lg);
  const i32x4 e4 = *(const i32x4*)(steps.ep + 16 * rows + 4 * lg);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int later = rows_later ? 16 * rows + 4 * lg + r - c : c - (16 * rows + 4 * lg + r);
    const float d = rows_later ? decay_of(h4[r], l4[r], hc, lc) : decay_of(hc, lc, h4[r], l4[r]);
    x[r] = later >= (strict ? 1 : 0) && e4[r] == ec ? x[r] * (scale * d) : 0.0f;
  }
  return x;
}

// One wave: a chunk's Steps, A^T and P (backwards P^T, without the scale) into LDS (pitch kMat).  Keys and queries are read as operands.
template <int DTYPE, int D, bool BACK, bool VEC>
__device__ inline void make_products(const DeltaArgs& g, int n, int h, int hk, int t0, int valid, int lane, Steps& steps, float* mA, float* mP) {
  typedef Num<DTYPE> M;
  const int li = lane & 15, lg = lane >> 4, dk = g.k.d;
  auto base = [&](const Strided& a) { return (const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes; };
  const unsigned char *const qb = base(g.q), *const kb = base(g.k);
  typename M::Raw q[2][D / 32], k[2][D / 32];
  const auto from_q = buffer(qb + (int64_t)t0 * g.q.st * M::kBytes, kWholeBuffer), from_k = buffer(kb + (int64_t)t0 * g.k.st * M::kBytes, kWholeBuffer);
#pragma unroll
  for (int I = 0; I < 2; ++I) {
    const int r = 16 * I + li;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const int col = 32 * s + 8 * lg;
      unsigned w[M::kPieceWords];
      if constexpr (VEC) {
        const bool there = r < valid && col < dk;
        load_words<M::kPieceWords>(w, from_k, there ? (unsigned)(r * (int)g.k.st + col) * M::kBytes : kOutside);
        __builtin_memcpy(&k[I][s], w, sizeof w);
        load_words<M::kPieceWords>(w, from_q, there ? (unsigned)(r * (int)g.q.st + col) * M::kBytes : kOutside);
      } else {
        const int64_t t = t0 + (r < valid ? r : 0);
        load_piece<DTYPE>(w, g.k, kb + t * g.k.st * M::kBytes, col, r < valid);
        __builtin_memcpy(&k[I][s], w, sizeof w);
        load_piece<DTYPE>(w, g.q, qb + t * g.q.st * M::kBytes, col, r < valid);
      }
      __builtin_memcpy(&q[I][s], w, sizeof w);
    }
  }
  const StepIn in = read_step(g, n, h, t0, valid, lane);
  const unsigned marks = (unsigned)__ballot(begins(in));
  put_steps(steps, in, marks, valid, lane);
  wave_order();
#pragma unroll
  for (int I = 0; I < 2; ++I)
#pragma unroll
    for (int J = 0; J < 2; ++J) {
      f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, p = a;
      if (J <= I) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
          if (32 * s >= dk) continue;
          a = M::mma(k[I][s], k[J][s], a);                                           // [i][j]
          p = BACK ? M::mma(q[I][s], k[J][s], p) : M::mma(k[J][s], q[I][s], p);  // [i][j], forwards [j][i]
        }
        a = decayed(steps, a, I, J, true, true, 1.0f, li, lg);
        p = BACK ? decayed(steps, p, I, J, true, false, 1.0f, li, lg) : decayed(steps, p, J, I, false, false, g.scale, li, lg);
      }
      *(f32x4*)(mA + (16 * J + li) * kMat + 16 * I + 4 * lg) = a;                // A^T [j][i]
      if (BACK) *(f32x4*)(mP + (16 * J + li) * kMat + 16 * I + 4 * lg) = p;      // P^T [j][i]
      else *(f32x4*)(mP + (16 * I + li) * kMat + 16 * J + 4 * lg) = p;           // P [i][j]
    }
  wave_order();
}

template <int DTYPE, int D>
struct Pitch {
  // of a row: 4 times an odd number of words, so that 16 rows' pieces of 16 bytes lie in different banks; of those 36 and 12
  // mod 64 also keep the transposing read's four rows of 32 bytes apart
  static constexpr int value = D * Num<DTYPE>::kBytes + (Num<DTYPE>::kBytes == 2 && D == 128 ? 48 : 16);
};

// Columns c0 + li of an array in LDS, K-slots its steps.
template <int DTYPE>
__device__ inline typename Num<DTYPE>::Raw columns(const unsigned char* tile, int pitch, int c0, int c_step, int li, int lg) {
  typedef Num<DTYPE> M;
  typename M::Raw r;
  if constexpr (DTYPE == SF_DTYPE_BF16) {
    const unsigned char* at = tile + (4 * lg + (li >> 2)) * pitch + (c0 + c_step * (li & 3)) * M::kBytes;
    const u32x2 x = M::column4(at), y = M::column4(at + 16 * pitch);
    r = u32x4{x[0], x[1], y[0], y[1]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      r.x[j] = M::element(tile + (4 * lg + (j & 3) + 16 * (j >> 2)) * pitch + (c0 + c_step * (li >> 2) + (li & 3)) * M::kBytes);
  }
  return r;
}

// One piece of a tile for thread `piece`.
template <int DTYPE>
__device__ inline void fetch(unsigned* w, const Strided& a, const unsigned char* base, int t0, int valid, int piece, int per_row, int c0) {
  const int r = piece / per_row, col = c0 + piece % per_row * 8;
  const bool live = r < valid;
  load_piece<DTYPE>(w, a, base + (int64_t)(live ? t0 + r : t0) * a.st * Num<DTYPE>::kBytes, col, live);
}
template <int DTYPE>
__device__ inline void put_piece(unsigned char* tile, int pitch, const unsigned* w, int piece, int per_row) {
  unsigned char* const at = tile + piece / per_row * pitch + piece % per_row * 8 * Num<DTYPE>::kBytes;
#pragma unroll
  for (int i = 0; i < Num<DTYPE>::kPieceWords; i += 4) *(u32x4*)(at + 4 * i) = *(const u32x4*)(w + i);
}

// How much of a call is known at compile time: kAny; kPieces: all rows are read and written in 16-byte pieces; kWhole: there are whole
// tiles besides, D columns of k and a multiple of 64 of v (else columns past theirs are left out, 32 of k, 16 of v at a time).
enum Known { kAny = 0, kPieces = 1, kWhole = 2 };

}  // namespace

}  // namespace sf
