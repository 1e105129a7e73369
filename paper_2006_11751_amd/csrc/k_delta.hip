// The gated delta rule (include/sf_memory.h), in chunks of C = 32 steps.  With G_i the sum of the logarithms of the decays up to
// step i of the chunk, D_ij = exp(G_i - G_j) for steps of one episode, E_i = exp(G_i) where no episode begins up to i, S the state that
// enters, and W_j = exp(G_last - G_j) where none begins behind j:
//   P_ij = D_ij (q_i . k_j), j <= i      A_ij = D_ij (k_i . k_j), j < i
//   e = (1 + A beta)^-1 (v - E k S)      u = beta e
//   o = scale (E q S + P u)              S <- exp(G_last) S + k^T W u
// so the steps' corrections e, each of which needs the one before, are one triangular system a chunk whose matrix does not depend on the
// state.  Its inverse T is made by substitution: blocks of 16 in registers, a lane for each column, joined by two products.
// (Substitution keeps the errors of a step to that step; powers of A would be larger than their sum where keys are alike.)
// Gradients, with R that of the state behind the chunk:
//   f = scale P^T do + W k R (of u)      z = T^T beta f (of v)        g = f - A^T z (of u, through later steps too)
//   dP = scale do u^T, dA = -z u^T       dbeta_i = g_i . e_i          R <- exp(G_last) R + scale q^T E do - k^T E z
//   dq = scale E do S^T + (dP D) k       dk = (dP D)^T q + (dA D + (dA D)^T) k - E z S^T + W u R^T
// and a step's decay has the sum over the later steps of its episode of  dP P + dA A (its row less its column), what the
// state gives it and what it gives the state.
// The backward pass goes over the chunks forwards for the states that enter them, backwards for the R's, and then makes all chunks'
// gradients at once (of at most 32 steps there is only this last part).
//
// Roundings.  What bf16 arrays hold enters the products as it is; fp32 numbers enter as sums of bf16 numbers: three terms (nothing is
// left out) where the result is fp32 or a state, two (2^-16 is left out) where it is rounded to bf16.  Products of two fp32 matrices
// (T, A and what they multiply) and all of fp32 arrays run on the fp32 matrix instruction.  G is summed in 64 bits
// and kept as two fp32 numbers, so that differences of steps close to each other do not lose to what came before.
//
// Zeros of masks are selected, but a product still multiplies them with the other operand's rows, and 0 x NaN is NaN.  So what enters
// a chunk is tested: one with a NaN or an infinity is taken again as chunks of one step (the gradients': number by number).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "sf_chunk.h"
#include "sf_internal.h"
#include "sf_memory.h"

namespace sf {

namespace {

constexpr int C = 32;    // steps of a chunk
constexpr int DV = 64;   // columns of v of a workgroup that goes over the chunks: 16 a wave
constexpr int kMat = 36; // a row of a matrix of the chunk's steps, in fp32: 32 and 4, so that 16 rows' pieces lie in different banks
// A decay that is zero in 32 bits begins the memory anew, as done does.
constexpr double kLeastLog2 = -126.0;

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
  float* seg_through;             // [N * H][n_seg][dk * dk] what a piece makes of the state that enters it
  int* seg_begin;                 // [N * H][n_seg] an episode begins in the piece
  int T, N, H, chunks, back;
  int blocks_v, blocks;           // workgroups of 64 columns of v; and of the identity besides
  float scale;
  Divisor heads, share, rows, round;  // H, heads that share one of q and k, N * H, 8 blocks
};

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
  const int64_t row = (int64_t)t0 * g.N + n;
  const int64_t last = (int64_t)(valid - 1) * g.N;  // (rows may lie far apart)
  StepIn s;
  if (last * g.H < (int64_t)1 << 28) {
    const unsigned at = (unsigned)(lane * g.N);
    const auto ld = buffer(g.log_decay + row * g.H + h, kWholeBuffer), be = buffer(g.beta + row * g.H + h, kWholeBuffer);
    const auto dn = buffer(g.done + (g.done ? row : 0), g.done ? kWholeBuffer : 0);
    s.ld = load_float(ld, lane < valid ? at * g.H * 4 : kOutside, 0);
    s.beta = load_float(be, lane < valid ? at * g.H * 4 : kOutside, 0);
    s.done = __builtin_amdgcn_raw_buffer_load_b8(dn, lane < valid ? at : kOutside, 0, 0) != 0;
  } else {
    const int64_t r = row + (int64_t)(lane < valid ? lane : 0) * g.N, at = r * g.H + h;
    s.ld = lane < valid ? g.log_decay[at] : 0.0f;
    s.beta = lane < valid ? g.beta[at] : 0.0f;
    s.done = lane < valid && g.done && g.done[r] != 0;
  }
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
        // rows are steps 16 R + 4 lg + r of tile R, columns are steps of the other one
        auto decayed = [&](f32x4 x, int rows, int columns, bool rows_later, bool strict, float scale) {
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
        };
        a = decayed(a, I, J, true, true, 1.0f);
        p = BACK ? decayed(p, I, J, true, false, 1.0f) : decayed(p, J, I, false, false, g.scale);
      }
      *(f32x4*)(mA + (16 * J + li) * kMat + 16 * I + 4 * lg) = a;                // A^T [j][i]
      if (BACK) *(f32x4*)(mP + (16 * J + li) * kMat + 16 * I + 4 * lg) = p;      // P^T [j][i]
      else *(f32x4*)(mP + (16 * I + li) * kMat + 16 * J + 4 * lg) = p;           // P [i][j]
    }
  wave_order();
}
// And T.
template <int DTYPE, int D, bool BACK, bool VEC>
__device__ inline void make_chunk(const DeltaArgs& g, int n, int h, int hk, int t0, int valid, int lane, Steps& steps, float* mA, float* mP, float* mT) {
  make_products<DTYPE, D, BACK, VEC>(g, n, h, hk, t0, valid, lane, steps, mA, mP);
  invert(mA, steps.beta, mT, lane);
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

template <int DTYPE, int D>
struct SweepLds {
  static constexpr int kPitch = Pitch<DTYPE, D>::value, kPitchV = Pitch<DTYPE, DV>::value;
  static constexpr int kK = C * kPitch, kV = 2 * C * kPitch, kP = kV + C * kPitchV, kT = kP + C * kMat * 4, kSteps = kT + C * kMat * 4,
                       kFlag = kSteps + (int)sizeof(Steps), kA = kFlag + 16, kBytes = kA, kBytesAlone = kA + C * kMat * 4;
};

// The matrices of every chunk, for the sweeps and the gradients: a wave makes one chunk's.
template <int DTYPE, int D, bool BACK, bool VEC>
__global__ __launch_bounds__(kThreads) void delta_chunks_kernel(DeltaArgs g) {
  constexpr int kWave = 2 * C * kMat * 4 + (int)sizeof(Steps);  // (T takes the place of P when that has left)
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned at = blockIdx.x * 4 + wave;
  if (at >= (unsigned)g.N * g.H * g.chunks) return;
  const int chunk = (int)g.rows.of(at), bh = (int)(at - (unsigned)chunk * (g.N * g.H));
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h), t0 = chunk * C, valid = min(C, g.T - t0);
  float *const mA = (float*)(lds + wave * kWave), *const mP = mA + C * kMat;
  Steps& steps = *(Steps*)(mP + C * kMat);
  float* const out = g.made + ((size_t)bh * g.chunks + chunk) * made_words(BACK);
  auto store = [&](float* to, const float* from) {
#pragma unroll
    for (int i = 0; i < kDense / 256; ++i) {
      const int e = (i * 64 + lane) * 4;
      *(f32x4*)(to + e) = *(const f32x4*)(from + e / C * kMat + e % C);
    }
  };
  make_products<DTYPE, D, BACK, VEC>(g, n, h, hk, t0, valid, lane, steps, mA, mP);
  store(out + kDense, mP);
  wave_order();
  invert(mA, steps.beta, mP, lane);
  wave_order();
  store(out, mP);
  if (BACK) store(out + 2 * kDense, mA);
  if (lane < kStepWords / 4) *(f32x4*)(out + (BACK ? 3 : 2) * kDense + 4 * lane) = *(const f32x4*)((const float*)&steps + 4 * lane);
}

enum Sweep { kResults = 0, kStates = 1, kBack = 2 };
// How much of a call is known at compile time: kAny; kPieces: all rows are read and written in 16-byte pieces; kWhole: there are whole
// tiles besides, D columns of k and a multiple of 64 of v (else columns past theirs are left out, 32 of k, 16 of v at a time).
enum Known { kAny = 0, kPieces = 1, kWhole = 2 };

// A workgroup of four waves goes over the chunks of one (row, head), or of one piece of T, for 64 columns of v, of which a wave owns 16: its part of
// the state stays in registers as the accumulator of the update.  The products are arranged so that accumulators feed the next
// product without a shuffle: a 16x16 accumulator holds rows 4 lg .. 4 lg + 3 of one column per lane (lg = lane / 16), two of them are
// the eight K-slots of an operand of 16x16x32, and the other operand follows the same numbering of the K axis.
//   kResults: o and the last state;  kStates: the states that enter the chunks, or the last one of a piece;  kBack: R, from the last chunk to the first
// ALONE: of one chunk, whose matrices the first wave makes (else they are read).
template <int DTYPE, int D, int SWEEP, bool ALONE, int KNOWN>
__global__ __launch_bounds__(kThreads, KNOWN != kAny ? (D == 64 ? 4 : 3) : 2) void delta_sweep_kernel(DeltaArgs g) {
  typedef Num<DTYPE> M;
  typedef SweepLds<DTYPE, D> L;
  constexpr int W = M::kPieceWords, NP = C * D / 8 / kThreads, ND = D / 16, kRow = D / 8, kRowV = DV / 8;
  constexpr bool kQ = SWEEP != kStates, kUp = SWEEP != kBack, VEC = KNOWN != kAny, WHOLE = KNOWN == kWhole;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  // the blocks of one (row, head) read the same arrays: one after another on one XCD (workgroups go to the 8 in turn)
  const unsigned round = g.round.of(blockIdx.x), in_round = blockIdx.x - round * (8 * g.blocks), turn8 = in_round >> 3;
  const int bh = (int)(round * 8 + (in_round & 7));
  if (bh >= g.N * g.H) return;
  // a piece has blocks of the identity's columns besides: what a state that enters becomes
  const bool identity = (int)turn8 >= g.blocks_v;
  const int v_block = DV * ((int)turn8 - (identity ? g.blocks_v : 0)), seg = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h);
  const int dk = WHOLE ? D : g.k.d, dv = identity ? dk : g.v.d;
  const int t_begin = seg * g.seg_len, t_end = min(g.T, t_begin + g.seg_len);
  auto base = [&](const Strided& a) { return (const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes; };
  const Strided third = SWEEP == kBack ? g.d_o : g.v;
  const unsigned char *const qb = base(g.q), *const kb = base(g.k), *const vb = base(third);
  unsigned char *const tq = lds, *const tk = lds + L::kK, *const tv = lds + L::kV;
  float *const mP = (float*)(lds + L::kP), *const mT = (float*)(lds + L::kT);
  Steps& steps = *(Steps*)(lds + L::kSteps);
  int* const flag = (int*)(lds + L::kFlag);

  if (tid < 2) flag[tid] = 0;
  if constexpr (ALONE) {
    __syncthreads();
    if (wave == 0) make_chunk<DTYPE, D, SWEEP == kBack, VEC>(g, n, h, hk, 0, g.T, lane, steps, (float*)(lds + L::kA), mP, mT);
  }

  const int v0 = v_block + 16 * wave, y = v0 + li;  // this wave's columns of v, this lane's
  const bool has_v = WHOLE || v0 < dv;
  auto has_k = [&](int s) { return WHOLE || 32 * s < dk; };
  // row of tile t of the state (two tiles are 32 rows: eight neighbours per lane group)
  auto col_k = [&](int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); };
  f32x4 S[ND];
  const unsigned y_at = WHOLE || y < dv ? (unsigned)(8 * lg * dv + y) * 4 : kOutside;  // (rows past dk lie past the end)
  {
    const float* s = nullptr;
    if (g.piece) s = nullptr;
    else if (g.n_seg > 1) s = g.seg_state + ((size_t)bh * g.n_seg + seg) * dk * dv;
    else if (g.s_in) s = g.s_in + (size_t)bh * dk * dv;
    const auto from = buffer(s, s ? (unsigned)(dk * dv) * 4 : 0);
#pragma unroll
    for (int a = 0; a < ND; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        S[a][r] = load_float(from, y_at, (32 * (a >> 1) + 4 * (a & 1) + r) * dv * 4);
        if (identity) S[a][r] = col_k(a, 4 * lg + r) == y ? 1.0f : 0.0f;
      }
  }
  auto store_state = [&](float* s) {
    int row = dv * 4;
    asm volatile("" : "+s"(row));  // (else the rows' offsets are kept in registers from here to there)
    const auto to = buffer(s, (unsigned)(dk * dv) * 4);
#pragma unroll
    for (int a = 0; a < ND; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)S[a][r]), to, y_at, (32 * (a >> 1) + 4 * (a & 1) + r) * row, 0);
  };

  // the chunk that is on its way: its rows, matrices and steps
  unsigned nq[NP][W], nk[NP][W], nv[W];
  f32x4 n_p, n_t, n_steps;
  unsigned at_q[NP], at_k[NP], at_v = kOutside;
  if constexpr (VEC) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int piece = tid + p * kThreads, r = piece / kRow, col = piece % kRow * 8;
      at_q[p] = WHOLE || col < dk ? (unsigned)(r * (int)g.q.st + col) * M::kBytes : kOutside;
      at_k[p] = WHOLE || col < dk ? (unsigned)(r * (int)g.k.st + col) * M::kBytes : kOutside;
    }
    const int col = v_block + tid % kRowV * 8;
    if ((WHOLE || col < third.d) && !identity) at_v = (unsigned)(tid / kRowV * (int)third.st + col) * M::kBytes;
  }
  const float* const made = g.made + (size_t)bh * g.chunks * made_words(!kUp || g.back);
  auto request = [&](int c) {
    const int t0 = c * C, valid = min(C, g.T - t0);
    if constexpr (VEC) {
      auto get = [&](unsigned* w, const Strided& a, const unsigned char* row, int r, unsigned at) {
        const auto from = buffer(row + (int64_t)t0 * a.st * M::kBytes, kWholeBuffer);
        load_words<W>(w, from, r < valid ? at : kOutside);
      };
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if constexpr (kQ) get(nq[p], g.q, qb, (tid + p * kThreads) / kRow, at_q[p]);
        get(nk[p], g.k, kb, (tid + p * kThreads) / kRow, at_k[p]);
      }
      get(nv, third, vb, tid / kRowV, at_v);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if constexpr (kQ) fetch<DTYPE>(nq[p], g.q, qb, t0, valid, tid + p * kThreads, kRow, 0);
        fetch<DTYPE>(nk[p], g.k, kb, t0, valid, tid + p * kThreads, kRow, 0);
      }
      fetch<DTYPE>(nv, third, vb, t0, identity ? 0 : valid, tid, kRowV, v_block);
    }
    if constexpr (!ALONE) {
      const float* const m = made + (size_t)c * made_words(!kUp || g.back);
      n_t = *(const f32x4*)(m + 4 * tid);
      if constexpr (kQ) n_p = *(const f32x4*)(m + kDense + 4 * tid);
      if (tid < kStepWords / 4) n_steps = *(const f32x4*)(m + (!kUp || g.back ? 3 : 2) * kDense + 4 * tid);
    }
  };
  unsigned at_o[2];  // of four neighbours of an output row
#pragma unroll
  for (int I = 0; I < 2; ++I) at_o[I] = WHOLE || v0 + 4 * lg < dv ? (unsigned)((16 * I + li) * (g.N * g.H * dv) + v0 + 4 * lg) * M::kBytes : kOutside;

  const int first = t_begin / C, last = (t_end - 1) / C;  // chunks
  if (t_begin < t_end) request(kUp ? first : last);
  bool any_begin = false;
  for (int c = kUp ? first : last, turn = 0; t_begin < t_end && (kUp ? c <= last : c >= first); c += kUp ? 1 : -1, turn ^= 1) {
    const int t0 = c * C, valid = min(C, g.T - t0);
    if (SWEEP != kResults && g.kept && has_v) store_state(g.kept + ((size_t)bh * g.chunks + c) * ((size_t)dk * dv));
    if constexpr (!ALONE) __syncthreads();  // the chunk before has been read
    float test = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if constexpr (kQ) put_piece<DTYPE>(tq, L::kPitch, nq[p], tid + p * kThreads, kRow);
      put_piece<DTYPE>(tk, L::kPitch, nk[p], tid + p * kThreads, kRow);
      if constexpr (SWEEP == kBack) test = finite_test<DTYPE>(nq[p], test);
      test = finite_test<DTYPE>(nk[p], test);
    }
    put_piece<DTYPE>(tv, L::kPitchV, nv, tid, kRowV);
    test = finite_test<DTYPE>(nv, test);
    if constexpr (!ALONE) {
      const int to = tid / 8 * kMat + tid % 8 * 4;
      *(f32x4*)(mT + to) = n_t;
      if constexpr (kQ) *(f32x4*)(mP + to) = n_p;
      if (tid < kStepWords / 4) *(f32x4*)((float*)&steps + 4 * tid) = n_steps;
    }
    if (test != 0.0f) flag[turn] = 1;
    __syncthreads();
    if (c != (kUp ? last : first)) request(kUp ? c + 1 : c - 1);
    // (marks of begins are where the episode's number grows)
    const int my_ep = steps.ep[lane & (C - 1)];
    const float my_steps = fmaf(steps.gh[lane & (C - 1)], 0.0f, steps.beta[lane & (C - 1)] * 0.0f);
    const int e_last = __builtin_amdgcn_readlane(my_ep, valid - 1);
    const bool marked = e_last != 0;
    any_begin = any_begin || marked;
    const bool odd = flag[turn] != 0 || __any(my_steps != 0.0f);
    if (tid == 0) flag[turn ^ 1] = 0;  // (read by all before the barrier above)
    if (!has_v) continue;

    // what the state gives the steps: k S, and q S
    f32x4 ks[2] = {}, qs[2] = {};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if (!has_k(s)) continue;
      float x[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = S[2 * s][r];
        x[4 + r] = S[2 * s + 1][r];
      }
      const typename M::Sum st = M::sum_terms(x);
#pragma unroll
      for (int J = 0; J < 2; ++J) {
        const int at = (16 * J + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes;
        ks[J] = M::mma(M::row(tk + at), st, ks[J]);                                               // [step][y]
        if constexpr (SWEEP == kResults) qs[J] = M::mma(leading<DTYPE>(st), M::row(tq + at), qs[J]);  // [y][step]
      }
    }
    // (of a state with something not finite every product is not finite: that an episode begins in the chunk does not stop it)
    if (odd || (marked && __any(ks[0][0] * 0.0f != 0.0f))) {
      // Step by step, each wave for its columns, so that nothing that is not finite meets a masked zero.
      auto element = [&](const unsigned char* tile, int pitch, int i, int x) { return M::element(tile + i * pitch + x * M::kBytes); };
      float s[ND][4];
#pragma unroll
      for (int a = 0; a < ND; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[a][r] = S[a][r];
      for (int at = 0; at < valid; ++at) {
        const int i = kUp ? at : valid - 1 - at;
        const StepIn in = read_step(g, n, h, t0 + i, 1, lane & 0);
        const bool begin = begins(in);
        const float keep = exp2f(in.ld * 1.44269504f), v = element(tv, L::kPitchV, i, 16 * wave + li);
        float sum = 0.0f;
#pragma unroll
        for (int a = 0; a < ND; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int x = col_k(a, 4 * lg + r);
            if (x >= dk) continue;
            if constexpr (kUp) s[a][r] = begin ? 0.0f : keep * s[a][r];
            else s[a][r] += g.scale * element(tq, L::kPitch, i, x) * v;
            sum += element(tk, L::kPitch, i, x) * s[a][r];
          }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const float u = in.beta * (kUp ? v - sum : -sum);
        float o = 0.0f;
#pragma unroll
        for (int a = 0; a < ND; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int x = col_k(a, 4 * lg + r);
            if (x >= dk) continue;
            s[a][r] += element(tk, L::kPitch, i, x) * u;
            if constexpr (SWEEP == kResults) o += element(tq, L::kPitch, i, x) * s[a][r];
            if constexpr (!kUp) s[a][r] = begin ? 0.0f : keep * s[a][r];
          }
        if constexpr (SWEEP == kResults) {
          o += __shfl_xor(o, 16);
          o += __shfl_xor(o, 32);
          if (lg == 0 && y < dv) M::store((unsigned char*)g.o + ((((int64_t)(t0 + i) * g.N + n) * g.H + h) * dv + y) * M::kBytes, g.scale * o);
        }
      }
#pragma unroll
      for (int a = 0; a < ND; ++a) S[a] = f32x4{s[a][0], s[a][1], s[a][2], s[a][3]};
      continue;
    }
    // columns of the third array: K-slots 0..3 are steps 4 lg .., 4..7 are 16 further on
    const typename M::Raw vt = columns<DTYPE>(tv, L::kPitchV, 16 * wave, 4, li, lg);
    float v[8];
    M::values(vt, v);
    f32x4 e4[2], w4[2], b4[2];
#pragma unroll
    for (int J = 0; J < 2; ++J) {
      const int j = 16 * J + 4 * lg;
      e4[J] = *(const f32x4*)(steps.enter + j);
      w4[J] = *(const f32x4*)(steps.leave + j);
      b4[J] = *(const f32x4*)(steps.beta + j);
    }
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const float keep = marked ? 0.0f : steps.enter[valid - 1];
    // (a state that is not finite is here only in a chunk that it all reaches: a factor of zero leaves out a finite number)
    if constexpr (kUp) {
      f32x4 x[2], e[2];
#pragma unroll
      for (int J = 0; J < 2; ++J)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[J][r] = v[4 * J + r] - e4[J][r] * ks[J][r];
      const Slots t1 = slots_of(mT, 16 + li, lg);
      e[0] = mm4(*(const f32x4*)(mT + li * kMat + 4 * lg), x[0], zero);
      e[1] = mm4(t1.b, x[1], mm4(t1.a, x[0], zero));
      float us[8];
#pragma unroll
      for (int J = 0; J < 2; ++J)
#pragma unroll
        for (int r = 0; r < 4; ++r) us[4 * J + r] = b4[J][r] * e[J][r];
      if constexpr (SWEEP == kResults) {
        const typename M::Out uo = M::out_terms(us);
        const auto to = buffer((unsigned char*)g.o + (((int64_t)t0 * g.N + n) * g.H + h) * dv * M::kBytes, kWholeBuffer);
#pragma unroll
        for (int I = 0; I < 2; ++I) {
          const int i = 16 * I + li;
          f32x4 own = (g.scale * steps.enter[i]) * qs[I];
          const Slots p = slots_of(mP, i, lg);
          float ps[8];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            ps[r] = p.a[r];
            ps[4 + r] = p.b[r];
          }
          own = mma_oo<DTYPE>(uo, M::out_terms(ps), own);  // [y][i]
          if constexpr (VEC) {
            const unsigned at = i < valid ? at_o[I] : kOutside;
            if constexpr (DTYPE == SF_DTYPE_BF16) __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(own[0], own[1]), pack_bf16(own[2], own[3])}, to, at, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, own), to, at, 0, 0);
          } else {
            if (i >= valid) continue;
            const int yo = v0 + 4 * lg;
            unsigned char* const out = (unsigned char*)g.o + ((((int64_t)(t0 + i) * g.N + n) * g.H + h) * dv + yo) * M::kBytes;
            if (yo + 4 <= dv) {
              if constexpr (DTYPE == SF_DTYPE_BF16) {
                const u32x2 two = {pack_bf16(own[0], own[1]), pack_bf16(own[2], own[3])};
                __builtin_memcpy(out, &two, 8);
              } else {
                __builtin_memcpy(out, &own, 16);
              }
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (yo + r < dv) M::store(out + r * M::kBytes, own[r]);
            }
          }
        }
      }
#pragma unroll
      for (int J = 0; J < 2; ++J)
#pragma unroll
        for (int r = 0; r < 4; ++r) us[4 * J + r] *= w4[J][r];
      const typename M::Sum uw = M::sum_terms(us);
#pragma unroll
      for (int a = 0; a < ND; ++a) {
        S[a] *= keep;
        if (has_k(a / 2)) S[a] = M::mma(columns<DTYPE>(tk, L::kPitch, col_k(a, 0), 8, li, lg), uw, S[a]);
      }
    } else {
      // f, and of it z = T^T beta f
      f32x4 f[2], z[2];
#pragma unroll
      for (int J = 0; J < 2; ++J) {
        f[J] = w4[J] * ks[J];
        const Slots p = slots_of(mP, 16 * J + li, lg);
        float ps[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ps[r] = g.scale * p.a[r];
          ps[4 + r] = g.scale * p.b[r];
        }
        f[J] = M::mma(M::sum_terms(ps), vt, f[J]);
        f[J] *= b4[J];
      }
      const Slots c0 = slots_down(mT, li, lg), c1 = slots_down(mT, 16 + li, lg);
      z[0] = mm4(c0.b, f[1], mm4(c0.a, f[0], zero));
      z[1] = mm4(c1.b, f[1], zero);
      float zs[8], os[8];
#pragma unroll
      for (int J = 0; J < 2; ++J)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          zs[4 * J + r] = -e4[J][r] * z[J][r];
          os[4 * J + r] = g.scale * e4[J][r] * v[4 * J + r];
        }
      const typename M::Sum zt = M::sum_terms(zs), ot = M::sum_terms(os);
#pragma unroll
      for (int a = 0; a < ND; ++a) {
        S[a] *= keep;
        if (has_k(a / 2)) {
          S[a] = M::mma(columns<DTYPE>(tk, L::kPitch, col_k(a, 0), 8, li, lg), zt, S[a]);
          S[a] = M::mma(columns<DTYPE>(tq, L::kPitch, col_k(a, 0), 8, li, lg), ot, S[a]);
        }
      }
    }
  }
  if (!has_v) return;
  if (g.piece) {
    const size_t at = (size_t)bh * g.n_seg + seg;
    if (identity) store_state(g.seg_through + at * dk * dk);
    else store_state(g.seg_state + at * dk * dv);
    if (!identity && v_block == 0 && tid == 0) g.seg_begin[at] = any_begin ? 1 : 0;
  } else if (g.s_out && seg == (kUp ? g.n_seg - 1 : 0)) {
    store_state(g.s_out + (size_t)bh * dk * dv);
  }
}

// What enters each piece of T, from the pieces' own states and what they make of one that enters:  S <- M S + own, backwards R <- M^T R + own;
// where an episode begins in the piece, own alone.  A workgroup has 16 columns of one (row, head), a wave 16 rows of the state; the state goes
// round through LDS.
template <bool BACK>
__global__ __launch_bounds__(512) void delta_join_kernel(DeltaArgs g) {
  constexpr int kPitch = 132;
  __shared__ __attribute__((aligned(16))) float state[2][16 * kPitch];  // [y][row]
  // the workgroups of one (row, head) read the same matrices: one after another on one XCD
  const unsigned round = g.round.of(blockIdx.x), in_round = blockIdx.x - round * (8 * g.blocks);
  const int dk = g.k.d, dv = g.v.d, bh = (int)(round * 8 + (in_round & 7)), y0 = (int)(in_round >> 3) * 16;
  if (bh >= g.N * g.H) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, lg = lane >> 4;
  const int x0 = 16 * wave, y = y0 + li;
  const unsigned size = (unsigned)(dk * dv) * 4, y_at = y < dv ? (unsigned)((x0 + 4 * lg) * dv + y) * 4 : kOutside;  // (rows past dk lie past the end)
  f32x4 in;  // rows x0 + 4 lg + r
  const auto from_in = buffer(g.s_in ? g.s_in + (size_t)bh * dk * dv : nullptr, g.s_in ? size : 0);
#pragma unroll
  for (int r = 0; r < 4; ++r) in[r] = load_float(from_in, y_at, r * dv * 4);
  struct Piece {
    f32x4 m[8], own;
    int begin;
  };
  auto request = [&](Piece& p, int i) {
    const size_t at = (size_t)bh * g.n_seg + (BACK ? g.n_seg - 1 - i : i);
    const auto from_m = buffer(g.seg_through + at * dk * dk, (unsigned)(dk * dk) * 4), from_o = buffer(g.seg_state + at * dk * dv, size);
    p.begin = g.seg_begin[at];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      // (of a matrix's row what lies behind its columns is the next row's or zero, and meets rows of the state that are zero)
      const int a = x0 + li, b = 16 * s + 4 * lg;
      if constexpr (BACK) {
#pragma unroll
        for (int r = 0; r < 4; ++r) p.m[s][r] = load_float(from_m, a < dk ? (unsigned)(b * dk + a) * 4 : kOutside, r * dk * 4);
      } else {
        p.m[s] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_m, b < dk ? (unsigned)(a * dk + b) * 4 : kOutside, 0, 0));
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) p.own[r] = load_float(from_o, y_at, r * dv * 4);
  };
  // what entered piece i is written to the place of its own state, which is in registers by then
  auto turn = [&](Piece& p, int i) {
    const auto to = buffer(g.seg_state + ((size_t)bh * g.n_seg + (BACK ? g.n_seg - 1 - i : i)) * dk * dv, size);
    float* const round_trip = state[i & 1];
    *(f32x4*)(round_trip + li * kPitch + x0 + 4 * lg) = in;
    __syncthreads();
    f32x4 next = p.own;
#pragma unroll
    for (int r = 0; r < 4; ++r) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)in[r]), to, y_at, r * dv * 4, 0);
    if (p.begin == 0)
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (16 * s < dk) next = mm4(p.m[s], *(const f32x4*)(round_trip + li * kPitch + 16 * s + 4 * lg), next);
    in = next;
    if (i + 2 < g.n_seg) request(p, i + 2);
  };
  Piece even, odd;
  request(even, 0);
  if (g.n_seg > 1) request(odd, 1);
  for (int i = 0; i < g.n_seg; i += 2) {
    turn(even, i);
    if (i + 1 < g.n_seg) turn(odd, i + 1);
  }
}

template <int DTYPE, int D>
struct GradLds {
  static constexpr int kPitch = Pitch<DTYPE, D>::value, kTile = C * kPitch, kPitchF = (D + 4) * 4, kTileF = C * kPitchF;
  static constexpr int kWaves = D / 16, kThreads = 64 * kWaves;
  // q, k, v, do; u and z in fp32; A^T, P^T and T, which make room for dP D and its like as operands
  static constexpr int kU = 4 * kTile, kZ = kU + kTileF, kA = kZ + kTileF, kP = kA + C * kMat * 4, kT = kP + C * kMat * 4,
                       kOperand = 4096, kM = kA;  // [3] of two terms (or halves) of 2 x 64 lanes x 16 bytes
  static_assert(3 * kOperand <= 3 * C * kMat * 4, "operands");
  static constexpr int kSteps = kT + C * kMat * 4, kFlag = kSteps + (int)sizeof(Steps);
  static constexpr int kSums = kFlag + 32;  // float [kWaves + 4][C] of each kind
  static constexpr int kSumRows = 2 * kWaves + 5;
  static constexpr int kBytes = kSums + kSumRows * C * 4;
};

// All gradients of one chunk, given the states S that enters it and R behind it: one workgroup for each (row, head, chunk), a wave for 16
// columns of v and then for 16 of k.
// ALONE: the only chunk, whose matrices the first wave makes (else they are read).
template <int DTYPE, int D, bool ALONE, int KNOWN>
__global__ __launch_bounds__(4 * D, D == 64 && DTYPE == SF_DTYPE_BF16 ? 3 : 2) void delta_grad_kernel(DeltaArgs g) {
  typedef Num<DTYPE> M;
  typedef GradLds<DTYPE, D> L;
  constexpr bool VEC = KNOWN != kAny, WHOLE = KNOWN == kWhole;
  constexpr int W = M::kPieceWords, ND = D / 16, kRow8 = D / 8, kT = L::kThreads;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  // (workgroups go round the XCDs: 16 neighbours, whose rows of a step are neighbours too, for each)
  const unsigned which = (blockIdx.x & ~127u) + (blockIdx.x & 7) * 16 + ((blockIdx.x >> 3) & 15);
  const int chunk = (int)g.rows.of(which), bh = (int)(which - (unsigned)chunk * (g.N * g.H));
  if (chunk >= g.chunks) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h);
  const int dk = WHOLE ? D : g.k.d, dv = WHOLE ? D : g.v.d, t0 = chunk * C, valid = min(C, g.T - t0);
  auto base = [&](const Strided& a) { return (const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes; };
  unsigned char *const tq = lds, *const tk = lds + L::kTile, *const tv = lds + 2 * L::kTile, *const to = lds + 3 * L::kTile;
  float *const mU = (float*)(lds + L::kU), *const mZ = (float*)(lds + L::kZ), *const mA = (float*)(lds + L::kA), *const mP = (float*)(lds + L::kP),
               *const mT = (float*)(lds + L::kT);
  constexpr int kF = D + 4;
  int* const flag = (int*)(lds + L::kFlag);  // by waves
  Steps& steps = *(Steps*)(lds + L::kSteps);
  // by waves: sums over their columns for each step; by tiles: of dP P + dA A along its rows and columns; a number of each wave
  float *const sum_b = (float*)(lds + L::kSums), *const sum_g = sum_b + L::kWaves * C, *const sum_m = sum_g + L::kWaves * C, *const sum_1 = sum_m + 4 * C;

  const size_t state = (size_t)dk * dv;
  const float* const s0 = g.kept_s ? g.kept_s + ((size_t)bh * g.chunks + chunk) * state : nullptr;
  const float* const r1 = g.kept_r ? g.kept_r + ((size_t)bh * g.chunks + chunk) * state : nullptr;

  // the arrays: one piece of each a thread
  unsigned w[4][W];
  const int row8 = tid / kRow8, col8 = tid % kRow8 * 8;
  auto array = [&](unsigned* to_w, const Strided& a) {
    if constexpr (VEC) {
      const auto from = buffer(base(a) + (int64_t)t0 * a.st * M::kBytes, kWholeBuffer);
      load_words<W>(to_w, from, row8 < valid && col8 < a.d ? (unsigned)(row8 * (int)a.st + col8) * M::kBytes : kOutside);
    } else {
      fetch<DTYPE>(to_w, a, base(a), t0, valid, tid, kRow8, 0);
    }
  };
  array(w[0], g.q);
  array(w[1], g.k);
  array(w[2], g.v);
  array(w[3], g.d_o);
  f32x4 n_m[(3 * kDense / 4 + kT - 1) / kT], n_steps;
  if constexpr (!ALONE) {
    const float* const from_steps = g.made + ((size_t)bh * g.chunks + chunk) * made_words(true);
#pragma unroll
    for (int i = 0; i < 3 * kDense / 4; i += kT)
      if (i + tid < 3 * kDense / 4) n_m[i / kT] = *(const f32x4*)(from_steps + 4 * (i + tid));
    if (tid < kStepWords / 4) n_steps = *(const f32x4*)(from_steps + 3 * kDense + 4 * tid);
  }

  StepIn in = {};
  if constexpr (ALONE) in = read_step(g, n, h, 0, valid, lane);
  // the states, 32 rows of both at a time: two pieces of four numbers of each a thread
  const int y0 = 16 * wave, y = y0 + li;  // this wave's columns of v, this lane's
  auto col_k = [&](int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); };
  const auto from_s = buffer(s0, s0 ? (unsigned)state * 4 : 0), from_r = buffer(r1, r1 ? (unsigned)state * 4 : 0);
  constexpr int kPer = D / 4;
  f32x4 ns[2], nr[2];
  auto request = [&](int s) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int row = 32 * s + (tid + p * kT) / kPer, c = (tid + p * kT) % kPer * 4;
      const unsigned at = WHOLE || c < dv ? (unsigned)(row * dv + c) * 4 : kOutside;  // (rows past dk lie past the end)
      ns[p] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_s, at, 0, 0));
      nr[p] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_r, at, 0, 0));
      if (!WHOLE && c + 4 > dv)  // (the next row's numbers)
#pragma unroll
        for (int i = 1; i < 4; ++i)
          if (c + i >= dv) ns[p][i] = nr[p][i] = 0.0f;
    }
  };
  request(0);
  float test = 0.0f;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    put_piece<DTYPE>(lds + a * L::kTile, L::kPitch, w[a], tid, kRow8);
    test = finite_test<DTYPE>(w[a], test);
  }
  if constexpr (!ALONE) {
#pragma unroll
    for (int i = 0; i < 3 * kDense / 4; i += kT) {
      const int e = i + tid, m = e / (kDense / 4), in = e % (kDense / 4);
      if (e < 3 * kDense / 4) *(f32x4*)((m == 0 ? mT : m == 1 ? mP : mA) + in / 8 * kMat + in % 8 * 4) = n_m[i / kT];
    }
    if (tid < kStepWords / 4) *(f32x4*)((float*)&steps + 4 * tid) = n_steps;
  } else if (wave == 0) {
    put_steps(steps, in, (unsigned)__ballot(begins(in)), valid, lane);
  }
  __syncthreads();
  const int my_ep = steps.ep[lane & (C - 1)];
  const float my_steps = fmaf(steps.gh[lane & (C - 1)], 0.0f, steps.beta[lane & (C - 1)] * 0.0f);
  const int e_last = __builtin_amdgcn_readlane(my_ep, valid - 1);
  const bool marked = e_last != 0;
  // steps that an episode begins with: another one's episode than the step before
  const unsigned begin = (unsigned)__ballot(lane < valid && my_ep != (lane ? __shfl_up(my_ep, 1) : 0));
  const float keep = marked ? 0.0f : steps.enter[valid - 1];

  // tiles of the chunk's matrices, [i][j] with i in tile I, j in tile J: the first four waves those of A, the last four those of P
  const int I = wave >> 1 & 1, J = wave & 1;
  float decays[4];  // of steps i = 16 I + 4 lg + r and j = 16 J + li
  {
    const int j = 16 * J + li, ej = steps.ep[j];
    const f32x4 h4 = *(const f32x4*)(steps.gh + 16 * I + 4 * lg), l4 = *(const f32x4*)(steps.gl + 16 * I + 4 * lg);
    const i32x4 e4 = *(const i32x4*)(steps.ep + 16 * I + 4 * lg);
#pragma unroll
    for (int r = 0; r < 4; ++r) decays[r] = 16 * I + 4 * lg + r >= j && e4[r] == ej ? decay_of(h4[r], l4[r], steps.gh[j], steps.gl[j]) : 0.0f;
  }
  if constexpr (ALONE) {
    auto product = [&](const unsigned char* rows, float* to_matrix, bool strict) {
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      if (J <= I) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
          const int at = (32 * s + 8 * lg) * M::kBytes;
          if (32 * s < dk) acc = M::mma(M::row(rows + (16 * I + li) * L::kPitch + at), M::row(tk + (16 * J + li) * L::kPitch + at), acc);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = decays[r] != 0.0f && (!strict || 16 * I + 4 * lg + r > 16 * J + li) ? acc[r] * decays[r] : 0.0f;
      }
      *(f32x4*)(to_matrix + (16 * J + li) * kMat + 16 * I + 4 * lg) = acc;  // [j][i]
    };
    if (wave < 4) product(tk, mA, true);
    if (L::kWaves == 4 || wave >= 4) product(tq, mP, false);
  }

  // what the states give the steps; the slabs go through the places of u and z
  f32x4 ks[2] = {}, qs[2] = {}, kr[2] = {};
  float through = 0.0f;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    if (32 * s >= dk) continue;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int at = (tid + p * kT) / kPer * kF + (tid + p * kT) % kPer * 4;
      *(f32x4*)(mU + at) = ns[p];
      *(f32x4*)(mZ + at) = nr[p];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        through = fmaf(ns[p][i], nr[p][i], through);
        test = fmaf(ns[p][i], 0.0f, fmaf(nr[p][i], 0.0f, test));
      }
    }
    __syncthreads();
    if (32 * (s + 1) < dk) request(s + 1);
    if constexpr (ALONE) {
      if (s == 0 && wave == L::kWaves - 1) invert(mA, steps.beta, mT, lane);
    }
    float xs[8], xr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      xs[i] = mU[(8 * lg + i) * kF + y];
      xr[i] = mZ[(8 * lg + i) * kF + y];
    }
    const typename M::Sum st = M::sum_terms(xs), rt = M::sum_terms(xr);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = (16 * t + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes;
      const auto kk = M::row(tk + at);
      ks[t] = M::mma(kk, st, ks[t]);
      kr[t] = M::mma(kk, rt, kr[t]);
      qs[t] = M::mma(M::row(tq + at), st, qs[t]);
    }
    __syncthreads();
  }
  {
    const bool odd = __any(test != 0.0f);
    if (lane == 0) flag[wave] = odd;
  }
  __syncthreads();

  const int64_t head_k = ((int64_t)n * g.H + h) * dk, head_v = ((int64_t)n * g.H + h) * dv, step_k = (int64_t)g.N * g.H * dk,
                step_v = (int64_t)g.N * g.H * dv;
  // One wave: the sums of dG over each step and the ones behind it in its episode, which is what a decay's gradient is (0 where none was made).
  auto decay_gradient = [&](float dG) {
    const int i = lane & (C - 1);
    const unsigned behind = (begin & ~((2u << i) - 1)) | (valid < C ? 1u << valid : 0u);
    const int reach = (behind ? __ffs((int)behind) - 1 : C) - 1 - i;  // steps behind it
    float s = i < valid ? dG : 0.0f;
    float b = row_left<1>(s);
    s += reach >= 1 ? b : 0.0f;
    b = row_left<2>(s);
    s += reach >= 2 ? b : 0.0f;
    b = row_left<4>(s);
    s += reach >= 4 ? b : 0.0f;
    b = row_left<8>(s);
    s += reach >= 8 ? b : 0.0f;
    b = __shfl(s, 16);
    s += i < 16 && reach >= 16 - i ? b : 0.0f;
    return begin >> i & 1 ? 0.0f : s;
  };
  const int64_t step_at = ((int64_t)t0 * g.N + n) * g.H + h;

  if (__any(lane < L::kWaves && flag[lane & 7] != 0) || __any(my_steps != 0.0f)) {
    // Number by number, so that nothing that is not finite meets a masked zero.
    auto at = [&](const unsigned char* tile, int r, int c) { return M::element(tile + r * L::kPitch + c * M::kBytes); };
    auto put = [&](void* out, bool f32, int64_t i, float v) {
      if (f32) ((float*)out)[i] = v;
      else M::store((unsigned char*)out + i * M::kBytes, v);
    };
    auto decay = [&](int i, int j) { return decay_of(steps.gh[i], steps.gl[i], steps.gh[j], steps.gl[j]); };
    float *const dP = mT, *const dA = (float*)tv;  // [i][j], in the places of T and, when e is made, of v
    for (int e = tid; e < C * C; e += kT) {
      const int i = e / C, j = e % C;
      float a = 0.0f, p = 0.0f;
      if (j <= i && i < valid && steps.ep[i] == steps.ep[j]) {
        for (int x = 0; x < dk; ++x) p += at(tq, i, x) * at(tk, j, x);
        p *= g.scale * decay(i, j);
        if (j < i) {
          for (int x = 0; x < dk; ++x) a += at(tk, i, x) * at(tk, j, x);
          a *= decay(i, j);
        }
      }
      mA[j * kMat + i] = a;
      mP[j * kMat + i] = p;
    }
    __syncthreads();
    // mU: e, mZ: g; a thread has a column of v
    auto sum_all = [&](float x) {
      x = wave_sum(x);
      __syncthreads();
      if (lane == 0) sum_1[wave] = x;
      __syncthreads();
      float s = 0.0f;
      for (int i = 0; i < L::kWaves; ++i) s += sum_1[i];
      return s;
    };
    float tail = 0.0f;  // of dG of the last step
    for (int i = 0; i < valid; ++i) {
      float ks = 0.0f, qs = 0.0f, e = 0.0f;
      if (tid < dv) {
        if (s0 && steps.ep[i] == 0)
          for (int x = 0; x < dk; ++x) {
            ks += at(tk, i, x) * s0[x * dv + tid];
            qs += at(tq, i, x) * s0[x * dv + tid];
          }
        ks *= steps.ep[i] == 0 ? steps.enter[i] : 0.0f;
        qs *= steps.ep[i] == 0 ? steps.enter[i] * g.scale : 0.0f;
        e = at(tv, i, tid) - ks;
        for (int j = 0; j < i; ++j)
          if (steps.ep[j] == steps.ep[i]) e -= mA[j * kMat + i] * steps.beta[j] * mU[j * kF + tid];
        mU[i * kF + tid] = e;
        mZ[i * kF + tid] = ks;  // (until z is made)
      }
      const float s = sum_all(tid < dv ? qs * at(to, i, tid) : 0.0f);
      if (tid == 0) sum_g[i] = s;
    }
    for (int j = valid - 1; j >= 0; --j) {
      float after = 0.0f, f = 0.0f, ks = 0.0f, b = 0.0f;
      if (tid < dv) {
        if (r1 && steps.ep[j] == e_last) {
          for (int x = 0; x < dk; ++x) after += at(tk, j, x) * r1[x * dv + tid];
          after *= steps.leave[j];
        }
        f = after;
        for (int i = j; i < valid; ++i)
          if (steps.ep[i] == steps.ep[j]) {
            f += mP[j * kMat + i] * at(to, i, tid);
            if (i > j) f -= mA[j * kMat + i] * steps.beta[i] * mZ[i * kF + tid];
          }
        ks = mZ[j * kF + tid];
        mZ[j * kF + tid] = f;
        b = f * mU[j * kF + tid];
        put(g.dv, DTYPE == SF_DTYPE_FP32, (t0 + j) * step_v + head_v + tid, steps.beta[j] * f);
      }
      const bool mine = tid < dv;
      const float sb = sum_all(b);
      const float sw = sum_all(mine ? after * steps.beta[j] * mU[j * kF + tid] : 0.0f);
      const float sk = sum_all(mine && steps.ep[j] == 0 ? steps.beta[j] * f * ks : 0.0f);
      tail += steps.ep[j] == e_last ? sw : 0.0f;
      if (tid == 0) {
        g.dbeta[step_at + (int64_t)j * g.N * g.H] = sb;
        sum_g[j] += -sk - (steps.ep[j] == e_last ? sw : 0.0f);
      }
    }
    if (s0 && r1 && !marked) {
      float rs = 0.0f;
      for (int e = tid; e < dk * dv; e += kT) rs += r1[e] * s0[e];
      tail += keep * sum_all(rs);
    }
    __syncthreads();
    for (int e = tid; e < C * C; e += kT) {
      const int i = e / C, j = e % C;
      float p = 0.0f, a = 0.0f;
      if (j <= i && i < valid && steps.ep[i] == steps.ep[j]) {
        for (int c = 0; c < dv; ++c) {
          p += at(to, i, c) * (steps.beta[j] * mU[j * kF + c]);
          a -= steps.beta[i] * mZ[i * kF + c] * (steps.beta[j] * mU[j * kF + c]);
        }
      }
      dP[i * C + j] = p;  // (without the scale, which is in P)
      dA[i * C + j] = j < i ? a : 0.0f;
    }
    __syncthreads();
    if (tid < valid) {
      float s = sum_g[tid];
      for (int j = 0; j <= tid; ++j)
        if (steps.ep[j] == steps.ep[tid])
          s += dP[tid * C + j] * mP[j * kMat + tid] + (j < tid ? dA[tid * C + j] * mA[j * kMat + tid] : 0.0f);
      for (int i = tid; i < valid; ++i)
        if (steps.ep[i] == steps.ep[tid])
          s -= dP[i * C + tid] * mP[tid * kMat + i] + (i > tid ? dA[i * C + tid] * mA[tid * kMat + i] : 0.0f);
      sum_b[tid] = s + (tid == valid - 1 ? tail : 0.0f);
    } else if (tid < C) {
      sum_b[tid] = 0.0f;
    }
    __syncthreads();
    if (wave == 0) {
      const float d = decay_gradient(sum_b[lane & (C - 1)]);
      if (lane < valid) g.dlog_decay[step_at + (int64_t)lane * g.N * g.H] = d;
    }
    for (int e = tid; e < valid * dk; e += kT) {
      const int t = e / dk, x = e % dk;
      float q = 0.0f, k = 0.0f, s = 0.0f;
      for (int j = 0; j <= t; ++j)
        if (steps.ep[j] == steps.ep[t]) {
          const float d = decay(t, j);
          q += g.scale * dP[t * C + j] * d * at(tk, j, x);
          if (j < t) k += dA[t * C + j] * d * at(tk, j, x);
        }
      for (int i = t; i < valid; ++i)
        if (steps.ep[i] == steps.ep[t]) {
          const float d = decay(i, t);
          k += g.scale * dP[i * C + t] * d * at(tq, i, x);
          if (i > t) k += dA[i * C + t] * d * at(tk, i, x);
        }
      if (s0 && steps.ep[t] == 0) {
        float z = 0.0f;
        for (int c = 0; c < dv; ++c) {
          s += s0[x * dv + c] * at(to, t, c);
          z += s0[x * dv + c] * mZ[t * kF + c];
        }
        q += g.scale * steps.enter[t] * s;
        k -= steps.enter[t] * steps.beta[t] * z;
      }
      if (r1 && steps.ep[t] == e_last) {
        s = 0.0f;
        for (int c = 0; c < dv; ++c) s += r1[x * dv + c] * mU[t * kF + c];
        k += steps.leave[t] * steps.beta[t] * s;
      }
      put(g.dq, DTYPE == SF_DTYPE_FP32 || g.f32, (t0 + t) * step_k + head_k + x, q);
      put(g.dk, DTYPE == SF_DTYPE_FP32 || g.f32, (t0 + t) * step_k + head_k + x, k);
    }
    if (g.dstate0)
      for (int e = tid; e < dk * dv; e += kT) {
        const int x = e / dv, c = e % dv;
        float s = r1 && !marked ? keep * r1[e] : 0.0f;
        for (int i = 0; i < valid; ++i)
          if (steps.ep[i] == 0) s += steps.enter[i] * (g.scale * at(tq, i, x) * at(to, i, c) - at(tk, i, x) * steps.beta[i] * mZ[i * kF + c]);
        g.dstate0[(size_t)bh * state + e] = s;
      }
    return;
  }

  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  f32x4 z[2];
  {
    const typename M::Raw vt = columns<DTYPE>(tv, L::kPitch, y0, 4, li, lg), ot = columns<DTYPE>(to, L::kPitch, y0, 4, li, lg);
    float v[8], o[8];
    M::values(vt, v);
    M::values(ot, o);
    f32x4 e4[2], w4[2], b4[2], x[2], e[2], f[2], bf[2], gu[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = 16 * t + 4 * lg;
      e4[t] = *(const f32x4*)(steps.enter + j);
      w4[t] = *(const f32x4*)(steps.leave + j);
      b4[t] = *(const f32x4*)(steps.beta + j);
      // (finite numbers only from here: a factor of zero leaves out what it multiplies)
      ks[t] *= e4[t];
      qs[t] *= e4[t];
      kr[t] *= w4[t];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[t][r] = v[4 * t + r] - ks[t][r];
    }
    const Slots t1 = slots_of(mT, 16 + li, lg);
    e[0] = mm4(*(const f32x4*)(mT + li * kMat + 4 * lg), x[0], zero);
    e[1] = mm4(t1.b, x[1], mm4(t1.a, x[0], zero));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const Slots p = slots_of(mP, 16 * t + li, lg);
      float ps[8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        ps[r] = g.scale * p.a[r];
        ps[4 + r] = g.scale * p.b[r];
      }
      f[t] = M::mma(M::sum_terms(ps), ot, kr[t]);
      bf[t] = b4[t] * f[t];
    }
    const Slots c0 = slots_down(mT, li, lg), c1 = slots_down(mT, 16 + li, lg);
    z[0] = mm4(c0.b, bf[1], mm4(c0.a, bf[0], zero));
    z[1] = mm4(c1.b, bf[1], zero);
    const Slots a0 = slots_of(mA, li, lg);
    gu[0] = f[0] - mm4(a0.b, z[1], mm4(a0.a, z[0], zero));
    gu[1] = f[1] - mm4(*(const f32x4*)(mA + (16 + li) * kMat + 16 + 4 * lg), z[1], zero);
    float rest = 0.0f;  // of dG of the last step: what the chunk's steps give the state behind it
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * t + 4 * lg + r;
        const float u = b4[t][r] * e[t][r], own = kr[t][r] * u;
        rest += own;
        const float sb = row_sum(gu[t][r] * e[t][r]), sg = row_sum(g.scale * qs[t][r] * o[4 * t + r] - z[t][r] * ks[t][r] - own);
        if (li == 0) {
          sum_b[wave * C + j] = sb;
          sum_g[wave * C + j] = sg;
        }
        mU[j * kF + y] = u;
        mZ[j * kF + y] = z[t][r];
      }
    rest = wave_sum(fmaf(keep, through, rest));
    if (lane == 0) sum_1[wave] = rest;
    if (g.dstate0 && y0 < dv) {
      float zs[8], os[8];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          zs[4 * t + r] = -e4[t][r] * z[t][r];
          os[4 * t + r] = g.scale * e4[t][r] * o[4 * t + r];
        }
      const typename M::Sum zt = M::sum_terms(zs), dt = M::sum_terms(os);
      const auto to_state = buffer(g.dstate0 + (size_t)bh * state, (unsigned)state * 4);
      const unsigned y_at = WHOLE || y < dv ? (unsigned)(8 * lg * dv + y) * 4 : kOutside;
#pragma unroll
      for (int a = 0; a < ND; ++a) {
        if (32 * (a >> 1) >= dk) continue;
        f32x4 acc;
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = keep * load_float(from_r, y_at, (32 * (a >> 1) + 4 * (a & 1) + r) * dv * 4);
        acc = M::mma(columns<DTYPE>(tk, L::kPitch, col_k(a, 0), 8, li, lg), zt, acc);
        acc = M::mma(columns<DTYPE>(tq, L::kPitch, col_k(a, 0), 8, li, lg), dt, acc);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)acc[r]), to_state, y_at, (32 * (a >> 1) + 4 * (a & 1) + r) * dv * 4, 0);
      }
    }
  }
  __syncthreads();

  // dP D, by i and by j, and dA D with its transpose, as operands; their sums for the decays
  unsigned char* const m = lds + L::kM;
  auto rows8 = [&](const float* tile, int row, int s) {  // eight neighbours of a row of u or z
    F32::Raw r;
    *(f32x4*)&r.x[0] = *(const f32x4*)(tile + row * kF + 32 * s + 8 * lg);
    *(f32x4*)&r.x[4] = *(const f32x4*)(tile + row * kF + 32 * s + 8 * lg + 4);
    return r;
  };
  float dt[4];  // D of steps i = 16 I + li and j = 16 J + 4 lg + r
  {
    const int i = 16 * I + li, ei = steps.ep[i];
    const f32x4 h4 = *(const f32x4*)(steps.gh + 16 * J + 4 * lg), l4 = *(const f32x4*)(steps.gl + 16 * J + 4 * lg);
    const i32x4 e4 = *(const i32x4*)(steps.ep + 16 * J + 4 * lg);
#pragma unroll
    for (int r = 0; r < 4; ++r) dt[r] = i >= 16 * J + 4 * lg + r && e4[r] == ei ? decay_of(steps.gh[i], steps.gl[i], h4[r], l4[r]) : 0.0f;
  }
  f32x4 made[4];  // dP [j][i], dP [i][j], dA + its transpose [j][i] (I, J as the tile's row and column), M [i][j]
  made[0] = made[1] = made[2] = made[3] = zero;
  if (L::kWaves == 4 || wave >= 4) {
    if (J <= I) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        if (32 * s >= dv) continue;
        const auto ut = M::sum_terms(rows8(mU, 16 * J + li, s).x);
        const auto oi = M::row(to + (16 * I + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes);
        made[0] = M::mma(ut, oi, made[0]);
        made[1] = M::mma(oi, ut, made[1]);
      }
      const f32x4 p = *(const f32x4*)(mP + (16 * J + li) * kMat + 16 * I + 4 * lg);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        made[0][r] *= g.scale * dt[r];
        made[1][r] *= g.scale;
        made[3][r] += made[1][r] * p[r];
        made[1][r] *= decays[r];
      }
    }
  }
  if (wave < 4) {
    f32x4 low = zero, high = zero;  // [i][j] of -z u^T and of -u z^T
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if (32 * s >= dv) continue;
      if (J <= I) low = F32::mma(rows8(mZ, 16 * I + li, s), rows8(mU, 16 * J + li, s), low);
      if (J >= I) high = F32::mma(rows8(mU, 16 * I + li, s), rows8(mZ, 16 * J + li, s), high);
    }
    const f32x4 a = *(const f32x4*)(mA + (16 * J + li) * kMat + 16 * I + 4 * lg);
    const int j = 16 * J + li, ej = steps.ep[j];
    const f32x4 h4 = *(const f32x4*)(steps.gh + 16 * I + 4 * lg), l4 = *(const f32x4*)(steps.gl + 16 * I + 4 * lg);
    const i32x4 e4 = *(const i32x4*)(steps.ep + 16 * I + 4 * lg);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * I + 4 * lg + r;
      made[3][r] -= low[r] * a[r];  // (a is zero where j is not before i)
      const float up = i < j && e4[r] == ej ? decay_of(steps.gh[j], steps.gl[j], h4[r], l4[r]) : 0.0f;
      made[2][r] = -(i > j ? low[r] * decays[r] : high[r] * up);
    }
  }
  // (on their way for what follows: rows y0 + li of both states, eight numbers at 32 s + 8 lg; past dv they are the next row's, or zero
  // behind the last one, and what they meet is zero)
  float row_s[D / 32][8], row_r[D / 32][8];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    load_words<8>((unsigned*)row_s[s], from_s, (unsigned)(y * dv + 32 * s + 8 * lg) * 4);
    load_words<8>((unsigned*)row_r[s], from_r, (unsigned)(y * dv + 32 * s + 8 * lg) * 4);
  }
  f32x4 row_sums = made[3];
  float col_sum = (made[3][0] + made[3][1]) + (made[3][2] + made[3][3]);
#pragma unroll
  for (int r = 0; r < 4; ++r) row_sums[r] = row_sum(row_sums[r]);
  col_sum += __shfl_xor(col_sum, 16);
  col_sum += __shfl_xor(col_sum, 32);
  __syncthreads();  // T has been read, and the sums of this part have a place of their own
  // (rows of tile I from tile J, less columns of tile J from tile I: both halves of the waves add up behind the barrier)
  float* const tile_sums = sum_m;
  if (L::kWaves == 4) {
    if (li == 0) *(f32x4*)(tile_sums + J * C + 16 * I + 4 * lg) = row_sums;
    if (lg == 0) tile_sums[2 * C + I * C + 16 * J + li] = col_sum;
  } else {
    float* const mine = (wave < 4 ? (float*)tv : (float*)tv + 4 * C);  // (v has been read)
    if (li == 0) *(f32x4*)(mine + J * C + 16 * I + 4 * lg) = row_sums;
    if (lg == 0) mine[2 * C + I * C + 16 * J + li] = col_sum;
  }
  if (L::kWaves == 4 || wave >= 4) {
    M::put4(m + I * 1024, 2048, lane, J, made[0]);
    M::put4(m + L::kOperand + J * 1024, 2048, lane, I, made[1]);
  }
  if (wave < 4) M::put4(m + 2 * L::kOperand + J * 1024, 2048, lane, I, made[2]);
  __syncthreads();

  if (wave == 0) {
    const int i = lane & (C - 1);
    float b = 0.0f, s = 0.0f, rest = 0.0f;
#pragma unroll
    for (int w = 0; w < L::kWaves; ++w) {
      b += sum_b[w * C + i];
      s += sum_g[w * C + i];
      rest += sum_1[w];
    }
    auto add = [&](const float* t) { s += (t[i] + t[C + i]) - (t[2 * C + i] + t[3 * C + i]); };
    if (L::kWaves == 4) {
      add(tile_sums);
    } else {
      add((float*)tv);
      add((float*)tv + 4 * C);
    }
    const float d = decay_gradient(i == valid - 1 ? s + rest : s);
    if (lane < valid) {
      g.dbeta[step_at + (int64_t)lane * g.N * g.H] = b;
      g.dlog_decay[step_at + (int64_t)lane * g.N * g.H] = d;
    }
  }

  // dq and dk, 16 columns a wave, [k][step]
  f32x4 dq[2] = {}, dkk[2] = {};
  if (y0 < dk) {
    f32x4 zs[2] = {}, us[2] = {};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if (32 * s >= dv) continue;
      const typename M::Out st = M::out_terms(row_s[s]), rt = M::out_terms(row_r[s]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int i = 16 * t + li;
        dq[t] = M::mma(st, M::row(to + i * L::kPitch + (32 * s + 8 * lg) * M::kBytes), dq[t]);
        zs[t] = mma_oo<DTYPE>(st, M::out_terms(rows8(mZ, i, s).x), zs[t]);
        us[t] = mma_oo<DTYPE>(rt, M::out_terms(rows8(mU, i, s).x), us[t]);
      }
    }
    const typename M::Raw kt = columns<DTYPE>(tk, L::kPitch, y0, 4, li, lg), qt = columns<DTYPE>(tq, L::kPitch, y0, 4, li, lg);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int i = 16 * t + li;
      const float e = steps.enter[i], l = steps.leave[i];
      dq[t] = M::mma(kt, M::get(m + t * 1024, 2048, lane), (g.scale * e) * dq[t]);
      dkk[t] = l * us[t] - e * zs[t];
      dkk[t] = M::mma(qt, M::get(m + L::kOperand + t * 1024, 2048, lane), dkk[t]);
      dkk[t] = M::mma(kt, M::get(m + 2 * L::kOperand + t * 1024, 2048, lane), dkk[t]);
    }
  }
  __syncthreads();
  // out by whole rows, through the places of q and k; dv from z
  constexpr bool kF32 = DTYPE == SF_DTYPE_FP32;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int i = 16 * t + li, c = y0 + 4 * lg;
    if (g.f32 && !kF32) {
      float* const at_q = (float*)g.dq + (t0 + i) * step_k + head_k + c;
      float* const at_k = (float*)g.dk + (t0 + i) * step_k + head_k + c;
      if (i < valid && c + 4 <= dk) {
        __builtin_memcpy(at_q, &dq[t], 16);
        __builtin_memcpy(at_k, &dkk[t], 16);
      } else if (i < valid) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (c + r < dk) {
            at_q[r] = dq[t][r];
            at_k[r] = dkk[t][r];
          }
      }
      continue;
    }
    unsigned char* const at = lds + i * L::kPitch + c * M::kBytes;
    if constexpr (kF32) {
      *(f32x4*)at = dq[t];
      *(f32x4*)(at + L::kTile) = dkk[t];
    } else {
      *(u32x2*)at = u32x2{pack_bf16(dq[t][0], dq[t][1]), pack_bf16(dq[t][2], dq[t][3])};
      *(u32x2*)(at + L::kTile) = u32x2{pack_bf16(dkk[t][0], dkk[t][1]), pack_bf16(dkk[t][2], dkk[t][3])};
    }
  }
  __syncthreads();
  if (row8 >= valid) return;
  auto store = [&](void* out, int64_t at, int d, const unsigned* piece) {
    if (col8 + 8 <= d) {
#pragma unroll
      for (int i = 0; i < W; i += 4) __builtin_memcpy((unsigned char*)out + at * M::kBytes + 4 * i, piece + i, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (col8 + i >= d) continue;
        if constexpr (kF32) ((unsigned*)out)[at + i] = piece[i];
        else ((uint16_t*)out)[at + i] = (uint16_t)(piece[i / 2] >> (16 * (i & 1)));
      }
    }
  };
  unsigned piece[W];
  if (kF32 || !g.f32) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
#pragma unroll
      for (int i = 0; i < W; i += 4) *(u32x4*)(piece + i) = *(const u32x4*)(lds + a * L::kTile + row8 * L::kPitch + col8 * M::kBytes + 4 * i);
      store(a == 0 ? g.dq : g.dk, (t0 + row8) * step_k + head_k + col8, dk, piece);
    }
  }
  {
    const float* const x = mZ + row8 * kF + col8;
    if constexpr (kF32) {
      *(u32x4*)piece = *(const u32x4*)x;
      *(u32x4*)(piece + 4) = *(const u32x4*)(x + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) piece[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
    store(g.dv, (t0 + row8) * step_v + head_v + col8, dv, piece);
  }
}

// Sums of the gradients of shared heads: in [rows][H][d] fp32, out [rows][H / share][d].
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void delta_share_kernel(const float* in, void* out, int64_t n_out, int d, int share) {
  for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < n_out; e += (int64_t)gridDim.x * kThreads) {
    const float* x = in + e / d * share * d + e % d;
    float sum = 0.0f;
    for (int i = 0; i < share; ++i) sum += x[(int64_t)i * d];
    Num<DTYPE>::store((unsigned char*)out + e * Num<DTYPE>::kBytes, sum);
  }
}

// One step of one (row, head): the state is read and decayed, multiplied with k and q in one go, corrected and written:
//   o = scale (S'^T q + (q . k) u).
// A thread holds four neighbours of every (256 / lanes)-th row, so that all its loads are under way at once.
template <int DTYPE, bool VEC>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(DeltaArgs g, float* table, int n_env, const int32_t* ids, int share, int lanes_log2) {
  typedef Num<DTYPE> M;
  __shared__ __attribute__((aligned(16))) float sq[128], sk[128], part[2][4][128], su[128];
  const int tid = threadIdx.x, n = blockIdx.x / g.H, h = blockIdx.x % g.H, dk = g.k.d, dv = g.v.d;
  const int id = ids ? ids[n] : n;
  const bool known = id >= 0 && id < n_env;
  const float l2 = g.log_decay[(int64_t)n * g.H + h] * 1.44269504f, beta = g.beta[(int64_t)n * g.H + h];
  const bool begin = !known || (g.done && g.done[n] != 0) || l2 < (float)kLeastLog2;
  const float keep = exp2f(l2);
  const int rows = kThreads >> lanes_log2, row0 = tid >> lanes_log2, c0 = (tid & ((1 << lanes_log2) - 1)) * 4;
  float* s = table + ((int64_t)(known ? id : 0) * g.H + h) * dk * dv;
  constexpr int kMost = 16;  // rows of a thread: 128 / (256 / 32)
  float x[kMost][4];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int r = row0 + i * rows;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i][j] = 0.0f;
    if (begin || r >= dk || c0 >= dv) continue;
    if constexpr (VEC) {
      *(f32x4*)x[i] = *(const f32x4*)(s + r * dv + c0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + j < dv) x[i][j] = s[r * dv + c0 + j];
    }
  }
  if (tid < 128) {
    sk[tid] = tid < dk ? M::element((const unsigned char*)g.k.p + (n * g.k.sn + h / share * g.k.sh + tid) * M::kBytes) : 0.0f;
  } else {
    sq[tid - 128] = tid - 128 < dk ? M::element((const unsigned char*)g.q.p + (n * g.q.sn + h / share * g.q.sh + tid - 128) * M::kBytes) : 0.0f;
  }
  const float v = tid < dv ? M::element((const unsigned char*)g.v.p + (n * g.v.sn + h * g.v.sh + tid) * M::kBytes) : 0.0f;
  __syncthreads();
  float a[4] = {}, b[4] = {};  // of S'^T k and S'^T q
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int r = row0 + i * rows;
    if (r >= dk || c0 >= dv) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[i][j] = begin ? 0.0f : keep * x[i][j];
      a[j] = begin ? 0.0f : fmaf(sk[r], x[i][j], a[j]);
      b[j] = begin ? 0.0f : fmaf(sq[r], x[i][j], b[j]);
    }
  }
  // over the rows: within the wave, then over the four waves
  for (int m = 1 << lanes_log2; m < 64; m <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] += __shfl_xor(a[j], m);
      b[j] += __shfl_xor(b[j], m);
    }
  if ((tid & 63) < 1 << lanes_log2 && c0 < 128) {
    *(f32x4*)&part[0][tid >> 6][c0] = f32x4{a[0], a[1], a[2], a[3]};
    *(f32x4*)&part[1][tid >> 6][c0] = f32x4{b[0], b[1], b[2], b[3]};
  }
  __syncthreads();
  if (tid < 128) {
    float qk = wave_sum(sq[tid & 63] * sk[tid & 63] + sq[64 + (tid & 63)] * sk[64 + (tid & 63)]);
    const float sum = tid < dv ? (part[0][0][tid] + part[0][1][tid]) + (part[0][2][tid] + part[0][3][tid]) : 0.0f;
    const float u = tid < dv ? beta * (v - sum) : 0.0f;
    su[tid] = u;
    if (tid < dv) {
      const float o = (part[1][0][tid] + part[1][1][tid]) + (part[1][2][tid] + part[1][3][tid]) + qk * u;
      M::store((unsigned char*)g.o + (((int64_t)n * g.H + h) * dv + tid) * M::kBytes, g.scale * o);
    }
  }
  __syncthreads();
  if (!known || c0 >= dv) return;
  const f32x4 u4 = *(const f32x4*)(su + c0);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int r = row0 + i * rows;
    if (r >= dk) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i][j] = fmaf(sk[r], u4[j], x[i][j]);
    if constexpr (VEC) {
      *(f32x4*)(s + r * dv + c0) = *(f32x4*)x[i];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + j < dv) s[r * dv + c0 + j] = x[i][j];
    }
  }
}

// ---- host side ---------------------------------------------------------------------------------

int check(const sf_deltarule_config* c, const char* fn) {
  if (!c || c->struct_size != sizeof(sf_deltarule_config)) {
    set_error("%s: null configuration or struct_size mismatch", fn);
    return SF_ERR_ARG;
  }
  if (c->dtype != SF_DTYPE_FP32 && c->dtype != SF_DTYPE_BF16) {
    set_error("%s: dtype = %d", fn, c->dtype);
    return SF_ERR_ARG;
  }
  if (c->T < 0 || c->N < 0 || c->H < 1 || c->Hk < 1 || c->H % c->Hk || c->dk < 1 || c->dk > 128 || c->dv < 1 || c->dv > 128) {
    set_error("%s: T = %d, N = %d, H = %d, Hk = %d, dk = %d, dv = %d out of range", fn, c->T, c->N, c->H, c->Hk, c->dk, c->dv);
    return SF_ERR_SHAPE;
  }
  if ((int64_t)c->T * c->N > INT32_MAX || (int64_t)c->N * c->H > 1 << 21 || (int64_t)c->N * c->H * ((c->T + (int64_t)C - 1) / C) > INT32_MAX - 128) {
    set_error("%s: T * N or N * H * T / 32 beyond 2^31 - 1, or N * H beyond 2^21", fn);
    return SF_ERR_SHAPE;
  }
  if (!isfinite(c->scale)) {
    set_error("%s: scale is not finite", fn);
    return SF_ERR_SHAPE;
  }
  return SF_OK;
}

int check_ptr(const char* fn, const char* name, const void* p, size_t align, bool optional = false) {
  if (!p && optional) return SF_OK;
  if (!p || (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0) {
    set_error("%s: %s is null or not %zu-byte aligned", fn, name, align);
    return SF_ERR_ARG;
  }
  return SF_OK;
}

// Whether two arrays of states (or null) have a number in common; of no rows, whether they begin at one address.
bool overlap(const sf_deltarule_config* c, const float* a, const float* b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), size = (uintptr_t)c->N * c->H * c->dk * c->dv * 4;
  return a && b && (x == y || (x < y ? y - x : x - y) < size);
}

int chunks_of(const sf_deltarule_config* c) { return (c->T + C - 1) / C; }

// Pieces of T where the workgroups that go over the chunks (one for each 64 columns of a head) leave CUs idle.
struct Split {
  int n_seg, seg_len;
};
Split split_of(const sf_deltarule_config* c) {
  const int64_t lanes = (int64_t)c->N * c->H * (c->dv > DV ? 2 : 1);
  const int chunks = chunks_of(c);
  if (lanes == 0 || lanes > 128 || chunks < 16) return Split{1, std::max(1, chunks) * C};
  const int want = (int)std::min<int64_t>((512 + lanes - 1) / lanes, 32);
  const int per = std::max(8, (chunks + want - 1) / want);
  return Split{(chunks + per - 1) / per, per * C};
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
struct Workspace {
  size_t made, seg_state, seg_through, seg_begin;  // bytes of each part, in this order
  size_t states, dq, dk, total;                    // the states that enter the chunks and as many R's; the shared heads' gradients
};
Workspace workspace_of(const sf_deltarule_config* c, int backward) {
  Workspace w = {};
  const size_t lanes = (size_t)c->N * c->H, chunks = chunks_of(c), state = (size_t)c->dk * c->dv * 4;
  const Split s = split_of(c);
  if (c->T > C) w.made = align256(lanes * chunks * made_words(backward) * 4);
  if (s.n_seg > 1) {
    w.seg_state = align256(lanes * s.n_seg * state);
    w.seg_through = align256(lanes * s.n_seg * c->dk * c->dk * 4);
    w.seg_begin = align256(lanes * s.n_seg * 4);
  }
  if (backward) {
    if (c->T > C) w.states = align256(lanes * chunks * state);
    if (c->H != c->Hk) w.dq = w.dk = align256((size_t)c->T * c->N * c->H * c->dk * 4);
  }
  w.total = w.made + w.seg_state + w.seg_through + w.seg_begin + 2 * w.states + w.dq + w.dk;
  return w;
}

// (a chunk's rows lie within 2^31 bytes then, and one behind the other)
bool near(int64_t st, int d) { return st >= d && st <= 1 << 23; }
Strided strided(const sf_deltarule_config* c, const void* p, const int64_t* s, bool shared, int d) {
  Strided a = {p, c->T == 1 ? 0 : s[0], s[1], s[2], shared, d, 0};  // (one step: any stride)
  const int per = 16 / (c->dtype == SF_DTYPE_BF16 ? 2 : 4);
  // (pieces are eight columns in both types)
  a.vec = d % 8 == 0 && (c->T == 1 || near(s[0], d)) && a.st % per == 0 && s[1] % per == 0 && s[2] % per == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
  return a;
}

DeltaArgs args_of(const sf_deltarule_config* c, const void* q, const void* k, const void* v, const float* log_decay, const float* beta,
                  const uint8_t* done) {
  DeltaArgs g = {};
  const int share = c->H / c->Hk;
  g.q = strided(c, q, c->q_stride, share > 1, c->dk);
  g.k = strided(c, k, c->k_stride, share > 1, c->dk);
  g.v = strided(c, v, c->v_stride, false, c->dv);
  g.log_decay = log_decay;
  g.beta = beta;
  g.done = done;
  g.T = c->T;
  g.N = c->N;
  g.H = c->H;
  g.chunks = std::max(1, chunks_of(c));
  g.blocks_v = g.blocks = c->dv > DV ? 2 : 1;
  g.n_seg = 1;
  g.seg_len = g.chunks * C;
  g.scale = c->scale;
  g.heads = divisor(c->H);
  g.share = divisor(share);
  g.rows = divisor((unsigned)std::max(1, c->N * c->H));
  return g;
}

// The parts of the workspace.
void with_pieces(const sf_deltarule_config* c, DeltaArgs& g, const Workspace& w, unsigned char* ws) {
  const Split s = split_of(c);
  g.made = (float*)ws;
  g.n_seg = s.n_seg;
  g.seg_len = s.seg_len;
  g.seg_state = (float*)(ws + w.made);
  g.seg_through = (float*)(ws + w.made + w.seg_state);
  g.seg_begin = (int*)(ws + w.made + w.seg_state + w.seg_through);
}

template <int DTYPE, int D, bool BACK>
void launch_chunks(const DeltaArgs& g, hipStream_t st) {
  const unsigned grid = (unsigned)(((int64_t)g.N * g.H * g.chunks + 3) / 4);
  constexpr int bytes = 4 * (2 * C * kMat * 4 + (int)sizeof(Steps));
  static_assert(bytes <= 64 * 1024, "no attribute needed");
  if (g.q.vec && g.k.vec) delta_chunks_kernel<DTYPE, D, BACK, true><<<grid, kThreads, bytes, st>>>(g);
  else delta_chunks_kernel<DTYPE, D, BACK, false><<<grid, kThreads, bytes, st>>>(g);
}
template <int DTYPE>
void launch_chunks(const DeltaArgs& g, hipStream_t st) {
  if (g.k.d > 64) g.back ? launch_chunks<DTYPE, 128, true>(g, st) : launch_chunks<DTYPE, 128, false>(g, st);
  else g.back ? launch_chunks<DTYPE, 64, true>(g, st) : launch_chunks<DTYPE, 64, false>(g, st);
}
hipError_t make_chunks(const sf_deltarule_config* c, const DeltaArgs& g, hipStream_t st) {
  if (c->dtype == SF_DTYPE_BF16) launch_chunks<SF_DTYPE_BF16>(g, st);
  else launch_chunks<SF_DTYPE_FP32>(g, st);
  return hipGetLastError();
}

template <int DTYPE, int D, int SWEEP, bool ALONE>
void launch_sweep(const DeltaArgs& g, bool vec, hipStream_t st) {
  typedef SweepLds<DTYPE, D> L;
  constexpr int bytes = ALONE ? L::kBytesAlone : L::kBytes;
  static_assert(bytes <= 64 * 1024, "no attribute needed");
  const dim3 grid((unsigned)((g.N * g.H + 7) / 8 * 8 * g.blocks), (unsigned)g.n_seg);
  if (!vec) delta_sweep_kernel<DTYPE, D, SWEEP, ALONE, kAny><<<grid, kThreads, bytes, st>>>(g);
  else if (g.k.d == D && g.v.d % DV == 0) delta_sweep_kernel<DTYPE, D, SWEEP, ALONE, kWhole><<<grid, kThreads, bytes, st>>>(g);
  else delta_sweep_kernel<DTYPE, D, SWEEP, ALONE, kPieces><<<grid, kThreads, bytes, st>>>(g);
}
template <int SWEEP, bool ALONE = false>
hipError_t sweep(const sf_deltarule_config* c, DeltaArgs g, hipStream_t st) {
  if (g.piece && SWEEP == kStates) g.blocks = g.blocks_v + (c->dk > DV ? 2 : 1);
  g.round = divisor(8 * g.blocks);
  const Strided& third = SWEEP == kBack ? g.d_o : g.v;
  const bool vec = g.k.vec && third.vec && (SWEEP == kStates || g.q.vec) &&
                   (SWEEP != kResults || ((reinterpret_cast<uintptr_t>(g.o) & 15) == 0 && (int64_t)c->N * c->H * c->dv * 4 * C < (int64_t)1 << 31));
  if (c->dtype == SF_DTYPE_BF16) {
    if (c->dk > 64) launch_sweep<SF_DTYPE_BF16, 128, SWEEP, ALONE>(g, vec, st);
    else launch_sweep<SF_DTYPE_BF16, 64, SWEEP, ALONE>(g, vec, st);
  } else {
    if (c->dk > 64) launch_sweep<SF_DTYPE_FP32, 128, SWEEP, ALONE>(g, vec, st);
    else launch_sweep<SF_DTYPE_FP32, 64, SWEEP, ALONE>(g, vec, st);
  }
  return hipGetLastError();
}
template <bool BACK>
hipError_t join(const sf_deltarule_config* c, DeltaArgs g, hipStream_t st) {
  g.blocks = (c->dv + 15) / 16;
  g.round = divisor(8 * g.blocks);
  delta_join_kernel<BACK><<<(unsigned)((c->N * c->H + 7) / 8 * 8 * g.blocks), 512, 0, st>>>(g);
  return hipGetLastError();
}

template <int DTYPE, int D, bool ALONE, int KNOWN>
hipError_t launch_grad(const DeltaArgs& g, hipStream_t st) {
  const auto kern = delta_grad_kernel<DTYPE, D, ALONE, KNOWN>;
  constexpr int bytes = GradLds<DTYPE, D>::kBytes;
  static_assert(bytes <= 160 * 1024, "LDS");
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)(((int64_t)g.N * g.H * g.chunks + 127) / 128 * 128), 4 * D, bytes, st>>>(g);
  return hipGetLastError();
}
template <int DTYPE, int D, bool ALONE>
hipError_t launch_grad(const DeltaArgs& g, hipStream_t st) {
  if (!(g.q.vec && g.k.vec && g.v.vec && g.d_o.vec)) return launch_grad<DTYPE, D, ALONE, kAny>(g, st);
  return launch_grad<DTYPE, D, ALONE, kPieces>(g, st);
}
template <int DTYPE, int D>
hipError_t launch_grad(const DeltaArgs& g, hipStream_t st) {
  return g.chunks == 1 ? launch_grad<DTYPE, D, true>(g, st) : launch_grad<DTYPE, D, false>(g, st);
}
hipError_t grad(const sf_deltarule_config* c, const DeltaArgs& g, hipStream_t st) {
  const bool wide = c->dk > 64 || c->dv > 64;
  if (c->dtype == SF_DTYPE_BF16) return wide ? launch_grad<SF_DTYPE_BF16, 128>(g, st) : launch_grad<SF_DTYPE_BF16, 64>(g, st);
  return wide ? launch_grad<SF_DTYPE_FP32, 128>(g, st) : launch_grad<SF_DTYPE_FP32, 64>(g, st);
}

int launched(const char* fn, hipError_t e) {
  if (e == hipSuccess) return SF_OK;
  set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
  return SF_ERR_DEVICE;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" int64_t sf_deltarule_workspace_bytes(const sf_deltarule_config* cfg, int backward) {
  if (check(cfg, "sf_deltarule_workspace_bytes") != SF_OK) return -1;
  return (int64_t)workspace_of(cfg, backward).total;
}

extern "C" int sf_deltarule(const sf_deltarule_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                            const float* beta, const uint8_t* done, const float* state0, void* o, float* state, void* workspace,
                            void* hip_stream) {
  static const char* fn = "sf_deltarule";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = (int64_t)cfg->T * cfg->N == 0;
  const Workspace w = workspace_of(cfg, 0);
  if ((rc = check_ptr(fn, "q", q, e, none)) || (rc = check_ptr(fn, "k", k, e, none)) || (rc = check_ptr(fn, "v", v, e, none)) ||
      (rc = check_ptr(fn, "o", o, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4, none)) ||
      (rc = check_ptr(fn, "beta", beta, 4, none)) || (rc = check_ptr(fn, "state0", state0, 4, true)) ||
      (rc = check_ptr(fn, "state", state, 4, true)) || (rc = check_ptr(fn, "workspace", workspace, 256, w.total == 0)))
    return rc;
  if (state != state0 && overlap(cfg, state, state0)) {
    set_error("%s: state overlaps state0", fn);
    return SF_ERR_ALIAS;
  }
  if (cfg->N == 0) return SF_OK;
  DeltaArgs g = args_of(cfg, q, k, v, log_decay, beta, done);
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  g.o = o;
  g.s_in = state0;
  g.s_out = state;
  if (cfg->T <= C) return launched(fn, sweep<kResults, true>(cfg, g, st));
  with_pieces(cfg, g, w, (unsigned char*)workspace);
  hipError_t err = make_chunks(cfg, g, st);
  if (err == hipSuccess && g.n_seg > 1) {
    g.piece = 1;
    err = sweep<kStates>(cfg, g, st);
    g.piece = 0;
    if (err == hipSuccess) err = join<false>(cfg, g, st);
  }
  if (err == hipSuccess) err = sweep<kResults>(cfg, g, st);
  return launched(fn, err);
}

extern "C" int sf_deltarule_backward(const sf_deltarule_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                                     const float* beta, const void* d_o, const uint8_t* done, const float* state0, const float* dstate,
                                     void* dq, void* dk, void* dv, float* dlog_decay, float* dbeta, float* dstate0, void* workspace,
                                     void* hip_stream) {
  static const char* fn = "sf_deltarule_backward";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = (int64_t)cfg->T * cfg->N == 0;
  const Workspace w = workspace_of(cfg, 1);
  if ((rc = check_ptr(fn, "q", q, e, none)) || (rc = check_ptr(fn, "k", k, e, none)) || (rc = check_ptr(fn, "v", v, e, none)) ||
      (rc = check_ptr(fn, "do", d_o, e, none)) || (rc = check_ptr(fn, "dq", dq, e, none)) || (rc = check_ptr(fn, "dk", dk, e, none)) ||
      (rc = check_ptr(fn, "dv", dv, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4, none)) ||
      (rc = check_ptr(fn, "beta", beta, 4, none)) || (rc = check_ptr(fn, "dlog_decay", dlog_decay, 4, none)) ||
      (rc = check_ptr(fn, "dbeta", dbeta, 4, none)) || (rc = check_ptr(fn, "state0", state0, 4, true)) ||
      (rc = check_ptr(fn, "dstate", dstate, 4, true)) || (rc = check_ptr(fn, "dstate0", dstate0, 4, true)) ||
      (rc = check_ptr(fn, "workspace", workspace, 256, w.total == 0)))
    return rc;
  if (overlap(cfg, dstate0, dstate) || overlap(cfg, dstate0, state0)) {
    set_error("%s: dstate0 overlaps dstate or state0", fn);
    return SF_ERR_ALIAS;
  }
  if (cfg->N == 0) return SF_OK;
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  unsigned char* const ws = (unsigned char*)workspace;
  const int share = cfg->H / cfg->Hk;
  DeltaArgs g = args_of(cfg, q, k, v, log_decay, beta, done);
  g.d_o = strided(cfg, d_o, cfg->do_stride, false, cfg->dv);
  with_pieces(cfg, g, w, ws);
  g.back = 1;
  const size_t at = w.made + w.seg_state + w.seg_through + w.seg_begin;
  hipError_t err = cfg->T <= C ? hipSuccess : make_chunks(cfg, g, st);
  if (cfg->T == 0 || cfg->T > C) {
    if (cfg->T > 0) {
      g.s_in = state0;
      if (err == hipSuccess && g.n_seg > 1) {
        g.piece = 1;
        err = sweep<kStates>(cfg, g, st);
        g.piece = 0;
        if (err == hipSuccess) err = join<false>(cfg, g, st);
      }
      g.kept = (float*)(ws + at);
      if (err == hipSuccess) err = sweep<kStates>(cfg, g, st);
      g.kept = nullptr;
    }
    g.s_in = dstate;
    if (err == hipSuccess && g.n_seg > 1) {
      g.piece = 1;
      err = sweep<kBack>(cfg, g, st);
      g.piece = 0;
      if (err == hipSuccess) err = join<true>(cfg, g, st);
    }
    g.s_out = dstate0;
    if (cfg->T > 0) g.kept = (float*)(ws + at + w.states);
    if (err == hipSuccess) err = sweep<kBack>(cfg, g, st);
    g.kept_s = (const float*)(ws + at);
    g.kept_r = g.kept;
  } else {
    g.kept_s = state0;
    g.kept_r = dstate;
    g.dstate0 = dstate0;
  }
  if (none || err != hipSuccess) return launched(fn, err);
  float* const part_q = (float*)(ws + at + 2 * w.states);
  float* const part_k = (float*)(ws + at + 2 * w.states + w.dq);
  g.dq = share > 1 ? part_q : dq;
  g.dk = share > 1 ? part_k : dk;
  g.dv = dv;
  g.dlog_decay = dlog_decay;
  g.dbeta = dbeta;
  g.f32 = share > 1;
  err = grad(cfg, g, st);
  if (err == hipSuccess && share > 1) {
    const int64_t count = (int64_t)cfg->T * cfg->N * cfg->Hk * cfg->dk;
    const unsigned grid = (unsigned)std::min<int64_t>((count + kThreads - 1) / kThreads, 1 << 20);
    const auto kern = cfg->dtype == SF_DTYPE_BF16 ? delta_share_kernel<SF_DTYPE_BF16> : delta_share_kernel<SF_DTYPE_FP32>;
    kern<<<grid, kThreads, 0, st>>>(part_q, dq, count, cfg->dk, share);
    kern<<<grid, kThreads, 0, st>>>(part_k, dk, count, cfg->dk, share);
    err = hipGetLastError();
  }
  return launched(fn, err);
}

extern "C" int sf_deltarule_step(const sf_deltarule_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                                 const float* beta, float* state_table, int32_t n_env, const int32_t* env_ids, const uint8_t* done, void* o,
                                 void* hip_stream) {
  static const char* fn = "sf_deltarule_step";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  if (cfg->T != 1 || n_env < 1) {
    set_error("%s: T = %d (1 is wanted), n_env = %d", fn, cfg->T, n_env);
    return SF_ERR_SHAPE;
  }
  if (!env_ids && cfg->N > n_env) {
    set_error("%s: %d rows, but %d states and no ids", fn, cfg->N, n_env);
    return SF_ERR_SHAPE;
  }
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = cfg->N == 0;
  if ((rc = check_ptr(fn, "q", q, e, none)) || (rc = check_ptr(fn, "k", k, e, none)) || (rc = check_ptr(fn, "v", v, e, none)) ||
      (rc = check_ptr(fn, "o", o, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4, none)) ||
      (rc = check_ptr(fn, "beta", beta, 4, none)) || (rc = check_ptr(fn, "state_table", state_table, 16)) ||
      (rc = check_ptr(fn, "env_ids", env_ids, 4, true)))
    return rc;
  if (none) return SF_OK;
  DeltaArgs g = args_of(cfg, q, k, v, log_decay, beta, done);
  g.o = o;
  // a thread has four columns; rows of a multiple of four floats are read 16 bytes at a time
  int lanes_log2 = 0;
  while ((4 << lanes_log2) < cfg->dv) ++lanes_log2;
  if (lanes_log2 < 4) lanes_log2 = 4;  // (256 threads then have 16 rows each of at most 256)
  const bool vec = cfg->dv % 4 == 0;
  const auto kern = cfg->dtype == SF_DTYPE_BF16 ? (vec ? delta_step_kernel<SF_DTYPE_BF16, true> : delta_step_kernel<SF_DTYPE_BF16, false>)
                                                : (vec ? delta_step_kernel<SF_DTYPE_FP32, true> : delta_step_kernel<SF_DTYPE_FP32, false>);
  kern<<<(unsigned)(cfg->N * cfg->H), kThreads, 0, reinterpret_cast<hipStream_t>(hip_stream)>>>(g, state_table, n_env, env_ids, cfg->H / cfg->Hk,
                                                                                            lanes_log2);
  return launched(fn, hipGetLastError());
}
