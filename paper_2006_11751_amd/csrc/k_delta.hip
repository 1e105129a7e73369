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
// a chunk is tested: one with a NaN or an infinity is taken step by step, by each wave for its own columns (the gradients': number by number).
#include <math.h>

#include <algorithm>

#include "sf_delta.h"
#include "sf_internal.h"

namespace sf {

namespace {

template <int DTYPE, int D, int NT>
struct SweepLds {
  static constexpr int kPitch = Pitch<DTYPE, D>::value, kPitchV = Pitch<DTYPE, DV * NT>::value;
  static constexpr int kK = C * kPitch, kV = 2 * C * kPitch, kP = kV + C * kPitchV, kT = kP + C * kMat * 4, kSteps = kT + C * kMat * 4,
                       kFlag = kSteps + (int)sizeof(Steps), kA = kFlag + 16, kBytes = kA, kBytesAlone = kA + C * kMat * 4;
};

// The matrices of every chunk, for the sweeps and the gradients: a wave makes one chunk's.  They do not depend on a state, so that all
// are made at once and the sweeps, whose chunks wait for one another, only read them: 9 KB a chunk (backwards 13) in fp32.  bf16, 128 columns of
// k: 4096 chunks 21 us, 8192 30 to 35 us, of which the products are little and a wave's chain (read, decays, substitution, write) most.
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

// Where element (x, y) of what a piece makes of a state lies: tiles of 16 x 16, of which a lane of the join has four neighbours of a row.
__host__ __device__ inline int up16(int d) { return (d + 15) & ~15; }
__host__ __device__ inline int64_t through_size(int dk) { return (int64_t)up16(dk) * up16(dk); }
__device__ inline int through_at(int dk, int x, int y) { return ((x >> 4) * (up16(dk) >> 4) + (y >> 4)) * 256 + ((y & 15) >> 2) * 64 + (x & 15) * 4 + (y & 3); }

enum Sweep { kResults = 0, kStates = 1, kBack = 2 };

// A workgroup of four waves goes over the chunks of one (row, head), or of one piece of T, for 64 NT columns of v, of which a wave owns 16 NT: its
// part of the state stays in registers as the accumulator of the update.  The products are arranged so that accumulators feed the next
// product without a shuffle: a 16x16 accumulator holds rows 4 lg .. 4 lg + 3 of one column per lane (lg = lane / 16), two of them are
// the eight K-slots of an operand of 16x16x32, and the other operand follows the same numbering of the K axis.
// Bound by the length of a chunk's chain, not by memory or the matrix units: k S (ks), T and its correction, o, the update of S, each of which
// waits for the one before: 7.2 thousand cycles a chunk with 16 columns a wave, 9.7 with 32 (k S 2.5, o 2.2, S 1.8, the rest staging and
// steps).  What fills the waits is other workgroups, so registers count, but a spill lies in the chain: bounds of 3 workgroups a CU with 64 columns of k and
// 2 with 128 spill nothing with one tile; of 4 and 3 they spilled up to 39 registers, forwards, gradients, us so | before: fp32, 512 steps of 8 heads, 16 rows
// of 64 columns 67 | 77, 190 | 203, 8 rows of 128 95 | 117, 289 | 302; bf16 the same within 2 %.  With two tiles and 128 columns of k, at 256 registers, fp32 spills 8 to 38 of
// them, bf16 with columns that are no whole tiles 15 to 28; a bound of one workgroup, which spills none, is slower (fp32, 64 rows 377 us, so 334).
// 512 steps of 64 rows, 8 heads of 128, bf16: 120 us, the vector units busy 0.51 of it, the matrix units 0.40.  A single chunk is bound by memory instead
// where rows are many: 32 steps of 2048 rows, 8 heads of 64, bf16 204 us (4.0 TB/s), of 128 569 (4.7); fp32 276 and 898.  With few rows it is the
// launch and one chain: 64 rows 10.1 us.
//   kResults: o and the last state;  kStates: the states that enter the chunks, or the last one of a piece;  kBack: R, from the last chunk to the first
// ALONE: of one chunk, whose products are made here, a tile by each wave, and T by the last one (else they are read).
template <int DTYPE, int D, int NT, int SWEEP, bool ALONE, int KNOWN>
__global__ __launch_bounds__(kThreads, KNOWN == kAny || NT == 2 || D == 128 ? 2 : 3) void delta_sweep_kernel(DeltaArgs g) {
  typedef Num<DTYPE> M;
  typedef SweepLds<DTYPE, D, NT> L;
  constexpr int W = M::kPieceWords, NP = C * D / 8 / kThreads, ND = D / 16, kRow = D / 8, kRowV = DV * NT / 8;
  constexpr bool kQ = SWEEP != kStates, kUp = SWEEP != kBack, VEC = KNOWN != kAny, WHOLE = KNOWN == kWhole;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  // the blocks of one (row, head) read the same arrays: one after another on one XCD (workgroups go to the 8 in turn)
  const unsigned round = g.round.of(blockIdx.x), in_round = blockIdx.x - round * (8 * g.blocks), turn8 = in_round >> 3;
  const int bh = (int)(round * 8 + (in_round & 7));
  if (bh >= g.N * g.H) return;
  // a piece has blocks of the identity's columns besides: what a state that enters becomes
  const bool identity = (int)turn8 >= g.blocks_v;
  const int v_block = DV * NT * ((int)turn8 - (identity ? g.blocks_v : 0)), seg = blockIdx.y;
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
  StepIn in = {};
  if constexpr (ALONE) in = read_step(g, n, h, 0, g.T, lane);

  const int v0 = v_block + 16 * NT * wave;  // this wave's columns of v, by tiles of 16; this lane's are v0 + 16 c + li
  const bool has_v = WHOLE || v0 < dv;
  auto has_k = [&](int s) { return WHOLE || 32 * s < dk; };
  // row of tile t of the state (two tiles are 32 rows: eight neighbours per lane group)
  auto col_k = [&](int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); };
  f32x4 S[NT][ND];
  unsigned y_at[NT];
#pragma unroll
  for (int c = 0; c < NT; ++c) y_at[c] = WHOLE || v0 + 16 * c + li < dv ? (unsigned)(8 * lg * dv + v0 + 16 * c + li) * 4 : kOutside;  // (rows past dk lie past the end)
  {
    const float* s = nullptr;
    if (g.piece) s = nullptr;
    else if (g.n_seg > 1) s = g.seg_state + ((size_t)bh * g.n_seg + seg) * dk * dv;
    else if (g.s_in) s = g.s_in + (size_t)bh * dk * dv;
    const auto from = buffer(s, s ? (unsigned)(dk * dv) * 4 : 0);
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int a = 0; a < ND; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          S[c][a][r] = load_float(from, y_at[c], (32 * (a >> 1) + 4 * (a & 1) + r) * dv * 4);
          if (identity) S[c][a][r] = col_k(a, 4 * lg + r) == v0 + 16 * c + li ? 1.0f : 0.0f;
        }
  }
  auto store_state = [&](float* s) {
    int row = dv * 4;
    asm volatile("" : "+s"(row));  // (else the rows' offsets are kept in registers from here to there)
    const auto to = buffer(s, (unsigned)(dk * dv) * 4);
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int a = 0; a < ND; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)S[c][a][r]), to, y_at[c], (32 * (a >> 1) + 4 * (a & 1) + r) * row, 0);
  };

  // the chunk that is on its way: its rows, matrices and steps
  unsigned nq[NP][W], nk[NP][W], nv[NT][W];
  f32x4 n_p, n_t, n_steps;
  unsigned at_q[NP], at_k[NP], at_v[NT];
  if constexpr (VEC) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int piece = tid + p * kThreads, r = piece / kRow, col = piece % kRow * 8;
      at_q[p] = WHOLE || col < dk ? (unsigned)(r * (int)g.q.st + col) * M::kBytes : kOutside;
      at_k[p] = WHOLE || col < dk ? (unsigned)(r * (int)g.k.st + col) * M::kBytes : kOutside;
    }
#pragma unroll
    for (int p = 0; p < NT; ++p) {
      const int piece = tid + p * kThreads, col = v_block + piece % kRowV * 8;
      at_v[p] = (WHOLE || col < third.d) && !identity ? (unsigned)(piece / kRowV * (int)third.st + col) * M::kBytes : kOutside;
    }
  }
  const int first = t_begin / C, last = (t_end - 1) / C, begin_c = kUp ? first : last, way = kUp ? 1 : -1;  // chunks
  constexpr int kMade = made_words(!kUp);  // (kStates: forwards' or backwards')
  const int made_size = SWEEP == kStates && g.back ? made_words(true) : kMade;
  // where the next chunk lies: its rows, and what is made of it
  const unsigned char *at_rows_q = qb + (int64_t)begin_c * C * g.q.st * M::kBytes, *at_rows_k = kb + (int64_t)begin_c * C * g.k.st * M::kBytes,
                      *at_rows_v = vb + (int64_t)begin_c * C * third.st * M::kBytes;
  const int64_t step_q = (int64_t)way * C * g.q.st * M::kBytes, step_k = (int64_t)way * C * g.k.st * M::kBytes, step_v = (int64_t)way * C * third.st * M::kBytes;
  const float* at_made = g.made + ((size_t)bh * g.chunks + begin_c) * made_size;
  auto request = [&](int c) {
    const int t0 = c * C, valid = min(C, g.T - t0);
    if constexpr (VEC) {
      auto get = [&](unsigned* w, const unsigned char* rows, int r, unsigned at) { load_words<W>(w, buffer(rows, kWholeBuffer), r < valid ? at : kOutside); };
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if constexpr (kQ) get(nq[p], at_rows_q, (tid + p * kThreads) / kRow, at_q[p]);
        get(nk[p], at_rows_k, (tid + p * kThreads) / kRow, at_k[p]);
      }
#pragma unroll
      for (int p = 0; p < NT; ++p) get(nv[p], at_rows_v, (tid + p * kThreads) / kRowV, at_v[p]);
      at_rows_q += step_q;
      at_rows_k += step_k;
      at_rows_v += step_v;
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if constexpr (kQ) fetch<DTYPE>(nq[p], g.q, qb, t0, valid, tid + p * kThreads, kRow, 0);
        fetch<DTYPE>(nk[p], g.k, kb, t0, valid, tid + p * kThreads, kRow, 0);
      }
#pragma unroll
      for (int p = 0; p < NT; ++p) fetch<DTYPE>(nv[p], third, vb, t0, identity ? 0 : valid, tid + p * kThreads, kRowV, v_block);
    }
    if constexpr (!ALONE) {
      n_t = *(const f32x4*)(at_made + 4 * tid);
      if constexpr (kQ) n_p = *(const f32x4*)(at_made + kDense + 4 * tid);
      if (tid < kStepWords / 4) n_steps = *(const f32x4*)(at_made + made_size - kStepWords + 4 * tid);
      at_made += way * made_size;
    }
  };
  // of four neighbours of an output row, tile c of the columns; a tile is 16 columns on
  unsigned at_o[2];
#pragma unroll
  for (int I = 0; I < 2; ++I) at_o[I] = (unsigned)((16 * I + li) * (g.N * g.H * dv) + v0 + 4 * lg) * M::kBytes;

  if (t_begin < t_end) request(begin_c);
  bool any_begin = false;
  for (int c = kUp ? first : last, turn = 0; t_begin < t_end && (ALONE ? turn == 0 : kUp ? c <= last : c >= first); c += kUp ? 1 : -1, turn ^= 1) {
    const int t0 = c * C, valid = min(C, g.T - t0);
    if (SWEEP != kResults && g.kept && has_v) store_state(g.kept + ((size_t)bh * g.chunks + c) * ((size_t)dk * dv));
    __syncthreads();  // the chunk before has been read
    float test = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if constexpr (kQ) put_piece<DTYPE>(tq, L::kPitch, nq[p], tid + p * kThreads, kRow);
      put_piece<DTYPE>(tk, L::kPitch, nk[p], tid + p * kThreads, kRow);
      if constexpr (SWEEP == kBack) test = finite_test<DTYPE>(nq[p], test);
      test = finite_test<DTYPE>(nk[p], test);
    }
#pragma unroll
    for (int p = 0; p < NT; ++p) {
      put_piece<DTYPE>(tv, L::kPitchV, nv[p], tid + p * kThreads, kRowV);
      test = finite_test<DTYPE>(nv[p], test);
    }
    if constexpr (!ALONE) {
      const int to = tid / 8 * kMat + tid % 8 * 4;
      *(f32x4*)(mT + to) = n_t;
      if constexpr (kQ) *(f32x4*)(mP + to) = n_p;
      if (tid < kStepWords / 4) *(f32x4*)((float*)&steps + 4 * tid) = n_steps;
    } else if (wave == 0) {
      put_steps(steps, in, (unsigned)__ballot(begins(in)), valid, lane);
    }
    if (test != 0.0f) flag[turn] = 1;
    __syncthreads();
    if constexpr (ALONE) {
      // A^T and P, a tile of 16 x 16 of each a wave
      const int I = wave >> 1, J = wave & 1;
      float* const mA = (float*)(lds + L::kA);
      f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, p = a;
      if (J <= I) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
          if (!has_k(s)) continue;
          const int at = (32 * s + 8 * lg) * M::kBytes;
          const auto ki = M::row(tk + (16 * I + li) * L::kPitch + at), kj = M::row(tk + (16 * J + li) * L::kPitch + at);
          a = M::mma(ki, kj, a);                                                 // [i][j]
          p = M::mma(kj, M::row(tq + (16 * I + li) * L::kPitch + at), p);  // [j][i]
        }
        a = decayed(steps, a, I, J, true, true, 1.0f, li, lg);
        p = decayed(steps, p, J, I, false, false, g.scale, li, lg);
      }
      *(f32x4*)(mA + (16 * J + li) * kMat + 16 * I + 4 * lg) = a;
      *(f32x4*)(mP + (16 * I + li) * kMat + 16 * J + 4 * lg) = p;
      __syncthreads();
      if (wave == 3) invert(mA, steps.beta, mT, lane);
    }
    if constexpr (!ALONE) {
      if (c != (kUp ? last : first)) request(kUp ? c + 1 : c - 1);
    }
    // (marks of begins are where the episode's number grows)
    const int my_ep = steps.ep[lane & (C - 1)];
    const float my_steps = fmaf(steps.gh[lane & (C - 1)], 0.0f, steps.beta[lane & (C - 1)] * 0.0f);
    const int e_last = __builtin_amdgcn_readlane(my_ep, valid - 1);
    const bool marked = e_last != 0;
    any_begin = any_begin || marked;
    const bool odd = flag[turn] != 0 || __any(my_steps != 0.0f);
    if (tid == 0) flag[turn ^ 1] = 0;  // (read by all before the barrier above)
    if (!has_v) {
      if constexpr (ALONE) __syncthreads();
      continue;
    }

    // what the state gives the steps: k S, and q S
    f32x4 ks[NT][2] = {}, qs[NT][2] = {};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      if (!has_k(s)) continue;
      typename M::Sum st[NT];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        float x[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = S[c][2 * s][r];
          x[4 + r] = S[c][2 * s + 1][r];
        }
        st[c] = three_terms<DTYPE, SWEEP == kResults>(x);
      }
#pragma unroll
      for (int J = 0; J < 2; ++J) {
        const int at = (16 * J + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes;
        const auto kk = M::row(tk + at);
#pragma unroll
        for (int c = 0; c < NT; ++c) ks[c][J] = M::mma(kk, st[c], ks[c][J]);  // [step][y]
        if constexpr (SWEEP == kResults) {
          const auto qq = M::row(tq + at);
#pragma unroll
          for (int c = 0; c < NT; ++c) qs[c][J] = M::mma(leading<DTYPE>(st[c]), qq, qs[c][J]);  // [y][step]
        }
      }
    }
    if constexpr (ALONE) __syncthreads();  // T is there
    // (of a state with something not finite every product is not finite: that an episode begins in the chunk does not stop it)
    float state_test = 0.0f;
#pragma unroll
    for (int c = 0; c < NT; ++c) state_test = fmaf(ks[c][0][0], 0.0f, state_test);
    if (odd || (marked && __any(state_test != 0.0f))) {
      // Step by step, each wave for its columns, so that nothing that is not finite meets a masked zero.
      auto element = [&](const unsigned char* tile, int pitch, int i, int x) { return M::element(tile + i * pitch + x * M::kBytes); };
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const int y = v0 + 16 * c + li;
        float s[ND][4];
#pragma unroll
        for (int a = 0; a < ND; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[a][r] = S[c][a][r];
        for (int at = 0; at < valid; ++at) {
          const int i = kUp ? at : valid - 1 - at;
          const StepIn in = read_step(g, n, h, t0 + i, 1, lane & 0);
          const bool begin = begins(in);
          const float keep = exp2f(in.ld * 1.44269504f), v = element(tv, L::kPitchV, i, y - v_block);
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
        for (int a = 0; a < ND; ++a) S[c][a] = f32x4{s[a][0], s[a][1], s[a][2], s[a][3]};
      }
      continue;
    }
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const float keep = marked ? 0.0f : steps.enter[valid - 1];
    f32x4 e4[2], w4[2], b4[2];
#pragma unroll
    for (int J = 0; J < 2; ++J) {
      const int j = 16 * J + 4 * lg;
      e4[J] = *(const f32x4*)(steps.enter + j);
      w4[J] = *(const f32x4*)(steps.leave + j);
      b4[J] = *(const f32x4*)(steps.beta + j);
    }
    // columns of the third array: K-slots 0..3 are steps 4 lg .., 4..7 are 16 further on
    typename M::Raw vt[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) vt[c] = columns<DTYPE>(tv, L::kPitchV, 16 * (NT * wave + c), 4, li, lg);
    // (a state that is not finite is here only in a chunk that it all reaches: a factor of zero leaves out a finite number)
    typename M::Sum add_k[NT], add_q[NT];  // what is multiplied with k^T, and backwards with q^T, for the state
    if constexpr (kUp) {
      float us[NT][8];
      const f32x4 t0_ = *(const f32x4*)(mT + li * kMat + 4 * lg);
      const Slots t1 = slots_of(mT, 16 + li, lg);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        float v[8];
        M::values(vt[c], v);
        f32x4 x[2], e[2];
#pragma unroll
        for (int J = 0; J < 2; ++J)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[J][r] = v[4 * J + r] - e4[J][r] * ks[c][J][r];
        e[0] = mm4(t0_, x[0], zero);
        e[1] = mm4(t1.b, x[1], mm4(t1.a, x[0], zero));
#pragma unroll
        for (int J = 0; J < 2; ++J)
#pragma unroll
          for (int r = 0; r < 4; ++r) us[c][4 * J + r] = b4[J][r] * e[J][r];
      }
      if constexpr (SWEEP == kResults) {
        typename M::Out uo[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) uo[c] = M::out_terms(us[c]);
        const auto to = buffer((unsigned char*)g.o + (((int64_t)t0 * g.N + n) * g.H + h) * dv * M::kBytes, kWholeBuffer);
#pragma unroll
        for (int I = 0; I < 2; ++I) {
          const int i = 16 * I + li;
          const float from_state = g.scale * steps.enter[i];
          const Slots p = slots_of(mP, i, lg);
          float ps[8];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            ps[r] = p.a[r];
            ps[4 + r] = p.b[r];
          }
          const typename M::Out pt = M::out_terms(ps);
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            const f32x4 own = mma_oo<DTYPE>(uo[c], pt, from_state * qs[c][I]);  // [y][i]
            const int yo = v0 + 16 * c + 4 * lg;
            if constexpr (VEC) {
              const unsigned at = i < valid && (WHOLE || yo < dv) ? at_o[I] + 16 * c * M::kBytes : kOutside;
              if constexpr (DTYPE == SF_DTYPE_BF16) __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(own[0], own[1]), pack_bf16(own[2], own[3])}, to, at, 0, 0);
              else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, own), to, at, 0, 0);
            } else {
              if (i >= valid) continue;
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
      }
#pragma unroll
      for (int c = 0; c < NT; ++c) {
#pragma unroll
        for (int J = 0; J < 2; ++J)
#pragma unroll
          for (int r = 0; r < 4; ++r) us[c][4 * J + r] *= w4[J][r];
        add_k[c] = three_terms<DTYPE>(us[c]);
      }
    } else {
      // f, and of it z = T^T beta f
      typename M::Sum pt[2];
#pragma unroll
      for (int J = 0; J < 2; ++J) {
        const Slots p = slots_of(mP, 16 * J + li, lg);
        float ps[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ps[r] = g.scale * p.a[r];
          ps[4 + r] = g.scale * p.b[r];
        }
        pt[J] = three_terms<DTYPE>(ps);
      }
      const Slots c0 = slots_down(mT, li, lg), c1 = slots_down(mT, 16 + li, lg);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        f32x4 f[2], z[2];
#pragma unroll
        for (int J = 0; J < 2; ++J) f[J] = b4[J] * M::mma(pt[J], vt[c], w4[J] * ks[c][J]);
        z[0] = mm4(c0.b, f[1], mm4(c0.a, f[0], zero));
        z[1] = mm4(c1.b, f[1], zero);
        float v[8], zs[8], os[8];
        M::values(vt[c], v);
#pragma unroll
        for (int J = 0; J < 2; ++J)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            zs[4 * J + r] = -e4[J][r] * z[J][r];
            os[4 * J + r] = g.scale * e4[J][r] * v[4 * J + r];
          }
        add_k[c] = three_terms<DTYPE>(zs);
        add_q[c] = three_terms<DTYPE>(os);
      }
    }
#pragma unroll
    for (int a = 0; a < ND; ++a) {
#pragma unroll
      for (int c = 0; c < NT; ++c) S[c][a] *= keep;
      if (!has_k(a / 2)) continue;
      const typename M::Raw kt = columns<DTYPE>(tk, L::kPitch, col_k(a, 0), 8, li, lg);
#pragma unroll
      for (int c = 0; c < NT; ++c) S[c][a] = M::mma(kt, add_k[c], S[c][a]);
      if constexpr (!kUp) {
        const typename M::Raw qt = columns<DTYPE>(tq, L::kPitch, col_k(a, 0), 8, li, lg);
#pragma unroll
        for (int c = 0; c < NT; ++c) S[c][a] = M::mma(qt, add_q[c], S[c][a]);
      }
    }
  }
  if (!has_v) return;
  if (g.piece) {
    const size_t at = (size_t)bh * g.n_seg + seg;
    if (identity) {
      // by tiles of 16 x 16 as the join reads them; for the gradients its transpose besides
      float* const to = g.seg_through + at * through_size(dk) * (g.back ? 2 : 1);
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int a = 0; a < ND; ++a)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int x = col_k(a, 4 * lg + r), y = v0 + 16 * c + li;
            if (x >= up16(dk) || y >= up16(dk)) continue;
            to[through_at(dk, x, y)] = S[c][a][r];
            if (g.back) to[through_size(dk) + through_at(dk, y, x)] = S[c][a][r];
          }
    } else store_state(g.seg_state + at * dk * dv);
    if (!identity && v_block == 0 && tid == 0) g.seg_begin[at] = any_begin ? 1 : 0;
  } else if (g.s_out && seg == (kUp ? g.n_seg - 1 : 0)) {
    store_state(g.s_out + (size_t)bh * dk * dv);
  }
}

// What enters each piece of T, from the pieces' own states and what they make of one that enters:  S <- M S + own, backwards R <- M^T R + own;
// where an episode begins in the piece, own alone.  A workgroup has 16 columns of one (row, head), a wave 16 rows of the state; the state goes
// round through LDS.  Two pieces' matrices are on their way at a time; on the fp32 matrix instruction, as this is where a state's errors would
// add up.  32 pieces of 8 heads of 128: 49 us, a piece's 1.5 is what a product of 128 x 128 with 16 columns takes after the one before.
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
    const float* const through = g.seg_through + at * through_size(dk) * (g.back ? 2 : 1) + (BACK ? through_size(dk) : 0);
    const auto from_m = buffer(through, (unsigned)through_size(dk) * 4), from_o = buffer(g.seg_state + at * dk * dv, size);
    p.begin = g.seg_begin[at];
    const int tiles = up16(dk) >> 4;
#pragma unroll
    for (int s = 0; s < 8; ++s)
      p.m[s] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                             from_m, wave < tiles && s < tiles ? (unsigned)((wave * tiles + s) * 256 + lane * 4) * 4 : kOutside, 0, 0));
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

// Sums of the gradients of shared heads, of dq and of dk: in [rows][H][d] fp32, out [rows][H / share][d], each in one order.  A thread has
// PER neighbours of a row of d; 2^lanes_log2 threads have a row.  (A gradients kernel that went over the heads of a group would need no sums,
// but has a group's share fewer workgroups, where they are few already.)  Bound by memory: 1024 steps of 8 rows, 8 heads of 128, two on each key, 14 us.
template <int DTYPE, int PER>
__global__ __launch_bounds__(kThreads) void delta_share_kernel(const float* in_q, const float* in_k, void* out_q, void* out_k, int64_t rows, int d, int share,
                                                               int lanes_log2) {
  typedef Num<DTYPE> M;
  const float* const in = blockIdx.y ? in_k : in_q;
  unsigned char* const out = (unsigned char*)(blockIdx.y ? out_k : out_q);
  const int col = (threadIdx.x & ((1 << lanes_log2) - 1)) * PER, in_block = kThreads >> lanes_log2;
  if (col >= d) return;
  for (int64_t row = (int64_t)blockIdx.x * in_block + (threadIdx.x >> lanes_log2); row < rows; row += (int64_t)gridDim.x * in_block) {
    const float* const x = in + row * share * d + col;
    float sum[PER] = {};
    for (int i = 0; i < share; ++i) {
      float y[PER];
      __builtin_memcpy(y, x + (int64_t)i * d, sizeof y);
#pragma unroll
      for (int j = 0; j < PER; ++j) sum[j] += y[j];
    }
    unsigned char* const to = out + (row * d + col) * M::kBytes;
    if constexpr (DTYPE == SF_DTYPE_BF16 && PER == 4) {
      const u32x2 two = {pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
      __builtin_memcpy(to, &two, 8);
    } else if constexpr (PER == 4) {
      __builtin_memcpy(to, sum, 16);
    } else {
      M::store(to, sum[0]);
    }
  }
}

// One step of one (row, head): the state is read and decayed, multiplied with k and q in one go, corrected and written:
//   o = scale (S'^T q + (q . k) u).
// A thread holds four neighbours of every (256 / lanes)-th row, MOST of them, so that all its loads are under way at once and the state
// passes through registers once.  Bound by memory: 2048 rows, 8 heads of 64, 113 us (4.85 TB/s of state read and written; a copy has
// 5.3; 90 us where the same rows come call after call and part of them is still in the last-level cache).  MOST is the smallest of 4, 8 and 16
// that does: with 16 always the registers left half the workgroups a CU, 127 us.  16 rows: 6 us, of which the launch is most.
template <int DTYPE, bool VEC, int MOST>
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
  float x[MOST][4];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
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
  for (int i = 0; i < MOST; ++i) {
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
  for (int i = 0; i < MOST; ++i) {
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

int check(const sf_deltarule_config* c, const char* fn, bool backward = false) {
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
  // (a launch's threads are counted in 32 bits: 64 a chunk forwards, up to 512 backwards, of 128 chunks at a time)
  if ((int64_t)c->T * c->N > INT32_MAX || (int64_t)c->N * c->H > kMostHeads ||
      (int64_t)c->N * c->H * ((c->T + (int64_t)C - 1) / C) > (backward ? 1 << 23 : 1 << 26) - 128) {
    set_error("%s: T * N beyond 2^31 - 1, N * H beyond 2^21, or N * H times chunks of 32 steps beyond %s - 128", fn, backward ? "2^23" : "2^26");
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

// Pieces of T where heads are few: a pass over the pieces with the identity's columns besides, and as many steps in a row to join them as there
// are pieces, for chunks in a row that are fewer by that factor.  Both grow together least at a number of pieces near the root of
// twice the chunks, while the workgroups (w, one for each 64 columns of a head) find CUs that are idle; at w = 128 no number pays for 1024 or 2048 steps (for
// 4096, four pieces save 4 % in bf16, 9 % in fp32).
// us with 1, 4, 8, 16, 32 pieces, bf16, forwards | backwards (H heads over all rows):
//   H x columns, T      w
//    8 x  64, 1024      8    67  45  36  39    -  | 146  103   83   87    -
//    8 x  64, 16384     8   933 436 237 146  119  | 2052 1049 600  392  323
//    8 x 128, 512      16    49  41  40   -    -  | 118  102   97    -    -
//    8 x 128, 4096     16   323 164 102  88  104  | 769  439  302  262  298
//    8 x 128, 16384    16  1270 586 322 221  212  | 3038 1618 1026 774  782
//   32 x  64, 1024     32    68  48  42  50    -  | 165  126  109  124    -
//   64 x  64, 2048     64   133  91  83  93  126  | 356  266  245  273  333
//   32 x 128, 1024     64    90  73  74  93    -  | 267  228  237  283    -
//   32 x 128, 4096     64   336 206 182 190  230  | 1020 747  713  733  855
//  128 x  64, 1024    128    76  82  90 117    -  | 237  246  267  315    -
//   64 x 128, 2048    128   182 184 190 224  335  | 694  716  731  847 1059
// fp32, with 1, 4, 8, 16:
//    8 x  64, 1024      8   109  63  47  46 | 212  144  111  108
//    8 x 128, 4096     16   643 293 173 142 | 1269 721  467  382
//   64 x  64, 2048     64   223 143 133 143 | 542  411  392  419
//   32 x 128, 1024     64   175 120 120 142 | 431  347  344  410
struct Split {
  int n_seg, seg_len;
};
Split split_of(const sf_deltarule_config* c) {
  const int64_t w = (int64_t)c->N * c->H * (std::max(c->dk, c->dv) > DV ? 2 : 1);
  const int chunks = chunks_of(c);
  if (w == 0 || w > 64 || chunks < std::max<int64_t>(16, w / 2)) return Split{1, std::max(1, chunks) * C};
  int want = 1;
  while ((want + 1) * (want + 1) <= 2 * chunks && want + 1 <= 512 / w && want < 32) ++want;
  const int per = (chunks + want - 1) / want;
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
    w.seg_through = align256(lanes * s.n_seg * through_size(c->dk) * (backward ? 8 : 4));
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

template <int DTYPE, int D, int NT, int SWEEP, bool ALONE, int KNOWN>
void launch_sweep(DeltaArgs& g, hipStream_t st) {
  typedef SweepLds<DTYPE, D, NT> L;
  constexpr int bytes = ALONE ? L::kBytesAlone : L::kBytes;
  static_assert(bytes <= 64 * 1024, "no attribute needed");
  const auto blocks = [](int d) { return (d + DV * NT - 1) / (DV * NT); };
  g.blocks_v = blocks(g.v.d);
  g.blocks = g.blocks_v + (g.piece && SWEEP == kStates ? blocks(g.k.d) : 0);
  g.round = divisor(8 * g.blocks);
  const dim3 grid((unsigned)((g.N * g.H + 7) / 8 * 8 * g.blocks), (unsigned)g.n_seg);
  delta_sweep_kernel<DTYPE, D, NT, SWEEP, ALONE, KNOWN><<<grid, kThreads, bytes, st>>>(g);
}
template <int DTYPE, int D, int SWEEP, bool ALONE>
void launch_sweep(DeltaArgs& g, bool vec, hipStream_t st) {
  if (!vec) return launch_sweep<DTYPE, D, 1, SWEEP, ALONE, kAny>(g, st);
  // Two tiles of 16 columns a wave read the chunk's rows and matrices half as often and have two chains of products to fill each other's
  // waits, but half the workgroups; of w workgroups of 64 columns, us with one | two tiles, 512 steps, heads of 128, forwards, gradients:
  //   bf16 w = 256 63 | 82, 262 | 303;  512 87 | 87, 444 | 453;  768 133 | 129, 650 | 657;  1024 165 | 147, 853 | 829;  4096 640 | 584, 3289 | 3262
  //   fp32 w = 256 113 | 167, 436 | 538;  512 174 | 184, 768 | 814;  768 267 | 306, 1142 | 1238;  1024 344 | 334, 1478 | 1496;  4096 1324 | 1261, 5948 | 5892
  // With whole tiles (KNOWN) the bounds of columns fold away.  512 steps of 8 heads, us with | without, forwards, gradients:
  //   bf16 16 rows of 64 44 | 48, 127 | 136;  8 rows of 128 52 | 63, 166 | 185;  64 rows of 128 148 | 152, 833 | 865
  //   fp32 16 rows of 64 67 | 75, 190 | 204;  8 rows of 128 95 | 110, 289 | 323;  64 rows of 128 332 | 354, 1484 | 1492
  if constexpr (!ALONE)
    if (g.v.d > DV && (int64_t)g.N * g.H * g.n_seg * (g.piece && SWEEP == kStates ? 4 : 2) >= 1024) {
      const bool whole = g.k.d == D && g.v.d == 2 * DV && !(g.piece && SWEEP == kStates && D == 64);  // (the identity has D columns)
      return whole ? launch_sweep<DTYPE, D, 2, SWEEP, ALONE, kWhole>(g, st) : launch_sweep<DTYPE, D, 2, SWEEP, ALONE, kPieces>(g, st);
    }
  if (g.k.d == D && g.v.d % DV == 0) launch_sweep<DTYPE, D, 1, SWEEP, ALONE, kWhole>(g, st);
  else launch_sweep<DTYPE, D, 1, SWEEP, ALONE, kPieces>(g, st);
}
template <int SWEEP, bool ALONE = false>
hipError_t sweep(const sf_deltarule_config* c, DeltaArgs g, hipStream_t st) {
  const Strided& third = SWEEP == kBack ? g.d_o : g.v;
  // (a chunk's results in reach of one buffer.  By pieces with addresses of 64 bits in place of that: 32 steps of 2^25 numbers of o 5 % more,
  // fp32, of 2^24, 8 %; 32 steps of 5462 rows of a projection of 1536 columns 3 %, gradients 8 %; 64 steps of those 28 and 11 %)
  const int64_t chunk_bytes = (int64_t)c->N * c->H * c->dv * (c->dtype == SF_DTYPE_BF16 ? 2 : 4) * C;
  const bool vec = g.k.vec && third.vec && (SWEEP == kStates || g.q.vec) &&
                   (SWEEP != kResults || ((reinterpret_cast<uintptr_t>(g.o) & 15) == 0 && chunk_bytes < (int64_t)1 << 31));
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

int launched(const char* fn, hipError_t e) {
  if (e == hipSuccess) return SF_OK;
  set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
  return SF_ERR_DEVICE;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" int64_t sf_deltarule_workspace_bytes(const sf_deltarule_config* cfg, int backward) {
  if (check(cfg, "sf_deltarule_workspace_bytes", backward != 0) != SF_OK) return -1;
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
  int rc = check(cfg, fn, true);
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
  err = delta_gradients(cfg, g, st);
  if (err == hipSuccess && share > 1) {
    const int64_t rows = (int64_t)cfg->T * cfg->N * cfg->Hk;
    const int per = cfg->dk % 4 == 0 ? 4 : 1;
    int lanes_log2 = 0;
    while (per << lanes_log2 < cfg->dk) ++lanes_log2;
    const int64_t in_block = kThreads >> lanes_log2, blocks = std::min<int64_t>((rows + in_block - 1) / in_block, 1 << 14);
    const auto kern = cfg->dtype == SF_DTYPE_BF16 ? (per == 4 ? delta_share_kernel<SF_DTYPE_BF16, 4> : delta_share_kernel<SF_DTYPE_BF16, 1>)
                                                  : (per == 4 ? delta_share_kernel<SF_DTYPE_FP32, 4> : delta_share_kernel<SF_DTYPE_FP32, 1>);
    kern<<<dim3((unsigned)blocks, 2), kThreads, 0, st>>>(part_q, part_k, dq, dk, rows, cfg->dk, share, lanes_log2);
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
  if (lanes_log2 < 4) lanes_log2 = 4;  // (256 threads then have at most 16 rows each)
  const int most = (cfg->dk + (kThreads >> lanes_log2) - 1) / (kThreads >> lanes_log2);  // rows of a thread
  const auto launch = [&](auto dtype, auto vec) {
    constexpr int kType = decltype(dtype)::value;
    constexpr bool kVec = decltype(vec)::value;
    const auto kern = most <= 4 ? delta_step_kernel<kType, kVec, 4> : most <= 8 ? delta_step_kernel<kType, kVec, 8> : delta_step_kernel<kType, kVec, 16>;
    kern<<<(unsigned)(cfg->N * cfg->H), kThreads, 0, reinterpret_cast<hipStream_t>(hip_stream)>>>(g, state_table, n_env, env_ids, cfg->H / cfg->Hk,
                                                                                              lanes_log2);
  };
  const auto by_type = [&](auto vec) {
    if (cfg->dtype == SF_DTYPE_BF16) launch(std::integral_constant<int, SF_DTYPE_BF16>(), vec);
    else launch(std::integral_constant<int, SF_DTYPE_FP32>(), vec);
  };
  if (cfg->dv % 4 == 0) by_type(std::true_type());
  else by_type(std::false_type());
  return launched(fn, hipGetLastError());
}
