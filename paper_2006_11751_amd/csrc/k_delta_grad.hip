// The gradients of the gated delta rule, chunk by chunk (k_delta.hip has the formulas and what goes before).
//
// A chunk's workgroup keeps all it makes in LDS and registers: q, k, v, do, both states and the chunk's matrices are read once, the
// gradients written once.  At 2048 rows of 32 steps, 8 heads of 64, bf16, that is 1.28 GB, 240 us at a copy's rate; it takes 436 us (2.9 TB/s).
// Bound by its chain: a dozen parts that each wait for the one before through LDS and a barrier, 42 thousand cycles, which only other workgroups
// of the CU fill.  (The vector units have an instruction half of the time, a third of them splits into bf16 terms, the matrix units a
// quarter.)  So LDS counts: 51 KB with 64 columns in bf16 are 3 workgroups a CU, with 2 it takes 536 us; and of 128 columns v
// leaves LDS before z comes, for 2 a CU.  Sizes are arguments: as constants the compiler kept all their offsets at once and spilled, 788 us.
// fp32, 64 rows: 29 us, 1024 steps of 8 rows, 8 heads of 128, bf16: 129 us of 330 (the others are the sweeps').
#include "sf_delta.h"
#include "sf_internal.h"

namespace sf {

namespace {

template <int DTYPE, int D>
struct GradLds {
  static constexpr int kPitch = Pitch<DTYPE, D>::value, kTile = C * kPitch, kPitchF = (D + 4) * 4, kTileF = C * kPitchF;
  static constexpr int kWaves = D / 16, kThreads = 64 * kWaves;
  // q, k, do, v; u and z in fp32, before them slabs of the states, and with 128 columns in the place of z first v (two workgroups a CU
  // then); A^T, P^T and T, which make room for dP D and its like as operands
  static constexpr bool kShared = D == 128;
  static constexpr int kU = (kShared ? 3 : 4) * kTile, kZ = kU + kTileF, kV = kShared ? kZ : 3 * kTile, kA = kZ + kTileF, kP = kA + C * kMat * 4, kT = kP + C * kMat * 4,
                       kOperand = 4096, kM = kA;  // [3] of two terms (or halves) of 2 x 64 lanes x 16 bytes
  static_assert(3 * kOperand <= 3 * C * kMat * 4 && kTile <= kTileF, "operands in the matrices' place, v in that of z");
  static constexpr int kSteps = kT + C * kMat * 4, kFlag = kSteps + (int)sizeof(Steps);
  static constexpr int kSums = kFlag + 32;
  static constexpr int kSumRows = 2 * kWaves + (kWaves == 4 ? 4 : 8) + 1;  // of C numbers
  static constexpr int kBytes = kSums + kSumRows * C * 4;
};

// All gradients of one chunk, given the states S that enters it and R behind it: one workgroup for each (row, head, chunk), a wave for 16
// columns of v and then for 16 of k.
// ALONE: the only chunk, whose products are made here by the first eight waves (of four: each) and T by the last one (else they are
// read).  VEC: all arrays are read in 16-byte pieces.
template <int DTYPE, int D, bool ALONE, bool VEC>
__global__ __launch_bounds__(4 * D, DTYPE == SF_DTYPE_FP32 ? 2 : D == 64 ? 3 : 4) void delta_grad_kernel(DeltaArgs g) {
  typedef Num<DTYPE> M;
  typedef GradLds<DTYPE, D> L;
  constexpr int W = M::kPieceWords, ND = D / 16, kRow8 = D / 8, kT = L::kThreads;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  // (workgroups go round the XCDs: 16 neighbours, whose rows of a step are neighbours too, for each)
  const unsigned which = (blockIdx.x & ~127u) + (blockIdx.x & 7) * 16 + ((blockIdx.x >> 3) & 15);
  const int chunk = (int)g.rows.of(which), bh = (int)(which - (unsigned)chunk * (g.N * g.H));
  if (chunk >= g.chunks) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h);
  const int dk = g.k.d, dv = g.v.d, t0 = chunk * C, valid = min(C, g.T - t0);
  auto base = [&](const Strided& a) { return (const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes; };
  unsigned char *const tq = lds, *const tk = lds + L::kTile, *const to = lds + 2 * L::kTile, *const tv = lds + L::kV;
  float *const mU = (float*)(lds + L::kU), *const mZ = (float*)(lds + L::kZ), *const mA = (float*)(lds + L::kA), *const mP = (float*)(lds + L::kP),
               *const mT = (float*)(lds + L::kT);
  constexpr int kF = D + 4;
  constexpr bool kF32 = DTYPE == SF_DTYPE_FP32;
  int* const flag = (int*)(lds + L::kFlag);  // by waves
  Steps& steps = *(Steps*)(lds + L::kSteps);
  // by waves: sums over their columns for each step; by tiles: of dP P + dA A along its rows and columns; a number of each wave
  float *const sum_b = (float*)(lds + L::kSums), *const sum_g = sum_b + L::kWaves * C, *const sum_m = sum_g + L::kWaves * C, *const sum_1 = sum_m + (L::kWaves == 4 ? 4 : 8) * C;

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
      const unsigned at = c < dv ? (unsigned)(row * dv + c) * 4 : kOutside;  // (rows past dk lie past the end)
      ns[p] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_s, at, 0, 0));
      nr[p] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from_r, at, 0, 0));
      if (c + 4 > dv)  // (the next row's numbers)
#pragma unroll
        for (int i = 1; i < 4; ++i)
          if (c + i >= dv) ns[p][i] = nr[p][i] = 0.0f;
    }
  };
  request(0);
  float test = 0.0f;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    put_piece<DTYPE>(a == 0 ? tq : a == 1 ? tk : a == 2 ? tv : to, L::kPitch, w[a], tid, kRow8);
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
  const int ep_before = __shfl_up(my_ep, 1);  // (by all lanes: one that does not take part gives nothing)
  const unsigned begin = (unsigned)__ballot(lane < valid && my_ep != (lane ? ep_before : 0));
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
        acc = decayed(steps, acc, I, J, true, strict, 1.0f, li, lg);
      }
      *(f32x4*)(to_matrix + (16 * J + li) * kMat + 16 * I + 4 * lg) = acc;  // [j][i]
    };
    if (wave < 4) product(tk, mA, true);
    if (L::kWaves == 4 || wave >= 4) product(tq, mP, false);
  }

  // this wave's columns of v and do
  typename M::Raw vt, ot;
  auto own_columns = [&]() {
    vt = columns<DTYPE>(tv, L::kPitch, y0, 4, li, lg);
    ot = columns<DTYPE>(to, L::kPitch, y0, 4, li, lg);
  };
  if constexpr (L::kShared) {
    own_columns();
    __syncthreads();  // v makes room
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
    const typename M::Sum st = three_terms<DTYPE>(xs), rt = three_terms<DTYPE>(xr);
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
    // dP and dA [i][j] lie where A^T and P^T [j][i] have nothing; dP's diagonal behind the rows
    auto dP = [&](int i, int j) -> float& { return mP[i * kMat + (i == j ? C : j)]; };
    auto dA = [&](int i, int j) -> float& { return mA[i * kMat + j]; };
    const unsigned char* const v_at = base(g.v) + (int64_t)t0 * g.v.st * M::kBytes;
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
      if (j > i) continue;
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
        e = M::element(v_at + (i * g.v.st + tid) * M::kBytes) - ks;
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
      if (j <= i) dP(i, j) = p;  // (without the scale, which is in P)
      if (j < i) dA(i, j) = a;
    }
    __syncthreads();
    if (tid < valid) {
      float s = sum_g[tid];
      for (int j = 0; j <= tid; ++j)
        if (steps.ep[j] == steps.ep[tid])
          s += dP(tid, j) * mP[j * kMat + tid] + (j < tid ? dA(tid, j) * mA[j * kMat + tid] : 0.0f);
      for (int i = tid; i < valid; ++i)
        if (steps.ep[i] == steps.ep[tid])
          s -= dP(i, tid) * mP[tid * kMat + i] + (i > tid ? dA(i, tid) * mA[tid * kMat + i] : 0.0f);
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
          q += g.scale * dP(t, j) * d * at(tk, j, x);
          if (j < t) k += dA(t, j) * d * at(tk, j, x);
        }
      for (int i = t; i < valid; ++i)
        if (steps.ep[i] == steps.ep[t]) {
          const float d = decay(i, t);
          k += g.scale * dP(i, t) * d * at(tq, i, x);
          if (i > t) k += dA(i, t) * d * at(tk, i, x);
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
    if constexpr (!L::kShared) own_columns();
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
      f[t] = M::mma(three_terms<DTYPE>(ps), ot, kr[t]);
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
      const typename M::Sum zt = three_terms<DTYPE>(zs), dt = three_terms<DTYPE>(os);
      const auto to_state = buffer(g.dstate0 + (size_t)bh * state, (unsigned)state * 4);
      const unsigned y_at = y < dv ? (unsigned)(8 * lg * dv + y) * 4 : kOutside;
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
        const auto ut = three_terms<DTYPE>(rows8(mU, 16 * J + li, s).x);
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
  auto store_dv = [&](const float* x) {
    if (row8 >= valid) return;
    unsigned piece[W];
    if constexpr (kF32) {
      __builtin_memcpy(piece, x, 32);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) piece[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    }
    store(g.dv, (t0 + row8) * step_v + head_v + col8, dv, piece);
  };
  // In bf16 u and z are kept from here as the two terms that they enter the products of dk with, else each wave would split all of them
  // (32 steps of 2048 rows, 8 heads of 64: 441 us, so 436; 1024 steps of 8 rows, 8 heads of 128, with the sweeps 337 and 332).
  float* const at_z = mZ + row8 * kF + col8;
  if constexpr (!kF32) {
    float* const at_u = mU + row8 * kF + col8;
    float z8[8], u8[8];
    __builtin_memcpy(z8, at_z, 32);
    __builtin_memcpy(u8, at_u, 32);
    store_dv(z8);
    const typename M::Out zt = M::out_terms(z8), ut = M::out_terms(u8);
    *(u32x4*)at_z = zt.t[0];
    *(u32x4*)(at_z + 4) = zt.t[1];
    *(u32x4*)at_u = ut.t[0];
    *(u32x4*)(at_u + 4) = ut.t[1];
  }
  // (rows of tile I from tile J, less columns of tile J from tile I: both halves of the waves add up behind the barrier)
  float* const tile_sums = sum_m;
  if (L::kWaves == 4) {
    if (li == 0) *(f32x4*)(tile_sums + J * C + 16 * I + 4 * lg) = row_sums;
    if (lg == 0) tile_sums[2 * C + I * C + 16 * J + li] = col_sum;
  } else {
    float* const mine = wave < 4 ? tile_sums : tile_sums + 4 * C;
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
      add(tile_sums);
      add(tile_sums + 4 * C);
    }
    const float d = decay_gradient(i == valid - 1 ? s + rest : s);
    if (lane < valid) {
      g.dbeta[step_at + (int64_t)lane * g.N * g.H] = b;
      g.dlog_decay[step_at + (int64_t)lane * g.N * g.H] = d;
    }
  }

  auto terms8 = [&](const float* tile, int row, int s) {  // of rows8
    if constexpr (kF32) {
      return M::out_terms(rows8(tile, row, s).x);
    } else {
      const u32x4* const at = (const u32x4*)(tile + row * kF + 32 * s + 8 * lg);
      return typename M::Out{{at[0], at[1]}};
    }
  };
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
        zs[t] = mma_oo<DTYPE>(st, terms8(mZ, i, s), zs[t]);
        us[t] = mma_oo<DTYPE>(rt, terms8(mU, i, s), us[t]);
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
  // out by whole rows, through the places of q and k
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
  if (kF32 || !g.f32) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      unsigned piece[W];
#pragma unroll
      for (int i = 0; i < W; i += 4) *(u32x4*)(piece + i) = *(const u32x4*)(lds + a * L::kTile + row8 * L::kPitch + col8 * M::kBytes + 4 * i);
      store(a == 0 ? g.dq : g.dk, (t0 + row8) * step_k + head_k + col8, dk, piece);
    }
  }
  if constexpr (kF32) store_dv(at_z);
}

template <int DTYPE, int D, bool ALONE, bool VEC>
hipError_t launch_grad(const DeltaArgs& g, hipStream_t st) {
  const auto kern = delta_grad_kernel<DTYPE, D, ALONE, VEC>;
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
  return g.q.vec && g.k.vec && g.v.vec && g.d_o.vec ? launch_grad<DTYPE, D, ALONE, true>(g, st) : launch_grad<DTYPE, D, ALONE, false>(g, st);
}
template <int DTYPE, int D>
hipError_t launch_grad(const DeltaArgs& g, hipStream_t st) {
  return g.chunks == 1 ? launch_grad<DTYPE, D, true>(g, st) : launch_grad<DTYPE, D, false>(g, st);
}
}  // namespace

hipError_t delta_gradients(const sf_deltarule_config* c, const DeltaArgs& g, hipStream_t st) {
  const bool wide = c->dk > 64 || c->dv > 64;
  if (c->dtype == SF_DTYPE_BF16) return wide ? launch_grad<SF_DTYPE_BF16, 128>(g, st) : launch_grad<SF_DTYPE_BF16, 64>(g, st);
  return wide ? launch_grad<SF_DTYPE_FP32, 128>(g, st) : launch_grad<SF_DTYPE_FP32, 64>(g, st);
}

}  // namespace sf
