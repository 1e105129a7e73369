// The gated feed-forward block (include/sf_memory.h): h = act(x Wg^T) * (x Wu^T), y = h Wd^T, and its gradients.
//
// Every product is C[m][f] = sum_k X[m][k] W[f][k].  An operand lies in memory with k along its rows or with k from row to
// row (the gradients' products take the same arrays the other way round); the latter is transposed by the read that
// takes it out of LDS.  Arrays that cannot be read in whole 16-byte pieces are laid out in the workspace first.  One kernel
// in three forms, all on the 16-bit matrix instruction 32x32x16 with fp32 accumulation:
//   kOne    C itself; two pairs of operands may follow one another in one sum (dx = dg Wg + du Wu)
//   kPair   both projections of one x, activation and product behind them: h
//   kTriple both projections computed again and dy Wd beside them: h, dg = dh u act'(g), du = dh act(g)
// Nothing of the forward pass is kept for the backward pass: g and u in fp32 would be twice the bytes of all other arrays
// together, and rounded they would put a second rounding into dg.
//
// Roundings.  bf16: h, dg and du are rounded to bf16 once (they are operands of the next product), the results once.  fp32:
// an operand is the exact sum of three bf16 numbers, and of the nine products the six largest are added, smallest first,
// as passes over K (what is dropped is 2^-27 of the product); nothing else is rounded to 16 bits.
//
// Tile: four waves, each with up to 256 accumulators per lane, so that a 16-byte operand read feeds four products; K in
// steps of BK through two buffers in LDS, the step after next under way in registers.  In LDS rows along k are 16 bytes
// longer than their numbers (16 neighbours then lie in different banks), rows across k are 16 words mod 64 apart (the
// transposing read takes 32 columns of four rows at once).  What lies past an array's end is read as zero by the
// buffer's bounds check.  Where tiles are too few for the chip, K is cut and the parts' sums are added by a second launch.
//
// Few rows (serving): the weights are what is read, so each wave takes 16 rows of them straight into operands, the
// waves of a workgroup share K, and their sums are added in LDS.
//
// Measured, bf16: 8192 x 2048 x 8192 forwards, both projections 460-518 us (1060 to 1200 TFLOP/s; the products alone 1470, the
// exponentials and the exchange of h behind them take 11 us a tile, and one workgroup a CU leaves nothing beside them), the
// last product 216-233 (1180 to 1270; the matrix pipe is busy 0.72 of the time, at 1.66 GHz under that load).  8192 x 1024 x
// 4096 backwards: kTriple 290 us (711 TFLOP/s: three operands a product more from LDS per accumulator than kPair, and 17 us
// behind a tile), dx 134 (1025), the weights 200 (1030).  fp32, 2048 x 512 x 1365 backwards, six products for one: 11 us to lay
// operands out, 94 + 44 + 7 + 82 + 7 for the products and sums (100 TFLOP/s, 600 counted six times).  13 x 512 x 2048: 4.3
// and 5.8 us, 6.3 MB: a launch and two trips to memory each.
#include <math.h>

#include <algorithm>

#include "sf_internal.h"
#include "sf_memory.h"
#include "sf_split.h"

namespace sf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
enum Form { kOne = 0, kPair = 1, kTriple = 2 };

__device__ inline unsigned pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ inline float from_bf16(unsigned h) { return __builtin_bit_cast(float, h << 16); }

// act(g) and its slope.  FINE: for fp32 results; else the native exponential (2^-20 of a result rounded to 2^-8).
template <int ACT, bool FINE, bool SLOPE>
__device__ inline float activation(float g, float& slope) {
  if constexpr (ACT == SF_ACT_GELU) {
    const float phi = 0.5f * erfcf(-g * 0.70710678f);  // (1 + erf has lost its digits in the lower tail)
    if (SLOPE) slope = phi + g * 0.39894228f * expf(-0.5f * g * g);
    return g * phi;
  } else {
    const float s = FINE ? 1.0f / (1.0f + expf(-g)) : __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    if constexpr (ACT == SF_ACT_SIGMOID) {
      if (SLOPE) slope = s * (1.0f - s);
      return s;
    } else {
      if (SLOPE) slope = s * (1.0f + g * (1.0f - s));
      return g * s;
    }
  }
}
template <int N>
struct Constant {
  static constexpr int value = N;
};
// f(A), f(A + 1), .. f(B - 1) with the number known at compile time
template <int A, int B, class Fn>
__device__ __attribute__((always_inline)) inline void each(const Fn& f) {
  if constexpr (A < B) {
    f(Constant<A>());
    each<A + 1, B>(f);
  }
}
// f(activation's number, whether it is fine) with both known at compile time
template <class Fn>
__device__ inline void with_activation(int act, bool fine, const Fn& f) {
  if (fine) {
    if (act == SF_ACT_SILU) f(Constant<SF_ACT_SILU>(), Constant<1>());
    else if (act == SF_ACT_GELU) f(Constant<SF_ACT_GELU>(), Constant<1>());
    else f(Constant<SF_ACT_SIGMOID>(), Constant<1>());
  } else {
    if (act == SF_ACT_SILU) f(Constant<SF_ACT_SILU>(), Constant<0>());
    else if (act == SF_ACT_GELU) f(Constant<SF_ACT_GELU>(), Constant<0>());
    else f(Constant<SF_ACT_SIGMOID>(), Constant<0>());
  }
}

struct Operand {
  const uint16_t* p;  // [planes][rows][pitch] bf16
  int64_t pitch, plane;
  int rows, cols;     // as it lies in memory
};
// Where numbers go that are operands of a later product: rows of `pitch`, one plane or three
struct Terms {
  uint16_t* p;
  int64_t pitch, plane;
};
struct GemmArgs {
  Operand w[3], x[2];
  int K;           // padded to 64 (operands along k: zeros there; across k: no rows there, read as zeros)
  int pairs;       // kOne: pairs of operands that follow one another
  int terms;       // planes of each operand: 1 or 3
  int F, M;        // of C
  int nf, nm;      // tiles
  int act;
  void* out;       // kOne: [M][F] (bf16 or, `out_f32`, fp32)
  int out_f32;
  int splits;      // parts of K, out is then fp32 [splits][M][F]
  int Fp;          // F padded to 64
  Terms h, dg, du; // [M][Fp]: kPair h; kTriple all
};
struct GemmGroup {
  GemmArgs g[3];
  int n, tiles[3];  // problems of one launch and their workgroups
};

// the planes of a product of two operands in three terms, smallest first
__device__ constexpr int kPlaneW[6] = {0, 1, 2, 0, 1, 0};
__device__ constexpr int kPlaneX[6] = {2, 1, 0, 1, 0, 0};

// (lanes of a wave exchange numbers through LDS: its accesses run in order, the compiler is kept from reordering them)
__device__ inline void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// eight neighbours rounded, or (exact) as three terms
__device__ inline void terms8(const float* v, u32x4* w, bool exact) {
  if (!exact) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[0][i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    return;
  }
  float left = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned a, b, c;
    split_pair(v[2 * i], v[2 * i + 1], a, b, c, left);
    w[0][i] = a;
    w[1][i] = b;
    w[2][i] = c;
  }
}
// the same at offset `at` (a multiple of 8)
__device__ inline void store_terms8(const Terms& t, bool exact, int64_t at, const float* v) {
  u32x4 w[3];
  terms8(v, w, exact);
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i == 0 || exact) *(u32x4*)(t.p + i * t.plane + at) = w[i];
}
// eight neighbours of a result's row (its first `left` ones)
__device__ inline void store_out8(void* out, int f32, int F, int64_t at, int left, const float* v) {
  if ((F & 7) == 0) {  // (out is 16-byte aligned)
    if (f32) {
      *(f32x4*)((float*)out + at) = *(const f32x4*)v;
      *(f32x4*)((float*)out + at + 4) = *(const f32x4*)(v + 4);
    } else {
      *(u32x4*)((uint16_t*)out + at) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    if (r >= left) break;
    if (f32) ((float*)out)[at + r] = v[r];
    else ((uint16_t*)out)[at + r] = (uint16_t)pack_bf16(v[r], 0.0f);
  }
}

// LDS of B rows of an operand, BK numbers of K: along k (0) or across (1)
constexpr int lds_pitch(int across, int B, int BK) { return !across ? BK * 2 + 16 : B == 64 ? 192 : B * 2 + 64; }
constexpr int lds_bytes(int across, int B, int BK) { return lds_pitch(across, B, BK) * (across ? BK : B); }

// BF rows of each w, BM rows of each x per workgroup; a wave has half of both.  ACROSS: bit a: w[a], bit 4: every x.
template <int FORM, int ACROSS, int BF, int BM, int BK>
struct Tile {
  static constexpr int kW = FORM == kOne ? 1 : FORM == kPair ? 2 : 3, kX = FORM == kTriple ? 2 : 1, kN = kW + kX;
  static constexpr int across(int n) { return n < kW ? ACROSS >> n & 1 : ACROSS >> 4 & 1; }
  static constexpr int rows(int n) { return n < kW ? BF : BM; }
  static constexpr int pitch(int n) { return lds_pitch(across(n), rows(n), BK); }
  static constexpr int at(int n) { return n == 0 ? 0 : at(n - 1) + lds_bytes(across(n - 1), rows(n - 1), BK); }
  static constexpr int kStage = at(kN);
  static constexpr int kEnd = 4 * kW * 32 * (BF / 2 + 4) * 4;  // behind the products: see there
  static constexpr int kBytes = 2 * kStage > kEnd ? 2 * kStage : kEnd;
  static constexpr int pieces(int n) { return rows(n) * BK / 8 / kThreads; }  // 16-byte pieces of a step per thread
  static constexpr int first(int n) { return n == 0 ? 0 : first(n - 1) + pieces(n - 1); }
  static constexpr int of(int i) {  // the array of piece i
    int n = 0;
    while (i >= first(n + 1)) ++n;
    return n;
  }
};

template <int FORM, int ACROSS, int BF, int BM, int BK, int WAVES>
__global__ __launch_bounds__(kThreads, WAVES) void ffn_gemm_kernel(GemmGroup group) {
  typedef Tile<FORM, ACROSS, BF, BM, BK> L;
  constexpr int W = L::kW, X = L::kX, N = L::kN, TF = BF / 64, TM = BM / 64;  // a wave's 32 x 32 tiles
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 31, lh = lane >> 5;
  const int wf = wave & 1, wm = wave >> 1;

  // tiles in runs of neighbours per XCD, in bands of four tiles of x: 32 CUs then share 4 tiles of x and 8 of w in their L2
  int total = 0;
  for (int i = 0; i < group.n; ++i) total += group.tiles[i];
  const int per_xcd = (total + 7) / 8;
  int tile = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (tile >= total || (int)(blockIdx.x >> 3) >= per_xcd) return;
  int which = 0;
  while (which + 1 < group.n && tile >= group.tiles[which]) tile -= group.tiles[which++];
  const GemmArgs& g = group.g[which];
  const int part = FORM == kOne ? tile / (g.nf * g.nm) : 0;
  if (FORM == kOne) tile -= part * (g.nf * g.nm);
  const int band = tile / (4 * g.nf), in_band = tile - band * 4 * g.nf, height = min(4, g.nm - 4 * band);
  const int f0 = in_band / height * BF, m0 = (4 * band + in_band % height) * BM;

  // this thread's pieces of the arrays' tiles: row (of the tile, or of K) and 16 bytes of it
  constexpr int NP = L::first(N), NK = BK / 16;
  auto row_of = [&](auto i) __attribute__((always_inline)) {
    constexpr int n = L::of(decltype(i)::value), per = L::across(n) ? L::rows(n) / 8 : BK / 8;
    return tid / per + kThreads / per * (decltype(i)::value - L::first(n));
  };
  auto col_of = [&](auto i) __attribute__((always_inline)) {
    constexpr int n = L::of(decltype(i)::value), per = L::across(n) ? L::rows(n) / 8 : BK / 8;
    return tid % per * 16;
  };
  // the step to be requested next: its pass (pair of operands, planes) and place in K
  const int passes = (g.terms == 1 ? 1 : 6) * g.pairs, steps_k = g.K / BK, all = steps_k * passes;
  const int s_begin = FORM == kOne ? (int)((int64_t)all * part / g.splits) : 0;
  const int steps = (FORM == kOne ? (int)((int64_t)all * (part + 1) / g.splits) : all) - s_begin;
  int pass = s_begin / steps_k, k = s_begin % steps_k * BK;
  const unsigned char* base[N];
  unsigned from[N], pitch[N];  // bytes to this thread's first piece of an array, between rows
  auto begin_pass = [&]() __attribute__((always_inline)) {
    const int pair = FORM == kOne && pass >= passes / g.pairs ? 1 : 0, term = g.terms == 1 ? 5 : pass - pair * 6;
    each<0, N>([&](auto i) __attribute__((always_inline)) {
      constexpr int n = decltype(i)::value;
      const Operand& o = n < W ? g.w[FORM == kOne ? pair : n] : g.x[FORM == kOne ? pair : n - W];
      const int64_t r0 = n < W ? f0 : m0;
      pitch[n] = (unsigned)o.pitch * 2;
      from[n] = row_of(Constant<L::first(n)>()) * pitch[n] + col_of(Constant<L::first(n)>());
      // (across K the bounds end only the step's last row: behind the others lie gaps or the next row.  All of a thread's pieces of an
      // array are of one column, the columns a multiple of eight; 63 rows of 2^23 bytes further on is still past the end.)
      if (L::across(n) && col_of(Constant<L::first(n)>()) >= 2 * (int)(o.cols - r0)) from[n] = 0x80000000u;
      base[n] = (const unsigned char*)(o.p + (n < W ? kPlaneW[term] : kPlaneX[term]) * o.plane + (L::across(n) ? r0 : r0 * o.pitch));
    });
  };
  // (the bounds: bytes from the tile's (along k) or the step's (across k) first number to the array's end)
  __amdgpu_buffer_rsrc_t source[N];
  int rows[N], cols[N];  // of each array, from the tile on
  each<0, N>([&](auto i) __attribute__((always_inline)) {
    constexpr int n = decltype(i)::value;
    const Operand& o = n < W ? g.w[n] : g.x[n - W];
    rows[n] = o.rows;
    cols[n] = o.cols - (n < W ? f0 : m0);
  });
  auto locate = [&]() __attribute__((always_inline)) {
    each<0, N>([&](auto i) __attribute__((always_inline)) {
      constexpr int n = decltype(i)::value;
      if constexpr (L::across(n)) {
        const int left = min(BK, rows[n] - k);  // (the last row ends with its numbers)
        source[n] = __builtin_amdgcn_make_buffer_rsrc((void*)(base[n] + (int64_t)k * pitch[n]), 0,
                                                      left > 0 ? (left - 1) * (int)pitch[n] + cols[n] * 2 : 0, 0x00027000);
      } else {
        source[n] = __builtin_amdgcn_make_buffer_rsrc((void*)base[n], 0, min(L::rows(n), rows[n] - (n < W ? f0 : m0)) * (int)pitch[n], 0x00027000);
      }
    });
  };
  auto advance = [&]() __attribute__((always_inline)) {  // (past the end: the last step again, for no use)
    k += BK;
    if (k == g.K) {
      if (pass + 1 < passes) {
        ++pass;
        k = 0;
        begin_pass();
      } else {
        k -= BK;
      }
    }
    locate();
  };
  u32x4 next[NP];
  auto request = [&](auto i) __attribute__((always_inline)) {
    constexpr int n = L::of(decltype(i)::value), per = L::across(n) ? L::rows(n) / 8 : BK / 8;
    next[decltype(i)::value] = __builtin_amdgcn_raw_buffer_load_b128(
        source[n], from[n] + (unsigned)(kThreads / per * (decltype(i)::value - L::first(n))) * pitch[n], L::across(n) ? 0 : 2 * k, 0);
  };
  auto put = [&](auto i, int stage) __attribute__((always_inline)) {
    constexpr int n = L::of(decltype(i)::value);
    *(u32x4*)(lds + stage + L::at(n) + row_of(i) * L::pitch(n) + col_of(i)) = next[decltype(i)::value];
  };
  // Operands of 16 numbers of K: row li of a 32-row tile, k = 8 lh .. 8 lh + 7.  Across k two transposing reads of four k
  // each: of 16 lanes, lane i names row i / 4 and four columns, and is given column i of the four rows.
  bf16x8 fr[2][W * TF + X * TM];
  auto operand = [&](auto array, int t, int stage, int kk) __attribute__((always_inline)) {
    constexpr int n = decltype(array)::value;
    const int half = n < W ? wf * (BF / 2) : wm * (BM / 2), r = half + 32 * t;
    const unsigned char* at = lds + stage + L::at(n);
    if constexpr (!L::across(n)) {
      return *(const bf16x8*)(at + (r + li) * L::pitch(n) + lh * 16 + kk * 32);
    } else {
      const int grp = lane >> 4, i = lane & 15;
      const unsigned char* p = at + (16 * kk + 8 * (grp >> 1) + (i >> 2)) * L::pitch(n) + (r + 16 * (grp & 1) + 4 * (i & 3)) * 2;
      typedef __attribute__((address_space(3))) s16x4* Lds4;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(p + 4 * L::pitch(n)));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  constexpr int FR = [] {  // LDS reads of them
    int r = 0;
    for (int n = 0; n < N; ++n) r += (n < W ? TF : TM) * (L::across(n) ? 2 : 1);
    return r;
  }();
  auto operands = [&](int to, int stage, int kk) __attribute__((always_inline)) {
    each<0, X>([&](auto n) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TM; ++t) fr[to][W * TF + decltype(n)::value * TM + t] = operand(Constant<W + decltype(n)::value>(), t, stage, kk);
    });
    each<0, W>([&](auto n) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < TF; ++t) fr[to][decltype(n)::value * TF + t] = operand(n, t, stage, kk);
    });
  };
  constexpr int MF = W * TF * TM;

  f32x16 acc[W][TF][TM];
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int b = 0; b < TF; ++b)
#pragma unroll
      for (int c = 0; c < TM; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[a][b][c][v] = 0.0f;

  begin_pass();
  locate();
  each<0, NP>(request);
  each<0, NP>([&](auto i) __attribute__((always_inline)) { put(i, 0); });
  advance();
  each<0, NP>(request);
  __syncthreads();
  operands(0, 0, 0);
  // One step: behind the products of 16 numbers of K the operands of the next 16 are read, and the pieces of the next step
  // go to LDS, each followed by the request for the step after that.  All reads of a step are done before its last products,
  // where the barrier stands: behind it the next step's first operands are read under these products.
  for (int s = 0; s < steps; ++s) {
    const int stage = (s & 1) * L::kStage, other = L::kStage - stage;
    advance();
    each<0, NK>([&](auto step) __attribute__((always_inline)) {
      constexpr int kk = decltype(step)::value, cur = kk & 1;
      constexpr bool last = kk == NK - 1;
      if constexpr (last) __syncthreads();
      operands(cur ^ 1, last ? other : stage, last ? 0 : kk + 1);
      constexpr int p0 = last ? NP : NP * kk / (NK - 1), p1 = last ? NP : NP * (kk + 1) / (NK - 1);
      each<p0, p1>([&](auto i) __attribute__((always_inline)) {
        put(i, other);
        request(i);
      });
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int b = 0; b < TF; ++b)
#pragma unroll
          for (int c = 0; c < TM; ++c)
            acc[a][b][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                fr[cur][a * TF + b], fr[cur][W * TF + (FORM == kTriple && a == 2 ? TM : 0) + c], acc[a][b][c], 0, 0, 0);
      // the order of all that: spread evenly behind the products
      constexpr int extra = FR + (p1 - p0);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
        for (int e = extra * i / MF; e < extra * (i + 1) / MF; ++e) {
          if (e < FR) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          } else {
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
          }
        }
      }
    });
  }
  __syncthreads();  // (the last step's needless reads are done: LDS is written again)

  // An accumulator has one column m = li per lane and, four at a time, neighbouring rows f = 8 q + 4 lh.  The wave's columns
  // go through LDS (its own part), 32 of x at a time, so that what is stored are whole pieces of neighbours.
  constexpr int FW = 32 * TF, EP = FW + 4;      // a wave's rows of w; row length there
  constexpr int LPR = FW / 8, NI = LPR / 2;     // lanes of a row m, rounds of 64 lanes over 32 rows
  float* const area = (float*)lds + wave * (W * 32 * EP);
  const int fwave = f0 + wf * FW;
  const GemmArgs a_ = g;  // (kept in registers: behind wave_order it would be read again and again)
#pragma unroll
  for (int c = 0; c < TM; ++c) {
    const int mw = m0 + wm * (BM / 2) + 32 * c;
    wave_order();
#pragma unroll
    for (int a = 0; a < W; ++a)
#pragma unroll
      for (int b = 0; b < TF; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(f32x4*)(area + (a * 32 + li) * EP + 32 * b + 8 * q + 4 * lh) =
              f32x4{acc[a][b][c][4 * q], acc[a][b][c][4 * q + 1], acc[a][b][c][4 * q + 2], acc[a][b][c][4 * q + 3]};
    wave_order();
    if constexpr (FORM == kOne) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = i * (64 / LPR) + lane / LPR, col = lane % LPR * 8, m = mw + row, f = fwave + col;
        if (m < a_.M && f < a_.F)
          store_out8(a_.out, a_.out_f32, a_.F, ((int64_t)part * a_.M + m) * a_.F + f, a_.F - f, area + row * EP + col);
      }
    } else {
      // (rows of w along K, columns of w across K past F and rows of x past M were read as zeros, so that gate, up and dh, and with them h,
      // dg and du, are zeros where they are padded)
      // (a piece that is not there has an offset past the end, so that no branch parts the rounds of the loop)
      const int64_t corner = (int64_t)mw * a_.h.pitch + fwave;  // (all three arrays have one shape)
      auto buffer = [&](const Terms& t, int plane) __attribute__((always_inline)) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)(t.p + plane * t.plane + corner), 0, 0x7FFFFFFF, 0x00027000);
      };
      with_activation(a_.act, a_.terms == 3, [&](auto act, auto exact) __attribute__((always_inline)) {
        constexpr bool kShort = decltype(act)::value != SF_ACT_GELU && !decltype(exact)::value;
#pragma unroll kShort ? NI : 1
        for (int i = 0; i < NI; ++i) {
          const int row = i * (64 / LPR) + lane / LPR, col = lane % LPR * 8;
          const float* const at = area + row * EP + col;
          float gate[8], up[8], h[8], dh[8], dg[8], du[8];
#pragma unroll
          for (int r = 0; r < 8; r += 4) {
            *(f32x4*)(gate + r) = *(const f32x4*)(at + r);
            *(f32x4*)(up + r) = *(const f32x4*)(at + 32 * EP + r);
            if constexpr (FORM == kTriple) *(f32x4*)(dh + r) = *(const f32x4*)(at + 64 * EP + r);
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            float slope = 0.0f;
            const float v = activation<decltype(act)::value, decltype(exact)::value, FORM == kTriple>(gate[r], slope);
            h[r] = v * up[r];
            if constexpr (FORM == kTriple) {
              dg[r] = dh[r] * up[r] * slope;
              du[r] = dh[r] * v;
            }
          }
          const unsigned to = mw + row < a_.M && fwave + col < a_.Fp ? (unsigned)(row * (int)a_.h.pitch + col) * 2 : 0x80000000u;
          auto store = [&](const Terms& t, const float* v) __attribute__((always_inline)) {
            u32x4 w[3];
            terms8(v, w, decltype(exact)::value);
            __builtin_amdgcn_raw_buffer_store_b128(w[0], buffer(t, 0), to, 0, 0);
            if constexpr (decltype(exact)::value) {
              __builtin_amdgcn_raw_buffer_store_b128(w[1], buffer(t, 1), to, 0, 0);
              __builtin_amdgcn_raw_buffer_store_b128(w[2], buffer(t, 2), to, 0, 0);
            }
          };
          store(a_.h, h);
          if constexpr (FORM == kTriple) {
            store(a_.dg, dg);
            store(a_.du, du);
          }
        }
      });
    }
  }
}

// The sums of the parts of K, four neighbours a thread.
struct SumGroup {
  const float* parts[3];
  void* out[3];
  int64_t size[3], threads[3];
  int n, splits;
};
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void ffn_sum_kernel(SumGroup g) {
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int which = 0;
  while (which + 1 < g.n && i >= g.threads[which]) i -= g.threads[which++];
  const float* const parts = g.parts[which];
  void* const out = g.out[which];
  const int64_t size = g.size[which];
  i *= 4;
  if (i >= size) return;
  if ((size & 3) == 0) {
    f32x4 v = *(const f32x4*)(parts + i);
    for (int j = 1; j < g.splits; ++j) v += *(const f32x4*)(parts + j * size + i);
    if (DTYPE == SF_DTYPE_BF16) *(u32x2*)((uint16_t*)out + i) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else *(f32x4*)((float*)out + i) = v;
    return;
  }
  for (int r = 0; r < 4 && i + r < size; ++r) {
    float v = parts[i + r];
    for (int j = 1; j < g.splits; ++j) v += parts[j * size + i + r];
    if (DTYPE == SF_DTYPE_BF16) ((uint16_t*)out)[i + r] = (uint16_t)pack_bf16(v, 0.0f);
    else ((float*)out)[i + r] = v;
  }
}

// ---- laying operands out -----------------------------------------------------------------------

struct Layout {
  const void* from;   // [rows][cols] of the calls' type, rows `pitch` elements apart
  int64_t pitch;
  int rows, cols, vec;
  Terms to;           // [rows][pitch], zeros up to the pitch
  int64_t pieces;     // eight numbers each
};
struct LayoutGroup {
  Layout l[5];
  int n;
};

template <int DTYPE>
__device__ inline void lay_piece(const Layout& l, int64_t piece) {
  const int per = (int)(l.to.pitch / 8), c = (int)(piece % per) * 8;
  const int64_t r = piece / per, at = r * l.pitch + c;
  float v[8];
  if (DTYPE == SF_DTYPE_FP32 && l.vec && c + 8 <= l.cols) {
    *(f32x4*)v = *(const f32x4*)((const float*)l.from + at);
    *(f32x4*)(v + 4) = *(const f32x4*)((const float*)l.from + at + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = c + i >= l.cols ? 0.0f : DTYPE == SF_DTYPE_BF16 ? from_bf16(((const uint16_t*)l.from)[at + i]) : ((const float*)l.from)[at + i];
  }
  store_terms8(l.to, DTYPE == SF_DTYPE_FP32, r * l.to.pitch + c, v);
}

template <int DTYPE>
__global__ __launch_bounds__(kThreads) void ffn_layout_kernel(LayoutGroup group) {
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;; at += (int64_t)gridDim.x * kThreads) {
    int64_t piece = at;
    int which = 0;
    while (which < group.n && piece >= group.l[which].pieces) piece -= group.l[which++].pieces;
    if (which == group.n) return;
    lay_piece<DTYPE>(group.l[which], piece);
  }
}

// ---- few rows ----------------------------------------------------------------------------------

// C[m][f] for 16 MT rows m: 16 rows of each w per workgroup, its waves share K.
struct RowsArgs {
  const void *w[2], *x;
  int64_t w_pitch[2], x_pitch;
  int K, F, M, act;
  void* out;  // [M][F]
  int vec;    // rows are read in 16-byte pieces
};
constexpr int kRowWaves = 8;

// Eight numbers from k on, zeros from K on (in pieces: K is a multiple of 8; the address stays inside the row).
template <int DTYPE, bool VEC>
__device__ inline void load8(float* v, u32x4& raw, const void* p, int64_t at, int k, int K) {
  if constexpr (DTYPE == SF_DTYPE_BF16) {
    const uint16_t* q = (const uint16_t*)p + at;
    if constexpr (VEC) {
      raw = *(const u32x4*)(q + min(k, K - 8));
      if (k >= K) raw = u32x4{0, 0, 0, 0};
    } else {
      raw = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < K) raw[i / 2] |= (unsigned)q[k + i] << (16 * (i & 1));
    }
  } else {
    const float* q = (const float*)p + at;
    if constexpr (VEC) {
      *(f32x4*)v = *(const f32x4*)(q + min(k, K - 8));
      *(f32x4*)(v + 4) = *(const f32x4*)(q + min(k, K - 8) + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = k < K ? v[i] : 0.0f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = k + i < K ? q[k + i] : 0.0f;
    }
  }
}

template <int DTYPE, int W, int MT, bool VEC>
__global__ __launch_bounds__(64 * kRowWaves) void ffn_rows_kernel(RowsArgs g) {
  __shared__ __attribute__((aligned(16))) f32x4 part[kRowWaves][W][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lg = lane >> 4;
  const int f0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
  const int f_row = min(f0 + li, g.F - 1);
  f32x4 acc[W][MT];
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int c = 0; c < MT; ++c) acc[a][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int U = VEC ? 2 : 1;  // steps whose loads are under way together (up to 8: no shorter)
  for (int k0 = wave * 32; k0 < g.K; k0 += U * kRowWaves * 32) {
    u32x4 rw[U][W], rx[U][MT];
    float vw[U][W][8], vx[U][MT][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kRowWaves * 32 + 8 * lg;
#pragma unroll
      for (int a = 0; a < W; ++a) load8<DTYPE, VEC>(vw[u][a], rw[u][a], g.w[a], f_row * g.w_pitch[a], k, g.K);
#pragma unroll
      for (int c = 0; c < MT; ++c) load8<DTYPE, VEC>(vx[u][c], rx[u][c], g.x, min(m0 + 16 * c + li, g.M - 1) * g.x_pitch, k, g.K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int c = 0; c < MT; ++c) {
          if constexpr (DTYPE == SF_DTYPE_BF16) {
            acc[a][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rw[u][a]), __builtin_bit_cast(bf16x8, rx[u][c]),
                                                                acc[a][c], 0, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[a][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[u][a][i], vx[u][c][i], acc[a][c], 0, 0, 0);
          }
        }
  }
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int c = 0; c < MT; ++c) part[wave][a][c][lane] = acc[a][c];
  __syncthreads();
  // a wave finishes tiles of 16 rows of x: lane (li, lg) has row li, neighbours f = 4 lg ..
  for (int c = wave; c < MT; c += kRowWaves) {
    f32x4 v[W];
#pragma unroll
    for (int a = 0; a < W; ++a) {
      v[a] = part[0][a][c][lane];
#pragma unroll
      for (int i = 1; i < kRowWaves; ++i) v[a] += part[i][a][c][lane];
    }
    const int m = m0 + 16 * c + li, f = f0 + 4 * lg;
    if (m >= g.M) continue;
    float y[4];
    if constexpr (W == 2) {
      with_activation(g.act, DTYPE == SF_DTYPE_FP32, [&](auto act, auto) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float slope;
          y[r] = activation<decltype(act)::value, DTYPE == SF_DTYPE_FP32, false>(v[0][r], slope) * v[W - 1][r];
        }
      });
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = v[0][r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (f + r >= g.F) continue;
      const int64_t at = (int64_t)m * g.F + f + r;
      if (DTYPE == SF_DTYPE_BF16) ((uint16_t*)g.out)[at] = (uint16_t)pack_bf16(y[r], 0.0f);
      else ((float*)g.out)[at] = y[r];
    }
  }
}

__global__ __launch_bounds__(kThreads) void ffn_zero_kernel(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) p[i] = 0;
}

// ---- host side ---------------------------------------------------------------------------------

// Whether the path for few rows takes a call: there the time grows with the rows of x that each wave reads beside its weights,
// the tiles fill few CUs where the weights are small, and in fp32 the weights' terms have to be laid out for them first.
// us, rows (by 64) and tiles:      bf16 512 x 2048      bf16 2048 x 8192     fp32 512 x 2048      fp32 2048 x 8192
//     1 row                         7.5                  23                   13                   58
//    16                             9.3                  30                   16                   65
//    32                            11.8                  40   50              21                   87
//    64                            16.8   25             62   50              33   73             135  358
bool few_rows(const sf_ffn_config* c) {
  return c->M <= 32 || (c->M <= 128 && (c->dtype == SF_DTYPE_FP32 || (int64_t)c->D * c->F <= 1 << 21));
}

int check(const sf_ffn_config* c, const char* fn) {
  if (!c || c->struct_size != sizeof(sf_ffn_config)) {
    set_error("%s: null configuration or struct_size mismatch", fn);
    return SF_ERR_ARG;
  }
  if ((c->dtype != SF_DTYPE_FP32 && c->dtype != SF_DTYPE_BF16) || c->act < SF_ACT_SILU || c->act > SF_ACT_SIGMOID) {
    set_error("%s: dtype = %d, act = %d", fn, c->dtype, c->act);
    return SF_ERR_ARG;
  }
  const int most = 1 << 20;
  if (c->M < 0 || c->D < 1 || c->F < 1 || c->D > most || c->F > most || c->M > 1 << 24) {
    set_error("%s: M = %d, D = %d, F = %d out of range", fn, c->M, c->D, c->F);
    return SF_ERR_SHAPE;
  }
  return SF_OK;
}
bool fits(const char* fn, const char* name, const void* p, size_t align, bool optional = false) {
  if (p ? (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0 : optional) return true;
  set_error("%s: %s is null or misaligned", fn, name);
  return false;
}

int64_t pad64(int64_t n) { return (n + 63) / 64 * 64; }

// The workspace, given out from the front; without a base only counted.
struct Arena {
  unsigned char* base;
  size_t at;
  void* bytes(size_t n) {
    void* p = base ? base + at : nullptr;
    at += (n + 255) / 256 * 256;
    return p;
  }
  Terms take(int64_t rows, int64_t pitch, int terms) {
    return Terms{(uint16_t*)bytes((size_t)(rows * pitch * terms) * 2), pitch, rows * pitch};
  }
};
Operand operand(const Terms& t, int rows) { return Operand{t.p, t.pitch, t.plane, rows, (int)t.pitch}; }

struct Job {
  const sf_ffn_config* c;
  hipStream_t st;
  LayoutGroup lay = {};
  int64_t lay_pieces = 0;
  int terms() const { return c->dtype == SF_DTYPE_BF16 ? 1 : 3; }
  // An array as an operand: itself where it can be read in whole pieces (`along`: and is one along its rows, which then have
  // to be whole steps of K), else laid out in the workspace.
  Operand array(Arena& a, const void* p, int64_t pitch, int rows, int cols, bool along) {
    if (terms() == 1 && cols % (along ? 64 : 8) == 0 && pitch % 8 == 0 && pitch >= cols && pitch < 1 << 22 &&
        (reinterpret_cast<uintptr_t>(p) & 15) == 0)
      return Operand{(const uint16_t*)p, pitch, 0, rows, cols};
    const Terms t = a.take(rows, pad64(cols), terms());
    Layout& l = lay.l[lay.n++];
    l = Layout{p, pitch, rows, cols, pitch % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0, t, rows * t.pitch / 8};
    lay_pieces += l.pieces;
    return operand(t, rows);
  }
  hipError_t run_layout() {
    if (!lay.n) return hipSuccess;
    const unsigned grid = (unsigned)std::min<int64_t>((lay_pieces + kThreads - 1) / kThreads, 1 << 20);
    if (c->dtype == SF_DTYPE_BF16) ffn_layout_kernel<SF_DTYPE_BF16><<<grid, kThreads, 0, st>>>(lay);
    else ffn_layout_kernel<SF_DTYPE_FP32><<<grid, kThreads, 0, st>>>(lay);
    lay.n = 0;
    lay_pieces = 0;
    return hipGetLastError();
  }
};

template <int FORM, int ACROSS, int BF, int BM, int BK, int WAVES>
hipError_t launch_t(GemmGroup& group, hipStream_t st) {
  const auto kern = ffn_gemm_kernel<FORM, ACROSS, BF, BM, BK, WAVES>;
  constexpr int bytes = Tile<FORM, ACROSS, BF, BM, BK>::kBytes;
  static const hipError_t attr = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  int total = 0;
  for (int i = 0; i < group.n; ++i) {
    GemmArgs& g = group.g[i];
    // (padded columns of the next product's operand are this one's rows of w)
    g.nf = ((FORM == kOne ? g.F : g.Fp) + BF - 1) / BF;
    g.nm = (g.M + BM - 1) / BM;
    total += group.tiles[i] = g.nf * g.nm * (FORM == kOne ? g.splits : 1);
  }
  kern<<<(total + 7) / 8 * 8, kThreads, bytes, st>>>(group);
  return hipGetLastError();
}
int64_t tiles_of(int F, int M, int BF, int BM) { return (int64_t)((F + BF - 1) / BF) * ((M + BM - 1) / BM); }
// The large tile where it leaves few CUs without one, the small one otherwise.  us, large and small, by large tiles (D = 1024):
// kPair 96 tiles 29 and 20, 128 29 and 22, 160 29.6 and 29.2, 208 32 and 37, 512 69 and 75; kTriple 128 32 and 25, 192 34 and
// 36, 256 36 and 41, 320 60 and 56 (a second round of large ones just begun), 416 62 and 72, 1024 135 and 148.  Whole backward passes in
// fp32: 64 tiles 259 and 201, 128 336 and 327, 160 377 and 428, 256 505 and 602, 320 715 and 756, 512 970 and 1157.
constexpr int kEnough = 160;
// And a smaller one still where a round of workgroups takes all of it (256).  us of whole calls, 64 x 128 and 64 x 64, forwards and
// backwards, by tiles of 64 x 64: fp32 1024 x 2048, 160 tiles backwards 179 and 171, 256 213 and 197, 480 301 and 314; 1920 x 576, 135 122
// and 104, 300 and 269, 288 141 and 156, 390 and 436; bf16 1024 x 2048, 160 28 and 25, 50 and 46, 256 backwards 55 and 50, 480 30 and 31,
// 70 and 72.
constexpr int kOneRound = 256;
template <int FORM>
hipError_t launch(GemmGroup& group, hipStream_t st) {
  const GemmArgs& g = group.g[0];
  const bool one_round = tiles_of(g.Fp, g.M, 64, 64) <= kOneRound;
  if constexpr (FORM == kPair) {
    if (tiles_of(g.Fp, g.M, 128, 256) >= kEnough) return launch_t<kPair, 0, 128, 256, 64, 1>(group, st);
    return one_round ? launch_t<kPair, 0, 64, 64, 64, 2>(group, st) : launch_t<kPair, 0, 64, 128, 64, 2>(group, st);
  } else {
    if (tiles_of(g.Fp, g.M, 128, 128) >= kEnough) return launch_t<kTriple, 4, 128, 128, 32, 1>(group, st);
    return one_round ? launch_t<kTriple, 4, 64, 64, 32, 2>(group, st) : launch_t<kTriple, 4, 64, 128, 32, 2>(group, st);
  }
}

// Products of form kOne that do not depend on one another, as one launch, and where K is cut a second one.
struct Products {
  GemmGroup group = {};
  bool large = false;
  int splits = 1;
  // Parts of K: as many workgroups of small tiles as run at once, each part 16 steps of 64 or more.
  void plan() {
    int64_t big = 0, small = 0;
    int steps = 1 << 30;
    for (int i = 0; i < group.n; ++i) {
      const GemmArgs& g = group.g[i];
      big += tiles_of(g.F, g.M, 256, 256);
      small += tiles_of(g.F, g.M, 128, 128);
      const int s = g.K / 64 * (g.terms == 1 ? 1 : 6) * g.pairs;
      if (s < steps) steps = s;
    }
    large = big >= kEnough;
    splits = large || small == 0 ? 1 : (int)(512 / small);
    if (splits > steps / 16) splits = steps / 16;
    if (splits > 8) splits = 8;
    if (splits < 1) splits = 1;
  }
  size_t part_bytes(int i) const { return splits > 1 ? (size_t)splits * group.g[i].M * group.g[i].F * 4 : 0; }
  template <int ACROSS>
  hipError_t run(Arena& a, int dtype, hipStream_t st) {
    void* out[3];
    for (int i = 0; i < group.n; ++i) {
      GemmArgs& g = group.g[i];
      g.splits = splits;
      out[i] = g.out;
      if (splits > 1) {
        g.out = a.bytes(part_bytes(i));
        g.out_f32 = 1;
      }
    }
    hipError_t e = large ? launch_t<kOne, ACROSS, 256, 256, 64, 1>(group, st) : launch_t<kOne, ACROSS, 128, 128, 64, 2>(group, st);
    if (splits > 1 && e == hipSuccess) {
      SumGroup sums = {};
      int64_t threads = 0;
      sums.n = group.n;
      sums.splits = splits;
      for (int i = 0; i < group.n; ++i) {
        sums.parts[i] = (const float*)group.g[i].out;
        sums.out[i] = out[i];
        sums.size[i] = (int64_t)group.g[i].M * group.g[i].F;
        threads += sums.threads[i] = (sums.size[i] + 3) / 4;
      }
      const unsigned grid = (unsigned)((threads + kThreads - 1) / kThreads);  // (few tiles: below 256 x 128 x 128 numbers)
      if (dtype == SF_DTYPE_BF16) ffn_sum_kernel<SF_DTYPE_BF16><<<grid, kThreads, 0, st>>>(sums);
      else ffn_sum_kernel<SF_DTYPE_FP32><<<grid, kThreads, 0, st>>>(sums);
      e = hipGetLastError();
    }
    return e;
  }
};

template <int DTYPE, int W, bool VEC>
hipError_t launch_rows(const RowsArgs& g, hipStream_t st) {
  const dim3 grid((unsigned)((g.F + 15) / 16), (unsigned)((g.M + 63) / 64));
  if (g.M <= 16) ffn_rows_kernel<DTYPE, W, 1, VEC><<<grid, 64 * kRowWaves, 0, st>>>(g);
  else if (g.M <= 32) ffn_rows_kernel<DTYPE, W, 2, VEC><<<grid, 64 * kRowWaves, 0, st>>>(g);
  else ffn_rows_kernel<DTYPE, W, 4, VEC><<<grid, 64 * kRowWaves, 0, st>>>(g);
  return hipGetLastError();
}
template <int W>
hipError_t launch_rows(int dtype, const RowsArgs& g, hipStream_t st) {
  if (dtype == SF_DTYPE_BF16) return g.vec ? launch_rows<SF_DTYPE_BF16, W, true>(g, st) : launch_rows<SF_DTYPE_BF16, W, false>(g, st);
  return g.vec ? launch_rows<SF_DTYPE_FP32, W, true>(g, st) : launch_rows<SF_DTYPE_FP32, W, false>(g, st);
}

GemmArgs gemm(const sf_ffn_config* c, int terms, int K, int F, int M) {
  GemmArgs g = {};
  g.K = (int)pad64(K);
  g.pairs = 1;
  g.splits = 1;
  g.terms = terms;
  g.F = F;
  g.M = M;
  g.Fp = (int)pad64(F);
  g.act = c->act;
  g.out_f32 = c->dtype == SF_DTYPE_FP32;
  return g;
}

// What a call consists of, for the call itself and for the size of its workspace.
struct Forward {
  GemmGroup up = {};
  Products down;
  Forward(Job& j, Arena& a, const void* x, const void* wg, const void* wu, const void* wd, void* y) {
    const sf_ffn_config* c = j.c;
    up.n = 1;
    GemmArgs& u = up.g[0] = gemm(c, j.terms(), c->D, c->F, c->M);
    u.x[0] = j.array(a, x, c->x_stride, c->M, c->D, true);
    u.w[0] = j.array(a, wg, c->w_gate_stride, c->F, c->D, true);
    u.w[1] = j.array(a, wu, c->w_up_stride, c->F, c->D, true);
    u.h = a.take(c->M, u.Fp, j.terms());
    down.group.n = 1;
    GemmArgs& d = down.group.g[0] = gemm(c, j.terms(), c->F, c->D, c->M);
    d.w[0] = j.array(a, wd, c->w_down_stride, c->D, c->F, true);
    d.x[0] = operand(u.h, c->M);
    d.out = y;
    down.plan();
  }
};
struct Backward {
  GemmGroup mid = {};
  Products in, weights;
  Backward(Job& j, Arena& a, const void* x, const void* wg, const void* wu, const void* wd, const void* dy, void* dx, void* dwg, void* dwu,
           void* dwd) {
    const sf_ffn_config* c = j.c;
    const int terms = j.terms();
    mid.n = 1;
    GemmArgs& t = mid.g[0] = gemm(c, terms, c->D, c->F, c->M);
    t.x[0] = j.array(a, x, c->x_stride, c->M, c->D, true);
    t.x[1] = j.array(a, dy, c->dy_stride, c->M, c->D, true);
    t.w[0] = j.array(a, wg, c->w_gate_stride, c->F, c->D, true);
    t.w[1] = j.array(a, wu, c->w_up_stride, c->F, c->D, true);
    t.w[2] = j.array(a, wd, c->w_down_stride, c->D, c->F, false);
    t.h = a.take(c->M, t.Fp, terms);
    t.dg = a.take(c->M, t.Fp, terms);
    t.du = a.take(c->M, t.Fp, terms);
    const Operand h = operand(t.h, c->M), dg = operand(t.dg, c->M), du = operand(t.du, c->M);
    in.group.n = 1;
    GemmArgs& i = in.group.g[0] = gemm(c, terms, c->F, c->D, c->M);
    i.pairs = 2;
    i.w[0] = t.w[0];
    i.w[1] = t.w[1];
    i.x[0] = dg;
    i.x[1] = du;
    i.out = dx;
    in.plan();
    weights.group.n = 3;
    GemmArgs* w = weights.group.g;
    w[0] = w[1] = gemm(c, terms, c->M, c->D, c->F);
    w[2] = gemm(c, terms, c->M, c->F, c->D);
    w[0].w[0] = w[1].w[0] = t.x[0];
    w[0].x[0] = dg;
    w[1].x[0] = du;
    w[2].w[0] = h;
    w[2].x[0] = t.x[1];
    w[0].out = dwg;
    w[1].out = dwu;
    w[2].out = dwd;
    weights.plan();
  }
};

int device_error(const char* fn, hipError_t e) {
  set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
  return SF_ERR_DEVICE;
}

}  // namespace

}  // namespace sf

using namespace sf;

// (Whether an array is read as it is depends on its address, which is not known here: the larger need is given.)
extern "C" int64_t sf_ffn_workspace_bytes(const sf_ffn_config* cfg, int backward) {
  if (check(cfg, "sf_ffn_workspace_bytes") != SF_OK) return -1;
  if (!backward && few_rows(cfg)) return (int64_t)pad64((int64_t)cfg->M * cfg->F) * 4;
  Job j{cfg, nullptr};
  Arena a = {nullptr, 0};
  void* const odd = (void*)2;
  if (backward) {
    const Backward p(j, a, odd, odd, odd, odd, odd, odd, odd, odd, odd);
    a.bytes(p.in.part_bytes(0));
    for (int i = 0; i < 3; ++i) a.bytes(p.weights.part_bytes(i));
  } else {
    const Forward p(j, a, odd, odd, odd, odd, odd);
    a.bytes(p.down.part_bytes(0));
  }
  return (int64_t)a.at;
}

extern "C" int sf_ffn(const sf_ffn_config* cfg, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y,
                      void* workspace, void* hip_stream) {
  static const char* fn = "sf_ffn";
  const int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = cfg->M == 0;
  if (!fits(fn, "x", x, e, none) || !fits(fn, "w_gate", w_gate, e) || !fits(fn, "w_up", w_up, e) || !fits(fn, "w_down", w_down, e) ||
      !fits(fn, "y", y, 16, none) || !fits(fn, "workspace", workspace, 256, none))
    return SF_ERR_ARG;
  if (none) return SF_OK;
  Job j{cfg, reinterpret_cast<hipStream_t>(hip_stream)};
  hipError_t err;
  if (few_rows(cfg)) {
    const auto whole = [&](const void* p, int64_t pitch, int cols) {
      return cols % 8 == 0 && pitch % (16 / (int64_t)e) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
    };
    RowsArgs g = {};
    g.w[0] = w_gate;
    g.w[1] = w_up;
    g.x = x;
    g.w_pitch[0] = cfg->w_gate_stride;
    g.w_pitch[1] = cfg->w_up_stride;
    g.x_pitch = cfg->x_stride;
    g.K = cfg->D;
    g.F = cfg->F;
    g.M = cfg->M;
    g.act = cfg->act;
    g.out = workspace;
    g.vec = whole(w_gate, g.w_pitch[0], cfg->D) && whole(w_up, g.w_pitch[1], cfg->D) && whole(x, g.x_pitch, cfg->D);
    err = launch_rows<2>(cfg->dtype, g, j.st);
    if (err != hipSuccess) return device_error(fn, err);
    RowsArgs d = {};
    d.w[0] = w_down;
    d.x = workspace;
    d.w_pitch[0] = cfg->w_down_stride;
    d.x_pitch = cfg->F;
    d.K = cfg->F;
    d.F = cfg->D;
    d.M = cfg->M;
    d.out = y;
    d.vec = whole(w_down, d.w_pitch[0], cfg->F) && whole(workspace, cfg->F, cfg->F);
    err = launch_rows<1>(cfg->dtype, d, j.st);
    return err == hipSuccess ? SF_OK : device_error(fn, err);
  }
  Arena a = {(unsigned char*)workspace, 0};
  Forward p(j, a, x, w_gate, w_up, w_down, y);
  if ((err = j.run_layout()) != hipSuccess || (err = launch<kPair>(p.up, j.st)) != hipSuccess ||
      (err = p.down.run<0>(a, cfg->dtype, j.st)) != hipSuccess)
    return device_error(fn, err);
  return SF_OK;
}

extern "C" int sf_ffn_backward(const sf_ffn_config* cfg, const void* x, const void* w_gate, const void* w_up, const void* w_down,
                               const void* dy, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                               void* hip_stream) {
  static const char* fn = "sf_ffn_backward";
  const int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = cfg->M == 0;
  if (!fits(fn, "x", x, e, none) || !fits(fn, "w_gate", w_gate, e) || !fits(fn, "w_up", w_up, e) || !fits(fn, "w_down", w_down, e) ||
      !fits(fn, "dy", dy, e, none) || !fits(fn, "dx", dx, 16, none) || !fits(fn, "dw_gate", dw_gate, 16) ||
      !fits(fn, "dw_up", dw_up, 16) || !fits(fn, "dw_down", dw_down, 16) || !fits(fn, "workspace", workspace, 256, none))
    return SF_ERR_ARG;
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t err;
  if (none) {  // sums over no rows
    const int64_t n = (int64_t)cfg->D * cfg->F * (e / 2);
    for (void* p : {dw_gate, dw_up, dw_down}) ffn_zero_kernel<<<256, kThreads, 0, st>>>((uint16_t*)p, n);
    err = hipGetLastError();
    return err == hipSuccess ? SF_OK : device_error(fn, err);
  }
  Job j{cfg, st};
  Arena a = {(unsigned char*)workspace, 0};
  Backward p(j, a, x, w_gate, w_up, w_down, dy, dx, dw_gate, dw_up, dw_down);
  // (dx: w across k; the weights' gradients: both operands)
  if ((err = j.run_layout()) != hipSuccess || (err = launch<kTriple>(p.mid, st)) != hipSuccess ||
      (err = p.in.run<1>(a, cfg->dtype, st)) != hipSuccess || (err = p.weights.run<17>(a, cfg->dtype, st)) != hipSuccess)
    return device_error(fn, err);
  return SF_OK;
}
