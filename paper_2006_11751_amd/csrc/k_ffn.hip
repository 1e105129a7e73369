// The gated feed-forward block (include/sf_memory.h): h = act(x Wg^T) * (x Wu^T), y = h Wd^T, and its gradients.
//
// Every product is C[m][f] = sum_k X[m][k] W[f][k] with both operands dense in k (arrays that are not are laid out so
// first, in the workspace: for the gradients the weights and, for those of the weights, the rows transposed).  One
// kernel in three forms, all on the 16-bit matrix instruction 32x32x16 with fp32 accumulation:
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
// steps of BK through two buffers in LDS, the step after next under way in registers.  Rows in LDS are 16 bytes longer
// than their numbers: 16 neighbouring rows then lie in different banks.
//
// Few rows (serving): the weights are what is read, so each wave takes 16 rows of them straight into operands, the
// waves of a workgroup share K, and their sums are added in LDS.
#include <math.h>

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
// f(activation's number, whether it is fine) with both known at compile time
template <int N>
struct Constant {
  static constexpr int value = N;
};
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
  const uint16_t* p;  // [planes][rows][pitch] bf16, k dense, zeros from the array's own K to the padded one
  int64_t pitch, plane;
};
// Where numbers go that are operands of a later product: rows of `pitch`, one plane or three
struct Terms {
  uint16_t* p;
  int64_t pitch, plane;
};
struct GemmArgs {
  Operand w[3], x[2];
  int K;           // padded: a multiple of 64
  int pairs;       // kOne: pairs of operands that follow one another
  int terms;       // planes of each operand: 1 or 3
  int F, M;        // rows of w, of x
  int nf, nm;      // tiles
  int act;
  void* out;       // kOne: [M][F] (bf16 or, `out_f32`, fp32)
  int out_f32;
  int Fp, Mp;      // F, M padded to 64
  Terms h, dg, du;            // [M][Fp]: kPair h; kTriple dg, du
  Terms ht, dgt, dut;         // kTriple: [F][Mp]
};
struct GemmGroup {
  GemmArgs g[3];
  int n, tiles[3];  // problems of one launch and their tiles
};

// the planes of a product of two operands in three terms, smallest first
__device__ constexpr int kPlaneW[6] = {0, 1, 2, 0, 1, 0};
__device__ constexpr int kPlaneX[6] = {2, 1, 0, 1, 0, 0};

// (lanes of a wave exchange numbers through LDS: its accesses run in order, the compiler is kept from reordering them)
__device__ inline void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// eight neighbours, or their terms, at offset `at` (a multiple of 8)
__device__ inline void store_terms8(const Terms& t, int terms, int64_t at, const float* v) {
  u32x4 w[3];
  if (terms == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[0][i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *(u32x4*)(t.p + at) = w[0];
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
#pragma unroll
  for (int i = 0; i < 3; ++i) *(u32x4*)(t.p + i * t.plane + at) = w[i];
}
// eight neighbours of a result's row (its first `left` ones)
__device__ inline void store_out8(const GemmArgs& g, int64_t at, int left, const float* v) {
  if ((g.F & 7) == 0) {  // (out is 16-byte aligned)
    if (g.out_f32) {
      *(f32x4*)((float*)g.out + at) = *(const f32x4*)v;
      *(f32x4*)((float*)g.out + at + 4) = *(const f32x4*)(v + 4);
    } else {
      *(u32x4*)((uint16_t*)g.out + at) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    if (r >= left) break;
    if (g.out_f32) ((float*)g.out)[at + r] = v[r];
    else ((uint16_t*)g.out)[at + r] = (uint16_t)pack_bf16(v[r], 0.0f);
  }
}

// BF rows of each w, BM rows of each x per workgroup; a wave has half of both.
template <int FORM, int BF, int BM, int BK>
struct Tile {
  static constexpr int kW = FORM == kOne ? 1 : FORM == kPair ? 2 : 3, kX = FORM == kTriple ? 2 : 1;
  static constexpr int kRows = kW * BF + kX * BM, kPitch = BK * 2 + 16, kStage = kRows * kPitch;
  static constexpr int kEnd = 4 * kW * 32 * (BF / 2 + 4) * 4;  // behind the products: see there
  static constexpr int kBytes = 2 * kStage > kEnd ? 2 * kStage : kEnd;
  static constexpr int kPieces = kRows * (BK / 8) / kThreads;  // 16-byte pieces of a step per thread
};

template <int FORM, int BF, int BM, int BK, int WAVES>
__global__ __launch_bounds__(kThreads, WAVES) void ffn_gemm_kernel(GemmGroup group) {
  typedef Tile<FORM, BF, BM, BK> L;
  constexpr int W = L::kW, X = L::kX, TF = BF / 64, TM = BM / 64;  // a wave's 32 x 32 tiles
  constexpr int PR = BK / 8, RS = kThreads / PR;                   // pieces of a row; rows that all threads take at once
  static_assert(BF % RS == 0 && BM % RS == 0, "a piece's array is known at compile time");
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
  const int band = tile / (4 * g.nf), in_band = tile - band * 4 * g.nf, height = min(4, g.nm - 4 * band);
  const int f0 = in_band / height * BF, m0 = (4 * band + in_band % height) * BM;

  // this thread's pieces: row (tid / PR + RS * i) of the step's rows, piece tid % PR; bytes from the tile's first row on
  constexpr int NP = L::kPieces, NK = BK / 16, MF = W * TF * TM, FR = W * TF + X * TM;  // products, operands of 16 numbers of K
  unsigned row_at[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int first = RS * i;  // of the array's tile
    const bool of_w = first < W * BF;
    const int r = (of_w ? first % BF : (first - W * BF) % BM) + tid / PR;
    const Operand& o = of_w ? g.w[first / BF] : g.x[(first - W * BF) / BM];
    row_at[i] = (unsigned)min(r, (of_w ? g.F - 1 - f0 : g.M - 1 - m0)) * (unsigned)o.pitch * 2 + (tid % PR) * 16;  // (past the end: the last row, never stored)
  }
  // the step to be requested next: its pass (pair of operands, planes) and place in K
  const int passes = (g.terms == 1 ? 1 : 6) * g.pairs, steps = g.K / BK * passes;
  int pass = 0, k = 0;
  const unsigned char *wb[W], *xb[X];
  auto begin_pass = [&]() __attribute__((always_inline)) {
    const int pair = FORM == kOne && pass >= passes / g.pairs ? 1 : 0, term = g.terms == 1 ? 5 : pass - pair * 6;
#pragma unroll
    for (int a = 0; a < W; ++a) {
      const Operand& o = g.w[FORM == kOne ? pair : a];
      wb[a] = (const unsigned char*)(o.p + kPlaneW[term] * o.plane + (int64_t)f0 * o.pitch);
    }
#pragma unroll
    for (int a = 0; a < X; ++a) {
      const Operand& o = g.x[FORM == kOne ? pair : a];
      xb[a] = (const unsigned char*)(o.p + kPlaneX[term] * o.plane + (int64_t)m0 * o.pitch);
    }
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
  };
  u32x4 next[NP];
  auto request = [&](int i) __attribute__((always_inline)) {
    const int first = RS * i;
    const unsigned char* base = first < W * BF ? wb[first / BF] : xb[(first - W * BF) / BM];
    next[i] = *(const u32x4*)(base + 2 * k + row_at[i]);
  };
  unsigned char* const put_at = lds + tid / PR * L::kPitch + (tid % PR) * 16;
  auto put = [&](int i, int stage) __attribute__((always_inline)) { *(u32x4*)(put_at + stage + RS * i * L::kPitch) = next[i]; };
  const unsigned char* const w_at = lds + (wf * (BF / 2) + li) * L::kPitch + lh * 16;
  const unsigned char* const x_at = lds + (W * BF + wm * (BM / 2) + li) * L::kPitch + lh * 16;
  bf16x8 fw[2][W * TF], fx[2][X * TM];
  auto operands = [&](int to, int stage, int kk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < X * TM; ++i) fx[to][i] = *(const bf16x8*)(x_at + stage + (i / TM * BM + 32 * (i % TM)) * L::kPitch + kk * 32);
#pragma unroll
    for (int i = 0; i < W * TF; ++i) fw[to][i] = *(const bf16x8*)(w_at + stage + (i / TF * BF + 32 * (i % TF)) * L::kPitch + kk * 32);
  };

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
#pragma unroll
  for (int i = 0; i < NP; ++i) request(i);
#pragma unroll
  for (int i = 0; i < NP; ++i) put(i, 0);
  advance();
#pragma unroll
  for (int i = 0; i < NP; ++i) request(i);
  __syncthreads();
  operands(0, 0, 0);
  // One step: behind the products of 16 numbers of K the operands of the next 16 are read, and the pieces of the next step
  // go to LDS, each followed by the request for the step after that.  All reads of a step are done before its last products,
  // where the barrier stands: behind it the next step's first operands are read under these products.
  for (int s = 0; s < steps; ++s) {
    const int stage = (s & 1) * L::kStage, other = L::kStage - stage;
    advance();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const int cur = kk & 1;
      const bool last = kk == NK - 1;
      if (last) __syncthreads();
      operands(cur ^ 1, last ? other : stage, last ? 0 : kk + 1);
      const int p0 = last ? NP : NP * kk / (NK - 1), p1 = last ? NP : NP * (kk + 1) / (NK - 1);
#pragma unroll
      for (int i = p0; i < p1; ++i) {
        put(i, other);
        request(i);
      }
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int b = 0; b < TF; ++b)
#pragma unroll
          for (int c = 0; c < TM; ++c)
            acc[a][b][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fw[cur][a * TF + b], fx[cur][(FORM == kTriple && a == 2 ? TM : 0) + c],
                                                                   acc[a][b][c], 0, 0, 0);
      // the order of all that: spread evenly behind the products
      const int extra = FR + (p1 - p0);
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
    }
  }
  __syncthreads();  // (the last step's needless reads are done: LDS is written again)

  // An accumulator has one column m = li per lane and, four at a time, neighbouring rows f = 8 q + 4 lh.  The wave's columns
  // go through LDS (its own part), 32 of x at a time, so that what is stored are whole pieces of neighbours.
  constexpr int FW = 32 * TF, EP = FW + 4;      // a wave's rows of w; row length there
  constexpr int LPR = FW / 8, NI = LPR / 2;     // lanes of a row m, rounds of 64 lanes over 32 rows
  float* const area = (float*)lds + wave * (W * 32 * EP);
  const int fwave = f0 + wf * FW;
  const GemmArgs a_ = g;  // (kept in registers: behind wave_order it would be read again and again)
  const bool fine = a_.terms == 3;
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
        if (m < a_.M && f < a_.F) store_out8(a_, (int64_t)m * a_.F + f, a_.F - f, area + row * EP + col);
      }
    } else {
      with_activation(a_.act, fine, [&](auto act, auto exact) __attribute__((always_inline)) {
#pragma unroll 2
        for (int i = 0; i < NI; ++i) {
          const int row = i * (64 / LPR) + lane / LPR, col = lane % LPR * 8, m = mw + row, f = fwave + col;
          float* const at = area + row * EP + col;
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
            const bool in = f + r < a_.F && m < a_.M;  // (zeros where a later product's K is padded)
            h[r] = in ? v * up[r] : 0.0f;
            if constexpr (FORM == kTriple) {
              dg[r] = in ? dh[r] * up[r] * slope : 0.0f;
              du[r] = in ? dh[r] * v : 0.0f;
            }
          }
          if constexpr (FORM == kPair) {
            if (m < a_.M && f < a_.Fp) store_terms8(a_.h, a_.terms, (int64_t)m * a_.h.pitch + f, h);
          } else {
            if (m < a_.M && f < a_.Fp) {
              store_terms8(a_.dg, a_.terms, (int64_t)m * a_.dg.pitch + f, dg);
              store_terms8(a_.du, a_.terms, (int64_t)m * a_.du.pitch + f, du);
            }
#pragma unroll
            for (int r = 0; r < 8; r += 4) {  // for the transposed ones
              *(f32x4*)(at + r) = *(f32x4*)(h + r);
              *(f32x4*)(at + 32 * EP + r) = *(f32x4*)(dg + r);
              *(f32x4*)(at + 64 * EP + r) = *(f32x4*)(du + r);
            }
          }
        }
      });
    }
    if constexpr (FORM == kTriple) {
      wave_order();
#pragma unroll 2
      for (int i = 0; i < FW / 16; ++i) {  // 16 rows f at a time, 4 lanes with 8 columns m each
        const int row = 16 * i + lane / 4, col = lane % 4 * 8, f = fwave + row, m = mw + col;
        if (f >= a_.Fp || m >= a_.Mp) continue;
#pragma unroll
        for (int a = 0; a < 3; ++a) {
          float v[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) v[r] = area[(a * 32 + col + r) * EP + row];
          const Terms& t = a == 0 ? a_.ht : a == 1 ? a_.dgt : a_.dut;
          store_terms8(t, a_.terms, (int64_t)f * t.pitch + m, v);
        }
      }
    }
  }
}

// ---- laying operands out -----------------------------------------------------------------------

struct Layout {
  const void* from;   // [rows][cols] of the calls' type, rows `pitch` elements apart
  int64_t pitch;
  int rows, cols;
  Terms to;           // [rows][pitch] or, transposed, [cols][pitch]; zeros up to the pitch
  int transpose;
  int tiles;          // 64 x 64 tiles
};
struct LayoutGroup {
  Layout l[5];
  int n;
};

template <int DTYPE>
__global__ __launch_bounds__(kThreads) void ffn_layout_kernel(LayoutGroup group) {
  __shared__ float s[64][65];
  int tile = blockIdx.x, which = 0;
  while (which + 1 < group.n && tile >= group.l[which].tiles) tile -= group.l[which++].tiles;
  const Layout& l = group.l[which];
  const int nc = (l.cols + 63) / 64, r0 = tile / nc * 64, c0 = tile % nc * 64;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = r0 + y + 4 * i, c = c0 + x;
    float v = 0.0f;
    if (r < l.rows && c < l.cols) {
      const int64_t at = r * l.pitch + c;
      v = DTYPE == SF_DTYPE_BF16 ? from_bf16(((const uint16_t*)l.from)[at]) : ((const float*)l.from)[at];
    }
    s[y + 4 * i][x] = v;
  }
  __syncthreads();
  // pairs of neighbours of the result
  const int n_out = l.transpose ? l.cols : l.rows, o0 = l.transpose ? c0 : r0, k0 = l.transpose ? r0 : c0;
  const int k = (threadIdx.x & 31) * 2, o1 = threadIdx.x >> 5;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int o = o1 + 8 * i;
    if (o0 + o >= n_out) continue;
    const float a = l.transpose ? s[k][o] : s[o][k], b = l.transpose ? s[k + 1][o] : s[o][k + 1];
    unsigned* to = (unsigned*)(l.to.p + (o0 + o) * l.to.pitch + k0 + k);
    if (DTYPE == SF_DTYPE_BF16) {
      *to = pack_bf16(a, b);
    } else {
      unsigned t[3];
      float left = 0.0f;
      split_pair(a, b, t[0], t[1], t[2], left);
#pragma unroll
      for (int j = 0; j < 3; ++j) to[j * l.to.plane / 2] = t[j];
    }
  }
}

// ---- few rows ----------------------------------------------------------------------------------

// C[m][f] for M <= 16 MT rows: 16 rows of each w per workgroup, its waves share K.
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
  const int f0 = blockIdx.x * 16;
  const int f_row = min(f0 + li, g.F - 1);
  f32x4 acc[W][MT];
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int c = 0; c < MT; ++c) acc[a][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int U = VEC ? 2 : 1;  // steps whose loads are under way together
  for (int k0 = wave * 32; k0 < g.K; k0 += U * kRowWaves * 32) {
    u32x4 rw[U][W], rx[U][MT];
    float vw[U][W][8], vx[U][MT][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kRowWaves * 32 + 8 * lg;
#pragma unroll
      for (int a = 0; a < W; ++a) load8<DTYPE, VEC>(vw[u][a], rw[u][a], g.w[a], f_row * g.w_pitch[a], k, g.K);
#pragma unroll
      for (int c = 0; c < MT; ++c) load8<DTYPE, VEC>(vx[u][c], rx[u][c], g.x, min(16 * c + li, g.M - 1) * g.x_pitch, k, g.K);
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
    const int m = 16 * c + li, f = f0 + 4 * lg;
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

constexpr int kFewRows = 64;

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
  Terms take(int64_t rows, int64_t pitch, int terms) {
    Terms t = {base ? (uint16_t*)(base + at) : nullptr, pitch, rows * pitch};
    at += ((size_t)(rows * pitch * terms) * 2 + 255) / 256 * 256;
    return t;
  }
};
Operand operand(const Terms& t) { return Operand{t.p, t.pitch, t.plane}; }

struct Job {
  const sf_ffn_config* c;
  hipStream_t st;
  LayoutGroup lay = {};
  int lay_tiles = 0;
  int terms() const { return c->dtype == SF_DTYPE_BF16 ? 1 : 3; }
  // An array as an operand, dense in its columns: itself where it can be read as it is, else laid out in the workspace.
  Operand rows(Arena& a, const void* p, int64_t pitch, int rows, int cols) {
    if (terms() == 1 && cols % 64 == 0 && pitch % 8 == 0 && pitch > 0 && pitch <= 1 << 22 && (reinterpret_cast<uintptr_t>(p) & 15) == 0)
      return Operand{(const uint16_t*)p, pitch, 0};
    return lay_out(a, p, pitch, rows, cols, 0);
  }
  Operand lay_out(Arena& a, const void* p, int64_t pitch, int rows, int cols, int transpose) {
    const Terms t = a.take(transpose ? cols : rows, pad64(transpose ? rows : cols), terms());
    lay.l[lay.n] = Layout{p, pitch, rows, cols, t, transpose, (int)(pad64(rows) / 64 * (pad64(cols) / 64))};
    lay_tiles += lay.l[lay.n++].tiles;
    return operand(t);
  }
  hipError_t run_layout() {
    if (!lay.n) return hipSuccess;
    if (c->dtype == SF_DTYPE_BF16) ffn_layout_kernel<SF_DTYPE_BF16><<<lay_tiles, kThreads, 0, st>>>(lay);
    else ffn_layout_kernel<SF_DTYPE_FP32><<<lay_tiles, kThreads, 0, st>>>(lay);
    lay.n = lay_tiles = 0;
    return hipGetLastError();
  }
};

template <int FORM, int BF, int BM, int BK, int WAVES>
hipError_t launch_t(GemmGroup& group, hipStream_t st) {
  const auto kern = ffn_gemm_kernel<FORM, BF, BM, BK, WAVES>;
  constexpr int bytes = Tile<FORM, BF, BM, BK>::kBytes;
  static const hipError_t attr = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  int total = 0;
  for (int i = 0; i < group.n; ++i) {
    GemmArgs& g = group.g[i];
    // (padded columns of the next product's operand are this one's rows of w)
    g.nf = ((FORM == kOne ? g.F : g.Fp) + BF - 1) / BF;
    g.nm = ((FORM == kTriple ? g.Mp : g.M) + BM - 1) / BM;
    total += group.tiles[i] = g.nf * g.nm;
  }
  kern<<<(total + 7) / 8 * 8, kThreads, bytes, st>>>(group);
  return hipGetLastError();
}
// The large tile where it leaves no CU without one, the small one otherwise.
template <int FORM>
hipError_t launch(GemmGroup& group, hipStream_t st) {
  int64_t large = 0;
  for (int i = 0; i < group.n; ++i) {
    const GemmArgs& g = group.g[i];
    if (FORM == kOne) large += (int64_t)((g.F + 255) / 256) * ((g.M + 255) / 256);
    else large += (int64_t)((g.Fp + 127) / 128) * ((g.M + (FORM == kPair ? 255 : 127)) / (FORM == kPair ? 256 : 128));
  }
  if constexpr (FORM == kOne) return large >= 192 ? launch_t<kOne, 256, 256, 64, 1>(group, st) : launch_t<kOne, 128, 128, 64, 2>(group, st);
  else if constexpr (FORM == kPair) return large >= 192 ? launch_t<kPair, 128, 256, 64, 1>(group, st) : launch_t<kPair, 64, 128, 64, 2>(group, st);
  else return large >= 192 ? launch_t<kTriple, 128, 128, 32, 1>(group, st) : launch_t<kTriple, 64, 128, 32, 2>(group, st);
}

template <int DTYPE, int W, bool VEC>
hipError_t launch_rows(const RowsArgs& g, hipStream_t st) {
  const unsigned grid = (unsigned)((g.F + 15) / 16);
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
  g.terms = terms;
  g.F = F;
  g.M = M;
  g.Fp = (int)pad64(F);
  g.Mp = (int)pad64(M);
  g.act = c->act;
  g.out_f32 = c->dtype == SF_DTYPE_FP32;
  return g;
}

struct ForwardPlan {
  Operand x, wg, wu, wd;
  Terms h;
};
ForwardPlan plan_forward(Job& j, Arena& a, const void* x, const void* wg, const void* wu, const void* wd) {
  const sf_ffn_config* c = j.c;
  ForwardPlan p;
  p.x = j.rows(a, x, c->x_stride, c->M, c->D);
  p.wg = j.rows(a, wg, c->w_gate_stride, c->F, c->D);
  p.wu = j.rows(a, wu, c->w_up_stride, c->F, c->D);
  p.wd = j.rows(a, wd, c->w_down_stride, c->D, c->F);
  p.h = a.take(c->M, pad64(c->F), j.terms());
  return p;
}
struct BackwardPlan {
  Operand x, wg, wu, dy, wd_t, wg_t, wu_t, x_t, dy_t;
  Terms dg, du, ht, dgt, dut;
};
// (the layouts are run in two launches: five fit one)
BackwardPlan plan_backward(Job& j, Job& j2, Arena& a, const void* x, const void* wg, const void* wu, const void* wd, const void* dy) {
  const sf_ffn_config* c = j.c;
  BackwardPlan p;
  p.x = j.rows(a, x, c->x_stride, c->M, c->D);
  p.wg = j.rows(a, wg, c->w_gate_stride, c->F, c->D);
  p.wu = j.rows(a, wu, c->w_up_stride, c->F, c->D);
  p.dy = j.rows(a, dy, c->dy_stride, c->M, c->D);
  p.wd_t = j.lay_out(a, wd, c->w_down_stride, c->D, c->F, 1);
  p.wg_t = j2.lay_out(a, wg, c->w_gate_stride, c->F, c->D, 1);
  p.wu_t = j2.lay_out(a, wu, c->w_up_stride, c->F, c->D, 1);
  p.x_t = j2.lay_out(a, x, c->x_stride, c->M, c->D, 1);
  p.dy_t = j2.lay_out(a, dy, c->dy_stride, c->M, c->D, 1);
  const int64_t Fp = pad64(c->F), Mp = pad64(c->M);
  p.dg = a.take(c->M, Fp, j.terms());
  p.du = a.take(c->M, Fp, j.terms());
  p.ht = a.take(Fp, Mp, j.terms());
  p.dgt = a.take(Fp, Mp, j.terms());
  p.dut = a.take(Fp, Mp, j.terms());
  return p;
}

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
  if (!backward && cfg->M <= kFewRows) return (int64_t)pad64((int64_t)cfg->M * cfg->F) * 4;
  Job j{cfg, nullptr}, j2{cfg, nullptr};
  Arena a = {nullptr, 0};
  const void* const odd = (const void*)2;
  if (backward) plan_backward(j, j2, a, odd, odd, odd, odd, odd);
  else plan_forward(j, a, odd, odd, odd, odd);
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
  if (cfg->M <= kFewRows) {
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
  const ForwardPlan p = plan_forward(j, a, x, w_gate, w_up, w_down);
  if ((err = j.run_layout()) != hipSuccess) return device_error(fn, err);
  GemmGroup up = {};
  up.n = 1;
  up.g[0] = gemm(cfg, j.terms(), cfg->D, cfg->F, cfg->M);
  up.g[0].w[0] = p.wg;
  up.g[0].w[1] = p.wu;
  up.g[0].x[0] = p.x;
  up.g[0].h = p.h;
  if ((err = launch<kPair>(up, j.st)) != hipSuccess) return device_error(fn, err);
  GemmGroup down = {};
  down.n = 1;
  down.g[0] = gemm(cfg, j.terms(), cfg->F, cfg->D, cfg->M);
  down.g[0].w[0] = p.wd;
  down.g[0].x[0] = operand(p.h);
  down.g[0].out = y;
  err = launch<kOne>(down, j.st);
  return err == hipSuccess ? SF_OK : device_error(fn, err);
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
  Job j{cfg, st}, j2{cfg, st};
  Arena a = {(unsigned char*)workspace, 0};
  const BackwardPlan p = plan_backward(j, j2, a, x, w_gate, w_up, w_down, dy);
  if ((err = j.run_layout()) != hipSuccess || (err = j2.run_layout()) != hipSuccess) return device_error(fn, err);
  const int terms = j.terms();
  GemmGroup mid = {};
  mid.n = 1;
  GemmArgs& t = mid.g[0];
  t = gemm(cfg, terms, cfg->D, cfg->F, cfg->M);
  t.w[0] = p.wg;
  t.w[1] = p.wu;
  t.w[2] = p.wd_t;
  t.x[0] = p.x;
  t.x[1] = p.dy;
  t.dg = p.dg;
  t.du = p.du;
  t.ht = p.ht;
  t.dgt = p.dgt;
  t.dut = p.dut;
  if ((err = launch<kTriple>(mid, st)) != hipSuccess) return device_error(fn, err);
  GemmGroup in = {};
  in.n = 1;
  in.g[0] = gemm(cfg, terms, cfg->F, cfg->D, cfg->M);
  in.g[0].pairs = 2;
  in.g[0].w[0] = p.wg_t;
  in.g[0].w[1] = p.wu_t;
  in.g[0].x[0] = operand(p.dg);
  in.g[0].x[1] = operand(p.du);
  in.g[0].out = dx;
  if ((err = launch<kOne>(in, st)) != hipSuccess) return device_error(fn, err);
  GemmGroup w = {};
  w.n = 3;
  for (int i = 0; i < 3; ++i) w.g[i] = i < 2 ? gemm(cfg, terms, cfg->M, cfg->D, cfg->F) : gemm(cfg, terms, cfg->M, cfg->F, cfg->D);
  w.g[0].w[0] = w.g[1].w[0] = p.x_t;
  w.g[0].x[0] = operand(p.dgt);
  w.g[1].x[0] = operand(p.dut);
  w.g[2].w[0] = operand(p.ht);
  w.g[2].x[0] = p.dy_t;
  w.g[0].out = dw_gate;
  w.g[1].out = dw_up;
  w.g[2].out = dw_down;
  err = launch<kOne>(w, st);
  return err == hipSuccess ? SF_OK : device_error(fn, err);
}
