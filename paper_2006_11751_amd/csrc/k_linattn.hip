// Linear attention with a decay for each head (include/sf_memory.h), in chunks of C = 32 steps:
//   inside a chunk  o_i += sum over j <= i, same episode: g^(i-j) (q_i . k_j) v_j
//   from before     o_i += g^(i+1) S q_i          where no episode begins up to i
//   the state       S <- g^n S + sum_j g^(n-1-j) k_j v_j^T   (terms from before the chunk's last episode begin: none)
// Every gradient is the same sum with other arrays in the three places and, for two of them, time reversed:
//   dq: (do, v, k) forwards with S transposed;  dk: (v, do, q) and dv: (k, q, do) backwards with the state
//   R_t = scale q_t do_t^T + g R_{t+1}.
// So there is one kernel, told by LinOp what stands where; a launch of the backward pass runs all three.  (Short trajectories
// have a kernel of their own for the gradients, a single step has one.)
//
// A workgroup of four waves walks the chunks of one (row, head), or of one piece of T, for 64 columns of v.  A wave owns 16
// of them: its part of the state stays in registers as the accumulator of the update.  The products are arranged
// so that accumulators feed the next product without a shuffle: a 16x16 accumulator holds rows 4g .. 4g+3 of one
// column per lane (g = lane / 16), two of them are the eight K-slots of an operand of 16x16x32, and the other operand
// follows the same numbering of the K axis.
//   P^T = K Q^T   [j][i]   masked and decayed in registers, shared by the waves through LDS in operand order
//   O^T = V^T P^T + S^T Q^T [dv][i]    the second product scaled per lane (a lane is a step i)
//   S  += K^T V~  [dk][dv]   V~: v times its step's weight
// K^T and V^T are read from row-major LDS with the transposing read (fp32: element by element).
//
// Roundings.  bf16 arrays enter the products as they are.  What is computed in fp32 and enters a product goes in as
// a sum of bf16 numbers: P and S for the output in two terms (2^-16 of them is left out at most, the output is
// rounded to 2^-8), V~ for the state, which is fp32, in three (nothing is left out).  fp32 arrays run on the fp32 matrix
// instruction throughout.
//
// Masked entries are selected, but a product still multiplies their zeros with the other operand's rows, and 0 x NaN
// is NaN.  So the chunk's k and v are tested as they are staged; a chunk with a NaN or an infinity in them is taken again as
// chunks of one step, which keeps it from earlier steps and from later episodes.
//
// Measured, bf16.  32 steps of 64 rows x 8 heads of 64 (25 MB): 8 us, of which a chunk's chain of load, two products and
// store is most (3.2 TB/s); 2048 rows: 186 us, 4.3 TB/s; 128 steps of 256 rows: 39 us, 5.1.  16384 steps of one row, 8 heads
// of 128, in 64 pieces: 26 us for the pieces' states, 16 to join them (70 MB written and read), 49 for the results: the
// eight chunks of a piece in sequence, each twice.  fp32, 333 steps of 30 rows x 6 heads of 40 and 72, gradients: 92 us for
// the sweeps, eleven chunks in sequence of 8 us each on the fp32 matrix instruction, 11 for the shared heads' sums.
// Columns that are no multiple of 8, and unaligned rows, are read and written by unaligned pieces (200 rows x 100 steps x 8 heads
// of 100: 167 us, 1.5 TB/s; number by number 245).  Forwards in fp32: 32 steps of 64 rows 9.0 us, of 2048 226, 4.8 TB/s; 128 steps of 256
// rows 87, 3.9, of heads of 128 238.  Gradients beyond 32 steps or 64 columns, by three sweeps that each read their arrays: 128 steps of
// 512 rows x 8 heads of 64 205 us in bf16 (3.3 TB/s of what has to move), 378 in fp32; 256 rows of heads of 128 277 and 615.
// The results' kernel for whole rows of 128 in bf16 has four workgroups a CU at the price of 20 bytes a lane in scratch memory.
#include <math.h>

#include <algorithm>

#include "sf_internal.h"
#include "sf_memory.h"
#include "sf_split.h"

namespace sf {

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

// n / d for 0 <= n < 2^31, without a division on the device
struct Divisor {
  unsigned mul, shift;
  __device__ unsigned of(unsigned n) const { return (__umulhi(mul, n) + n) >> shift; }
};
Divisor divisor(unsigned d) {
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

struct LinOp {
  Strided q, k, v;
  void* o;
  int64_t ot, on, oh;
  int o_f32, o_vec;     // the output is fp32 whatever the arrays are (partial sums of shared heads); 16-byte pieces
  const float* s_in;    // state before the first step, or null; [N][H] matrices of d(k) x d(v), element (a, b) at
  float* s_out;         //   a * s_a + b * s_b; state behind the last one, or null
  int64_t s_a, s_b;
  float w_scale, alpha; // of the terms k v^T (in state and output), of the output
  int reverse;          // time runs backwards: an episode boundary lies behind its step, the state
                        //   enters the first step undecayed and leaves decayed
};
struct LinArgs {
  LinOp op[3];
  const float* log_decay;
  const uint8_t* done;  // or null
  int T, N, H, ops;
  int blocks_v;         // of 64 columns of the widest v
  Divisor round, heads, share;  // 8 ops blocks_v, H, heads that share one of k and v
  int n_seg, seg_len;   // pieces of T (seg_len a multiple of every C)
  float* seg_state;     // n_seg > 1: [op][N * H][n_seg][dk * dv], first the pieces' own states, then what enters them
  float* seg_keep;      // [op][N * H][n_seg] g^length, -1 if an episode begins in the piece
};

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
// The decay's binary logarithm: no -infinity (times zero it would be NaN), but a NaN stays one.
__device__ inline float log2_decay(float log_decay) {
  const float l2 = log_decay * 1.44269504f;
  return l2 < -1e30f ? -1e30f : l2;
}

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

constexpr int C = 32;   // steps of a chunk
constexpr int DV = 64;  // columns of v of a workgroup: 16 a wave

template <int DTYPE, int D>
struct Lds {
  typedef Num<DTYPE> M;
  // of a row: 4 times an odd number of words, so that 16 rows' pieces of 16 bytes lie in different banks; of those 36 and 12
  // mod 64 also keep the transposing read's four rows of 32 bytes apart
  static constexpr int pitch(int columns) { return columns * M::kBytes + (M::kBytes == 2 && columns == 128 ? 48 : 16); }
  static constexpr int kPitch = pitch(D), kPitchV = pitch(DV);
  static constexpr int kK = C * kPitch, kV = 2 * C * kPitch;
  static constexpr int kFrags = C / 16;                     // operands of P: 32 steps j, 16 steps i
  static constexpr int kTermPitch = kFrags * 1024;
  static constexpr int kP = kV + C * kPitchV;               // two terms (or halves) of kFrags x 64 lanes x 16 bytes
  static constexpr int kEp = kP + 2 * kTermPitch;           // int [C]: episode of the step, counted in the chunk
  static constexpr int kW = kEp + C * 4;                    // float [C]: weight of the step's term in the state
  static constexpr int kFlag = kW + C * 4;                  // int [2]: the chunk holds something not finite
  static constexpr int kBytes = kFlag + 16;
};

// STATE: only the piece's own state (from zero) and whether an episode begins in it.
// How much of a call is known at compile time: kAny; kPieces: all rows are read and written in 16-byte pieces; kWhole: k and v
// have whole tiles besides, D and a multiple of 64 columns (else columns past theirs are left out, 32 of k, 16 of v at a time).
enum Known { kAny = 0, kPieces = 1, kWhole = 2 };
template <int DTYPE, int D, bool STATE, int KNOWN>
__global__ __launch_bounds__(kThreads, KNOWN == kAny ? 2 : D == 64 || DTYPE == SF_DTYPE_BF16 ? 4 : 3) void linattn_kernel(LinArgs g) {
  typedef Num<DTYPE> M;
  typedef Lds<DTYPE, D> L;
  constexpr int W = M::kPieceWords, NP = C * D / 8 / kThreads;  // pieces of a tile of q or k per thread; one of v's
  constexpr int ND = D / 16;                                    // tiles of k
  static_assert(C * DV / 8 == kThreads && C == 32, "a piece of v per thread, one operand for the chunk's steps");
  constexpr bool WHOLE = KNOWN == kWhole;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  // the ops of one (row, head) read the same arrays: one after another on one XCD (workgroups go to the 8 in turn)
  const unsigned round = g.round.of(blockIdx.x), in_round = blockIdx.x - round * (8 * g.ops * g.blocks_v), turn8 = in_round >> 3;
  const int v_block = (int)turn8 >= g.ops ? DV : 0, which = (int)turn8 - (v_block ? g.ops : 0);
  const int bh = (int)(round * 8 + (in_round & 7));
  const LinOp op = g.op[which];
  if (bh >= g.N * g.H || v_block >= op.v.d) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h), seg = blockIdx.y;
  const int t_begin = seg * g.seg_len, t_end = min(g.T, t_begin + g.seg_len);  // in the op's own direction
  const int dk = op.k.d, dv = op.v.d;
  const float l2 = log2_decay(g.log_decay[h]);
  const bool scan = g.n_seg > 1;
  const size_t seg_at = ((size_t)which * g.N * g.H + bh) * g.n_seg + seg;

  auto row_of = [&](const Strided& a) { return (const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes; };
  const unsigned char *const qrow = row_of(op.q), *const krow = row_of(op.k), *const vrow = row_of(op.v);

  const int v0 = v_block + 16 * wave;  // this wave's columns of v (past dv: nothing to do)
  const bool has_v = WHOLE || v0 < dv;
  auto has_k = [&](int s) { return WHOLE || 32 * s < dk; };  // columns 32 s .. of k
  // column of k of tile t (two tiles are 32 columns: eight neighbours per lane group)
  auto col_k = [&](int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); };

  // Memory is read and written through buffers that begin at a uniform address: what differs from lane to lane is an offset
  // that stays the same from chunk to chunk, what is not there has an offset past the end (it is read as zero, not written).
  constexpr unsigned kOutside = 0x80000000u;
  auto buffer = [&](const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000); };
  f32x4 S[ND];
  {
    const float* s = nullptr;
    int sa = (int)op.s_a, sb = (int)op.s_b;
    if constexpr (!STATE) {
      if (scan) {
        s = g.seg_state + seg_at * ((size_t)dk * dv);
        sa = dv;
        sb = 1;
      } else if (op.s_in) {
        s = op.s_in + (size_t)bh * dk * dv;
      }
    }
    const auto from = buffer(s, s ? dk * dv * 4 : 0);
    const int y = v0 + li;
    if (KNOWN != kAny && sa == 1) {  // neighbours of k lie side by side (their columns are a multiple of eight)
#pragma unroll
      for (int a = 0; a < ND; ++a) {
        const int x = col_k(a, 4 * lg);
        const unsigned at = WHOLE || (x < dk && y < dv) ? (unsigned)(y * sb + x) * 4 : kOutside;
        S[a] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0));
      }
    } else {
#pragma unroll
      for (int a = 0; a < ND; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int x = col_k(a, 4 * lg + r);
          const unsigned at = WHOLE || (x < dk && y < dv) ? (unsigned)(8 * lg * sa + y * sb) * 4 : kOutside;
          S[a][r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, at, (32 * (a >> 1) + 4 * (a & 1) + r) * sa * 4, 0));
        }
    }
  }

  // the chunk that is on its way: its rows and its episode marks
  unsigned nq[NP][W], nk[NP][W], nv[W];
  int n_done = 0;
  auto step_of = [&](int i) { return op.reverse ? g.T - 1 - i : i; };
  int alone_to = t_begin;  // steps before this one are chunks of their own
  auto width = [&](int c0) { return c0 < alone_to ? 1 : min(C, t_end - c0); };
  // row r of a chunk, in its order in memory
  auto place = [&](int r) { return op.reverse ? C - 1 - r : r; };
  auto first_of = [&](int c0) { return (int64_t)(op.reverse ? g.T - C - c0 : c0); };  // (may lie outside: its row is not there then)
  constexpr int kPieceRow = D / 8, kPieceRowV = DV / 8;  // pieces of a row
  unsigned at_q[NP], at_k[NP], at_v = kOutside;
  if constexpr (KNOWN != kAny) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int piece = tid + p * kThreads, r = piece / kPieceRow, col = piece % kPieceRow * 8;
      const bool in = WHOLE || col < dk;
      at_q[p] = in ? (unsigned)(place(r) * (int)op.q.st + col) * M::kBytes : kOutside;
      at_k[p] = in ? (unsigned)(place(r) * (int)op.k.st + col) * M::kBytes : kOutside;
    }
    const int col = v_block + tid % kPieceRowV * 8;
    if (WHOLE || col < dv) at_v = (unsigned)(place(tid / kPieceRowV) * (int)op.v.st + col) * M::kBytes;
  }
  auto fetch = [&](unsigned* w, __amdgpu_buffer_rsrc_t from, unsigned at) {
#pragma unroll
    for (int i = 0; i < W; i += 4) *(u32x4*)(w + i) = __builtin_amdgcn_raw_buffer_load_b128(from, at + 4 * i, 0, 0);
  };
  auto request = [&](int c0) {
    const int valid = width(c0);
    if constexpr (KNOWN != kAny) {
      const int64_t t = first_of(c0);
      const auto bq = buffer(qrow + t * op.q.st * M::kBytes, 0x7FFFFFFF), bk = buffer(krow + t * op.k.st * M::kBytes, 0x7FFFFFFF),
                 bv = buffer(vrow + t * op.v.st * M::kBytes, 0x7FFFFFFF);
      const bool all = valid == C;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const bool live = all || (tid + p * kThreads) / kPieceRow < valid;
        if constexpr (!STATE) fetch(nq[p], bq, live ? at_q[p] : kOutside);
        fetch(nk[p], bk, live ? at_k[p] : kOutside);
      }
      fetch(nv, bv, all || tid / kPieceRowV < valid ? at_v : kOutside);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int piece = tid + p * kThreads, r = piece / kPieceRow, col = piece % kPieceRow * 8;
        const bool live = r < valid;
        const int64_t t = step_of(live ? c0 + r : t_end - 1);
        if constexpr (!STATE) load_piece<DTYPE>(nq[p], op.q, qrow + t * op.q.st * M::kBytes, col, live);
        load_piece<DTYPE>(nk[p], op.k, krow + t * op.k.st * M::kBytes, col, live);
      }
      const int r = tid / kPieceRowV;
      const bool live = r < valid;
      const int64_t t = step_of(live ? c0 + r : t_end - 1);
      load_piece<DTYPE>(nv, op.v, vrow + t * op.v.st * M::kBytes, v_block + tid % kPieceRowV * 8, live);
    }
    n_done = 0;
    if (g.done && lane < C && lane < valid) {
      const int i = c0 + lane;  // backwards the boundary before step i is the mark of the step after it in time
      if (!op.reverse) n_done = g.done[(size_t)i * g.N + n];
      else if (i > 0) n_done = g.done[(size_t)(g.T - i) * g.N + n];
    }
  };
  unsigned at_o[C / 16];  // of four neighbours of an output row
#pragma unroll
  for (int I = 0; I < C / 16; ++I) {
    const int y = v0 + 4 * lg;
    at_o[I] = y < dv ? (unsigned)(place(16 * I + li) * (int)op.ot + y) * (op.o_f32 ? 4 : M::kBytes) : kOutside;
  }
  unsigned char* const orow = (unsigned char*)op.o + (n * op.on + h * op.oh) * (op.o_f32 ? 4 : M::kBytes);
  unsigned char* const tq = lds;
  unsigned char* const tk = lds + L::kK;
  unsigned char* const tv = lds + L::kV;
  int* const ep = (int*)(lds + L::kEp);
  float* const wgt = (float*)(lds + L::kW);
  int* const flag = (int*)(lds + L::kFlag);
  if (tid < 2) flag[tid] = 0;

  bool any_done = false;
  request(t_begin);
  for (int c0 = t_begin, turn = 0, step; c0 < t_end; c0 += step, turn ^= 1) {
    const int valid = width(c0);
    const int late = c0 == 0 && op.reverse ? 1 : 0;  // the state enters undecayed
    const unsigned marks = (unsigned)__ballot(n_done != 0);  // (lanes below C)
    __syncthreads();  // the chunk before has been read
    float test = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int piece = tid + p * kThreads, at = piece / kPieceRow * L::kPitch + piece % kPieceRow * 8 * M::kBytes;
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        if constexpr (!STATE) *(u32x4*)(tq + at + 4 * i) = *(u32x4*)(nq[p] + i);
        *(u32x4*)(tk + at + 4 * i) = *(u32x4*)(nk[p] + i);
      }
      test = finite_test<DTYPE>(nk[p], test);
    }
    {
      const int at = tid / kPieceRowV * L::kPitchV + tid % kPieceRowV * 8 * M::kBytes;
#pragma unroll
      for (int i = 0; i < W; i += 4) *(u32x4*)(tv + at + 4 * i) = *(u32x4*)(nv + i);
      test = finite_test<DTYPE>(nv, test);
    }
    if (test != 0.0f) flag[turn] = 1;
    if (tid < C) {
      const int e = __popc(marks & ((2u << tid) - 1));
      ep[tid] = e;
      wgt[tid] = e == __popc(marks) && tid < valid ? op.w_scale * pow2(l2 * (float)(valid - 1 - tid)) : 0.0f;
    }
    __syncthreads();
    if (tid == 0) flag[turn ^ 1] = 0;  // (read by all before the barrier above)
    if (flag[turn] != 0 && valid > 1 && c0 >= alone_to) {  // again, step by step
      alone_to = c0 + valid;
      request(c0);
      step = 0;
      continue;
    }
    step = valid;
    if (c0 + valid < t_end) request(c0 + valid);
    any_done |= marks != 0;

    if constexpr (!STATE) {
      // P^T: 16 x 16 tiles [j tile J][i tile I], J <= I; a pair of tiles is one operand
      auto tile_p = [&](int I, int J) __attribute__((always_inline)) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        if (J <= I) {
#pragma unroll
          for (int s = 0; s < D / 32; ++s) {
            const int at = (32 * s + 8 * lg) * M::kBytes;
            if (has_k(s)) acc = M::mma(M::row(tk + (16 * J + li) * L::kPitch + at), M::row(tq + (16 * I + li) * L::kPitch + at), acc);
          }
          const int lag = 16 * (I - J) + li - 4 * lg;  // i - j of r = 0
          const float p_scale = op.w_scale * op.alpha;
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[r] = I > J || lag >= r ? acc[r] * (p_scale * pow2(l2 * (float)(lag - r))) : 0.0f;
          if (marks) {
            const int e = ep[16 * I + li];
            const i32x4 ej = *(const i32x4*)(ep + 16 * J + 4 * lg);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] = ej[r] == e ? acc[r] : 0.0f;
          }
        }
        M::put4(lds + L::kP + I * 1024, L::kTermPitch, lane, J, acc);
      };
      tile_p(wave >> 1, wave & 1);
    }
    __syncthreads();

    // V^T of this wave's columns: K-slots 0..3 are steps 4 g .., 4..7 are 16 further on
    typename M::Raw vt;
    if (has_v) {
      if constexpr (DTYPE == SF_DTYPE_BF16) {
        const unsigned char* at = tv + (4 * lg + (li >> 2)) * L::kPitchV + (16 * wave + 4 * (li & 3)) * M::kBytes;
        const u32x2 x = M::column4(at), y = M::column4(at + 16 * L::kPitchV);
        vt = u32x4{x[0], x[1], y[0], y[1]};
      } else {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          vt.x[r] = M::element(tv + (4 * lg + (r & 3) + 16 * (r >> 2)) * L::kPitchV + (16 * wave + li) * M::kBytes);
      }
    }

    if (!STATE && has_v) {
      // what the state gives all steps (two accumulator tiles of it are one operand), scaled per step, and on top of it what
      // the chunk's own steps give
      f32x4 out[C / 16];
#pragma unroll
      for (int I = 0; I < C / 16; ++I) out[I] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        if (!has_k(s)) continue;
        float x[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = S[2 * s][r];
          x[4 + r] = S[2 * s + 1][r];
        }
        const typename M::Out st = M::out_terms(x);
#pragma unroll
        for (int I = 0; I < C / 16; ++I)
          out[I] = M::mma(st, M::row(tq + (16 * I + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes), out[I]);
      }
#pragma unroll
      for (int I = 0; I < C / 16; ++I) {
        const int i = 16 * I + li;
        const float c = op.alpha * pow2(l2 * (float)(i + 1 - late));
        f32x4 own = out[I];
#pragma unroll
        for (int r = 0; r < 4; ++r) own[r] *= c;
        if (marks) {
          const bool reach = (marks & ((2u << i) - 1)) == 0;  // no episode has begun: the state is this step's
#pragma unroll
          for (int r = 0; r < 4; ++r) own[r] = reach ? own[r] : 0.0f;
        }
        own = M::mma(vt, M::get(lds + L::kP + I * 1024, L::kTermPitch, lane), own);
        if constexpr (KNOWN != kAny) {
          const unsigned at = i < valid ? at_o[I] : kOutside;
          const auto to = buffer(orow + first_of(c0) * op.ot * (op.o_f32 ? 4 : M::kBytes), 0x7FFFFFFF);
          if (op.o_f32) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, own), to, at, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16(own[0], own[1]), pack_bf16(own[2], own[3])}, to, at, 0, 0);
        } else {
          const int y = v0 + 4 * lg;
          const int64_t at = n * op.on + h * op.oh + step_of(c0 + i) * op.ot + y;
          if (i < valid && y + 4 <= dv) {
            if (op.o_f32) {
              __builtin_memcpy((float*)op.o + at, &own, 16);
            } else {
              const u32x2 two = {pack_bf16(own[0], own[1]), pack_bf16(own[2], own[3])};
              __builtin_memcpy((unsigned char*)op.o + at * 2, &two, 8);
            }
            continue;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (i >= valid || y + r >= dv) continue;
            if (op.o_f32) ((float*)op.o)[at + r] = own[r];
            else M::store((unsigned char*)op.o + (at + r) * M::kBytes, own[r]);
          }
        }
      }
    }

    const float keep = pow2(l2 * (float)(valid - late));
    if (marks) {
#pragma unroll
      for (int a = 0; a < ND; ++a) S[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    } else {
#pragma unroll
      for (int a = 0; a < ND; ++a)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[a][r] *= keep;
    }
    if (has_v) {
      const f32x4 w0 = *(const f32x4*)(wgt + 4 * lg), w1 = *(const f32x4*)(wgt + 16 + 4 * lg);
      float x[8];
      M::values(vt, x);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] *= w0[r];
        x[4 + r] *= w1[r];
      }
      const typename M::Sum vw = M::sum_terms(x);
#pragma unroll
      for (int a = 0; a < ND; ++a) {
        if (!has_k(a / 2)) continue;
        typename M::Raw kt;
        if constexpr (DTYPE == SF_DTYPE_BF16) {
          const unsigned char* at = tk + (4 * lg + (li >> 2)) * L::kPitch + col_k(a, 4 * (li & 3)) * M::kBytes;
          const u32x2 y = M::column4(at), z = M::column4(at + 16 * L::kPitch);
          kt = u32x4{y[0], y[1], z[0], z[1]};
        } else {
#pragma unroll
          for (int r = 0; r < 8; ++r)
            kt.x[r] = M::element(tk + (4 * lg + (r & 3) + 16 * (r >> 2)) * L::kPitch + col_k(a, li) * M::kBytes);
        }
        S[a] = M::mma(kt, vw, S[a]);
      }
    }
  }

  // (a state that is written lies [dk][dv])
  float* s = nullptr;
  float f = 1.0f;
  bool zero = false;
  if constexpr (STATE) {
    s = g.seg_state + seg_at * ((size_t)dk * dv);
    if (tid == 0 && v_block == 0)
      g.seg_keep[seg_at] = any_done ? -1.0f : pow2(l2 * (float)(t_end - t_begin - (seg == 0 && op.reverse ? 1 : 0)));
  } else if (op.s_out && seg == g.n_seg - 1) {
    s = op.s_out + (size_t)bh * dk * dv;
    if (op.reverse) {  // one step further back: to before the first step
      f = t_end > t_begin ? pow2(l2) : 1.0f;
      zero = g.done && t_end > t_begin && g.done[n] != 0;
    }
  }
  if (!s) return;
  const auto to = buffer(s, dk * dv * 4);
  const int y = v0 + li;
#pragma unroll
  for (int a = 0; a < ND; ++a)
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // (rows past dk lie past the end)
      const unsigned at = WHOLE || y < dv ? (unsigned)(8 * lg * dv + y) * 4 : kOutside;
      __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, zero ? 0.0f : f * S[a][r]), to, at, (32 * (a >> 1) + 4 * (a & 1) + r) * dv * 4, 0);
    }
}

// What enters each piece of T, from the pieces' own states: one thread per element of a state, kAhead pieces read ahead.
// Bound by those bytes' latency: 8 heads of 128 x 128, 64 pieces, 34 MB read and written: 15.7 us, 4.3 TB/s.
__global__ __launch_bounds__(kThreads) void linattn_join_kernel(LinArgs g) {
  constexpr int kAhead = 16;
  const LinOp& op = g.op[blockIdx.z];
  const int bh = blockIdx.y, dk = op.k.d, dv = op.v.d, e = blockIdx.x * kThreads + threadIdx.x;
  if (e >= dk * dv) return;
  const size_t at = ((size_t)blockIdx.z * g.N * g.H + bh) * g.n_seg, size = (size_t)dk * dv;
  float* s = g.seg_state + at * size + e;
  float in = op.s_in ? op.s_in[(size_t)bh * dk * dv + e / dv * op.s_a + e % dv * op.s_b] : 0.0f;
  for (int i0 = 0; i0 < g.n_seg; i0 += kAhead) {
    float own[kAhead], keep[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int j = min(i0 + i, g.n_seg - 1);
      own[i] = s[j * size];
      keep[i] = g.seg_keep[at + j];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= g.n_seg) break;
      s[(i0 + i) * size] = in;
      in = own[i] + (keep[i] < 0.0f ? 0.0f : keep[i] * in);  // (a decay may be zero: times NaN or infinity it is not)
    }
  }
}

// The whole backward pass of a trajectory of at most C steps and heads of at most 64 columns, one workgroup for each (row,
// head): a learner's rollouts (32 steps) fit.  Nothing has to be carried, so both directions of time are made from one copy
// of the arrays in LDS, where the three sweeps above read each array two or three times:
//   A = do v^T, P = q k^T, masked and decayed, A in both orders
//   dq^T = k^T A^T + state0 do^T,  dk^T = q^T A + dstate v^T,  dv^T = do^T P + dstate^T k^T,  dstate0 = q~^T do + g^T dstate
// (q~: q times what a step's term has decayed to before the first).  Roundings as above: what comes from fp32 enters a product
// in two terms, for dstate0 in three.  Bound by memory; 2048 rows x 8 heads of 64, 32 steps, bf16, both states: 1.28 GB in
// 265 us, 4.8 TB/s (three sweeps: 355; a row stride of 2 MB costs a tenth: 2000 rows reach 5.3).  What it took: results
// through LDS and out by whole rows (the accumulators' own 32 bytes a row: 331 us), states read 64 bytes of a row at a time
// (32, in two halves: 375), 16 neighbours to an XCD (one: 341).
struct ShortArgs {
  Strided q, k, v, d_o;
  void *dq, *dk, *dv;              // [T][N] rows of H heads
  const float *state0, *dstate;    // or null
  float* dstate0;                  // or null
  const float* log_decay;
  const uint8_t* done;             // or null
  int T, N, H, f32;                // f32: dk and dv are fp32 whatever the arrays are (partial sums of shared heads)
  float scale;
  Divisor heads, share;
};

template <int DTYPE>
struct ShortLds {
  static constexpr int kPitch = Lds<DTYPE, 64>::kPitch, kTile = C * kPitch;
  static constexpr int kM = 4 * kTile, kMatrix = 4096;  // three matrices of two operands in two terms (or halves)
  static constexpr int kEp = kM + 3 * kMatrix;          // int [C]
  static constexpr int kFirst = kEp + C * 4;            // float [C]: the decay from before the first step to this one; 0 past an episode begin
  static constexpr int kLast = kFirst + C * 4;          // float [C]: from this step to the last one; 0 if an episode begins between
  static constexpr int kFlag = kLast + C * 4;
  // at the end: dstate0 and the gradients, to go out by whole rows
  static constexpr int kStatePitch = 68 * 4, kOut = 64 * kStatePitch, kOutBytes = kOut + 3 * kTile;
  static constexpr int kBytes = kFlag + 16 > kOutBytes ? kFlag + 16 : kOutBytes;
};

template <int DTYPE>
__global__ __launch_bounds__(kThreads, DTYPE == SF_DTYPE_BF16 ? 4 : 3) void linattn_short_kernel(ShortArgs g) {
  typedef Num<DTYPE> M;
  typedef ShortLds<DTYPE> L;
  constexpr int W = M::kPieceWords;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  // (workgroups go round the XCDs: 16 neighbours, whose rows of a step are neighbours too, for each)
  const int bh = (blockIdx.x & ~127) + (blockIdx.x & 7) * 16 + ((blockIdx.x >> 3) & 15);
  if (bh >= g.N * g.H) return;
  const int n = (int)g.heads.of(bh), h = bh - n * g.H, hk = (int)g.share.of(h);
  const int T = g.T, dk = g.q.d, dv = g.v.d;
  const float l2 = log2_decay(g.log_decay[h]);
  constexpr unsigned kOutside = 0x80000000u;
  auto buffer = [&](const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000); };

  // the arrays: one piece of each a thread
  unsigned w[4][W];
  const int row = tid >> 3, col = (tid & 7) * 8;
  auto fetch = [&](unsigned* to, const Strided& a) {
    const auto from = buffer((const unsigned char*)a.p + (n * a.sn + (a.shared ? hk : h) * a.sh) * M::kBytes, 0x7FFFFFFF);
    const unsigned at = row < T && col < a.d ? (unsigned)(row * (int)a.st + col) * M::kBytes : kOutside;
#pragma unroll
    for (int i = 0; i < W; i += 4) *(u32x4*)(to + i) = __builtin_amdgcn_raw_buffer_load_b128(from, at + 4 * i, 0, 0);
  };
  fetch(w[0], g.q);
  fetch(w[1], g.k);
  fetch(w[2], g.v);
  fetch(w[3], g.d_o);
  const bool begin = g.done && lane < T && g.done[(size_t)lane * g.N + n] != 0;
  const unsigned marks = (unsigned)__ballot(begin);
  // the states as operands: rows 16 wave + li, eight K-slots 32 s + 16 (j / 4) + 4 lg + j % 4, so that four lanes read 64
  // bytes of a row together and the columns' slots are the rows of an accumulator too
  const size_t state_at = (size_t)bh * dk * dv;
  const int state_bytes = dk * dv * 4, mine = 16 * wave + li;
  const auto s0 = buffer(g.state0 + (g.state0 ? state_at : 0), g.state0 ? state_bytes : 0);
  const auto ds = buffer(g.dstate + (g.dstate ? state_at : 0), g.dstate ? state_bytes : 0);
  float in[2][8], end[2][8], end_t[2][8];  // state0 and dstate by rows of k, dstate by rows of v
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int x = 16 * s + 4 * lg;
    const unsigned at = x < dv ? (unsigned)(mine * dv + x) * 4 : kOutside;  // (rows past dk lie past the end)
    *(f32x4*)(in[s >> 1] + 4 * (s & 1)) = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(s0, at, 0, 0));
    *(f32x4*)(end[s >> 1] + 4 * (s & 1)) = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(ds, at, 0, 0));
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const unsigned at = mine < dv ? (unsigned)((16 * s + 4 * lg) * dv + mine) * 4 : kOutside;
#pragma unroll
    for (int j = 0; j < 4; ++j) end_t[s >> 1][4 * (s & 1) + j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ds, at, j * dv * 4, 0));
  }

  unsigned char *const tq = lds, *const tk = lds + L::kTile, *const tv = lds + 2 * L::kTile, *const to = lds + 3 * L::kTile;
  int* const ep = (int*)(lds + L::kEp);
  float *const first = (float*)(lds + L::kFirst), *const last = (float*)(lds + L::kLast);
  int* const flag = (int*)(lds + L::kFlag);
  if (tid == 0) *flag = 0;
  if (tid < C) {
    const int e = __popc(marks & ((2u << tid) - 1));
    ep[tid] = e;
    first[tid] = e == 0 ? pow2(l2 * (float)(tid + 1)) : 0.0f;
    last[tid] = tid < T && e == __popc(marks) ? pow2(l2 * (float)(T - 1 - tid)) : 0.0f;
  }
  __syncthreads();
  float test = 0.0f;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
#pragma unroll
    for (int i = 0; i < W; i += 4) *(u32x4*)(lds + a * L::kTile + row * L::kPitch + col * M::kBytes + 4 * i) = *(u32x4*)(w[a] + i);
    test = finite_test<DTYPE>(w[a], test);
  }
  if (test != 0.0f) *flag = 1;
  __syncthreads();

  const int64_t head_k = ((int64_t)n * g.H + h) * dk, head_v = ((int64_t)n * g.H + h) * dv, step_k = (int64_t)g.N * g.H * dk,
                step_v = (int64_t)g.N * g.H * dv;
  if (*flag) {
    // Element by element, so that nothing that is not finite meets a masked zero.
    float *const A = (float*)(lds + L::kM), *const P = A + C * C;
    auto at = [&](const unsigned char* tile, int r, int c) { return M::element(tile + r * L::kPitch + c * M::kBytes); };
    for (int e = tid; e < C * C; e += kThreads) {
      const int i = e / C, j = e % C;
      float a = 0.0f, p = 0.0f;
      if (j <= i && ep[i] == ep[j]) {
        for (int y = 0; y < dv; ++y) a += at(to, i, y) * at(tv, j, y);
        for (int x = 0; x < dk; ++x) p += at(tq, i, x) * at(tk, j, x);
        const float c = g.scale * pow2(l2 * (float)(i - j));
        a *= c;
        p *= c;
      }
      A[e] = a;
      P[e] = p;
    }
    __syncthreads();
    auto put = [&](void* out, bool f32, int64_t i, float v) {
      if (f32) ((float*)out)[i] = v;
      else M::store((unsigned char*)out + i * M::kBytes, v);
    };
    for (int e = tid; e < T * dk; e += kThreads) {
      const int t = e / dk, x = e % dk;
      float q = 0.0f, k = 0.0f, v = 0.0f;
      for (int j = 0; j <= t; ++j)
        if (ep[j] == ep[t]) q += A[t * C + j] * at(tk, j, x);
      for (int i = t; i < T; ++i)
        if (ep[i] == ep[t]) k += A[i * C + t] * at(tq, i, x);
      if (g.state0 && ep[t] == 0) {
        for (int y = 0; y < dv; ++y) v += g.state0[state_at + x * dv + y] * at(to, t, y);
        q += g.scale * first[t] * v;
      }
      if (g.dstate && ep[t] == ep[T - 1]) {
        v = 0.0f;
        for (int y = 0; y < dv; ++y) v += g.dstate[state_at + x * dv + y] * at(tv, t, y);
        k += last[t] * v;
      }
      put(g.dq, DTYPE == SF_DTYPE_FP32, t * step_k + head_k + x, q);
      put(g.dk, g.f32, t * step_k + head_k + x, k);
    }
    for (int e = tid; e < T * dv; e += kThreads) {
      const int t = e / dv, y = e % dv;
      float v = 0.0f, k = 0.0f;
      for (int i = t; i < T; ++i)
        if (ep[i] == ep[t]) v += P[i * C + t] * at(to, i, y);
      if (g.dstate && ep[t] == ep[T - 1]) {
        for (int x = 0; x < dk; ++x) k += g.dstate[state_at + x * dv + y] * at(tk, t, x);
        v += last[t] * k;
      }
      put(g.dv, g.f32, t * step_v + head_v + y, v);
    }
    if (g.dstate0)
      for (int e = tid; e < dk * dv; e += kThreads) {
        float v = 0.0f;
        for (int i = 0; i < T; ++i)
          if (ep[i] == 0) v += g.scale * first[i] * at(tq, i, e / dv) * at(to, i, e % dv);
        if (g.dstate && marks == 0) v += pow2(l2 * (float)T) * g.dstate[state_at + e];
        g.dstate0[state_at + e] = v;
      }
    return;
  }

  // the matrices: wave (I, J) makes its tile of each, i in tile I, j in tile J
  {
    const int I = wave >> 1, J = wave & 1;
    f32x4 m1 = {0.0f, 0.0f, 0.0f, 0.0f}, m2 = m1, m3 = m1;
    if (J <= I) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int at_i = (16 * I + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes, at_j = (16 * J + li) * L::kPitch + (32 * s + 8 * lg) * M::kBytes;
        if (32 * s < dv) {
          const auto o = M::row(to + at_i), v = M::row(tv + at_j);
          m1 = M::mma(v, o, m1);  // [j][i]
          m2 = M::mma(o, v, m2);  // [i][j]
        }
        if (32 * s < dk) m3 = M::mma(M::row(tq + at_i), M::row(tk + at_j), m3);
      }
      const int ahead = 16 * (I - J);
      const int ei = ep[16 * I + li], ej = ep[16 * J + li];
      const i32x4 eis = *(const i32x4*)(ep + 16 * I + 4 * lg), ejs = *(const i32x4*)(ep + 16 * J + 4 * lg);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int lag1 = ahead + li - 4 * lg - r, lag2 = ahead + 4 * lg + r - li;
        m1[r] = lag1 >= 0 && ejs[r] == ei ? m1[r] * (g.scale * pow2(l2 * (float)lag1)) : 0.0f;
        const float c = g.scale * pow2(l2 * (float)lag2);
        const bool in2 = lag2 >= 0 && eis[r] == ej;
        m2[r] = in2 ? m2[r] * c : 0.0f;
        m3[r] = in2 ? m3[r] * c : 0.0f;
      }
    }
    unsigned char* const m = lds + L::kM;
    M::put4(m + I * 1024, 2048, lane, J, m1);
    M::put4(m + L::kMatrix + J * 1024, 2048, lane, I, m2);
    M::put4(m + 2 * L::kMatrix + J * 1024, 2048, lane, I, m3);
  }
  __syncthreads();

  // columns 16 wave .. (or, c0, others) of an array, K-slots its steps
  auto columns = [&](const unsigned char* tile, int c0) {
    typename M::Raw r;
    if constexpr (DTYPE == SF_DTYPE_BF16) {
      const unsigned char* at = tile + (4 * lg + (li >> 2)) * L::kPitch + (c0 + 4 * (li & 3)) * M::kBytes;
      const u32x2 x = M::column4(at), y = M::column4(at + 16 * L::kPitch);
      r = u32x4{x[0], x[1], y[0], y[1]};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) r.x[j] = M::element(tile + (4 * lg + (j & 3) + 16 * (j >> 2)) * L::kPitch + (c0 + li) * M::kBytes);
    }
    return r;
  };
  constexpr bool kF32 = DTYPE == SF_DTYPE_FP32;
  f32x4 kept[3][2] = {}, kept0[4] = {};
  // the K-slots of the states, of a row
  auto slots = [&](const unsigned char* at) {
    typename M::Raw r;
    if constexpr (DTYPE == SF_DTYPE_BF16) {
      const u32x2 x = *(const u32x2*)at, y = *(const u32x2*)(at + 32);
      r = u32x4{x[0], x[1], y[0], y[1]};
    } else {
      *(f32x4*)&r.x[0] = *(const f32x4*)at;
      *(f32x4*)&r.x[4] = *(const f32x4*)(at + 64);
    }
    return r;
  };
  // one gradient: what the state gives (its rows by the other array's rows), scaled per step, and on top what the steps give
  auto gradient = [&](const float (*state)[8], bool has_state, const unsigned char* rows, int d_rows, const float* weight, float scale,
                      const typename M::Raw& by_step, int matrix, void* out, bool f32, int64_t step, int64_t head, int d) {
    if (16 * wave >= d) return;
#pragma unroll
    for (int I = 0; I < 2; ++I) {
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      const int t = 16 * I + li;
      if (has_state) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (32 * s < d_rows) acc = M::mma(M::out_terms(state[s]), slots(rows + t * L::kPitch + (32 * s + 4 * lg) * M::kBytes), acc);
        const float c = scale * weight[t];
        const bool reach = weight == first ? ep[t] == 0 : ep[t] == __popc(marks);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = reach ? acc[r] * c : 0.0f;
      }
      acc = M::mma(by_step, M::get(lds + L::kM + matrix * L::kMatrix + I * 1024, 2048, lane), acc);
      const int y = 16 * wave + 4 * lg;
      kept[matrix][I] = acc;
      if (f32 && !kF32 && t < T && y < d) *(f32x4*)((float*)out + t * step + head + y) = acc;
    }
  };
  gradient(in, g.state0 != nullptr, to, dv, first, g.scale, columns(tk, 16 * wave), 0, g.dq, kF32, step_k, head_k, dk);
  gradient(end, g.dstate != nullptr, tv, dv, last, 1.0f, columns(tq, 16 * wave), 1, g.dk, kF32 || g.f32, step_k, head_k, dk);
  const typename M::Raw o = columns(to, 16 * wave);
  gradient(end_t, g.dstate != nullptr, tk, dk, last, 1.0f, o, 2, g.dv, kF32 || g.f32, step_v, head_v, dv);

  if (g.dstate0 && 16 * wave < dv) {
    f32x4 w0 = *(const f32x4*)(first + 4 * lg), w1 = *(const f32x4*)(first + 16 + 4 * lg);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      w0[r] *= g.scale;
      w1[r] *= g.scale;
    }
    const float keep = pow2(l2 * (float)T);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (16 * s >= dk) break;
      float x[8];
      M::values(columns(tq, 16 * s), x);
      f32x4 acc;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] *= w0[r];
        x[4 + r] *= w1[r];
        acc[r] = marks ? 0.0f : keep * end_t[s >> 1][4 * (s & 1) + r];
      }
      kept0[s] = M::mma(M::sum_terms(x), o, acc);
    }
  }

  __syncthreads();
#pragma unroll
  for (int m = 0; m < 3; ++m)
#pragma unroll
    for (int I = 0; I < 2; ++I) {
      unsigned char* const at = lds + L::kOut + m * L::kTile + (16 * I + li) * L::kPitch + (16 * wave + 4 * lg) * M::kBytes;
      if constexpr (kF32) *(f32x4*)at = kept[m][I];
      else *(u32x2*)at = u32x2{pack_bf16(kept[m][I][0], kept[m][I][1]), pack_bf16(kept[m][I][2], kept[m][I][3])};
    }
  if (g.dstate0) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) *(float*)(lds + (16 * s + 4 * lg + r) * L::kStatePitch + mine * 4) = kept0[s][r];
  }
  __syncthreads();
  auto store = [&](void* out, int m, int64_t at, int d) {
    if (row >= T || col >= d) return;
#pragma unroll
    for (int i = 0; i < W; i += 4)
      *(u32x4*)((unsigned char*)out + at * M::kBytes + 4 * i) = *(const u32x4*)(lds + L::kOut + m * L::kTile + row * L::kPitch + col * M::kBytes + 4 * i);
  };
  store(g.dq, 0, row * step_k + head_k + col, dk);
  if (kF32 || !g.f32) {
    store(g.dk, 1, row * step_k + head_k + col, dk);
    store(g.dv, 2, row * step_v + head_v + col, dv);
  }
  if (!g.dstate0) return;
  const auto put = buffer(g.dstate0 + state_at, state_bytes);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = 16 * i + (tid >> 4), y = 4 * (tid & 15);
    __builtin_amdgcn_raw_buffer_store_b128(*(const u32x4*)(lds + x * L::kStatePitch + y * 4), put, y < dv ? (unsigned)(x * dv + y) * 4 : kOutside, 0, 0);
  }
}

// Sums of the gradients of shared heads: in [rows][H][d] fp32, out [rows][H / share][d].  (In a launch of their own, in one
// order: 9990 rows, 6 heads of 40 to 2: 4.9 us.)
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void linattn_share_kernel(const float* in, void* out, int64_t n_out, int d, int share) {
  for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < n_out; e += (int64_t)gridDim.x * kThreads) {
    const float* x = in + e / d * share * d + e % d;
    float sum = 0.0f;
    for (int i = 0; i < share; ++i) sum += x[(int64_t)i * d];
    Num<DTYPE>::store((unsigned char*)out + e * Num<DTYPE>::kBytes, sum);
  }
}

// One step of one (row, head): the state is read, decayed, added to, written and multiplied with q.  Bound by those
// bytes; a thread holds four neighbours of every (256 / lanes)-th row, so that all its loads are under way at once.  2048 rows
// x 8 heads of 64 (546 MB): 112 us, 4.9 TB/s; 16 rows: 5.5 us, a launch and one trip to memory.
template <int DTYPE, bool VEC>
__global__ __launch_bounds__(kThreads) void linattn_step_kernel(LinOp op, const float* log_decay, const uint8_t* done, float* table,
                                                                int n_env, const int32_t* ids, int H, int share, int lanes_log2) {
  typedef Num<DTYPE> M;
  __shared__ float sq[128], sk[128];
  __shared__ __attribute__((aligned(16))) float part[4][128];
  const int tid = threadIdx.x, n = blockIdx.x / H, h = blockIdx.x % H, dk = op.k.d, dv = op.v.d;
  const int id = ids ? ids[n] : n;
  const bool known = id >= 0 && id < n_env;
  const bool begin = !known || (done && done[n] != 0);
  const float gam = exp2f(log2_decay(log_decay[h]));
  const int rows = kThreads >> lanes_log2, row0 = tid >> lanes_log2, c0 = (tid & ((1 << lanes_log2) - 1)) * 4;
  float* s = table + ((int64_t)(known ? id : 0) * H + h) * dk * dv;
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
    if (tid < dk) sk[tid] = M::element((const unsigned char*)op.k.p + (n * op.k.sn + h / share * op.k.sh + tid) * M::kBytes);
  } else if (tid - 128 < dk) {
    sq[tid - 128] = M::element((const unsigned char*)op.q.p + (n * op.q.sn + h * op.q.sh + tid - 128) * M::kBytes);
  }
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    v[j] = c0 + j < dv ? M::element((const unsigned char*)op.v.p + (n * op.v.sn + h / share * op.v.sh + c0 + j) * M::kBytes) : 0.0f;
  __syncthreads();
  float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int r = row0 + i * rows;
    if (r >= dk || c0 >= dv) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[i][j] = sk[r] * v[j] + (begin ? 0.0f : gam * x[i][j]);
      o[j] += sq[r] * x[i][j];
    }
    if (!known) continue;
    if constexpr (VEC) {
      *(f32x4*)(s + r * dv + c0) = *(f32x4*)x[i];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c0 + j < dv) s[r * dv + c0 + j] = x[i][j];
    }
  }
  // over the rows: within the wave, then over the four waves
  for (int m = 1 << lanes_log2; m < 64; m <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], m);
  if ((tid & 63) < 1 << lanes_log2 && c0 < 128)
    *(f32x4*)&part[tid >> 6][c0] = f32x4{o[0], o[1], o[2], o[3]};
  __syncthreads();
  if (tid < dv) {
    const float sum = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
    M::store((unsigned char*)op.o + (n * op.on + h * op.oh + tid) * M::kBytes, op.alpha * sum);
  }
}

// ---- host side ---------------------------------------------------------------------------------

int check(const sf_linattn_config* c, const char* fn) {
  if (!c || c->struct_size != sizeof(sf_linattn_config)) {
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
  if ((int64_t)c->T * c->N > INT32_MAX || (int64_t)c->N * c->H > 1 << 21) {
    set_error("%s: T * N beyond 2^31 - 1 or N * H beyond 2^21", fn);
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
bool overlap(const sf_linattn_config* c, const float* a, const float* b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), size = (uintptr_t)c->N * c->H * c->dk * c->dv * 4;
  return a && b && (x == y || (x < y ? y - x : x - y) < size);
}

struct Split {
  int n_seg, seg_len;
};
// Pieces of T where the workgroups (one for each 64 columns of a head, and backwards for each of the three gradients) leave CUs
// idle, each with at least 256 steps.  The pieces' states cost a pass over k and v more, two launches and their own bytes, so T has
// to be longer the more heads and the larger states there are, and from 384 workgroups on no length pays.
// us whole and cut, heads of 64 and 128 columns, H of them over all rows:
//                     bf16 64, 1024 steps   4096       128, 1024    4096        fp32 64, 1024   4096       128, 1024    4096
//   forwards    8     52 30                 199 32     75 40        291 46      87 42           342 45     133 62       550 74
//              96     59 43                 225 86     85 87        361 250     98 70           440 180    144 153      616 513
//             192     59 58                 262 178    98 153       413 444     100 98          449 347    224 292      867 944
//             240     60 68                 264 222    108 189      419 540     104 119         455 410    226 375      871 1234
//   backwards   8     52 31                 200 41     75 49        308 72      88 44           363 65     134 71       544 146
//              48     58 52                 223 116    95 123       388 320     96 88           406 240    209 231      846 731
//              96     66 78                 286 229    114 200      474 595     130 141         567 473    299 440      1185 1447
Split split_of(const sf_linattn_config* c, int ops) {
  const int64_t lanes = (int64_t)c->N * c->H * ops;
  const int columns = std::max(c->dk, c->dv);
  const bool cut = lanes > 0 && lanes * (columns > DV ? 2 : 1) < 384 && c->T > 512 + lanes * columns / 24;
  const int64_t want = cut ? (768 + lanes - 1) / lanes : 1;
  int64_t len = (c->T + want - 1) / want;
  len = (len + 63) / 64 * 64;
  if (len < 256) len = 256;
  if (len >= c->T) return Split{1, c->T > 0 ? c->T : 1};
  return Split{(int)((c->T + len - 1) / len), (int)len};
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
struct Workspace {
  size_t state, keep, dk, dv, total;  // bytes of each part, in this order
};
Workspace workspace_of(const sf_linattn_config* c, int backward) {
  const int ops = backward ? 3 : 1;
  const Split s = split_of(c, ops);
  Workspace w = {0, 0, 0, 0, 0};
  const size_t rows = (size_t)c->T * c->N * c->H;
  if (s.n_seg > 1) {
    w.state = align256((size_t)ops * c->N * c->H * s.n_seg * c->dk * c->dv * 4);
    w.keep = align256((size_t)ops * c->N * c->H * s.n_seg * 4);
  }
  if (backward && c->H != c->Hk) {
    w.dk = align256(rows * c->dk * 4);
    w.dv = align256(rows * c->dv * 4);
  }
  w.total = w.state + w.keep + w.dk + w.dv;
  return w;
}

// (a chunk's rows lie within 2^31 bytes then, and one behind the other)
bool near(int64_t st, int d) { return st >= d && st <= 1 << 23; }
Strided strided(const sf_linattn_config* c, const void* p, const int64_t* s, bool shared, int d) {
  Strided a = {p, c->T == 1 ? 0 : s[0], s[1], s[2], shared, d, 0};  // (one step: any stride)
  const int per = 16 / (c->dtype == SF_DTYPE_BF16 ? 2 : 4);
  // (pieces are eight columns in both types)
  a.vec = d % 8 == 0 && (c->T == 1 || near(s[0], d)) && (a.st % per) == 0 && (s[1] % per) == 0 && (s[2] % per) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
  return a;
}
void put_out(const sf_linattn_config* c, LinOp& op, void* p, int64_t t, int64_t n, int64_t h, int d, bool f32) {
  op.o = p;
  op.ot = c->T == 1 ? 0 : t;
  op.on = n;
  op.oh = h;
  op.o_f32 = f32 || c->dtype == SF_DTYPE_FP32;
  const int per = op.o_f32 ? 4 : 8;
  op.o_vec = d % 8 == 0 && (c->T == 1 || near(t, d)) && op.ot % per == 0 && n % per == 0 && h % per == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

template <int DTYPE, int D, bool STATE, int KNOWN>
hipError_t launch_k(const LinArgs& g, hipStream_t st) {
  const auto kern = linattn_kernel<DTYPE, D, STATE, KNOWN>;
  constexpr int bytes = Lds<DTYPE, D>::kBytes;
  static_assert(bytes <= 64 * 1024, "no attribute needed");
  kern<<<dim3((unsigned)((g.N * g.H + 7) / 8 * 8 * g.ops * g.blocks_v), (unsigned)g.n_seg), kThreads, bytes, st>>>(g);
  return hipGetLastError();
}
template <int DTYPE, int D, bool STATE>
hipError_t launch_t(const LinArgs& g, hipStream_t st) {
  bool pieces = true, whole = true;
  for (int i = 0; i < g.ops; ++i) {
    const LinOp& o = g.op[i];
    pieces = pieces && o.q.vec && o.k.vec && o.v.vec && o.o_vec;
    whole = whole && o.k.d == D && o.v.d % DV == 0;
  }
  if (!pieces) return launch_k<DTYPE, D, STATE, kAny>(g, st);
  return whole ? launch_k<DTYPE, D, STATE, kWhole>(g, st) : launch_k<DTYPE, D, STATE, kPieces>(g, st);
}
template <bool STATE>
hipError_t launch(const sf_linattn_config* c, LinArgs& g, hipStream_t st) {
  bool wide = false;
  g.blocks_v = 1;
  for (int i = 0; i < g.ops; ++i) {
    wide = wide || g.op[i].k.d > 64;
    if (g.op[i].v.d > DV) g.blocks_v = 2;
  }
  g.round = divisor(8 * g.ops * g.blocks_v);
  g.heads = divisor(g.H);
  g.share = divisor(c->H / c->Hk);
  if (c->dtype == SF_DTYPE_FP32) return wide ? launch_t<SF_DTYPE_FP32, 128, STATE>(g, st) : launch_t<SF_DTYPE_FP32, 64, STATE>(g, st);
  return wide ? launch_t<SF_DTYPE_BF16, 128, STATE>(g, st) : launch_t<SF_DTYPE_BF16, 64, STATE>(g, st);
}

int run(const char* fn, const sf_linattn_config* c, LinArgs& g, int ops, const Workspace& w, unsigned char* ws, hipStream_t st) {
  if (c->N == 0) return SF_OK;
  const Split s = split_of(c, ops);
  g.T = c->T;
  g.N = c->N;
  g.H = c->H;
  g.ops = ops;
  g.n_seg = s.n_seg;
  g.seg_len = s.seg_len;
  hipError_t e = hipSuccess;
  if (s.n_seg > 1) {
    g.seg_state = (float*)ws;
    g.seg_keep = (float*)(ws + w.state);
    e = launch<true>(c, g, st);
    if (e == hipSuccess) {
      linattn_join_kernel<<<dim3((unsigned)((c->dk * c->dv + kThreads - 1) / kThreads), (unsigned)(c->N * c->H), (unsigned)ops), kThreads, 0,
                            st>>>(g);
      e = hipGetLastError();
    }
  }
  if (e == hipSuccess) e = launch<false>(c, g, st);
  if (e != hipSuccess) {
    set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
    return SF_ERR_DEVICE;
  }
  return SF_OK;
}

// The sums over the heads that share one of k and v.
int add_shared(const char* fn, const sf_linattn_config* c, const float* part_k, const float* part_v, void* dk, void* dv, hipStream_t st) {
  const int share = c->H / c->Hk;
  const int64_t nk = (int64_t)c->T * c->N * c->Hk * c->dk, nv = (int64_t)c->T * c->N * c->Hk * c->dv;
  const auto grid = [](int64_t n) { return (unsigned)std::min<int64_t>((n + kThreads - 1) / kThreads, 1 << 20); };
  if (c->dtype == SF_DTYPE_BF16) {
    linattn_share_kernel<SF_DTYPE_BF16><<<grid(nk), kThreads, 0, st>>>(part_k, dk, nk, c->dk, share);
    linattn_share_kernel<SF_DTYPE_BF16><<<grid(nv), kThreads, 0, st>>>(part_v, dv, nv, c->dv, share);
  } else {
    linattn_share_kernel<SF_DTYPE_FP32><<<grid(nk), kThreads, 0, st>>>(part_k, dk, nk, c->dk, share);
    linattn_share_kernel<SF_DTYPE_FP32><<<grid(nv), kThreads, 0, st>>>(part_v, dv, nv, c->dv, share);
  }
  const hipError_t err = hipGetLastError();
  if (err == hipSuccess) return SF_OK;
  set_error("%s: launch failed: %s", fn, hipGetErrorString(err));
  return SF_ERR_DEVICE;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" int64_t sf_linattn_workspace_bytes(const sf_linattn_config* cfg, int backward) {
  if (check(cfg, "sf_linattn_workspace_bytes") != SF_OK) return -1;
  return (int64_t)workspace_of(cfg, backward).total;
}

extern "C" int sf_linattn(const sf_linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                          const uint8_t* done, const float* state0, void* o, float* state, void* workspace, void* hip_stream) {
  static const char* fn = "sf_linattn";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = (int64_t)cfg->T * cfg->N == 0;
  const Workspace w = workspace_of(cfg, 0);
  if ((rc = check_ptr(fn, "q", q, e, none)) || (rc = check_ptr(fn, "k", k, e, none)) || (rc = check_ptr(fn, "v", v, e, none)) ||
      (rc = check_ptr(fn, "o", o, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4)) ||
      (rc = check_ptr(fn, "state0", state0, 4, true)) || (rc = check_ptr(fn, "state", state, 4, true)) ||
      (rc = check_ptr(fn, "workspace", workspace, 256, w.total == 0)))
    return rc;
  if (state != state0 && overlap(cfg, state, state0)) {
    set_error("%s: state overlaps state0", fn);
    return SF_ERR_ALIAS;
  }
  LinArgs g = {};
  g.log_decay = log_decay;
  g.done = done;
  LinOp& op = g.op[0];
  const int share = cfg->H / cfg->Hk;
  op.q = strided(cfg, q, cfg->q_stride, false, cfg->dk);
  op.k = strided(cfg, k, cfg->k_stride, share > 1, cfg->dk);
  op.v = strided(cfg, v, cfg->v_stride, share > 1, cfg->dv);
  put_out(cfg, op, o, cfg->o_stride[0], cfg->o_stride[1], cfg->o_stride[2], cfg->dv, false);
  op.s_in = state0;
  op.s_out = state;
  op.s_a = cfg->dv;
  op.s_b = 1;
  op.w_scale = 1.0f;
  op.alpha = cfg->scale;
  return run(fn, cfg, g, 1, w, (unsigned char*)workspace, reinterpret_cast<hipStream_t>(hip_stream));
}

extern "C" int sf_linattn_backward(const sf_linattn_config* cfg, const void* q, const void* k, const void* v,
                                   const float* log_decay, const void* d_o, const uint8_t* done, const float* state0,
                                   const float* dstate, void* dq, void* dk, void* dv, float* dstate0, void* workspace,
                                   void* hip_stream) {
  static const char* fn = "sf_linattn_backward";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = (int64_t)cfg->T * cfg->N == 0;
  const Workspace w = workspace_of(cfg, 1);
  if ((rc = check_ptr(fn, "q", q, e, none)) || (rc = check_ptr(fn, "k", k, e, none)) || (rc = check_ptr(fn, "v", v, e, none)) ||
      (rc = check_ptr(fn, "do", d_o, e, none)) || (rc = check_ptr(fn, "dq", dq, e, none)) || (rc = check_ptr(fn, "dk", dk, e, none)) ||
      (rc = check_ptr(fn, "dv", dv, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4)) ||
      (rc = check_ptr(fn, "state0", state0, 4, true)) || (rc = check_ptr(fn, "dstate", dstate, 4, true)) ||
      (rc = check_ptr(fn, "dstate0", dstate0, 4, true)) || (rc = check_ptr(fn, "workspace", workspace, 256, w.total == 0)))
    return rc;
  if (overlap(cfg, dstate0, dstate) || overlap(cfg, dstate0, state0)) {
    set_error("%s: dstate0 overlaps dstate or state0", fn);
    return SF_ERR_ALIAS;
  }
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const int H = cfg->H, Hk = cfg->Hk, share = H / Hk, Dk = cfg->dk, Dv = cfg->dv;
  unsigned char* ws = (unsigned char*)workspace;
  float* part_k = (float*)(ws + w.state + w.keep);
  float* part_v = (float*)(ws + w.state + w.keep + w.dk);
  const Strided sq = strided(cfg, q, cfg->q_stride, false, Dk), sk = strided(cfg, k, cfg->k_stride, share > 1, Dk),
                sv = strided(cfg, v, cfg->v_stride, share > 1, Dv), so = strided(cfg, d_o, cfg->o_stride, false, Dv);
  const auto sixteen = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
  if (cfg->T >= 1 && cfg->T <= C && Dk <= 64 && Dv <= 64 && sq.vec && sk.vec && sv.vec && so.vec && sixteen(dq) && sixteen(dk) && sixteen(dv)) {
    ShortArgs a = {};
    a.q = sq;
    a.k = sk;
    a.v = sv;
    a.d_o = so;
    a.dq = dq;
    a.dk = share > 1 ? part_k : dk;
    a.dv = share > 1 ? part_v : dv;
    a.state0 = state0;
    a.dstate = dstate;
    a.dstate0 = dstate0;
    a.log_decay = log_decay;
    a.done = done;
    a.T = cfg->T;
    a.N = cfg->N;
    a.H = H;
    a.f32 = share > 1 || cfg->dtype == SF_DTYPE_FP32;
    a.scale = cfg->scale;
    a.heads = divisor(H);
    a.share = divisor(share);
    if (!none) {
      if (cfg->dtype == SF_DTYPE_BF16) linattn_short_kernel<SF_DTYPE_BF16><<<(cfg->N * H + 127) / 128 * 128, kThreads, ShortLds<SF_DTYPE_BF16>::kBytes, st>>>(a);
      else linattn_short_kernel<SF_DTYPE_FP32><<<(cfg->N * H + 127) / 128 * 128, kThreads, ShortLds<SF_DTYPE_FP32>::kBytes, st>>>(a);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) {
      set_error("%s: launch failed: %s", fn, hipGetErrorString(err));
      return SF_ERR_DEVICE;
    }
    return share == 1 || none ? SF_OK : add_shared(fn, cfg, part_k, part_v, dk, dv, st);
  }
  LinArgs g = {};
  g.log_decay = log_decay;
  g.done = done;
  LinOp &oq = g.op[0], &ok = g.op[1], &ov = g.op[2];
  oq.q = so;
  oq.k = sv;
  oq.v = sk;
  put_out(cfg, oq, dq, (int64_t)cfg->N * H * Dk, (int64_t)H * Dk, Dk, Dk, false);
  oq.s_in = state0;
  oq.s_a = 1;
  oq.s_b = Dv;
  oq.w_scale = 1.0f;
  oq.alpha = cfg->scale;
  ok.q = sv;
  ok.k = so;
  ok.v = sq;
  put_out(cfg, ok, share > 1 ? part_k : dk, (int64_t)cfg->N * H * Dk, (int64_t)H * Dk, Dk, Dk, share > 1);
  ok.s_in = dstate;
  ok.s_a = 1;
  ok.s_b = Dv;
  ok.w_scale = cfg->scale;
  ok.alpha = 1.0f;
  ok.reverse = 1;
  ov.q = sk;
  ov.k = sq;
  ov.v = so;
  put_out(cfg, ov, share > 1 ? part_v : dv, (int64_t)cfg->N * H * Dv, (int64_t)H * Dv, Dv, Dv, share > 1);
  ov.s_in = dstate;
  ov.s_out = dstate0;
  ov.s_a = Dv;
  ov.s_b = 1;
  ov.w_scale = cfg->scale;
  ov.alpha = 1.0f;
  ov.reverse = 1;
  rc = run(fn, cfg, g, 3, w, ws, st);
  return rc != SF_OK || share == 1 || none ? rc : add_shared(fn, cfg, part_k, part_v, dk, dv, st);
}

extern "C" int sf_linattn_step(const sf_linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                               float* state_table, int32_t n_env, const int32_t* env_ids, const uint8_t* done, void* o,
                               void* hip_stream) {
  static const char* fn = "sf_linattn_step";
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
      (rc = check_ptr(fn, "o", o, e, none)) || (rc = check_ptr(fn, "log_decay", log_decay, 4)) ||
      (rc = check_ptr(fn, "state_table", state_table, 16)) || (rc = check_ptr(fn, "env_ids", env_ids, 4, true)))
    return rc;
  if (none) return SF_OK;
  const int share = cfg->H / cfg->Hk;
  LinOp op = {};
  op.q = strided(cfg, q, cfg->q_stride, false, cfg->dk);
  op.k = strided(cfg, k, cfg->k_stride, share > 1, cfg->dk);
  op.v = strided(cfg, v, cfg->v_stride, share > 1, cfg->dv);
  put_out(cfg, op, o, 0, cfg->o_stride[1], cfg->o_stride[2], cfg->dv, false);
  op.alpha = cfg->scale;
  // a thread has four columns; rows of a multiple of four floats are read 16 bytes at a time
  int lanes_log2 = 0;
  while ((4 << lanes_log2) < cfg->dv) ++lanes_log2;
  if (lanes_log2 < 4) lanes_log2 = 4;  // (256 threads then have 16 rows each of at most 256)
  const unsigned grid = (unsigned)(cfg->N * cfg->H);
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const bool vec = cfg->dv % 4 == 0;
  const auto kern = cfg->dtype == SF_DTYPE_BF16
                        ? (vec ? linattn_step_kernel<SF_DTYPE_BF16, true> : linattn_step_kernel<SF_DTYPE_BF16, false>)
                        : (vec ? linattn_step_kernel<SF_DTYPE_FP32, true> : linattn_step_kernel<SF_DTYPE_FP32, false>);
  kern<<<grid, kThreads, 0, st>>>(op, log_decay, done, state_table, n_env, env_ids, cfg->H, share, lanes_log2);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) {
    set_error("%s: launch failed: %s", fn, hipGetErrorString(err));
    return SF_ERR_DEVICE;
  }
  return SF_OK;
}
