// The norms behind and before a block with its gate, residual scale and residual stream (include/sf_memory.h), in
// one pass over the rows, forwards and backwards:
//   u = N_post(b) post_w,  y = x + scale act(gate) u,  n = N_pre(y) pre_w
// What bounds it is memory: each array is read or written once.  A row stays in the registers of LPR lanes (8 .. 64, or
// the workgroup's 256), eight neighbours of a lane at a time; its sums go over the lanes, and with 256 of them over
// LDS.  A group of lanes walks rows a grid apart, with the weights of its columns in registers and the next row's loads
// under way.  The norm over groups of channels (post only) makes a row of each group.
//
// Backwards everything is computed again from b, x and the gate, which costs no byte more than reading y would.
// Gradients of the weights are sums over rows: a lane adds its rows up in registers, the workgroup's lanes of one
// column are added, and a second launch adds the workgroups', always in the same order.
//
// Measured, bf16: 2048 x 512 forwards (8.4 MB) 4.6 us, a launch and one trip to memory; 16384 x 2048 with a gate backwards
// (537 MB) 108-113 us, 4.9 TB/s, and 4.8 for the sums of 512 workgroups.  fp32 calls, forwards and backwards: 2048 x 512 8.0 and 13.8 us,
// 16384 x 2048 129 and 219 (5.2 and 4.9 TB/s), 8192 x 4096 128 and 232.  Above 4096 columns a lane has four pieces, and backwards these
// do not fit its registers (scratch memory, bytes a lane: 388-432 in bf16, 732-768 in fp32): 4096 x 8192 95 and 547 us in bf16, 174 and
// 822 in fp32 (backwards 1.0 and 1.3 TB/s).
//
// All arithmetic is fp32; results are rounded once, n from the y that is not rounded.
#include <math.h>

#include "sf_internal.h"
#include "sf_memory.h"

namespace sf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

struct NormArgs {
  const void *b, *x, *gate, *dy, *dn;  // rows of D; all but b may be null
  int64_t b_s, x_s, gate_s, dy_s, dn_s;
  void *y, *n, *dx, *db, *dgate;       // dense rows; null where not wanted
  const float *post_w, *pre_w, *scale; // [D] or null
  float* part;                         // backwards: [slots / groups][3][D], see the second kernel
  int64_t rows;                        // M
  int D, Dg, groups;                   // columns, columns of a group
  int post, pre, act;
  float eps;
};

template <int DTYPE>
struct Io;
template <>
struct Io<SF_DTYPE_BF16> {
  static constexpr int kBytes = 2, kWords = 4;
  __device__ static void values(const unsigned* w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
    }
  }
  __device__ static void words(const float* v, unsigned* w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 p = {v[2 * i], v[2 * i + 1]};
      w[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
    }
  }
  __device__ static void put(unsigned* w, int j, const unsigned char* p) { w[j / 2] |= (unsigned)*(const uint16_t*)p << (16 * (j & 1)); }
  __device__ static void store(unsigned char* p, const unsigned* w, int j) { *(uint16_t*)p = (uint16_t)(w[j / 2] >> (16 * (j & 1))); }
  // (native exponential and reciprocal: 2^-21, the result is rounded to 2^-8)
  __device__ static float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }
};
template <>
struct Io<SF_DTYPE_FP32> {
  static constexpr int kBytes = 4, kWords = 8;
  __device__ static void values(const unsigned* w, float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, w[i]);
  }
  __device__ static void words(const float* v, unsigned* w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_bit_cast(unsigned, v[i]);
  }
  __device__ static void put(unsigned* w, int j, const unsigned char* p) { w[j] = *(const unsigned*)p; }
  __device__ static void store(unsigned char* p, const unsigned* w, int j) { *(unsigned*)p = w[j]; }
  __device__ static float sigmoid(float g) { return 1.0f / (1.0f + expf(-g)); }
};

// The lane's numbers of a row: number j of piece v is column (v * LPR + lane) * 8 + j where rows are read 16 bytes at a
// time, else column (8 v + j) * LPR + lane, so that neighbouring lanes still read neighbours.
template <int DTYPE, int LPR, int V, bool VEC>
struct Row {
  typedef Io<DTYPE> I;
  unsigned w[V][I::kWords];

  __device__ static int col(int v, int j, int lane) { return VEC ? (v * LPR + lane) * 8 + j : (8 * v + j) * LPR + lane; }
  __device__ void load(const void* base, int64_t at, int lane, int Dg) {
    const unsigned char* p = (const unsigned char*)base + at * I::kBytes;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (VEC) {
        const int c = col(v, 0, lane);
#pragma unroll
        for (int i = 0; i < I::kWords; i += 4)
          *(u32x4*)&w[v][i] = c < Dg ? *(const u32x4*)(p + (size_t)c * I::kBytes + 4 * i) : u32x4{0, 0, 0, 0};
      } else {
#pragma unroll
        for (int i = 0; i < I::kWords; ++i) w[v][i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = col(v, j, lane);
          if (c < Dg) I::put(w[v], j, p + (size_t)c * I::kBytes);
        }
      }
    }
  }
  __device__ void values(float (*x)[8]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) I::values(w[v], x[v]);
  }
  __device__ static void store(void* base, int64_t at, int lane, int Dg, float (*x)[8]) {
    unsigned char* p = (unsigned char*)base + at * I::kBytes;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      unsigned w[I::kWords];
      I::words(x[v], w);
      if constexpr (VEC) {
        const int c = col(v, 0, lane);
        if (c < Dg)
#pragma unroll
          for (int i = 0; i < I::kWords; i += 4) *(u32x4*)(p + (size_t)c * I::kBytes + 4 * i) = *(u32x4*)&w[i];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = col(v, j, lane);
          if (c < Dg) I::store(p + (size_t)c * I::kBytes, w, j);
        }
      }
    }
  }
  __device__ static void weights(float (*x)[8], const float* w, int lane, int Dg) {
    const bool whole = VEC && (reinterpret_cast<uintptr_t>(w) & 15) == 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (whole) {
        const int c = col(v, 0, lane);
#pragma unroll
        for (int j = 0; j < 8; j += 4)
          *(f32x4*)&x[v][j] = c >= Dg ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : w ? *(const f32x4*)(w + c + j) : f32x4{1.0f, 1.0f, 1.0f, 1.0f};
      } else
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = col(v, j, lane);
        x[v][j] = c >= Dg ? 0.0f : w ? w[c] : 1.0f;
      }
  }
};

// x plus what another lane of its 16 has: quad_perm, mirrored halves of 8, mirrored 16 (no trip through LDS)
template <int CONTROL>
__device__ inline float plus_lane(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xF, 0xF, false));
}
// Sums over the lanes of a row, of two numbers at once; with 256 lanes over LDS (two areas in turn: one barrier a sum).
template <int LPR>
struct Sum {
  float (*area)[8];
  int turn;
  __device__ void operator()(float& a, float& b) {
    a = plus_lane<0x141>(plus_lane<0x4E>(plus_lane<0xB1>(a)));  // lanes 1, 2 apart, then the other four of eight
    b = plus_lane<0x141>(plus_lane<0x4E>(plus_lane<0xB1>(b)));
    if constexpr (LPR > 8) {
      a = plus_lane<0x140>(a);
      b = plus_lane<0x140>(b);
    }
    if constexpr (LPR > 16) {
      a += __shfl_xor(a, 16);
      b += __shfl_xor(b, 16);
    }
    if constexpr (LPR > 32) {
      a += __shfl_xor(a, 32);
      b += __shfl_xor(b, 32);
    }
    if constexpr (LPR == 256) {
      float* s = area[turn];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        s[threadIdx.x >> 6] = a;
        s[4 + (threadIdx.x >> 6)] = b;
      }
      __syncthreads();
      a = (s[0] + s[1]) + (s[2] + s[3]);
      b = (s[4] + s[5]) + (s[6] + s[7]);
    }
  }
};

// x becomes the normalised row; what is returned is the inverse of its size.  Columns past Dg stay zero.
template <int V, class Row, class Sum>
__device__ inline float normalise(float (*x)[8], int how, int Dg, float eps, int lane, Sum& sum) {
  if (how == SF_NORM_NONE) return 1.0f;
  const float inv = 1.0f / (float)Dg;
  float a = 0.0f, b = 0.0f;
  if (how == SF_NORM_LAYER) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) a += x[v][j];
    sum(a, b);
    a *= inv;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[v][j] = Row::col(v, j, lane) < Dg ? x[v][j] - a : 0.0f;
  }
  a = b = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) a += x[v][j] * x[v][j];
  sum(a, b);
  const float r = __builtin_amdgcn_rsqf(a * inv + eps);  // (its result is off by one unit in the last place at most)
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) x[v][j] *= r;
  return r;
}
// d, the gradient of the normalised row `unit`, becomes that of the row
template <int V, class Row, class Sum>
__device__ inline void normalise_back(float (*d)[8], float (*unit)[8], float r, int how, int Dg, int lane, Sum& sum) {
  if (how == SF_NORM_NONE) return;
  float a = 0.0f, b = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      a += d[v][j] * unit[v][j];
      b += d[v][j];
    }
  sum(a, b);
  const float inv = 1.0f / (float)Dg;
  a *= inv * r;
  b *= inv;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // (past Dg both are zero)
      if (how == SF_NORM_LAYER) d[v][j] = Row::col(v, j, lane) < Dg ? d[v][j] - b : 0.0f;
      d[v][j] = r * d[v][j] - unit[v][j] * a;
    }
}

template <int DTYPE, int LPR, int V, bool VEC, bool BACK>
__global__ __launch_bounds__(kThreads, BACK && V == 1 ? 2 : 1) void resnorm_kernel(NormArgs g) {
  typedef Row<DTYPE, LPR, V, VEC> R;
  typedef Io<DTYPE> I;
  constexpr int RPW = kThreads / LPR;  // rows of a workgroup at a time
  __shared__ float area[2][8];
  extern __shared__ float columns[];   // backwards: [4 waves][3][Dg], where several groups of lanes are added
  const int lane = threadIdx.x % LPR;
  const int64_t slot = (int64_t)blockIdx.x * RPW + threadIdx.x / LPR, slots = (int64_t)gridDim.x * RPW;
  // (slots is a multiple of groups: a slot's rows are of one group, and `next` apart)
  const int group = (int)(slot % g.groups), Dg = g.Dg, c0 = group * Dg;
  const int64_t first = slot / g.groups, next = slots / g.groups;
  Sum<LPR> sum = {area, 0};

  R rb, rx, rg, rdy, rdn;
  auto request = [&](int64_t m) {
    rb.load(g.b, m * g.b_s + c0, lane, Dg);
    if (g.x) rx.load(g.x, m * g.x_s + c0, lane, Dg);
    if (g.gate) rg.load(g.gate, m * g.gate_s + c0, lane, Dg);
    if constexpr (BACK) {
      if (g.dy) rdy.load(g.dy, m * g.dy_s + c0, lane, Dg);
      if (g.dn) rdn.load(g.dn, m * g.dn_s + c0, lane, Dg);
    }
  };
  // (with 256 lanes a row is the workgroup's, so that all of it leaves the loop together)
  if (first < g.rows) request(first);
  float wpost[V][8], wpre[V][8], ws[V][8];
  R::weights(wpost, g.post_w ? g.post_w + c0 : nullptr, lane, Dg);
  R::weights(wpre, g.pre_w ? g.pre_w + c0 : nullptr, lane, Dg);
  R::weights(ws, g.scale ? g.scale + c0 : nullptr, lane, Dg);
  float spost[V][8], spre[V][8], ss[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) spost[v][j] = spre[v][j] = ss[v][j] = 0.0f;

  for (int64_t m = first; m < g.rows; m += next) {
    float u[V][8], y[V][8], gt[V][8], d[V][8], e[V][8];
    rb.values(u);
    if (g.x) rx.values(y);
    if (g.gate) rg.values(gt);
    if constexpr (BACK) {
      if (g.dy) rdy.values(d);
      if (g.dn) rdn.values(e);
    }
    if (m + next < g.rows) request(m + next);
    const int64_t to = m * g.D + c0;

    const float r = normalise<V, R>(u, g.post, Dg, g.eps, lane, sum);
    float a[V][8];  // scale times the gate's activation
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        a[v][j] = 1.0f;
        if (g.gate) {
          const float x = gt[v][j], s = I::sigmoid(x);
          a[v][j] = g.act == SF_GATE_SILU ? s * x : s;
          if constexpr (BACK) gt[v][j] = g.act == SF_GATE_SILU ? s * (1.0f + x * (1.0f - s)) : s * (1.0f - s);  // the slope
        }
        const float out = ws[v][j] * a[v][j] * (wpost[v][j] * u[v][j]);
        y[v][j] = g.x ? y[v][j] + out : out;
      }
    if constexpr (!BACK) {
      if (g.y) R::store(g.y, to, lane, Dg, y);
      if (g.n) {
        normalise<V, R>(y, g.pre, Dg, g.eps, lane, sum);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) y[v][j] *= wpre[v][j];
        R::store(g.n, to, lane, Dg, y);
      }
    } else {
      if (g.dn) {
        const float r2 = normalise<V, R>(y, g.pre, Dg, g.eps, lane, sum);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            spre[v][j] += e[v][j] * y[v][j];
            e[v][j] *= wpre[v][j];
          }
        normalise_back<V, R>(e, y, r2, g.pre, Dg, lane, sum);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) d[v][j] = g.dy ? d[v][j] + e[v][j] : e[v][j];
      }
      if (g.dx) R::store(g.dx, to, lane, Dg, d);
      // e: the gradient of the gate, then of b
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float wu = wpost[v][j] * u[v][j], da = d[v][j] * a[v][j], dsa = da * ws[v][j];
          ss[v][j] += da * wu;
          if (g.post != SF_NORM_NONE) spost[v][j] += dsa * u[v][j];
          if (g.gate) e[v][j] = d[v][j] * ws[v][j] * gt[v][j] * wu;
          d[v][j] = dsa * wpost[v][j];
        }
      if (g.dgate) R::store(g.dgate, to, lane, Dg, e);
      normalise_back<V, R>(d, u, r, g.post, Dg, lane, sum);
      if (g.db) R::store(g.db, to, lane, Dg, d);
    }
  }

  if constexpr (BACK) {
    if (!g.part) return;
    auto put = [&](float* p, int pitch) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = R::col(v, j, lane);
          if (c >= Dg) continue;
          p[c] = spost[v][j];
          p[pitch + c] = ss[v][j];
          p[2 * pitch + c] = spre[v][j];
        }
    };
    if (g.groups > 1) {  // the lanes of a workgroup are of different groups
      put(g.part + slot / g.groups * 3 * g.D + c0, g.D);
    } else if constexpr (LPR == 256) {
      put(g.part + (size_t)blockIdx.x * 3 * g.D, g.D);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int m = LPR; m < 64; m <<= 1) {
            spost[v][j] += __shfl_xor(spost[v][j], m);
            ss[v][j] += __shfl_xor(ss[v][j], m);
            spre[v][j] += __shfl_xor(spre[v][j], m);
          }
      if ((threadIdx.x & 63) < LPR) put(columns + (threadIdx.x >> 6) * 3 * Dg, Dg);
      __syncthreads();
      for (int c = threadIdx.x; c < 3 * Dg; c += kThreads)
        g.part[(size_t)blockIdx.x * 3 * Dg + c] = (columns[c] + columns[3 * Dg + c]) + (columns[6 * Dg + c] + columns[9 * Dg + c]);
    }
  }
}

// Sums of the workgroups' partial sums: 32 columns by 32 lanes per workgroup, eight loads of a lane under way.
__global__ __launch_bounds__(1024) void resnorm_sum_kernel(const float* part, int parts, int D, float* post, float* scale, float* pre) {
  __shared__ float s[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float a = 0.0f;
  if (c < 3 * D) {
    const float* p = part + c;
    const size_t pitch = (size_t)3 * D;
    int i = y;
    for (; i + 224 < parts; i += 256) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = p[(i + 32 * j) * pitch];
#pragma unroll
      for (int j = 0; j < 8; ++j) a += v[j];
    }
    for (; i < parts; i += 32) a += p[i * pitch];
  }
  s[y][x] = a;
  __syncthreads();
  if (y != 0 || c >= 3 * D) return;
  a = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) a += s[i][x];
  float* const to = c < D ? post : c < 2 * D ? scale : pre;
  if (to) to[c % D] = a;
}

// ---- host side ---------------------------------------------------------------------------------

constexpr int kMaxD = 8192;

struct Shape {
  int lpr, v;
};
// The lanes of a row: as few as hold it in one piece of eight numbers each, up to a wave, which takes two pieces, and then
// the workgroup.  (A wave with four pieces, 2048 columns, would need more registers backwards than two waves leave.)
Shape shape_of(int Dg) {
  for (int lpr = 8; lpr <= 64; lpr *= 2)
    if (Dg <= lpr * 8) return Shape{lpr, 1};
  if (Dg <= 1024) return Shape{64, 2};
  return Dg <= 2048 ? Shape{256, 1} : Dg <= 4096 ? Shape{256, 2} : Shape{256, 4};
}

int check(const sf_resnorm_config* c, const char* fn) {
  if (!c || c->struct_size != sizeof(sf_resnorm_config)) {
    set_error("%s: null configuration or struct_size mismatch", fn);
    return SF_ERR_ARG;
  }
  if ((c->dtype != SF_DTYPE_FP32 && c->dtype != SF_DTYPE_BF16) || c->post < SF_NORM_NONE || c->post > SF_NORM_LAYER ||
      c->pre < SF_NORM_NONE || c->pre > SF_NORM_LAYER || c->gate_act < SF_GATE_NONE || c->gate_act > SF_GATE_SILU) {
    set_error("%s: dtype = %d, post = %d, pre = %d, gate_act = %d", fn, c->dtype, c->post, c->pre, c->gate_act);
    return SF_ERR_ARG;
  }
  if (c->M < 0 || c->D < 1 || c->groups < 1 || c->groups > 1024 || c->D % c->groups || c->D / c->groups > kMaxD) {
    set_error("%s: M = %d, D = %d, groups = %d out of range", fn, c->M, c->D, c->groups);
    return SF_ERR_SHAPE;
  }
  if (c->groups > 1 && c->pre != SF_NORM_NONE) {
    set_error("%s: groups = %d with a norm of the whole row behind it", fn, c->groups);
    return SF_ERR_SHAPE;
  }
  if (!(c->eps >= 0.0f) || !isfinite(c->eps)) {
    set_error("%s: eps must be >= 0", fn);
    return SF_ERR_SHAPE;
  }
  return SF_OK;
}
int bad_ptr(const char* fn, const char* name) {
  set_error("%s: %s is null or misaligned", fn, name);
  return SF_ERR_ARG;
}
bool fits(const void* p, size_t align, bool optional) {
  return p ? (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0 : optional;
}

// Workgroups: every lane group a row, but backwards no more than leave few partial sums (512: two for each CU; the
// next row's loads are under way besides), and a multiple of the groups.
int grid_of(const sf_resnorm_config* c, bool back) {
  const int rpw = kThreads / shape_of(c->D / c->groups).lpr;
  int64_t n = ((int64_t)c->M * c->groups + rpw - 1) / rpw;
  const int64_t most = back ? 512 : 2048;
  if (n > most) n = most;
  if (n < 1) n = 1;
  return (int)((n + c->groups - 1) / c->groups * c->groups);
}
int parts_of(const sf_resnorm_config* c) {
  const int grid = grid_of(c, true);
  return c->groups > 1 ? grid / c->groups * (kThreads / shape_of(c->D / c->groups).lpr) : grid;
}

bool piecewise(const NormArgs& g, int e) {
  const int per = 16 / e;
  const void* const p[] = {g.b, g.x, g.gate, g.dy, g.dn, g.y, g.n, g.dx, g.db, g.dgate};
  for (const void* q : p)
    if (reinterpret_cast<uintptr_t>(q) & 15) return false;
  return g.Dg % 8 == 0 && g.b_s % per == 0 && g.x_s % per == 0 && g.gate_s % per == 0 && g.dy_s % per == 0 && g.dn_s % per == 0;
}

template <int DTYPE, int LPR, int V, bool BACK>
hipError_t launch_t(const sf_resnorm_config* c, const NormArgs& g, hipStream_t st) {
  const size_t lds = BACK && g.part && LPR < 256 && g.groups == 1 ? (size_t)12 * g.Dg * sizeof(float) : 0;  // at most 48 KB
  if (piecewise(g, Io<DTYPE>::kBytes)) resnorm_kernel<DTYPE, LPR, V, true, BACK><<<grid_of(c, BACK), kThreads, lds, st>>>(g);
  else resnorm_kernel<DTYPE, LPR, V, false, BACK><<<grid_of(c, BACK), kThreads, lds, st>>>(g);
  return hipGetLastError();
}
template <int DTYPE, bool BACK>
hipError_t launch(const sf_resnorm_config* c, const NormArgs& g, hipStream_t st) {
  const Shape s = shape_of(g.Dg);
  if (s.lpr == 8) return launch_t<DTYPE, 8, 1, BACK>(c, g, st);
  if (s.lpr == 16) return launch_t<DTYPE, 16, 1, BACK>(c, g, st);
  if (s.lpr == 32) return launch_t<DTYPE, 32, 1, BACK>(c, g, st);
  if (s.lpr == 64) return s.v == 1 ? launch_t<DTYPE, 64, 1, BACK>(c, g, st) : launch_t<DTYPE, 64, 2, BACK>(c, g, st);
  return s.v == 1 ? launch_t<DTYPE, 256, 1, BACK>(c, g, st)
                  : s.v == 2 ? launch_t<DTYPE, 256, 2, BACK>(c, g, st) : launch_t<DTYPE, 256, 4, BACK>(c, g, st);
}
template <bool BACK>
int run(const char* fn, const sf_resnorm_config* c, const NormArgs& g, hipStream_t st) {
  const hipError_t e = c->dtype == SF_DTYPE_BF16 ? launch<SF_DTYPE_BF16, BACK>(c, g, st) : launch<SF_DTYPE_FP32, BACK>(c, g, st);
  if (e != hipSuccess) {
    set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
    return SF_ERR_DEVICE;
  }
  return SF_OK;
}

NormArgs common(const sf_resnorm_config* c, const void* b, const void* x, const void* gate, const float* post_w,
                const float* scale, const float* pre_w) {
  NormArgs g = {};
  g.b = b;
  g.x = x;
  g.gate = c->gate_act == SF_GATE_NONE ? nullptr : gate;
  g.b_s = c->b_stride;
  g.x_s = x ? c->x_stride : 0;
  g.gate_s = g.gate ? c->gate_stride : 0;
  g.post_w = c->post == SF_NORM_NONE ? nullptr : post_w;
  g.scale = scale;
  g.pre_w = pre_w;
  g.rows = c->M;
  g.D = c->D;
  g.groups = c->groups;
  g.Dg = c->D / c->groups;
  g.post = c->post;
  g.pre = c->pre;
  g.act = c->gate_act;
  g.eps = c->eps;
  return g;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" int sf_resnorm(const sf_resnorm_config* cfg, const void* b, const void* x, const void* gate, const float* post_w,
                          const float* scale, const float* pre_w, void* y, void* n, void* hip_stream) {
  static const char* fn = "sf_resnorm";
  const int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = cfg->M == 0, pre = cfg->pre != SF_NORM_NONE;
  if (!fits(b, e, none)) return bad_ptr(fn, "b");
  if (!fits(x, e, true)) return bad_ptr(fn, "x");
  if (!fits(gate, e, none || cfg->gate_act == SF_GATE_NONE)) return bad_ptr(fn, "gate");
  if (!fits(post_w, 4, true)) return bad_ptr(fn, "post_w");
  if (!fits(scale, 4, true)) return bad_ptr(fn, "scale");
  if (!fits(pre_w, 4, true)) return bad_ptr(fn, "pre_w");
  if (!fits(y, e, none || pre)) return bad_ptr(fn, "y");
  if (!fits(n, e, none || !pre)) return bad_ptr(fn, "n");
  if (none) return SF_OK;
  NormArgs g = common(cfg, b, x, gate, post_w, scale, pre_w);
  g.y = y;
  g.n = pre ? n : nullptr;
  return run<false>(fn, cfg, g, reinterpret_cast<hipStream_t>(hip_stream));
}

extern "C" int64_t sf_resnorm_workspace_bytes(const sf_resnorm_config* cfg) {
  if (check(cfg, "sf_resnorm_workspace_bytes") != SF_OK) return -1;
  return (int64_t)parts_of(cfg) * 3 * cfg->D * (int64_t)sizeof(float);
}

extern "C" int sf_resnorm_backward(const sf_resnorm_config* cfg, const void* b, const void* x, const void* gate,
                                   const float* post_w, const float* scale, const float* pre_w, const void* dy,
                                   const void* dn, void* dx, void* db, void* dgate, float* dpost_w, float* dscale,
                                   float* dpre_w, void* workspace, void* hip_stream) {
  static const char* fn = "sf_resnorm_backward";
  int rc = check(cfg, fn);
  if (rc != SF_OK) return rc;
  const size_t e = cfg->dtype == SF_DTYPE_BF16 ? 2 : 4;
  const bool none = cfg->M == 0, pre = cfg->pre != SF_NORM_NONE, sums = dpost_w || dscale || dpre_w;
  if (!fits(b, e, none)) return bad_ptr(fn, "b");
  if (!fits(x, e, true)) return bad_ptr(fn, "x");
  if (!fits(gate, e, none || cfg->gate_act == SF_GATE_NONE)) return bad_ptr(fn, "gate");
  if (!fits(post_w, 4, true)) return bad_ptr(fn, "post_w");
  if (!fits(scale, 4, true)) return bad_ptr(fn, "scale");
  if (!fits(pre_w, 4, true)) return bad_ptr(fn, "pre_w");
  if (!fits(dy, e, none || pre)) return bad_ptr(fn, "dy");
  if (!fits(dn, e, none || !pre)) return bad_ptr(fn, "dn");
  if (!fits(dx, e, true)) return bad_ptr(fn, "dx");
  if (!fits(db, e, true)) return bad_ptr(fn, "db");
  if (!fits(dgate, e, true)) return bad_ptr(fn, "dgate");
  if (dgate && cfg->gate_act == SF_GATE_NONE) {
    set_error("%s: dgate without a gate", fn);
    return SF_ERR_ARG;
  }
  if (!fits(dpost_w, 4, true)) return bad_ptr(fn, "dpost_w");
  if (!fits(dscale, 4, true)) return bad_ptr(fn, "dscale");
  if (!fits(dpre_w, 4, true)) return bad_ptr(fn, "dpre_w");
  if (!fits(workspace, 256, !sums)) return bad_ptr(fn, "workspace");
  NormArgs g = common(cfg, b, x, gate, post_w, scale, pre_w);
  g.dy = dy;
  g.dy_s = dy ? cfg->dy_stride : 0;
  g.dn = pre ? dn : nullptr;
  g.dn_s = g.dn ? cfg->dn_stride : 0;
  g.dx = dx;
  g.db = db;
  g.dgate = g.gate ? dgate : nullptr;
  g.part = sums ? (float*)workspace : nullptr;
  if (none && !sums) return SF_OK;
  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  rc = run<true>(fn, cfg, g, st);  // (no rows: the partial sums are zeros)
  if (rc != SF_OK || !sums) return rc;
  resnorm_sum_kernel<<<(3 * cfg->D + 31) / 32, 1024, 0, st>>>(g.part, parts_of(cfg), cfg->D, dpost_w, dscale, dpre_w);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) {
    set_error("%s: launch failed: %s", fn, hipGetErrorString(err));
    return SF_ERR_DEVICE;
  }
  return SF_OK;
}
