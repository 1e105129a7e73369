// The global norm of a list of gradients, and the gradients scaled down to a largest norm (include/sf_memory.h):
//   norm = sqrt(sum over all numbers g of g^2),  g <- min(1, max_norm / (norm + eps)) g
// Two passes over the gradients, since the factor needs all of them: one adds the squares, the other reads again and writes.  The
// list is cut into chunks of one size, none across two tensors; a workgroup has one chunk in both passes.  Squares are
// added in 64 bits: exact to 2^-53 whatever the list's length, and no square of an fp32 number leaves their range.  Every workgroup
// of the second pass adds up all chunks' sums in the same order, which costs it the reading of some kilobytes from L2 and saves a launch
// in between (1 us of 38 or 68 with 1000 or 2000 chunks); of a list that takes several launches, whose chunks can be any number, one workgroup
// adds them up first, in the same order (300 tensors of all sizes 71 us, so 69; of 32 numbers each: 1000 60 and 55, 8000 435 and 309, 30000
// 2160 and 1120).  Nothing is added with atomics, so the same gradients give the same bits.
//
// Tensors are described in the launches' arguments, up to kTensors of them in one; no table has to be copied to the device, and a
// recorded graph holds its own.
//
// Bound by memory.  54 tensors, 856 MB: 184 us for the squares (4.7 TB/s), 319 to read again and write (5.4); half the chunks 203 and 339, four
// pieces ahead in place of eight 187 and 318.  Few numbers: 16 tensors of 11.5 MB 4.2 and 6.1 us, 300 tensors of all sizes, 67 MB, in three
// launches a pass 24 and 33 us, and 3 for the sums in between.
#include <math.h>

#include <algorithm>
#include <vector>

#include "sf_internal.h"
#include "sf_memory.h"

namespace sf {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kTensors = 120;      // of one launch: its arguments stay under 4 KB
constexpr int kChunks = 2048;      // of the whole list, and one more for each tensor's rest
constexpr int64_t kLeast = 16384;  // numbers of a chunk, and what it is a multiple of
constexpr int kAhead = 8;          // pieces of 16 bytes that a thread has on their way

struct ClipTensor {
  const void* in;
  void* out;
  int64_t n;
};
struct ClipArgs {
  const double* total;        // the sum of all chunks' sums, or null: each workgroup adds them up
  double* sums;               // one of each chunk
  float* norm;                // or null: written by another launch
  float max_norm, eps;
  int64_t chunk;              // numbers
  int n, chunks, all_chunks;  // tensors and chunks of this launch, chunks of the list
  int first;                  // this launch's first chunk
  unsigned bf16[(kTensors + 31) / 32];
  int begin[kTensors + 1];    // each tensor's first chunk, in this launch
  ClipTensor t[kTensors];
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

__device__ inline float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
__device__ inline float as_float(unsigned w) { return __builtin_bit_cast(float, w); }  // (of a vector's element the builtin takes the first)
__device__ inline unsigned pack(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// Which tensor a chunk belongs to: the last one that begins at it or before (tensors of nothing have no chunk, and begin where the
// next one does).
__device__ inline int tensor_of(const ClipArgs& g, int chunk) {
  int lo = 0, hi = g.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (g.begin[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

template <bool BF16>
__device__ inline double squares(const unsigned char* p, int64_t n) {
  constexpr int kPer = BF16 ? 8 : 4;  // numbers of a piece
  double sum[kAhead] = {};
  auto add = [&](double& s, const u32x4& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const double a = bf16_lo(w[i]), b = bf16_hi(w[i]);
        s = fma(a, a, s);
        s = fma(b, b, s);
      } else {
        const double a = as_float(w[i]);
        s = fma(a, a, s);
      }
    }
  };
  const int64_t pieces = n / kPer;
  int64_t at = threadIdx.x;
  for (; at + (kAhead - 1) * kThreads < pieces; at += kAhead * kThreads) {
    u32x4 w[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) __builtin_memcpy(&w[a], p + (at + a * kThreads) * 16, 16);
#pragma unroll
    for (int a = 0; a < kAhead; ++a) add(sum[a], w[a]);
  }
  for (; at < pieces; at += kThreads) {
    u32x4 w;
    __builtin_memcpy(&w, p + at * 16, 16);
    add(sum[0], w);
  }
  const int64_t e = pieces * kPer + threadIdx.x;  // (fewer than a piece are left)
  if (e < n) {
    const double a = BF16 ? bf16_lo(((const uint16_t*)p)[e]) : ((const float*)p)[e];
    sum[1] = fma(a, a, sum[1]);
  }
  double all = 0.0;
#pragma unroll
  for (int a = 0; a < kAhead; ++a) all += sum[a];
  return all;
}

__global__ __launch_bounds__(kThreads) void clip_squares_kernel(ClipArgs g) {
  __shared__ double part[kThreads / 64];
  const int i = tensor_of(g, blockIdx.x);
  const ClipTensor t = g.t[i];
  const int64_t e0 = (int64_t)(blockIdx.x - g.begin[i]) * g.chunk, n = min(g.chunk, t.n - e0);
  const bool bf16 = g.bf16[i >> 5] >> (i & 31) & 1;
  const double mine = wave_sum(bf16 ? squares<true>((const unsigned char*)t.in + e0 * 2, n) : squares<false>((const unsigned char*)t.in + e0 * 4, n));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) g.sums[g.first + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// From the chunk's end to its begin: what the pass before read last is read first.
template <bool BF16>
__device__ inline void scale(const unsigned char* in, unsigned char* out, int64_t n, float by) {
  constexpr int kPer = BF16 ? 8 : 4;
  auto times = [&](u32x4 w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) w[i] = pack(by * bf16_lo(w[i]), by * bf16_hi(w[i]));
      else w[i] = __builtin_bit_cast(unsigned, by * as_float(w[i]));
    }
    return w;
  };
  const int64_t pieces = n / kPer, e = pieces * kPer + threadIdx.x;
  if (e < n) {
    if constexpr (BF16) ((uint16_t*)out)[e] = (uint16_t)pack(by * bf16_lo(((const uint16_t*)in)[e]), 0.0f);
    else ((float*)out)[e] = by * ((const float*)in)[e];
  }
  int64_t at = pieces - 1 - threadIdx.x;
  for (; at - (kAhead - 1) * kThreads >= 0; at -= kAhead * kThreads) {
    u32x4 w[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) __builtin_memcpy(&w[a], in + (at - a * kThreads) * 16, 16);
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      w[a] = times(w[a]);
      __builtin_memcpy(out + (at - a * kThreads) * 16, &w[a], 16);
    }
  }
  for (; at >= 0; at -= kThreads) {
    u32x4 w;
    __builtin_memcpy(&w, in + at * 16, 16);
    w = times(w);
    __builtin_memcpy(out + at * 16, &w, 16);
  }
}

// One workgroup: the sum over all chunks, in one order whoever adds.
__device__ inline double sum_of_chunks(const double* sums, int n) {
  __shared__ double part[kThreads / 64];
  double sum = 0.0;
  int c = threadIdx.x;
  for (; c + (kAhead - 1) * kThreads < n; c += kAhead * kThreads) {
    double x[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) x[a] = sums[c + a * kThreads];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) sum += x[a];
  }
  for (; c < n; c += kThreads) sum += sums[c];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(kThreads) void clip_sum_kernel(double* sums, int n) {
  const double sum = sum_of_chunks(sums, n);
  if (threadIdx.x == 0) sums[n] = sum;
}

__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipArgs g) {
  const double norm = sqrt(g.total ? *g.total : sum_of_chunks(g.sums, g.all_chunks));
  if (g.norm && blockIdx.x == 0 && threadIdx.x == 0) *g.norm = (float)norm;
  if ((int)blockIdx.x >= g.chunks) return;  // (a list of nothing)
  const double q = (double)g.max_norm / (norm + (double)g.eps);
  const float by = q >= 1.0 ? 1.0f : (float)q;  // (NaN stays NaN)
  const int i = tensor_of(g, blockIdx.x);
  const ClipTensor t = g.t[i];
  if (by == 1.0f && t.in == t.out) return;
  const int64_t e0 = (int64_t)(blockIdx.x - g.begin[i]) * g.chunk, n = min(g.chunk, t.n - e0);
  const bool bf16 = g.bf16[i >> 5] >> (i & 31) & 1;
  const int64_t b0 = e0 * (bf16 ? 2 : 4);
  if (bf16) scale<true>((const unsigned char*)t.in + b0, (unsigned char*)t.out + b0, n, by);
  else scale<false>((const unsigned char*)t.in + b0, (unsigned char*)t.out + b0, n, by);
}

// ---- host side ---------------------------------------------------------------------------------

// Numbers of a chunk, from the whole list's.
int64_t chunk_of(int64_t total) {
  const int64_t c = (total + kChunks - 1) / kChunks;
  return std::max<int64_t>(kLeast, (c + kLeast - 1) / kLeast * kLeast);
}

struct Chunks {
  int64_t size, count;                                // numbers of a chunk, chunks of the list
  bool total;                                         // several launches: the chunks' sums are added up in between
  int64_t sums() const { return count + (total ? 1 : 0); }  // numbers of the workspace
};

// false: an error has been set.
bool chunks_of(const char* fn, int32_t n, const int64_t* sizes, Chunks* c, int* rc) {
  if (n < 0 || n > 1 << 20 || (n > 0 && !sizes)) {
    set_error("%s: %d tensors%s", fn, n, n > 0 ? ", sizes is null" : "");
    *rc = n < 0 || n > 1 << 20 ? SF_ERR_SHAPE : SF_ERR_ARG;
    return false;
  }
  int64_t total = 0, tensors = 0;
  for (int i = 0; i < n; ++i) {
    if (sizes[i] < 0 || sizes[i] > (int64_t)1 << 40) {
      set_error("%s: tensor %d of %lld numbers", fn, i, (long long)sizes[i]);
      *rc = SF_ERR_SHAPE;
      return false;
    }
    total += sizes[i];
    tensors += sizes[i] > 0;
  }
  c->size = chunk_of(total);
  c->count = 0;
  for (int i = 0; i < n; ++i) c->count += (sizes[i] + c->size - 1) / c->size;
  c->total = tensors > kTensors;
  return true;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" int64_t sf_gradclip_workspace_bytes(int32_t n, const int64_t* sizes) {
  Chunks c;
  int rc;
  if (!chunks_of("sf_gradclip_workspace_bytes", n, sizes, &c, &rc)) return -1;
  return (c.sums() * (int64_t)sizeof(double) + 255) / 256 * 256;
}

extern "C" int sf_gradclip(const sf_gradclip_config* cfg, const void* const* grads, const int64_t* sizes, const int32_t* dtypes, void* const* out,
                           float* norm, void* workspace, void* hip_stream) {
  static const char* fn = "sf_gradclip";
  if (!cfg || cfg->struct_size != sizeof(sf_gradclip_config)) {
    set_error("%s: null configuration or struct_size mismatch", fn);
    return SF_ERR_ARG;
  }
  Chunks chunks;
  int rc;
  if (!chunks_of(fn, cfg->n, sizes, &chunks, &rc)) return rc;
  const int64_t chunk = chunks.size, count = chunks.count;
  if (!(cfg->max_norm >= 0.0f) || !(cfg->eps > 0.0f) || !isfinite(cfg->eps)) {
    set_error("%s: max_norm = %g, eps = %g", fn, cfg->max_norm, cfg->eps);
    return SF_ERR_SHAPE;
  }
  if (cfg->n > 0 && (!grads || !dtypes || !out)) {
    set_error("%s: grads, dtypes or out is null", fn);
    return SF_ERR_ARG;
  }
  if (!norm || (reinterpret_cast<uintptr_t>(norm) & 3) != 0) {
    set_error("%s: norm is null or not 4-byte aligned", fn);
    return SF_ERR_ARG;
  }
  if (count > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)) {
    set_error("%s: workspace is null or not 256-byte aligned", fn);
    return SF_ERR_ARG;
  }
  for (int i = 0; i < cfg->n; ++i) {
    if (dtypes[i] != SF_DTYPE_FP32 && dtypes[i] != SF_DTYPE_BF16) {
      set_error("%s: dtype of tensor %d = %d", fn, i, dtypes[i]);
      return SF_ERR_ARG;
    }
    const uintptr_t mask = dtypes[i] == SF_DTYPE_BF16 ? 1 : 3;
    if (sizes[i] > 0 && (!grads[i] || !out[i] || ((reinterpret_cast<uintptr_t>(grads[i]) | reinterpret_cast<uintptr_t>(out[i])) & mask) != 0)) {
      set_error("%s: tensor %d or its result is null or not aligned to its type", fn, i);
      return SF_ERR_ARG;
    }
  }
  // A result may be its own gradient and lie on nothing else: all tensors and results by their addresses, one behind the other.
  struct Span {
    uintptr_t at, end;
    int i;
    bool written;
  };
  try {
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)cfg->n + 2);
    for (int i = 0; i < cfg->n; ++i) {
      if (sizes[i] == 0) continue;
      const uintptr_t size = (uintptr_t)sizes[i] * (dtypes[i] == SF_DTYPE_BF16 ? 2 : 4), a = reinterpret_cast<uintptr_t>(grads[i]),
                      b = reinterpret_cast<uintptr_t>(out[i]);
      spans.push_back(Span{a, a + size, i, a == b});
      if (a != b) spans.push_back(Span{b, b + size, i, true});
    }
    spans.push_back(Span{reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm) + 4, -1, true});
    if (count > 0)
      spans.push_back(Span{reinterpret_cast<uintptr_t>(workspace), reinterpret_cast<uintptr_t>(workspace) + (uintptr_t)chunks.sums() * sizeof(double), -1, true});
    const auto before = [](const Span& a, const Span& b) { return a.at < b.at; };
    if (!std::is_sorted(spans.begin(), spans.end(), before)) std::sort(spans.begin(), spans.end(), before);
    uintptr_t end = 0, end_written = 0;  // of all spans before, of those that are written
    for (const Span& s : spans) {
      if (s.at < end_written || (s.written && s.at < end)) {
        set_error("%s: what is written overlaps another tensor of the list, the norm or the workspace (at tensor %d)", fn, s.i);
        return SF_ERR_ALIAS;
      }
      end = std::max(end, s.end);
      if (s.written) end_written = std::max(end_written, s.end);
    }
  } catch (const std::bad_alloc&) {
    set_error("%s: out of host memory", fn);
    return SF_ERR_OOM;
  }

  const hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  // the list twice: first the squares of all tensors, then the results of all
  for (int pass = 0; pass < 2; ++pass) {
    int i = 0;
    int64_t first = 0;
    bool named = false;  // the norm has a launch that writes it
    if (pass == 1 && chunks.total) clip_sum_kernel<<<1, kThreads, 0, st>>>((double*)workspace, (int)count);
    do {
      ClipArgs g = {};
      g.sums = (double*)workspace;
      g.total = chunks.total ? g.sums + count : nullptr;
      g.max_norm = cfg->max_norm;
      g.eps = cfg->eps;
      g.chunk = chunk;
      g.all_chunks = (int)count;
      g.first = (int)first;
      for (; i < cfg->n && g.n < kTensors; ++i) {
        if (sizes[i] == 0) continue;
        g.t[g.n] = ClipTensor{grads[i], out[i], sizes[i]};
        if (dtypes[i] == SF_DTYPE_BF16) g.bf16[g.n >> 5] |= 1u << (g.n & 31);
        g.begin[g.n] = g.chunks;
        g.chunks += (int)((sizes[i] + chunk - 1) / chunk);
        ++g.n;
      }
      g.begin[g.n] = g.chunks;
      first += g.chunks;
      if (pass == 0) {
        if (g.chunks > 0) clip_squares_kernel<<<(unsigned)g.chunks, kThreads, 0, st>>>(g);
      } else if (g.chunks > 0 || !named) {
        g.norm = named ? nullptr : norm;
        named = true;
        clip_scale_kernel<<<(unsigned)std::max(g.chunks, 1), kThreads, 0, st>>>(g);
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) {
        set_error("%s: launch failed: %s", fn, hipGetErrorString(e));
        return SF_ERR_DEVICE;
      }
    } while (i < cfg->n);
  }
  return SF_OK;
}
