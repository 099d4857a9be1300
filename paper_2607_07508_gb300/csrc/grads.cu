// Global norm of many gradient tensors, and their clipped copies.
//
//   sumsq = sum over tensors and elements of g^2,   norm = sqrt(sumsq)
//   coef  = max_norm / norm where norm > max_norm, else 1,   out = coef g
//
// Both kernels read every element once and the second one writes it: bound by HBM. 1.85 GB in 146 tensors: squares 282 us
// (6.5 TB/s), clipped copies 544 us (3.7 GB at 6.8 TB/s). The second read cannot be saved, as the norm is known only after
// the first, but it begins with what the first read last, which the L2 still has. The tensors are cut into chunks
// that a grid of fixed size takes in turn, whatever their sizes and types; a chunk's tensor is found in the kernel's
// arguments, so that a call copies nothing to the device and can be captured. Small lists take the host 14 to 18 us
// for the two calls' three launches. Tensors off 16 bytes go by single elements: 800 MB of fp32 in ten tensors 167 us for
// the squares and 730 for the copies, where aligned ones take 112 and 241.
//
// The squares' range: a batch of a thread's loads is summed in fp32 where that sum is a normal number far from both
// ends, else (an element past 2^57 or so, or all of them tiny) again in fp64, and batches are added in fp64. No order
// depends on timing.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "grads.cuh"
#include "sao_common.cuh"

namespace sao {
namespace {

constexpr int kThreads = 256;
constexpr int kLoads = 8;                                 // of 16 bytes, in flight in a thread
constexpr int kChunkBytes = kThreads * kLoads * 16;       // 32 KB of a tensor
// clip_kernel writes what it loads: 512 threads of 64 registers, two CTAs to an SM, which took 544 us for 3.7 GB where
// 256 threads of 156 registers took 710 and three CTAs 715
constexpr int kClipThreads = 512;
constexpr int kClipLoads = kChunkBytes / (kClipThreads * 16);
constexpr int kMaxGrid = 8 * 160;                         // CTAs of a launch, at most

// The tensors of one launch. n: elements, with the types in its top bits.
constexpr int64_t kBf16Src = int64_t(1) << 62, kBf16Dst = int64_t(1) << 61;
constexpr int64_t kCount = kBf16Dst - 1;
template <int kCap>
struct List {
  const void *src[kCap];
  void *dst[kCap];
  int64_t n[kCap];
  int64_t first[kCap + 1];  // the tensor's first chunk; [count]: all chunks
  int count;
};

__host__ __device__ constexpr int64_t chunk_elements(bool bf16) { return kChunkBytes / (bf16 ? 2 : 4); }

// The tensor that holds chunk c.
template <int kCap>
__device__ __forceinline__ int tensor_of(const List<kCap> &l, int64_t c) {
  int lo = 0, n = l.count;  // the last one that starts at or before c: one of lo .. lo + n - 1
  while (n > 1) {
    const int half = n / 2;
    if (l.first[lo + half] <= c) {
      lo += half;
      n -= half;
    } else {
      n = half;
    }
  }
  return lo;
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 16 bytes' squares, in chains of four.
template <bool kBf16>
__device__ __forceinline__ float squares(const uint4 &v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kBf16) {
      const float a = bf16_low(w[i]), b = bf16_high(w[i]);
      s = fmaf(a, a, s);
      t = fmaf(b, b, t);
    } else {
      const float a = __uint_as_float(w[i]);
      s = fmaf(a, a, s);
    }
  }
  return kBf16 ? s + t : s;
}
template <bool kBf16>
__device__ __noinline__ double squares64(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  double s = 0.0;
  for (int i = 0; i < 4; ++i) {
    if constexpr (kBf16) {
      const double a = bf16_low(w[i]), b = bf16_high(w[i]);
      s += a * a + b * b;
    } else {
      const double a = __uint_as_float(w[i]);
      s += a * a;
    }
  }
  return s;
}

// An element as it lies in memory, as the first of a vector whose others are 0.
template <bool kBf16>
__device__ __forceinline__ uint4 load_one(const void *p, int64_t i) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if constexpr (kBf16)
    v.x = ld(static_cast<const uint16_t *>(p) + i);
  else
    v.x = ld(static_cast<const uint32_t *>(p) + i);
  return v;
}

// One chunk of n elements from p on: vectors, or single elements where p lies off 16 bytes.
template <bool kBf16>
__device__ __forceinline__ double chunk_squares(const void *p, int n) {
  constexpr int kPer = kBf16 ? 8 : 4;
  double total = 0.0;
  const bool wide = (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
  const int vectors = wide ? n / kPer : 0;
  const auto batch = [&](const uint4(&v)[kLoads]) {
    float s[2] = {0.f, 0.f};
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      s[i & 1] += squares<kBf16>(v[i]);
      any |= v[i].x | v[i].y | v[i].z | v[i].w;
    }
    const float sum = s[0] + s[1];
    if (sum > 0x1p-90f && sum < 0x1p120f) {
      total += double(sum);
    } else if ((any & (kBf16 ? 0x7fff7fffu : 0x7fffffffu)) != 0u) {
      for (int i = 0; i < kLoads; ++i) total += squares64<kBf16>(v[i]);
    }
  };
  uint4 v[kLoads];
  if (vectors > 0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = threadIdx.x + i * kThreads;
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (at < vectors) v[i] = ld(static_cast<const uint4 *>(p) + at);
    }
    batch(v);
  }
  for (int at = vectors * kPer + threadIdx.x; at < n; at += kThreads * kLoads) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (at + i * kThreads < n) v[i] = load_one<kBf16>(p, at + i * kThreads);
    }
    batch(v);
  }
  return total;
}

template <int kCap>
__global__ void __launch_bounds__(kThreads) sumsq_kernel(const __grid_constant__ List<kCap> l, double *partial,
                                                         int add) {
  grid_wait();
  __shared__ double warp_sum[kThreads / 32];
  const int64_t chunks = l.first[l.count];
  double total = 0.0;
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = tensor_of(l, c);
    const bool bf16 = l.n[t] & kBf16Src;
    const int64_t from = (c - l.first[t]) * chunk_elements(bf16), left = (l.n[t] & kCount) - from;
    const char *p = static_cast<const char *>(l.src[t]) + from * (bf16 ? 2 : 4);
    const int n = int(left < chunk_elements(bf16) ? left : chunk_elements(bf16));
    total += bf16 ? chunk_squares<true>(p, n) : chunk_squares<false>(p, n);
  }
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x / 32] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) total += warp_sum[w];
    if (add) total += partial[blockIdx.x];
    partial[blockIdx.x] = total;
  }
}

// The partials' sum, in an order of its own.
__global__ void __launch_bounds__(kThreads) sumsq_finish(const double *partial, int parts, double *sumsq) {
  grid_wait();
  __shared__ double warp_sum[kThreads / 32];
  double total = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) total += ld(partial + i);
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x / 32] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) total += warp_sum[w];
    *sumsq = total;
  }
}

// Elements [0, n) of a chunk, scaled (by 1 into the same type: their bits, which a conversion of a NaN changes).
template <bool kBf16Src_, bool kBf16Dst_>
__device__ __forceinline__ void chunk_scale(const void *src, void *dst, int n, float coef) {
  constexpr int kPer = kBf16Src_ ? 8 : 4;
  const bool wide = ((reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst)) & 15u) == 0;
  const int vectors = wide ? n / kPer : 0;
  if (vectors > 0) {
    uint4 v[kClipLoads];
#pragma unroll
    for (int i = 0; i < kClipLoads; ++i) {
      const int at = threadIdx.x + i * kClipThreads;
      if (at < vectors) v[i] = ld(static_cast<const uint4 *>(src) + at);
    }
#pragma unroll
    for (int i = 0; i < kClipLoads; ++i) {
      const int at = threadIdx.x + i * kClipThreads;
      if (at >= vectors) continue;
      if constexpr (kBf16Src_ == kBf16Dst_) {
        if (coef == 1.f) {
          __stcs(static_cast<uint4 *>(dst) + at, v[i]);
          continue;
        }
      }
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      float f[kPer];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kBf16Src_) {
          f[2 * j] = bf16_low(w[j]) * coef;
          f[2 * j + 1] = bf16_high(w[j]) * coef;
        } else {
          f[j] = __uint_as_float(w[j]) * coef;
        }
      }
      if constexpr (kBf16Dst_) {
        uint32_t o[kPer / 2];
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
          o[j] = *reinterpret_cast<const uint32_t *>(&b);
        }
        if constexpr (kPer == 8)
          __stcs(static_cast<uint4 *>(dst) + at, make_uint4(o[0], o[1], o[2], o[3]));
        else
          __stcs(static_cast<uint2 *>(dst) + at, make_uint2(o[0], o[1]));
      } else {
#pragma unroll
        for (int j = 0; j < kPer / 4; ++j)
          __stcs(static_cast<float4 *>(dst) + at * (kPer / 4) + j,
                 make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]));
      }
    }
  }
  for (int at = vectors * kPer + threadIdx.x; at < n; at += kClipThreads) {
    const uint32_t w = load_one<kBf16Src_>(src, at).x;
    if constexpr (kBf16Src_ == kBf16Dst_) {
      if (coef == 1.f) {
        if constexpr (kBf16Dst_)
          static_cast<uint16_t *>(dst)[at] = uint16_t(w);
        else
          static_cast<uint32_t *>(dst)[at] = w;
        continue;
      }
    }
    const float f = __uint_as_float(kBf16Src_ ? w << 16 : w) * coef;
    if constexpr (kBf16Dst_)
      static_cast<__nv_bfloat16 *>(dst)[at] = __float2bfloat16_rn(f);
    else
      static_cast<float *>(dst)[at] = f;
  }
}

template <int kCap>
__global__ void __launch_bounds__(kClipThreads, 2)
    clip_kernel(const __grid_constant__ List<kCap> l, const double *sumsq, float max_norm, int in_place, float *norm,
                float *coef) {
  grid_wait();
  __shared__ float factor;
  if (threadIdx.x == 0) {
    const double x = sqrt(ld(sumsq));
    // a norm that is not finite clips nothing: the caller sees it and drops the step
    const double c = x > double(max_norm) && x < INFINITY ? double(max_norm) / x : 1.0;
    factor = float(c);
    if (blockIdx.x == 0) {
      *norm = float(x);
      *coef = x < INFINITY ? float(c) : NAN;
    }
  }
  __syncthreads();
  const float f = factor;
  if (in_place && f == 1.f) return;
  const int64_t chunks = l.first[l.count];
  // from the end: what sumsq_kernel read last is still in L2
  for (int64_t c = chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
    const int t = tensor_of(l, c);
    const bool from16 = l.n[t] & kBf16Src, to16 = l.n[t] & kBf16Dst;
    const int64_t from = (c - l.first[t]) * chunk_elements(from16), left = (l.n[t] & kCount) - from;
    const char *p = static_cast<const char *>(l.src[t]) + from * (from16 ? 2 : 4);
    char *q = static_cast<char *>(l.dst[t]) + from * (to16 ? 2 : 4);
    const int n = int(left < chunk_elements(from16) ? left : chunk_elements(from16));
    if (from16)
      to16 ? chunk_scale<true, true>(p, q, n, f) : chunk_scale<true, false>(p, q, n, f);
    else
      to16 ? chunk_scale<false, true>(p, q, n, f) : chunk_scale<false, false>(p, q, n, f);
  }
}

// A few tensors and many: the kernel's arguments are copied by each launch.
constexpr int kFew = 48, kMany = 512;

// Lists of up to kCap tensors that are not empty, one after another: launch(list, chunks).
template <int kCap, class F>
sao_status for_lists(const sao_tensor *src, const sao_tensor *dst, int32_t count, F launch) {
  List<kCap> l;
  for (int32_t i = 0; i < count;) {
    l.count = 0;
    int64_t chunks = 0;
    for (; i < count && l.count < kCap; ++i) {
      if (src[i].n == 0) continue;
      const int at = l.count++;
      const bool bf16 = src[i].dt == SAO_BF16;
      l.src[at] = src[i].data;
      l.dst[at] = dst[i].data;
      l.n[at] = src[i].n | (bf16 ? kBf16Src : 0) | (dst[i].dt == SAO_BF16 ? kBf16Dst : 0);
      l.first[at] = chunks;
      chunks += (src[i].n + chunk_elements(bf16) - 1) / chunk_elements(bf16);
    }
    l.first[l.count] = chunks;
    SAO_TRY(launch(l, chunks));
  }
  return SAO_OK;
}

int live(const sao_tensor *t, int32_t count) {
  int n = 0;
  for (int32_t i = 0; i < count; ++i) n += t[i].n > 0;
  return n;
}

sao_status grid_of(int64_t chunks, int *grid) {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  int64_t g = int64_t(di.sm_count) * 8;
  g = g < chunks ? g : chunks;
  *grid = int(g < 1 ? 1 : g > kMaxGrid ? kMaxGrid : g);
  return SAO_OK;
}

template <int kCap>
sao_status sumsq_of(const sao_tensor *grads, int32_t count, double *sumsq, double *partial, cudaStream_t s) {
  int parts = 0;
  SAO_TRY(for_lists<kCap>(grads, grads, count, [&](const List<kCap> &l, int64_t chunks) {
    // the first list's CTAs write partials, those of later ones add to them (or write where there is none yet)
    int grid;
    SAO_TRY(grid_of(chunks, &grid));
    if (parts > 0 && grid > parts) grid = parts;
    const int slot = launch_begin("grad_sumsq", s);
    pdl(sumsq_kernel<kCap>, unsigned(grid), kThreads, 0, s)(l, partial, parts > 0 ? 1 : 0);
    if (parts == 0) parts = grid;
    return launch_end(slot, s);
  }));
  const int slot = launch_begin("grad_sumsq_finish", s);
  pdl(sumsq_finish, 1, kThreads, 0, s)(partial, parts, sumsq);
  return launch_end(slot, s);
}

template <int kCap>
sao_status clip_of(const sao_tensor *grads, const sao_tensor *out, int32_t count, const double *sumsq, float max_norm,
                   float *norm, float *coef, cudaStream_t s) {
  const int in_place = out == nullptr;
  bool any = false;
  const auto launch = [&](const List<kCap> &l, int64_t chunks) {
    int grid;
    SAO_TRY(grid_of(chunks, &grid));
    const int slot = launch_begin("grad_clip", s);
    pdl(clip_kernel<kCap>, unsigned(grid), kClipThreads, 0, s)(l, sumsq, max_norm, in_place, norm, coef);
    any = true;
    return launch_end(slot, s);
  };
  SAO_TRY(for_lists<kCap>(grads, out ? out : grads, count, launch));
  if (any) return SAO_OK;
  List<kCap> none;
  none.count = 0;
  none.first[0] = 0;
  return launch(none, 0);
}

}  // namespace

size_t grad_ws_bytes() { return round256(kMaxGrid * sizeof(double)); }

sao_status check_disjoint(const sao_tensor *grads, const sao_tensor *out, int32_t count) {
  using Span = std::pair<uintptr_t, uintptr_t>;
  const auto span = [](const sao_tensor &t) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(t.data);
    return Span{p, p + uintptr_t(t.n) * (t.dt == SAO_BF16 ? 2 : 4)};
  };
  try {
    std::vector<Span> spans;
    spans.reserve(2 * size_t(count));
    for (int32_t i = 0; i < count; ++i) {
      if (grads[i].n == 0) continue;
      spans.push_back(span(grads[i]));
      if (out && (out[i].data != grads[i].data || out[i].dt != grads[i].dt)) spans.push_back(span(out[i]));
    }
    std::sort(spans.begin(), spans.end());
    for (size_t i = 1; i < spans.size(); ++i)
      if (spans[i].first < spans[i - 1].second) return fail(SAO_ERR_INVALID_ARG, "two of the tensors overlap");
  } catch (const std::bad_alloc &) {
    return fail(SAO_ERR_INVALID_ARG, "no memory for a list of %d tensors", count);
  }
  return SAO_OK;
}

sao_status grad_sumsq_launch(const sao_tensor *grads, int32_t count, double *sumsq, void *ws, size_t ws_bytes,
                             cudaStream_t s) {
  Carver c(ws, ws_bytes);
  double *partial = c.take<double>(kMaxGrid);
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace of the gradient norm too small");
  return live(grads, count) <= kFew ? sumsq_of<kFew>(grads, count, sumsq, partial, s)
                                    : sumsq_of<kMany>(grads, count, sumsq, partial, s);
}

sao_status grad_clip_launch(const sao_tensor *grads, const sao_tensor *out, int32_t count, const double *sumsq,
                            float max_norm, float *norm, float *coef, cudaStream_t s) {
  return live(grads, count) <= kFew ? clip_of<kFew>(grads, out, count, sumsq, max_norm, norm, coef, s)
                                    : clip_of<kMany>(grads, out, count, sumsq, max_norm, norm, coef, s);
}

}  // namespace sao
