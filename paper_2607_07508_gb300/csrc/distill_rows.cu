// Distillation of one or two rows of a bf16 head, or up to eight of an fp32 one, on the fp32 units.
//
// One token's products with W are matrix-vector products: 2 h V operations for the
// 2 h V bytes of W, so the bytes are the time. The tensor-core path goes through W
// three times (logits, dZ, dH) and through dZ again for dW; here the backward holds a
// few vocabulary rows of W in registers, and while they are there forms their logits, dZ, what
// they add to dH, and their rows of dW: W is read once, dW written once.
//
// A CTA takes a contiguous range of the vocabulary, kR rows of it at a time. Each of its
// 256 threads holds kNV units of 8 (bf16) or 4 (fp32) columns of the rows, and of H; the kR x kN dot products are
// added over the CTA (a reduce-scatter in each warp, then 8 partials each through shared
// memory), and one thread per product finishes it. All sums in fp32, dZ in fp32: the
// outputs are rounded once. One row of the moe head, V = 151,936, h = 2,048: forward 104 us
// (622 MB, 6.0 TB/s), backward 209 us (1.24 GB, 5.9 TB/s), of 6.8 TB/s for a copy.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "distill.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"
#include "tc_ptx.cuh"

namespace sao {
namespace {

constexpr int kBlock = 256, kWarps = kBlock / 32;
constexpr int kMostRange = 1024;  // vocabulary rows of a CTA: its table of entries in shared memory
constexpr float kLog2e = 1.4426950408889634f;

template <class T>
struct GemvArgs {
  const T *H, *W;
  int64_t V;
  int N, h, range;
};

// A unit of a row: kCols columns in four words. kVec: they lie side by side (rows start on 16
// bytes), and unit k of a thread is the (thread + k kBlock)th of the row; else they are
// single fp32 columns, kBlock apart.
template <class T>
constexpr int kCols = 16 / int(sizeof(T));
struct Unit {
  uint32_t w[4];
};
template <class T>
__device__ __forceinline__ float value(const Unit &u, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(u.w[i]);
  return __uint_as_float(i & 1 ? u.w[i / 2] & 0xffff0000u : u.w[i / 2] << 16);
}
// The column of element i of unit k.
template <class T, bool kVec>
__device__ __forceinline__ int column(int k, int i) {
  return kVec ? (int(threadIdx.x) + k * kBlock) * kCols<T> + i : int(threadIdx.x) + (k * kCols<T> + i) * kBlock;
}
template <class T, bool kVec>
__device__ __forceinline__ Unit load_unit(const T *row, int k, int h) {
  Unit u{};
  if constexpr (kVec) {
    const int c = column<T, kVec>(k, 0);
    if (c < h) {
      const uint4 x = __ldcs(reinterpret_cast<const uint4 *>(row + c));
      u = Unit{{x.x, x.y, x.z, x.w}};
    }
  } else {
    static_assert(sizeof(T) == 4, "single columns of 4 bytes");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column<T, kVec>(k, i);
      if (c < h) u.w[i] = __ldcs(reinterpret_cast<const uint32_t *>(row + c));
    }
  }
  return u;
}

// This thread's columns of the rows of H with live[t] (0 on the others).
template <class T, bool kVec, int kNV, int kN>
__device__ __forceinline__ void load_h(const GemvArgs<T> &a, const bool (&live)[kN], float (&hf)[kN][kNV * kCols<T>]) {
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      const Unit u = live[t] ? load_unit<T, kVec>(a.H + int64_t(t) * a.h, k, a.h) : Unit{};
#pragma unroll
      for (int i = 0; i < kCols<T>; ++i) hf[t][kCols<T> * k + i] = value<T>(u, i);
    }
}
// And of kR rows of W from v0 on (0 from `end` on).
template <class T, bool kVec, int kNV, int kR>
__device__ __forceinline__ void load_w(const GemvArgs<T> &a, int64_t v0, int64_t end, Unit (&w)[kR][kNV]) {
#pragma unroll
  for (int r = 0; r < kR; ++r)
#pragma unroll
    for (int k = 0; k < kNV; ++k)
      w[r][k] = v0 + r < end ? load_unit<T, kVec>(a.W + (v0 + r) * a.h, k, a.h) : Unit{};
}

// The kR x kN products, value r kN + t in p[0] of the lanes whose upper bits are its
// number; summed over the warp.
template <int kP>
__device__ __forceinline__ void reduce_scatter(float (&p)[kP]) {
  const int lane = threadIdx.x & 31;
  int n = kP;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool up = lane & o;
#pragma unroll
      for (int i = 0; i < kP / 2; ++i)
        if (i < n) {
          const float mine = up ? p[i + n] : p[i], other = up ? p[i] : p[i + n];
          p[i] = mine + __shfl_xor_sync(0xffffffffu, other, o);
        }
    } else {
      p[0] += __shfl_xor_sync(0xffffffffu, p[0], o);
    }
  }
}

// Logits of rows [v0, v0 + kR) (in sh: 8 warps' parts of each), after which a barrier is due.
template <class T, int kNV, int kN, int kR>
__device__ __forceinline__ void products(const Unit (&w)[kR][kNV], const float (&hf)[kN][kNV * kCols<T>],
                                         float (&sh)[kWarps][kR * kN]) {
  constexpr int kP = kR * kN;
  float p[kP];
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    float s[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) s[t] = 0.f;
#pragma unroll
    for (int k = 0; k < kNV; ++k)
#pragma unroll
      for (int i = 0; i < kCols<T>; ++i) {
        const float f = value<T>(w[r][k], i);
#pragma unroll
        for (int t = 0; t < kN; ++t) s[t] = fmaf(f, hf[t][kCols<T> * k + i], s[t]);
      }
#pragma unroll
    for (int t = 0; t < kN; ++t) p[r * kN + t] = s[t];
  }
  reduce_scatter(p);
  const int lane = threadIdx.x & 31;
  if (lane % (32 / kP) == 0) sh[threadIdx.x >> 5][lane / (32 / kP)] = p[0];
}

// Elements of H (in the backward of dH too) that a thread holds; fewer leave room for more CTAs an SM.
template <class T, int kNV, int kN>
constexpr int kHeld = kNV * kN * kCols<T>;

template <class T, bool kVec, int kNV, int kN, int kR>
__global__ void __launch_bounds__(kBlock, kHeld<T, kNV, kN> <= 16 ? 3 : 2)
    distill_gemv_fwd_kernel(const GemvArgs<T> a, const TopRef top, const uint8_t *row_mask, float2 *part) {
  constexpr int kP = kR * kN;
  static_assert((kP & (kP - 1)) == 0 && kP <= 32, "a lane per product");
  __shared__ float sh[2][kWarps][kP];
  __shared__ float2 sh_part[kP];
  grid_wait();
  bool live[kN];
#pragma unroll
  for (int t = 0; t < kN; ++t) live[t] = t < a.N && (row_mask == nullptr || row_mask[t] != 0);
  float hf[kN][kNV * kCols<T>];
  load_h<T, kVec, kNV, kN>(a, live, hf);
  const int64_t begin = int64_t(blockIdx.x) * a.range, end = begin + a.range < a.V ? begin + a.range : a.V;
  // thread i < kP: product i = r kN + t of each batch; its row's entries from the range on, ascending
  const int r = threadIdx.x / kN, t = threadIdx.x % kN;
  const bool mine = threadIdx.x < kP && t < a.N && (row_mask == nullptr || row_mask[t] != 0);
  float m = -INFINITY, s = 0.f;
  const float scale = top.inv_t * kLog2e;
  int q = 0, q_end = 0;
  if (mine) {
    const uint16_t *off = top.off + int64_t(t) * (top.tiles + 1);
    q = ld(off + begin / kTopTile);
    q_end = ld(off + top.tiles);
  }
  const int32_t *ids = top.id + int64_t(t) * top.K;
  int64_t next = q < q_end ? ld(ids + q) : a.V;
  int buf = 0;
  for (int64_t v0 = begin; v0 < end; v0 += kR, buf ^= 1) {
    Unit w[kR][kNV];
    load_w<T, kVec, kNV, kR>(a, v0, end, w);
    products<T, kNV, kN, kR>(w, hf, sh[buf]);
    __syncthreads();
    const int64_t v = v0 + r;
    if (mine && v < end) {
      float z = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) z += sh[buf][k][threadIdx.x];
      while (next < v) next = ++q < q_end ? ld(ids + q) : a.V;
      if (next == v) {
        top.z[int64_t(t) * top.K + q] = z * top.inv_t;
      } else {
        const float mn = !(z <= m) ? z : m;  // (NaN stays in s)
        if (mn != -INFINITY) {
          s = s * tc::ex2_approx((m - mn) * scale) + tc::ex2_approx((z - mn) * scale);
          m = mn;
        }
      }
    }
  }
  if (threadIdx.x < kP) sh_part[threadIdx.x] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x < kN && threadIdx.x < a.N) {
    float2 x = sh_part[threadIdx.x];
    for (int k = 1; k < kR; ++k) {
      const float2 y = sh_part[k * kN + threadIdx.x];
      const float mn = fmaxf(x.x, y.x);
      if (mn == -INFINITY) continue;
      x = make_float2(mn, x.y * tc::ex2_approx((x.x - mn) * scale) + y.y * tc::ex2_approx((y.x - mn) * scale));
    }
    part[int64_t(blockIdx.x) * a.N + threadIdx.x] = make_float2(x.x * top.inv_t, x.y);
  }
}

template <class T, bool kVec, int kNV, int kN, int kR, class TW>
__global__ void __launch_bounds__(kBlock, kHeld<T, kNV, kN> <= (sizeof(T) == 2 ? 16 : 32) ? 2 : 1)
    distill_gemv_bwd_kernel(const GemvArgs<T> a, const TopGrad g, TW *dW, int accumulate, float *dh_part) {
  constexpr int kP = kR * kN;
  extern __shared__ float table[];  // [range][kN]: the entries' dZ; below, a bit for each that there is
  __shared__ float sh[2][kWarps][kP], sh_dz[2][kP];
  grid_wait();
  bool live[kN];
#pragma unroll
  for (int t = 0; t < kN; ++t) live[t] = t < a.N && g.mask[t] != 0;
  constexpr int kC = kCols<T>;
  float hf[kN][kNV * kC], dh[kN][kNV * kC];
  load_h<T, kVec, kNV, kN>(a, live, hf);
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int j = 0; j < kNV * kC; ++j) dh[t][j] = 0.f;
  const int64_t begin = int64_t(blockIdx.x) * a.range, end = begin + a.range < a.V ? begin + a.range : a.V;
  uint32_t *bits = reinterpret_cast<uint32_t *>(table + a.range * kN);
  const int words = (a.range * kN + 31) / 32;
  for (int i = threadIdx.x; i < words; i += kBlock) bits[i] = 0u;
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kN; ++t) {
    if (!live[t]) continue;
    for (int i = threadIdx.x; i < g.K; i += kBlock) {
      const int64_t id = ld(g.ids + int64_t(t) * g.K + i);
      if (id < begin || id >= end) continue;
      const int at = int(id - begin) * kN + t;
      table[at] = ld(g.dz_top + int64_t(t) * g.K + i);
      atomicOr(bits + at / 32, 1u << (at % 32));
    }
  }
  const int r = threadIdx.x / kN, t = threadIdx.x % kN;
  const bool mine = threadIdx.x < kP && t < a.N && g.mask[t] != 0;
  const float gr = mine ? ld(g.g + t) : 0.f, rest = mine ? ld(g.rest + t) : 0.f;
  int buf = 0;
  for (int64_t v0 = begin; v0 < end; v0 += kR, buf ^= 1) {
    Unit w[kR][kNV];
    load_w<T, kVec, kNV, kR>(a, v0, end, w);
    products<T, kNV, kN, kR>(w, hf, sh[buf]);
    __syncthreads();
    if (threadIdx.x < kP) {
      float dz = 0.f;
      if (mine && v0 + r < end) {
        const int at = int(v0 - begin + r) * kN + t;
        if (bits[at / 32] >> (at % 32) & 1u) {
          dz = table[at];
        } else if (gr != 0.f) {
          float z = 0.f;
#pragma unroll
          for (int k = 0; k < kWarps; ++k) z += sh[buf][k][threadIdx.x];
          dz = gr * tc::ex2_approx(fmaf(z, g.inv_t, -rest) * kLog2e);
        }
      }
      sh_dz[buf][threadIdx.x] = dz;
    }
    __syncthreads();
#pragma unroll
    for (int rr = 0; rr < kR; ++rr) {
      float dz[kN];
#pragma unroll
      for (int tt = 0; tt < kN; ++tt) dz[tt] = sh_dz[buf][rr * kN + tt];
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        float o[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) {
          const float f = value<T>(w[rr][k], i);
          o[i] = 0.f;
#pragma unroll
          for (int tt = 0; tt < kN; ++tt) {
            dh[tt][kC * k + i] = fmaf(dz[tt], f, dh[tt][kC * k + i]);
            o[i] = fmaf(dz[tt], hf[tt][kC * k + i], o[i]);
          }
        }
        if (v0 + rr >= end) continue;
        TW *row = dW + (v0 + rr) * a.h;
        const int c = column<T, kVec>(k, 0);
        if constexpr (!kVec) {
#pragma unroll
          for (int i = 0; i < kC; ++i) {
            const int ci = column<T, kVec>(k, i);
            if (ci < a.h) row[ci] = accumulate ? o[i] + row[ci] : o[i];
          }
        } else if (c < a.h) {
          if constexpr (sizeof(TW) == 2) {
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const __nv_bfloat162 y = __floats2bfloat162_rn(o[2 * i], o[2 * i + 1]);
              b[i] = *reinterpret_cast<const uint32_t *>(&y);
            }
            __stcs(reinterpret_cast<uint4 *>(row + c), make_uint4(b[0], b[1], b[2], b[3]));
          } else {
#pragma unroll
            for (int i = 0; i < kC; i += 4) {
              float4 *d4 = reinterpret_cast<float4 *>(row + c + i);
              float4 y = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
              if (accumulate) {
                const float4 old = *d4;
                y = make_float4(y.x + old.x, y.y + old.y, y.z + old.z, y.w + old.w);
              }
              *d4 = y;
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int tt = 0; tt < kN; ++tt) {
    if (tt >= a.N) continue;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      float *row = dh_part + (int64_t(blockIdx.x) * a.N + tt) * a.h;
      if constexpr (kVec) {
        const int c = column<T, kVec>(k, 0);
        if (c >= a.h) continue;
#pragma unroll
        for (int i = 0; i < kC; i += 4)
          *reinterpret_cast<float4 *>(row + c + i) =
              make_float4(dh[tt][kC * k + i], dh[tt][kC * k + i + 1], dh[tt][kC * k + i + 2], dh[tt][kC * k + i + 3]);
      } else {
#pragma unroll
        for (int i = 0; i < kC; ++i)
          if (column<T, kVec>(k, i) < a.h) row[column<T, kVec>(k, i)] = dh[tt][kC * k + i];
      }
    }
  }
}

// dH = the sum of the CTAs' parts, rounded once: 32 columns and 32 slices of the parts per CTA, in a fixed order.
template <class T>
__global__ void __launch_bounds__(1024) distill_gemv_dH_kernel(const float *part, int parts, int64_t elements, T *dH) {
  __shared__ float sh[32][33];
  grid_wait();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t e = int64_t(blockIdx.x) * 32 + lane;
  float s = 0.f;
  if (e < elements) {
#pragma unroll 8
    for (int k = slice; k < parts; k += 32) s += ld(part + k * elements + e);
  }
  sh[slice][lane] = s;
  __syncthreads();
  if (slice != 0 || e >= elements) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 32; ++k) s += sh[k][lane];
  if constexpr (sizeof(T) == 4)
    dH[e] = s;
  else
    dH[e] = __float2bfloat16_rn(s);
}

// Units that a thread holds of a row.
int units_of(sao_dtype dt, int32_t h) {
  const int columns = dt == SAO_BF16 ? 8 * kBlock : 4 * kBlock;
  return (h + columns - 1) / columns;
}

// Vocabulary rows of a CTA: as many CTAs as two fit on each of 152 SMs, whole batches, at most
// kMostRange. From V alone: the same sums on every device.
int range_of(int32_t V) {
  int r = (V + 303) / 304;
  r = (r + 7) / 8 * 8;
  return r > kMostRange ? kMostRange : r;
}
int grid_of(int32_t V) {
  const int r = range_of(V);
  return (V + r - 1) / r;
}

// f(units a thread, rows of H, rows of W at a time): what gemv_takes() lets in.
template <int kValue>
struct Int {
  static constexpr int value = kValue;
};
template <class F>
void with_bf16_sizes(int64_t N, int32_t h, F f) {
  switch (units_of(SAO_BF16, h)) {
    case 1:
      if (N == 1) return f(Int<1>{}, Int<1>{}, Int<8>{});
      return f(Int<1>{}, Int<2>{}, Int<8>{});
    case 2:
      return f(Int<2>{}, Int<1>{}, Int<4>{});
    default:
      return f(Int<3>{}, Int<1>{}, Int<4>{});
  }
}
template <class F>
void with_f32_sizes(int64_t N, int32_t h, F f) {
  switch (units_of(SAO_F32, h)) {
    case 1:
      if (N == 1) return f(Int<1>{}, Int<1>{}, Int<8>{});
      if (N <= 4) return f(Int<1>{}, Int<4>{}, Int<8>{});
      return f(Int<1>{}, Int<8>{}, Int<4>{});
    case 2:
      if (N == 1) return f(Int<2>{}, Int<1>{}, Int<8>{});
      return f(Int<2>{}, Int<4>{}, Int<4>{});
    default:
      return f(Int<4>{}, Int<1>{}, Int<4>{});
  }
}
// Rows of H and W (and dW) start on 16 bytes.
bool vectors(sao_dtype dt, const void *H, const void *W, const void *dW, int32_t h) {
  return dt == SAO_BF16 || (h % 4 == 0 && aligned16(H) && aligned16(W) && aligned16(dW));
}

template <class T, bool kVec, class S>
void launch_fwd(const void *H, const void *W, const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                const TopRef &top, float2 *part, cudaStream_t s, S with_sizes) {
  const GemvArgs<T> a{static_cast<const T *>(H), static_cast<const T *>(W), V, int(N), h, range_of(V)};
  with_sizes([&](auto nv, auto n, auto r) {
    pdl(distill_gemv_fwd_kernel<T, kVec, nv.value, n.value, r.value>, unsigned(grid_of(V)), kBlock, 0, s)(
        a, top, row_mask, part);
  });
}
template <class T, bool kVec, class TW, class S>
void launch_bwd(const void *H, const void *W, const TopGrad &t, int64_t N, int32_t h, int32_t V, void *dW,
                int accumulate, float *part, cudaStream_t s, S with_sizes) {
  const GemvArgs<T> a{static_cast<const T *>(H), static_cast<const T *>(W), V, int(N), h, range_of(V)};
  with_sizes([&](auto nv, auto n, auto r) {
    const size_t smem = size_t(a.range) * n.value * 4 + (size_t(a.range) * n.value + 31) / 32 * 4;
    pdl(distill_gemv_bwd_kernel<T, kVec, nv.value, n.value, r.value, TW>, unsigned(grid_of(V)), kBlock, smem, s)(
        a, t, static_cast<TW *>(dW), accumulate, part);
  });
}

}  // namespace

// bf16: one row of up to 6,144 columns, two of up to 2,048. Against the tensor-core path, forward
// and backward (us): moe head 322 / 460 for one row, 347 / 462 for two, but 467 / 461
// for four, which leave registers for one CTA an SM; h = 1,024, V = 32,000 67 / 85, 76 / 85,
// 105 / 85; h = 6,144 1,023 / 1,244 for one.
// fp32, where that path splits W into three planes and multiplies them six times: eight rows of up to
// 1,024 columns, four of up to 2,048, one of up to 4,096: h = 1,024, V = 32,000 88 / 357 for one row,
// 100 / 359 for two to four, 135 / 360 for eight; h = 515, V = 20,000 44 / 204, 63 / 207, 94 / 208.
int64_t gemv_rows(int32_t h, sao_dtype dt) {
  const int u = units_of(dt, h);
  if (dt == SAO_BF16) return u == 1 ? 2 : u <= 3 ? 1 : 0;
  return u == 1 ? 8 : u == 2 ? 4 : u <= 4 ? 1 : 0;
}
bool gemv_takes(int64_t N, int32_t h, sao_dtype dt) { return N <= gemv_rows(h, dt); }

size_t gemv_fwd_bytes(int64_t N, int32_t V) { return round256(sizeof(float2) * size_t(grid_of(V)) * size_t(N)); }
size_t gemv_bwd_bytes(int64_t N, int32_t h, int32_t V) {
  return round256(sizeof(float) * size_t(grid_of(V)) * size_t(N) * size_t(h));
}

sao_status gemv_distill_fwd(const void *H, const void *W, sao_dtype dt, const uint8_t *row_mask, int64_t N, int32_t h,
                            int32_t V, const TopRef &top, const TopFinish &f, Carver &c, cudaStream_t s) {
  const int grid = grid_of(V);
  float2 *part = c.take<float2>(size_t(grid) * size_t(N));
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the distillation forward");
  int slot = launch_begin("distill_gemv_fwd", s);
  auto bf16 = [&](auto g) { with_bf16_sizes(N, h, g); };
  auto f32 = [&](auto g) { with_f32_sizes(N, h, g); };
  if (dt == SAO_BF16)
    launch_fwd<__nv_bfloat16, true>(H, W, row_mask, N, h, V, top, part, s, bf16);
  else if (vectors(dt, H, W, nullptr, h))
    launch_fwd<float, true>(H, W, row_mask, N, h, V, top, part, s, f32);
  else
    launch_fwd<float, false>(H, W, row_mask, N, h, V, top, part, s, f32);
  SAO_TRY(launch_end(slot, s));
  return distill_finish(top, f, part, grid, nullptr, N, s);
}

sao_status gemv_distill_bwd(const void *H, const void *W, sao_dtype dt, const TopGrad &t, int64_t N, int32_t h,
                            int32_t V, void *dH, void *dW, sao_dtype dw_dt, int accumulate, Carver &c, cudaStream_t s) {
  const int grid = grid_of(V);
  float *part = c.take<float>(size_t(grid) * size_t(N) * size_t(h));
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the distillation backward");
  int slot = launch_begin("distill_gemv_bwd", s);
  auto bf16 = [&](auto g) { with_bf16_sizes(N, h, g); };
  auto f32 = [&](auto g) { with_f32_sizes(N, h, g); };
  if (dt == SAO_BF16 && dw_dt == SAO_BF16)
    launch_bwd<__nv_bfloat16, true, __nv_bfloat16>(H, W, t, N, h, V, dW, 0, part, s, bf16);
  else if (dt == SAO_BF16)
    launch_bwd<__nv_bfloat16, true, float>(H, W, t, N, h, V, dW, accumulate, part, s, bf16);
  else if (vectors(dt, H, W, dW, h))
    launch_bwd<float, true, float>(H, W, t, N, h, V, dW, accumulate, part, s, f32);
  else
    launch_bwd<float, false, float>(H, W, t, N, h, V, dW, accumulate, part, s, f32);
  SAO_TRY(launch_end(slot, s));
  slot = launch_begin("distill_gemv_dH", s);
  const unsigned ctas = unsigned((N * h + 31) / 32);
  if (dt == SAO_BF16)
    pdl(distill_gemv_dH_kernel<__nv_bfloat16>, ctas, 1024, 0, s)(part, grid, N * h, static_cast<__nv_bfloat16 *>(dH));
  else
    pdl(distill_gemv_dH_kernel<float>, ctas, 1024, 0, s)(part, grid, N * h, static_cast<float *>(dH));
  return launch_end(slot, s);
}

}  // namespace sao
