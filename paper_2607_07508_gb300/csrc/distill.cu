// Distillation from a teacher's top logits: the per-row work around the LM head's
// products (logprobs_tc.cu, logprobs_f32.cu).
//
// Row t has student logits z_v = H_t . W_v / T, teacher entries S = {id_k >= 0} with
// logits a_k (divided by T here), and the loss is the Kullback-Leibler divergence
// between the two distributions with the vocabulary outside S as one outcome:
//   la  = log sum_S e^{a_k}, or the teacher's log-sum-exp over its vocabulary
//   p_k = e^{a_k - la},  rho = max(0, 1 - sum p)   (0 where the entries are renormalised)
//   loss = sum_S p_k (a_k - la - z_k + lse) + rho (log rho - (lse_R - lse))
// with lse over all columns and lse_R over those outside S. The forward's epilogues
// sum e^z outside S and keep z_k, so lse_R comes from a sum of its own terms: as
// 1 - sum q_k it would have no digits left where the student puts its mass on S.
//   d loss / d z_k = m q_k - p_k on S,  e^{z_v - lse_R} (m q_R - rho) outside,
// m = sum p + rho, q_k = e^{z_k - lse}, q_R = e^{lse_R - lse}: the second is
// q_v (m - rho / q_R) without a quotient that overflows as q_R vanishes. The teacher's
// mass m is 1 but where the entries' p add up to more (logits rounded to bf16 against the
// log-sum-exp of the exact ones), or are the whole vocabulary and do not add up to 1.
#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

#include "distill.cuh"
#include "f32_planes.cuh"
#include "logprobs_common.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"

namespace sao {
namespace {

constexpr int kSortWarps = 4;  // rows (one per warp) per CTA of the sort

__device__ __forceinline__ float teacher_logit(const void *a, sao_dtype adt, int64_t i) {
  return adt == SAO_BF16 ? __bfloat162float(ld(static_cast<const __nv_bfloat16 *>(a) + i))
                         : ld(static_cast<const float *>(a) + i);
}

// Sorts each row's entries by id (bitonic, in shared memory, a warp per row) and counts
// those below each 256-column tile. Entries with a negative id go last. A row with an id
// of V or more, or one id twice, is marked and raises SAO_DEVERR_TOP_ID.
__global__ void __launch_bounds__(32 * kSortWarps)
    distill_sort_kernel(const int32_t *ids, const uint8_t *row_mask, int64_t N, int K, int kp, int V, int tiles,
                        int32_t *sid, uint16_t *slot, uint16_t *off, int32_t *entries, unsigned int *range,
                        unsigned int *err) {
  extern __shared__ uint64_t sort_smem[];
  grid_wait();
  if (blockIdx.x == 0 && threadIdx.x < kRangeWords) range[threadIdx.x] = 0u;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = int64_t(blockIdx.x) * kSortWarps + warp;
  if (t >= N) return;
  if (row_mask && row_mask[t] == 0) {  // an fp32 forward of few rows runs over the masked ones too
    for (int j = lane; j <= tiles; j += 32) off[t * (tiles + 1) + j] = 0;
    return;
  }
  uint64_t *key = sort_smem + warp * kp;
  bool bad = false;
  int n = 0;
  for (int i = lane; i < kp; i += 32) {
    uint32_t id = 0xffffffffu;
    if (i < K) {
      const int32_t v = ld(ids + t * K + i);
      if (v >= V) bad = true;
      if (v >= 0) {
        id = uint32_t(v);
        ++n;
      }
    }
    key[i] = uint64_t(id) << 32 | uint32_t(i);
  }
  n = __reduce_add_sync(0xffffffffu, n);
  __syncwarp();
  for (int size = 2; size <= kp; size <<= 1) {
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      for (int i = lane; i < kp / 2; i += 32) {
        const int lo = 2 * i - (i & (stride - 1)), hi = lo + stride;
        const uint64_t x = key[lo], y = key[hi];
        if ((x > y) == ((lo & size) == 0)) {
          key[lo] = y;
          key[hi] = x;
        }
      }
      __syncwarp();
    }
  }
  for (int i = lane; i < K; i += 32) {
    const uint64_t x = key[i];
    if (i > 0 && i < n && uint32_t(key[i - 1] >> 32) == uint32_t(x >> 32)) bad = true;
    sid[t * K + i] = int32_t(x >> 32);
    slot[t * K + i] = uint16_t(x);
  }
  bad = __any_sync(0xffffffffu, bad);
  for (int j = lane; j <= tiles; j += 32) {
    int lo = 0, hi = n;  // entries with ids below 256 j
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((key[mid] >> 32) < uint64_t(j) * kTopTile)
        lo = mid + 1;
      else
        hi = mid;
    }
    off[t * (tiles + 1) + j] = uint16_t(bad ? 0 : lo);
  }
  if (lane == 0) {
    entries[t] = bad ? -1 : n;
    if (bad) raise_device_error(err, SAO_DEVERR_TOP_ID);
  }
}

// (m, s) pairs of a running maximum and a sum of exp(x - m). A NaN stays in s.
struct MaxSum {
  float m = -INFINITY, s = 0.f;
  __device__ __forceinline__ void add(float pm, float ps) {
    const bool up = !(pm <= m);
    const float mn = up ? pm : m;
    if (mn == -INFINITY) return;
    const float e = expf((up ? m : pm) - mn);
    s = up ? fmaf(s, e, ps) : fmaf(ps, e, s);
    m = mn;
  }
  __device__ __forceinline__ float log() const { return s > 0.f || s != s ? m + logf(s) : -INFINITY; }
};
template <int kSub>
__device__ __forceinline__ MaxSum sub_merge(MaxSum a) {
#pragma unroll
  for (int o = 1; o < kSub; o <<= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, a.m, o), os = __shfl_xor_sync(0xffffffffu, a.s, o);
    a.add(om, os);
  }
  return a;
}
template <int kSub>
__device__ __forceinline__ float sub_sum(float x) {
#pragma unroll
  for (int o = 1; o < kSub; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// kSub threads per row, as in the merge of the log-probs: thread k of a row takes the
// partials and the entries k, k + kSub, ...
template <int kSub>
__global__ void __launch_bounds__(256) distill_finish_kernel(const TopRef top, const TopFinish f, const float2 *part,
                                                             int nvt, const int *pos, int64_t N) {
  grid_wait();
  const int64_t tid = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t row = tid / kSub;
  const int sub = int(tid % kSub);
  const bool live = row < N;
  bool skip = !live || (f.row_mask != nullptr && f.row_mask[row] == 0);
  int64_t src = row;
  if (!skip && pos != nullptr) src = pos[row];
  const int n = skip ? 0 : ld(f.entries + row);  // (-1: no loop below runs)
  MaxSum rest;
  if (!skip) {
    constexpr int kU = kSub == 32 ? 8 : 4;  // loads in flight
    int j = sub;
    for (; j + (kU - 1) * kSub < nvt; j += kU * kSub) {
      float2 p[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) p[u] = __ldcs(part + int64_t(j + u * kSub) * N + src);
#pragma unroll
      for (int u = 0; u < kU; ++u) rest.add(p[u].x, p[u].y);
    }
    for (; j < nvt; j += kSub) {
      const float2 p = __ldcs(part + int64_t(j) * N + src);
      rest.add(p.x, p.y);
    }
  }
  rest = sub_merge<kSub>(rest);
  MaxSum student, teacher;
  const int64_t base = row * top.K;
  for (int i = sub; i < n; i += kSub) {
    student.add(ld(top.z + base + i), 1.f);
    teacher.add(teacher_logit(f.a, f.adt, base + ld(f.slot + base + i)) * top.inv_t, 1.f);
  }
  student = sub_merge<kSub>(student);
  teacher = sub_merge<kSub>(teacher);
  student.add(rest.m, rest.s);
  const float lse = student.log(), lse_rest = rest.log();
  const bool whole = f.teacher_lse != nullptr && !skip;
  const float la = whole ? ld(f.teacher_lse + row) : teacher.log();
  float psum = 0.f, loss = 0.f;
  for (int i = sub; i < n; i += kSub) {
    const float a = teacher_logit(f.a, f.adt, base + ld(f.slot + base + i)) * top.inv_t - la;
    const float p = expf(a);
    psum += p;
    if (p != 0.f) loss += p * ((a - ld(top.z + base + i)) + lse);
  }
  psum = sub_sum<kSub>(psum);
  loss = sub_sum<kSub>(loss);
  if (live) {
    for (int i = sub; i < top.K; i += kSub) {
      const bool entry = i < n;
      const int64_t at = skip || n < 0 ? base + i : base + ld(f.slot + base + i);
      f.z_top[at] = entry ? ld(top.z + base + i) : 0.f;
    }
  }
  if (!live || sub != 0) return;
  const float nan = __int_as_float(0x7fc00000);
  if (skip) {
    f.loss[row] = 0.f;
    f.lse[row] = 0.f;
    f.lse_rest[row] = nan;
    return;
  }
  float l = loss;
  bool grad = true;
  if (whole) {
    // the teacher's mass outside its entries; there is none where they are all columns
    const float rho = lse_rest == -INFINITY ? 0.f : 1.f - psum;
    if (rho > 0.f) l += rho * (logf(rho) - (lse_rest - lse));
    if (psum != psum || la != la) l = nan;
  } else if (teacher.m == -INFINITY) {
    l = 0.f;  // no entry, or none with a finite logit: nothing to learn
    grad = false;
  }
  if (n < 0) l = nan;
  f.loss[row] = l;
  f.lse[row] = lse;
  f.lse_rest[row] = grad && isfinite(l) ? lse_rest : nan;
}

// What the backward's products need of each row (kSub threads per row): the factor and
// the log-sum-exp of the columns outside the entries, and the entries' dZ.
template <int kSub>
__global__ void __launch_bounds__(256)
    distill_rows_kernel(const int32_t *ids, const void *a, sao_dtype adt, const float *teacher_lse, const float *lse,
                        const float *lse_rest, const float *z_top, const float *grad, int64_t N, int K, float inv_t,
                        uint8_t *mask, float *g_rest, float *rest, float *dz_top, unsigned int *range, float *lost) {
  grid_wait();
  if (blockIdx.x == 0 && threadIdx.x < kRangeWords) range[threadIdx.x] = 0u;
  if (lost != nullptr && blockIdx.x == 0 && threadIdx.x < kExtraRows) {
    mask[N + threadIdx.x] = 1;
    g_rest[N + threadIdx.x] = 0.f;
    rest[N + threadIdx.x] = 0.f;
  }
  const int64_t tid = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t row = tid / kSub;
  const int sub = int(tid % kSub);
  const bool live = row < N;
  const float g = live ? ld(grad + row) : 0.f, lr = live ? ld(lse_rest + row) : 0.f;
  const bool on = live && g != 0.f && lr == lr;
  const int64_t base = row * K;
  const int n = on ? K : 0;
  const bool whole = teacher_lse != nullptr;
  MaxSum teacher;
  if (!whole) {
    for (int i = sub; i < n; i += kSub)
      if (ld(ids + base + i) >= 0) teacher.add(teacher_logit(a, adt, base + i) * inv_t, 1.f);
    teacher = sub_merge<kSub>(teacher);
  }
  const float la = whole ? (on ? ld(teacher_lse + row) : 0.f) : teacher.log();
  const float l = on ? ld(lse + row) : 0.f, gt = g * inv_t;
  const bool none = lr == -INFINITY;  // the entries are all columns
  float mass = 1.f, rho = 0.f;        // of the teacher: in all, and outside the entries
  if (whole) {
    float psum = 0.f;
    for (int i = sub; i < n; i += kSub)
      if (ld(ids + base + i) >= 0) psum += expf(teacher_logit(a, adt, base + i) * inv_t - la);
    psum = sub_sum<kSub>(psum);
    mass = none ? psum : fmaxf(psum, 1.f);
    rho = none ? 0.f : fmaxf(1.f - psum, 0.f);
  }
  float off = 0.f;  // what rounding the entries to bf16 takes
  for (int i = sub; i < n; i += kSub) {
    if (ld(ids + base + i) < 0) continue;
    const float p = expf(teacher_logit(a, adt, base + i) * inv_t - la);
    const float d = gt * (mass * expf(ld(z_top + base + i) - l) - p);
    dz_top[base + i] = d;
    off += fabsf(d - __bfloat162float(__float2bfloat16_rn(d)));
  }
  off = sub_sum<kSub>(off);
  if (!live || sub != 0) return;
  if (lost != nullptr) lost[row] = off;
  mask[row] = on ? 1 : 0;
  if (!on) return;
  g_rest[row] = none ? 0.f : gt * (mass * expf(lr - l) - rho);
  rest[row] = none ? 0.f : lr;
}

// The block's exclusive sums of v, and *total (every thread; `sh` of 33).
__device__ __forceinline__ int block_before(int v, int *sh, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += up;
  }
  __syncthreads();
  if (lane == 31) sh[warp] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 32; ++w) {
    if (w < warp) before += sh[w];
    all += sh[w];
  }
  *total = all;
  return before + s - v;
}

// extra[j]: the kExtraRows tokens with the largest lost[] (none with 0), one CTA. The least value that
// is among them is found bit by bit, to 2^-11 of itself; where more tokens have it than
// there is room for, the first ones. Bound by its barriers.
__global__ void __launch_bounds__(1024) distill_extra_kernel(const float *lost, int N, int *extra) {
  constexpr int kEach = int(kExtraMost / 1024), kLowBit = 12;
  __shared__ int sh[32], counts[2][32];
  grid_wait();
  uint32_t key[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int t = int(threadIdx.x) * kEach + i;
    key[i] = t < N ? __float_as_uint(ld(lost + t)) : 0u;
  }
  auto among = [&](uint32_t low, uint32_t high) {  // keys in [low, high) of this thread
    int n = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) n += key[i] >= low && key[i] < high;
    return n;
  };
  constexpr uint32_t kMost = 0x80000000u;
  uint32_t least = 0u;
  for (int bit = 30; bit >= kLowBit; --bit) {
    const int n = __reduce_add_sync(0xffffffffu, among(least | 1u << bit, kMost));
    if ((threadIdx.x & 31) == 0) counts[bit & 1][threadIdx.x >> 5] = n;
    __syncthreads();
    if (__reduce_add_sync(0xffffffffu, counts[bit & 1][threadIdx.x & 31]) >= kExtraRows) least |= 1u << bit;
  }
  if (threadIdx.x < kExtraRows) extra[threadIdx.x] = -1;
  int taken = 0;
  uint32_t low = least + (1u << kLowBit), high = kMost;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {  // those above the least one, then those at it
    int total, at = taken + block_before(among(low, high), sh, &total);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (key[i] >= low && key[i] < high) {
        if (at < kExtraRows) extra[at] = int(threadIdx.x) * kEach + i;
        ++at;
      }
    taken += total;
    high = low;
    low = least > 0u ? least : 1u;
  }
}

// CTA (j, 1,024 columns, part): acc[part][row of its token] += acc[part][extra row j].
__global__ void __launch_bounds__(256) distill_fold_kernel(const TopGrad t, float *acc, const DhParts d, int h,
                                                           const int *pos, const int *count) {
  grid_wait();
  const int token = ld(t.extra + blockIdx.x);
  if (token < 0) return;
  const int rows = *count, parts = d.cap_rows ? dh_parts(d, rows) : 1;
  const int64_t to = ld(pos + token), from = ld(pos + t.tokens + blockIdx.x);
  const int c = int(blockIdx.y * 256 + threadIdx.x) * 4;  // (h is a multiple of 8)
  if (c >= h) return;
  for (int k = blockIdx.z; k < parts; k += gridDim.z) {
    float *part = acc + int64_t(k) * rows * h + c;
    float4 x = *reinterpret_cast<const float4 *>(part + to * h);
    const float4 y = *reinterpret_cast<const float4 *>(part + from * h);
    x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
    *reinterpret_cast<float4 *>(part + to * h) = x;
  }
}

// A warp per compacted row.
enum Patch : int { kOnePiece = 0, kFewPieces = 1, kThreePlanes = 2 };
template <int kPatch>
__global__ void __launch_bounds__(256)
    distill_patch_kernel(const TopGrad g, const int *idx, const int *count, int v0, int vc, __nv_bfloat16 *dz,
                         int64_t ldz, int64_t plane, unsigned int *range) {
  grid_wait();
  const int64_t i = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (i >= *count) return;
  int64_t t = ld(idx + i);
  bool second = kPatch == kFewPieces && i >= kFewRows;
  if (kPatch == kOnePiece && g.extra != nullptr && t >= g.tokens) {
    t = ld(g.extra + (t - g.tokens));
    second = true;
  }
  if (t < 0) return;
  const int64_t base = t * g.K;
  float most = 0.f;
  for (int k = threadIdx.x & 31; k < g.K; k += 32) {
    const int id = ld(g.ids + base + k);
    if (id < v0 || id - v0 >= vc) continue;
    const int c = id - v0;
    const float d = ld(g.dz_top + base + k);
    __nv_bfloat16 *dst = dz + i * ldz + c;
    if constexpr (kPatch == kThreePlanes) {
      most = larger(most, d);
      float p0, p1, p2;
      split3(d, p0, p1, p2);
      dst[0] = __float2bfloat16_rn(p0);
      dst[plane] = __float2bfloat16_rn(p1);
      dst[2 * plane] = __float2bfloat16_rn(p2);
    } else {
      const __nv_bfloat16 b = __float2bfloat16_rn(d);
      dst[0] = second ? __float2bfloat16_rn(d - __bfloat162float(b)) : b;
    }
  }
  if constexpr (kPatch == kThreePlanes) raise_class(range, most);
}

template <int kPatch>
sao_status patch(const TopGrad &t, const int *idx, const int *count, int64_t rows, int v0, int vc, __nv_bfloat16 *dz,
                 int64_t ldz, int64_t plane, unsigned int *range, cudaStream_t s) {
  int slot = launch_begin("distill_patch", s);
  pdl(distill_patch_kernel<kPatch>, unsigned((rows + 7) / 8), 256, 0, s)(t, idx, count, v0, vc, dz, ldz, plane, range);
  return launch_end(slot, s);
}

// CTA r: row r of Hc.
__global__ void __launch_bounds__(128) distill_few_rows_kernel(const uint8_t *mask, int N, const __nv_bfloat16 *H,
                                                               int h, int *idx, int *pos, int *count,
                                                               __nv_bfloat16 *Hc) {
  grid_wait();
  const int lane = threadIdx.x & 31;
  const unsigned lo = __ballot_sync(0xffffffffu, lane < N && mask[lane] != 0);
  const unsigned hi = __ballot_sync(0xffffffffu, lane + 32 < N && mask[lane + 32] != 0);
  const int n = __popc(lo) + __popc(hi), p = blockIdx.x % kFewRows;
  int t = -1;  // the p-th active token
  if (p < __popc(lo))
    t = __fns(lo, 0, p + 1);
  else if (p < n)
    t = 32 + __fns(hi, 0, p + 1 - __popc(lo));
  if (threadIdx.x == 0) idx[blockIdx.x] = t;
  if (blockIdx.x == 0 && threadIdx.x < N) {
    const int i = threadIdx.x;
    const unsigned word = i < 32 ? lo : hi, bit = 1u << (i & 31);
    pos[i] = word & bit ? __popc(word & (bit - 1u)) + (i < 32 ? 0 : __popc(lo)) : -1;
    if (i == 0) *count = n > 0 ? kFewRows + n : 0;
  }
  const uint4 *src = reinterpret_cast<const uint4 *>(H + int64_t(t) * h);
  uint4 *dst = reinterpret_cast<uint4 *>(Hc + int64_t(blockIdx.x) * h);
  for (int v = threadIdx.x; v < h / 8; v += 128) dst[v] = t >= 0 ? src[v] : make_uint4(0u, 0u, 0u, 0u);
}

__global__ void __launch_bounds__(256) distill_few_dH_kernel(const float *acc, const DhParts d, int h, const int *pos,
                                                             const int *count, int64_t N, __nv_bfloat16 *dH) {
  grid_wait();
  const int rows = *count, parts = dh_parts(d, rows);
  const int64_t part = int64_t(rows) * h, e = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (e >= N * h) return;
  const int64_t t = e / h, i = pos[t];
  float x = 0.f;
  if (i >= 0)
    for (int k = 0; k < parts; ++k) {
      const float *src = acc + k * part + i * h + (e - t * h);
      x += src[0] + src[int64_t(kFewRows) * h];
    }
  dH[e] = __float2bfloat16_rn(x);
}

// Rows up to which a warp takes one (see the merge of the log-probs).
constexpr int64_t kWarpRows = 8192;
int row_threads(int64_t N) { return N <= kWarpRows ? 32 : 8; }

struct FwdArrays {
  int32_t *sid, *entries;
  uint16_t *slot, *off;
  float *z;
  unsigned int *range;
};
FwdArrays take_fwd(Carver &c, int64_t N, int32_t V, int32_t K) {
  const size_t nk = size_t(N) * size_t(K), tiles = (size_t(V) + kTopTile - 1) / kTopTile;
  FwdArrays f;
  f.sid = c.take<int32_t>(nk);
  f.entries = c.take<int32_t>(size_t(N));
  f.slot = c.take<uint16_t>(nk);
  f.off = c.take<uint16_t>(size_t(N) * (tiles + 1));
  f.z = c.take<float>(nk);
  f.range = c.take<unsigned int>(kRangeWords);
  return f;
}
struct BwdArrays {
  uint8_t *mask;
  float *g, *rest, *dz_top, *lost;
  int *extra;
  unsigned int *range;
};
BwdArrays take_bwd(Carver &c, int64_t N, int32_t K) {
  BwdArrays b;
  b.mask = c.take<uint8_t>(size_t(N + kExtraRows));
  b.g = c.take<float>(size_t(N + kExtraRows));
  b.rest = c.take<float>(size_t(N + kExtraRows));
  b.lost = c.take<float>(size_t(N < kExtraMost ? N : kExtraMost));
  b.extra = c.take<int>(kExtraRows);
  b.dz_top = c.take<float>(size_t(N) * size_t(K));
  b.range = c.take<unsigned int>(kRangeWords);
  return b;
}

}  // namespace

sao_status patch_top_bf16(const TopGrad &t, const int *idx, const int *count, int64_t rows, bool few, int v0, int vc,
                          __nv_bfloat16 *dz, int64_t ldz, cudaStream_t s) {
  if (few) return patch<kFewPieces>(t, idx, count, rows, v0, vc, dz, ldz, 0, nullptr, s);
  return patch<kOnePiece>(t, idx, count, rows, v0, vc, dz, ldz, 0, nullptr, s);
}
sao_status patch_top_f32(const TopGrad &t, const int *idx, const int *count, int64_t rows, int v0, int vc,
                         __nv_bfloat16 *dz, int64_t ldz, int64_t plane, unsigned int *range, cudaStream_t s) {
  return patch<kThreePlanes>(t, idx, count, rows, v0, vc, dz, ldz, plane, range, s);
}

sao_status distill_few_rows(const uint8_t *mask, int64_t N, const __nv_bfloat16 *H, int32_t h, CompactRows *out,
                            Carver &c, cudaStream_t s) {
  out->idx = c.take<int>(2 * kFewRows);
  out->pos = c.take<int>(kFewRows);
  out->count = c.take<int>(1);
  out->Hc = c.take<__nv_bfloat16>(size_t(2 * kFewRows) * size_t(h));
  out->cap = 2 * kFewRows;
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for row compaction");
  int slot = launch_begin("distill_few_rows", s);
  pdl(distill_few_rows_kernel, 2 * kFewRows, 128, 0, s)(mask, int(N), H, h, out->idx, out->pos, out->count, out->Hc);
  return launch_end(slot, s);
}

sao_status distill_few_dH(const float *acc, const DhParts &parts, int32_t h, const int *pos, const int *count,
                          int64_t N, __nv_bfloat16 *dH, cudaStream_t s) {
  int slot = launch_begin("distill_few_dH", s);
  pdl(distill_few_dH_kernel, unsigned((N * h + 255) / 256), 256, 0, s)(acc, parts, h, pos, count, N, dH);
  return launch_end(slot, s);
}

sao_status distill_fold_extra(const TopGrad &t, float *acc, const DhParts &parts, int32_t h, const int *pos,
                              const int *count, cudaStream_t s) {
  int slot = launch_begin("distill_fold", s);
  const dim3 grid(unsigned(kExtraRows), unsigned((h + 1023) / 1024), parts.cap_rows ? 8u : 1u);
  pdl(distill_fold_kernel, grid, 256, 0, s)(t, acc, parts, h, pos, count);
  return launch_end(slot, s);
}

sao_status distill_finish(const TopRef &top, const TopFinish &f, const float2 *part, int nvt, const int *pos,
                          int64_t N, cudaStream_t s) {
  const int sub = row_threads(N);
  int slot = launch_begin("distill_finish", s);
  pdl(sub == 32 ? distill_finish_kernel<32> : distill_finish_kernel<8>, unsigned((N * sub + 255) / 256), 256, 0, s)(
      top, f, part, nvt, pos, N);
  return launch_end(slot, s);
}

size_t distill_ws_bytes(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt) {
  if (N <= 0) return 0;
  Carver f(nullptr, ~size_t(0)), b(nullptr, ~size_t(0));
  take_fwd(f, N, V, K);
  take_bwd(b, N, K);
  const bool rows = gemv_takes(N, h, dt);
  const size_t head_f = rows             ? gemv_fwd_bytes(N, V)
                        : dt == SAO_BF16 ? tc_distill_fwd_bytes(N, h, V)
                                         : f32_ws_bytes(N, h, V);
  const size_t head_b = rows             ? gemv_bwd_bytes(N, h, V)
                        : dt == SAO_BF16 ? tc_distill_bwd_bytes(N, h, V)
                                         : f32_ws_bytes(N, h, V);
  return f.off + head_f > b.off + head_b ? f.off + head_f : b.off + head_b;
}

size_t distill_ws_most(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt) {
  if (N <= 0) return 0;
  Carver f(nullptr, ~size_t(0)), b(nullptr, ~size_t(0));
  take_fwd(f, N, V, K);
  take_bwd(b, N, K);
  const int64_t few = gemv_rows(h, dt), n = N < few ? N : few;
  size_t head_f = n > 0 ? gemv_fwd_bytes(n, V) : 0, head_b = n > 0 ? gemv_bwd_bytes(n, h, V) : 0;
  if (N > few) {
    const size_t more_f = dt == SAO_BF16 ? tc_distill_fwd_bytes(N, h, V) : f32_ws_most(N, h, V);
    const size_t more_b = dt == SAO_BF16 ? tc_distill_bwd_most(N, h, V) : f32_ws_most(N, h, V);
    head_f = more_f > head_f ? more_f : head_f;
    head_b = more_b > head_b ? more_b : head_b;
  }
  return f.off + head_f > b.off + head_b ? f.off + head_f : b.off + head_b;
}

sao_status distill_fwd_launch(const void *H, const void *W, sao_dtype dt, const int32_t *ids, const void *a,
                              sao_dtype adt, const float *teacher_lse, const uint8_t *row_mask, int64_t N, int32_t h,
                              int32_t V, int32_t K, float temperature, float *loss, float *lse, float *lse_rest,
                              float *z_top, unsigned int *err, void *ws, size_t ws_bytes, cudaStream_t s) {
  Carver c(ws, ws_bytes);
  const FwdArrays w = take_fwd(c, N, V, K);
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the distillation forward");
  const int tiles = (V + kTopTile - 1) / kTopTile;
  int kp = 32;
  while (kp < K) kp <<= 1;
  int slot = launch_begin("distill_sort", s);
  pdl(distill_sort_kernel, unsigned((N + kSortWarps - 1) / kSortWarps), 32 * kSortWarps,
      size_t(kSortWarps) * kp * sizeof(uint64_t), s)(ids, row_mask, N, K, kp, V, tiles, w.sid, w.slot, w.off,
                                                     w.entries, w.range, err);
  SAO_TRY(launch_end(slot, s));
  const TopRef top{w.sid, w.off, w.z, K, tiles, 1.f / temperature, w.range};
  const TopFinish f{a, adt, teacher_lse, w.slot, w.entries, row_mask, loss, lse, lse_rest, z_top, V};
  if (gemv_takes(N, h, dt)) return gemv_distill_fwd(H, W, dt, row_mask, N, h, V, top, f, c, s);
  if (dt == SAO_BF16) return tc_distill_fwd(H, W, row_mask, N, h, V, top, f, err, c, s);
  return f32_distill_fwd(static_cast<const float *>(H), static_cast<const float *>(W), row_mask, N, h, V, top, f, err,
                         c, s);
}

sao_status distill_bwd_launch(const void *H, const void *W, sao_dtype dt, const int32_t *ids, const void *a,
                              sao_dtype adt, const float *teacher_lse, const float *lse, const float *lse_rest,
                              const float *z_top, const float *grad, int64_t N, int32_t h, int32_t V, int32_t K,
                              float temperature, void *dH, void *dW, sao_dtype dw_dt, int accumulate,
                              unsigned int *err, void *ws, size_t ws_bytes, cudaStream_t s) {
  Carver c(ws, ws_bytes);
  const BwdArrays w = take_bwd(c, N, K);
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the distillation backward");
  const float inv_t = 1.f / temperature;
  const int sub = row_threads(N);
  const bool extra = dt == SAO_BF16 && extra_rows(N);
  int slot = launch_begin("distill_rows", s);
  pdl(sub == 32 ? distill_rows_kernel<32> : distill_rows_kernel<8>, unsigned((N * sub + 255) / 256), 256, 0, s)(
      ids, a, adt, teacher_lse, lse, lse_rest, z_top, grad, N, K, inv_t, w.mask, w.g, w.rest, w.dz_top, w.range,
      extra ? w.lost : nullptr);
  SAO_TRY(launch_end(slot, s));
  if (extra) {
    slot = launch_begin("distill_extra", s);
    pdl(distill_extra_kernel, 1, 1024, 0, s)(w.lost, int(N), w.extra);
    SAO_TRY(launch_end(slot, s));
  }
  const TopGrad t{w.mask, w.g, w.rest, w.dz_top, ids, K, inv_t, w.range, extra ? w.extra : nullptr, N};
  if (gemv_takes(N, h, dt))
    return gemv_distill_bwd(H, W, dt, t, N, h, V, dH, dW, dw_dt, accumulate, c, s);
  if (dt == SAO_BF16) return tc_distill_bwd(H, W, t, N, h, V, dH, dW, dw_dt, accumulate, err, c, s);
  return f32_distill_bwd(static_cast<const float *>(H), static_cast<const float *>(W), t, N, h, V,
                         static_cast<float *>(dH), static_cast<float *>(dW), accumulate, err, c, s);
}

}  // namespace sao
