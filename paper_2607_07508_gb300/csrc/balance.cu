// Load-balance loss of a mixture of experts, with per-expert counts and gradients.
//
// Scores of token t: s_te = softmax(x_t)_e, or sigmoid(x_te) / sum_j sigmoid(x_tj). Over
// the n counted rows of a segment (the batch, or one packed trajectory), with k experts
// chosen per token:
//   c_e = how often e was chosen, P_e = sum_t s_te
//   loss = E / (k n^2) sum_e c_e P_e                (1 when both are even)
// and the mean of it over the segments that have a counted row. c is not
// differentiated, so with w_e = g E c_e / (k n^2 segments):
//   d x_te = s_te (w_e - sum_j s_tj w_j)            (sigmoid: times 1 - sigmoid(x_te))
//
// Rows are cut into chunks of equal size whatever the trajectories. A chunk writes one
// partial for each segment that it meets, at slot chunk + segment (along the batch
// either number grows, so the slots differ), and a segment's partials are added in the
// order of its chunks: no atomics on floating-point sums, the same bits every time.
#include <cuda_bf16.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "balance.cuh"
#include "per_device.h"
#include "sao_common.cuh"
#include "sao_internal.h"
#include "tc_ptx.cuh"

namespace sao {
namespace {

// A lane takes kC columns of a row, in loads of kVec columns (16 bytes, or one column).
// Rows on their way lie in shared memory (asynchronous copies), for single columns in registers
// (fp32 98,301 x 63 in 96 trajectories, forward / backward: 18 / 16 us, by copies of 4 bytes
// 20 / 25; 200,000 x 21 15 / 14, 19 / 33. Copying a warp's rows as one span of 16-byte pieces
// and picking the columns out of it took 20 / 22 and 18 / 20.)
template <int kVec>
constexpr bool kAsync = kVec > 1;
// Threads of a CTA, one to an SM: as many as the registers for the columns' scores and
// sums, and for the words that stay in them, allow. One CTA, not several: its partials are a
// launch's whole scratch, and the reduction reads them all.
constexpr int threads_of(bool async, int columns) {
  const int n = 65536 / ((async ? 2 : 4) * columns + 56) / 64 * 64;
  return n > 1024 ? 1024 : n;
}
template <class T, int kVec, int kC>
constexpr int kThreads = threads_of(kAsync<kVec>, kC);
// Rows that a thread has on their way.
constexpr int depth_of(bool async, int size, int columns) {
  const int n = (112 << 10) / (threads_of(async, columns) * columns * size);
  return !async ? 2 : n < 2 ? 2 : n > 6 ? 6 : n;
}
template <class T, int kVec, int kC>
constexpr int kDepthOf = depth_of(kAsync<kVec>, int(sizeof(T)), kC);
// Bytes of a thread's slots, and of its expert ids' (kIds a row).
constexpr int kIds = 2;
template <class T, int kVec, int kC>
constexpr int kRing = kAsync<kVec> ? kC * int(sizeof(T)) * kDepthOf<T, kVec, kC> : 0;
template <class T, int kVec, int kC>
constexpr int kIdRing = kIds * 4 * kDepthOf<T, kVec, kC>;

constexpr float kLog2e = 1.4426950408889634f;

struct BalanceArgs {
  const void *x;
  const int32_t *ids;
  const uint8_t *mask;   // or null
  const int32_t *cu;     // or null: one segment
  int B;
  int64_t N;
  int E, k;
  int chunk;             // rows per chunk
  int chunks;
  unsigned int *err;
};

// Segment b's first row and the row after its last, inside [0, N] whatever cu holds.
__device__ __forceinline__ int64_t seg_at(const BalanceArgs &a, int b) {
  if (a.cu == nullptr) return b == 0 ? 0 : a.N;
  const int64_t v = ld(a.cu + b);
  return v < 0 ? 0 : v > a.N ? a.N : v;
}
// The segment that holds row r, the last one that starts at or before it (whole warps; 32
// starts a round, where a search by halves would wait for memory five times).
__device__ __forceinline__ int seg_of(const BalanceArgs &a, int64_t r) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  for (int n = a.B; n > 1;) {  // it is one of lo .. lo + n - 1
    const int stride = (n + 31) / 32, at = lane * stride;
    const unsigned after = ~__ballot_sync(0xffffffffu, at < n && (at == 0 || seg_at(a, lo + at) <= r));
    const int k = after == 0u ? 31 : __ffs(after) - 2;  // the last lane of the leading ones that start before
    lo += k * stride;
    n = n - k * stride < stride ? n - k * stride : stride;
  }
  return lo;
}

// A row's words in one lane: load v is columns (l + v lanes) kVec .. + kVec.
template <class T, int kVec, int kC>
struct Row {
  static constexpr int kLoads = kC / kVec;
  static constexpr int kWords = kVec == 1 ? kLoads : kLoads * 4;
  uint32_t raw[kWords];
  __device__ __forceinline__ float at(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
    if constexpr (kVec == 1) return __uint_as_float(raw[j] << 16);
    return __uint_as_float(j & 1 ? raw[j / 2] & 0xffff0000u : raw[j / 2] << 16);
  }
  static __device__ __forceinline__ int column(int j, int l, int lanes) {
    return (l + j / kVec * lanes) * kVec + j % kVec;
  }
  static __device__ __forceinline__ void store(T *row, const float (&v)[kC], int E, int l, int lanes) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int c = (l + k * lanes) * kVec;
      if (c >= E) continue;
      if constexpr (kVec == 1) {
        if constexpr (sizeof(T) == 2)
          row[c] = __float2bfloat16_rn(v[k]);
        else
          row[c] = v[k];
      } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(row + c) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * k + 2 * i], v[8 * k + 2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
};

// The rows of a warp: first, first + step, ... (of its first lane group) below end.
struct Rows {
  int64_t first, end;
  int step;
};
// Of [r0, r1) within a CTA.
__device__ __forceinline__ Rows cta_rows(int64_t r0, int64_t r1, int warp, int warps, int groups) {
  return Rows{r0 + warp * groups, r1, warps * groups};
}
// Of the whole batch, the CTAs side by side: spans of masked rows fall on all of them (a
// contiguous part each left SMs idle for a sixth of the time).
__device__ __forceinline__ Rows grid_rows(const BalanceArgs &a, int warp, int warps, int groups) {
  return Rows{(int64_t(warp) * gridDim.x + blockIdx.x) * groups, a.N, warps * groups * int(gridDim.x)};
}

// 4 or 16 bytes into shared memory, asynchronously.
template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// The rows first, first + step, ... that a group of lanes goes through, those ahead
// already on their way into slots of the thread's own (no barrier). The words of rows that
// are not counted are anything (but for the first few rows they are not read), and
// columns past E read as -inf: they have no score. What a row needs is asked for kDepth rows
// before, its expert ids too, and the mask 32 rows at a time: with one row ahead, or a byte of the
// mask read per row, the kernels waited for memory half of their time (2^20 x 160 bf16 forward
// 93-128 us).
template <class T, int kVec, int kC>
struct Stream {
  static constexpr bool kSlots = kAsync<kVec>;
  static constexpr int kDepth = kDepthOf<T, kVec, kC>, kLoads = kC / kVec;
  static constexpr int kBytes = kVec * int(sizeof(T));
  // from a load's slots to the next one's
  __device__ __forceinline__ uint32_t pitch() const { return blockDim.x * uint32_t(kBytes); }
  const T *src;         // this lane's first column of the row kDepth steps ahead
  const int32_t *ids;   // this lane's first id of that row, or null
  const uint8_t *mask;  // of the warp's first row 64 steps after the last refill, or null
  int64_t src_step, ids_step;
  int left;             // rows from the warp's first row of this step to the end
  int step, k, l, lanes, cur = 0, seen = 0;
  int loads;            // this lane's loads that are in the row
  uint64_t on_bits;     // bit d: the row d steps ahead is counted
  uint32_t slots, id_slots;  // shared-memory addresses of this thread's first ones
  Row<T, kVec, kC> reg[kSlots ? 1 : kDepth];

  // Bit i of the result: this group's row i steps on is counted, `from` the warp's first row.
  // (Several groups' bytes asked for before the first is waited for saved 0.3 us of a short
  // launch, but took registers: 2^20 x 160 bf16 backward 113 -> 127 us.)
  __device__ __forceinline__ uint32_t counted32(const uint8_t *from, int rows) const {
    const int groups = 32 / lanes, lane = threadIdx.x & 31, mine = lane / lanes;
    uint32_t bits = 0;
    for (int g = 0; g < groups; ++g) {
      const int64_t at = int64_t(lane) * step + g;
      const uint32_t b = __ballot_sync(0xffffffffu, at < rows && (from == nullptr || ld(from + at) != 0));
      if (g == mine) bits = b;
    }
    return bits;
  }
  // Rows left after `steps` more (0 or less: none).
  __device__ __forceinline__ int past(int steps) const {
    const int64_t n = left - int64_t(steps) * step;
    return n > 0 ? int(n) : 0;
  }
  __device__ __forceinline__ void fetch(int slot, bool live) {
    if (live) {
      if constexpr (kSlots) {
        const uint32_t dst = slots + uint32_t(slot * kLoads) * pitch();
#pragma unroll
        for (int v = 0; v < kLoads; ++v)
          if (v < loads) copy_async<kBytes>(dst + v * pitch(), src + v * lanes * kVec);
      }
      if (ids) {
#pragma unroll
        for (int i = 0; i < kIds; ++i)
          if (l + i * lanes < k)
            copy_async<4>(id_slots + uint32_t(slot * kIds + i) * (blockDim.x * 4u), ids + i * lanes);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if constexpr (!kSlots) {
      using Word = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
      constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80u;  // -inf
#pragma unroll
      for (int v = 0; v < kLoads; ++v) {
        uint32_t w = none;
        if (live && v < loads) w = ld(reinterpret_cast<const Word *>(src) + v * lanes);
        reg[kDepth - 1].raw[v] = w;
      }
    }
  }
  // `lane_ids`: expert ids [N, k], or null.
  __device__ __forceinline__ Stream(const BalanceArgs &a, const Rows &rows, int lane, int group,
                                    const int32_t *lane_ids, const void *ring, const void *id_ring)
      : left(int(rows.end > rows.first ? rows.end - rows.first : 0)), step(rows.step), k(a.k), l(lane),
        lanes(group), loads((a.E / kVec - lane + group - 1) / group) {
    const int64_t warp_first = rows.first, first = warp_first + (threadIdx.x & 31) / group;
    src = static_cast<const T *>(a.x) + first * a.E + lane * kVec;
    src_step = int64_t(step) * a.E;
    ids_step = int64_t(step) * a.k;
    ids = lane_ids ? lane_ids + first * a.k + lane : nullptr;
    id_slots = tc::smem_u32(id_ring) + threadIdx.x * 4u;
    slots = 0;
    if constexpr (kSlots) {
      slots = tc::smem_u32(ring) + threadIdx.x * uint32_t(kBytes);
      constexpr uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
      for (int v = 0; v < kLoads; ++v)
        if (v >= loads)
          for (int d = 0; d < kDepth; ++d)
#pragma unroll
            for (int w = 0; w < kBytes; w += 4)
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(slots + uint32_t(d * kLoads + v) * pitch() + w), "r"(none)
                           : "memory");
    }
    // the first rows, counted or not: the mask is on its way as well
    const int mine = (threadIdx.x & 31) / group;
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if constexpr (!kSlots)
        if (d > 0) reg[d - 1] = reg[kDepth - 1];
      fetch(d, mine < past(d));
      src += src_step;
      if (ids) ids += ids_step;
    }
    mask = a.mask ? a.mask + warp_first : nullptr;
    on_bits = counted32(mask, left) |
              uint64_t(counted32(mask ? mask + 32 * int64_t(step) : nullptr, past(32))) << 32;
    if (mask) mask += 64 * int64_t(step);
  }
  __device__ __forceinline__ bool on() const { return on_bits & 1u; }
  __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory"); }
  // This row's words (again, until advance()).
  __device__ __forceinline__ Row<T, kVec, kC> row() const {
    if constexpr (kSlots) {
      Row<T, kVec, kC> x;
      const uint32_t at = slots + uint32_t(cur * kLoads) * pitch();
#pragma unroll
      for (int v = 0; v < kLoads; ++v) {
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(x.raw[4 * v]), "=r"(x.raw[4 * v + 1]), "=r"(x.raw[4 * v + 2]), "=r"(x.raw[4 * v + 3])
                     : "r"(at + v * pitch())
                     : "memory");
      }
      return x;
    } else {
      return reg[0];
    }
  }
  // Expert id l + i lanes of this row (i < kIds; below k only).
  __device__ __forceinline__ int id(int i) const {
    int v;
    asm volatile("ld.shared.b32 %0, [%1];"
                 : "=r"(v)
                 : "r"(id_slots + uint32_t(cur * kIds + i) * (blockDim.x * 4u))
                 : "memory");
    return v;
  }
  // To the next row; the words and ids of this one have been used.
  __device__ __forceinline__ void advance() {
    if constexpr (!kSlots) {
#pragma unroll
      for (int d = 1; d < kDepth; ++d) reg[d - 1] = reg[d];
    }
    fetch(cur, on_bits >> kDepth & 1u);
    src += src_step;
    if (ids) ids += ids_step;
    on_bits >>= 1;
    left = left > step ? left - step : 0;
    if (++cur == kDepth) cur = 0;
    if (++seen == 32) {
      seen = 0;
      on_bits |= uint64_t(counted32(mask, past(32))) << 32;
      if (mask) mask += 32 * int64_t(step);
    }
  }
};

__device__ __forceinline__ float lanes_max(float v, int lanes) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < lanes) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
    if (o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// q = e^(x - m), or e^-m sigmoid(x) = 1 / (e^m + e^(m - x)), and their sum over the row.
// kShift: m is given; else it is 0. (The difference is taken before it is scaled, so an
// exponent is off by 2^-24 of itself.) With `w` (sigmoids' backward): dot = sum q w too, and q
// becomes q (1 - sigmoid(x)), the last factor as e^(m - x) q: from a q near 1 the difference
// has no digits (5e-4 of it lost at x = 10, all at 17).
template <bool kSigmoid, bool kShift, class R, int kC>
__device__ __forceinline__ float scores(const R &x, float (&q)[kC], int lanes, float m, float em, const float *w,
                                        float *dot) {
  constexpr float kScale = kSigmoid ? -kLog2e : kLog2e;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kC; ++j) {
    const float v = x.at(j);
    const float p = tc::ex2_approx((kShift ? v - m : v) * kScale);
    q[j] = kSigmoid ? rcp_approx(em + p) : p;
    s[j & 3] += q[j];
    if (kSigmoid && w) {
      d[j & 3] = fmaf(q[j], w[j], d[j & 3]);
      q[j] *= fminf(p, FLT_MAX) * q[j];  // (p of infinity: q = 0)
    }
  }
  if (kSigmoid && w) *dot = lanes_sum((d[0] + d[1]) + (d[2] + d[3]), lanes);
  return lanes_sum((s[0] + s[1]) + (s[2] + s[3]), lanes);
}

// A row's scores q, up to a factor that the normalisation takes out, and 1 / their sum
// (0 for a row of -inf alone, which has no probabilities). Rows whose sum without a
// shift is near 1 need none: their largest logit is
// within 12 of 0, so exponents lose no more than with the largest subtracted. The
// search for it and its exchanges between lanes were a third of the instructions, and
// those bound the kernels. A warp with another row takes m = the largest logit, for sigmoids
// only where it is below 0 (the sigmoids themselves would vanish with it). w, dot: see scores().
template <bool kSigmoid, class S, int kC>
__device__ __forceinline__ float row_scores(const S &stream, float (&q)[kC], const float *w = nullptr,
                                            float *dot = nullptr) {
  const int lanes = stream.lanes;
  float s = scores<kSigmoid, false>(stream.row(), q, lanes, 0.f, 1.f, w, dot);
  const bool fine = kSigmoid ? s > 0x1p-10f : s > 0x1p-10f && s < 0x1p17f;
  if (!__all_sync(0xffffffffu, fine || !stream.on())) {
    const auto x = stream.row();
    float m = x.at(0), em = 1.f;
#pragma unroll
    for (int j = 1; j < kC; ++j) m = fmaxf(m, x.at(j));
    m = lanes_max(m, lanes);
    if (m == -INFINITY) m = 0.f;
    if constexpr (kSigmoid) {
      m = fminf(m, 0.f);
      em = tc::ex2_approx(m * kLog2e);
    }
    s = scores<kSigmoid, true>(x, q, lanes, m, em, w, dot);
  }
  return s == 0.f ? 0.f : rcp_approx(s);
}

// Runs f(segment, first row, row after the last) for the segments of chunk c (all threads).
template <class F>
__device__ __forceinline__ void for_segments(const BalanceArgs &a, int c, F f) {
  if (a.cu == nullptr) {
    f(0, 0, a.N);
    return;
  }
  int64_t r = int64_t(c) * a.chunk;
  const int64_t end = r + a.chunk < a.N ? r + a.chunk : a.N;
  for (int b = seg_of(a, r); b < a.B && r < end; ++b) {
    int64_t e = seg_at(a, b + 1);
    e = e < end ? e : end;
    if (e <= r) continue;
    f(b, r, e);
    r = e;
  }
}

// Where one cluster's forward writes its results; loss null: partials for the reduction.
struct BalanceOut {
  float *loss, *prob_sums;
  int64_t *counts, *rows;
};

constexpr int kCluster = 8;
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same shared variable in the CTA of cluster rank `rank`.
template <class T>
__device__ __forceinline__ T *peer_shared(T *p, unsigned rank) {
  uint64_t out;
  asm("mapa.u64 %0, %1, %2;" : "=l"(out) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<T *>(out);
}

// The end of a forward by one cluster (kCluster CTAs, the whole batch): each CTA has its sums
// and counts of every column, and its rows; CTA r adds those of columns r, r + 8, ...
__device__ __forceinline__ void cluster_finish(const BalanceArgs &a, const BalanceOut &o, float *sums, int *counts,
                                               int n) {
  __shared__ int my_rows;
  __shared__ float my_term, warp_term[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) my_rows = n;
  cluster_barrier();
  const int nr = __reduce_add_sync(0xffffffffu, lane < kCluster ? *peer_shared(&my_rows, lane) : 0);
  const float f = nr > 0 ? float(a.E) / (float(a.k) * float(nr)) / float(nr) : 0.f;
  float term = 0.f;
  for (int e = int(blockIdx.x) + kCluster * int(threadIdx.x); e < a.E; e += kCluster * int(blockDim.x)) {
    float ps[kCluster];
    int pc[kCluster];
#pragma unroll
    for (int p = 0; p < kCluster; ++p) {
      ps[p] = *peer_shared(sums + e, p);
      pc[p] = *peer_shared(counts + e, p);
    }
    float v = 0.f;
    int64_t c = 0;
#pragma unroll
    for (int p = 0; p < kCluster; ++p) {
      v += ps[p];
      c += pc[p];
    }
    o.prob_sums[e] = v;
    o.counts[e] = c;
    term += v * (float(c) * f);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) term += __shfl_xor_sync(0xffffffffu, term, d);
  if (lane == 0) warp_term[warp] = term;
  __syncthreads();
  if (threadIdx.x == 0) {
    term = 0.f;
    for (int w = 0; w < int(blockDim.x >> 5); ++w) term += warp_term[w];
    my_term = term;
  }
  cluster_barrier();
  if (blockIdx.x == 0 && warp == 0) {
    term = lane < kCluster ? *peer_shared(&my_term, lane) : 0.f;
#pragma unroll
    for (int d = kCluster / 2; d > 0; d >>= 1) term += __shfl_xor_sync(0xffffffffu, term, d);
    if (lane == 0) {
      o.loss[0] = term;
      o.rows[0] = nr;
    }
  }
  cluster_barrier();  // no CTA leaves while its shared memory may still be read
}

// Each group of `lanes` lanes takes a row at a time, the next ones' logits in flight, and
// keeps the sums of its columns in registers. One pass over the logits. 2^20 x 160 bf16:
// (a quarter masked) 94 us, 3.0 TB/s, bound by instructions (2.7 a cycle and SM);
// 2^20 x 128 fp32: 92 us, 5.8 TB/s.
template <class T, int kVec, int kC, bool kSigmoid>
__global__ void __launch_bounds__(kThreads<T, kVec, kC>)
    balance_partial_kernel(const BalanceArgs a, int lanes, const BalanceOut out, float *psum, int *pcount, int *prows,
                           unsigned int *ticket) {
  extern __shared__ uint4 smem[];  // the stream's slots, ids', sums [warps][E], counts [E]
  __shared__ int n_rows[32];
  const int block = blockDim.x, warps = block >> 5;
  grid_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  const uint4 *id_ring = smem + block * kRing<T, kVec, kC> / 16;
  float *sums = reinterpret_cast<float *>(const_cast<uint4 *>(id_ring) + block * kIdRing<T, kVec, kC> / 16);
  int *counts = reinterpret_cast<int *>(sums + warps * a.E);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int groups = 32 / lanes, l = lane & (lanes - 1);
  for_segments(a, blockIdx.x, [&](int b, int64_t r0, int64_t r1) {
    for (int e = threadIdx.x; e < a.E; e += block) counts[e] = 0;
    __syncthreads();
    float acc[kC];
#pragma unroll
    for (int j = 0; j < kC; ++j) acc[j] = 0.f;
    int n = 0;
    auto count = [&](int id) {
      if (unsigned(id) < unsigned(a.E))
        atomicAdd(counts + id, 1);
      else if (id >= 0)
        raise_device_error(a.err, SAO_DEVERR_EXPERT_ID);
    };
    const Rows rows = a.cu ? cta_rows(r0, r1, warp, warps, groups) : grid_rows(a, warp, warps, groups);
    Stream<T, kVec, kC> x(a, rows, l, lanes, a.ids, smem, id_ring);
    for (int64_t r = rows.first + lane / lanes; x.left > 0; r += rows.step) {  // the warp's lanes stay together
      x.wait();
      const bool on = x.on();
      if (__any_sync(0xffffffffu, on)) {  // (not in spans of masked rows)
        float q[kC];
        const float inv = row_scores<kSigmoid>(x, q);
        if (on) {
          if (l == 0) ++n;
#pragma unroll
          for (int i = 0; i < kIds; ++i)
            if (l + i * lanes < a.k) count(x.id(i));
          for (int j = l + kIds * lanes; j < a.k; j += lanes) count(ld(a.ids + r * a.k + j));
#pragma unroll
          for (int j = 0; j < kC; ++j) acc[j] = fmaf(q[j], inv, acc[j]);
        }
        __syncwarp();
      }
      x.advance();
    }
    for (int o = lanes; o < 32; o <<= 1) {  // the warp's groups
#pragma unroll
      for (int j = 0; j < kC; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
    }
    if (lane < lanes) {
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        const int c = Row<T, kVec, kC>::column(j, l, lanes);
        if (c < a.E) sums[warp * a.E + c] = acc[j];
      }
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) n_rows[warp] = n;
    __syncthreads();
    const int64_t slot = int64_t(blockIdx.x) + b;
    for (int e = threadIdx.x; e < a.E; e += block) {
      float v = 0.f;
#pragma unroll 4
      for (int w = 0; w < warps; ++w) v += sums[w * a.E + e];
      if (out.loss) {
        sums[e] = v;
      } else {
        psum[slot * a.E + e] = v;
        pcount[slot * a.E + e] = counts[e];
      }
    }
    int t = 0;
    if (threadIdx.x == 0)
      for (int w = 0; w < warps; ++w) t += n_rows[w];
    if (out.loss) {
      cluster_finish(a, out, sums, counts, t);
      return;
    }
    if (threadIdx.x == 0) prows[slot] = t;
    __syncthreads();
  });
}

// CTA (b, 32 columns): adds the segment's partials, kSlices warps side by side; the
// CTAs of a batch of up to 256 experts are one cluster, whose first CTA adds their products
// (2 us less than by the ticket); else the last CTA adds those of all. Bound by latency: a batch's
// 152 partials are asked for at once (in three rounds a forward of 65,536 x 128 was 1 us longer). (The
// sums are of positive numbers, in a fixed order, in fp32; fp64, on which GB300 has few units,
// took longer than the loads.)
template <int kSlices>
__global__ void __launch_bounds__(32 * kSlices)
    balance_reduce_kernel(const BalanceArgs a, int cols, bool cluster, const float *psum, const int *pcount,
                          const int *prows, float *loss, int64_t *counts, float *prob_sums, int64_t *rows, float *terms,
                          unsigned int *ticket) {
  __shared__ float sh_sum[kSlices][32], sh_term[kSlices];
  __shared__ long long sh_count[kSlices][32], sh_rows[kSlices];
  __shared__ int sh_used[kSlices];
  __shared__ bool last;
  __shared__ float my_term;
  grid_wait();
  const int b = blockIdx.x / cols, g = blockIdx.x % cols;
  const int slice = threadIdx.x >> 5, lane = threadIdx.x & 31, e = g * 32 + lane;
  const int64_t r0 = seg_at(a, b), r1 = seg_at(a, b + 1);
  float s = 0.f;
  long long n = 0, nr = 0;
  if (r1 > r0) {
    const int c0 = int(r0 / a.chunk), c1 = int((r1 - 1) / a.chunk);
    constexpr int kU = 10;  // partials in flight
    for (int c = c0 + slice; c <= c1; c += kU * kSlices) {
      float ps[kU];
      int pn[kU], pr[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t slot = int64_t(c) + u * kSlices + b;
        const bool in = c + u * kSlices <= c1;
        ps[u] = in && e < a.E ? ld(psum + slot * a.E + e) : 0.f;
        pn[u] = in && e < a.E ? ld(pcount + slot * a.E + e) : 0;
        pr[u] = in ? ld(prows + slot) : 0;
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        s += ps[u];
        n += pn[u];
        nr += pr[u];
      }
    }
  }
  sh_sum[slice][lane] = s;
  sh_count[slice][lane] = n;
  if (lane == 0) sh_rows[slice] = nr;
  __syncthreads();
  if (slice == 0) {
    s = 0.f;
    n = nr = 0;
#pragma unroll
    for (int k = 0; k < kSlices; ++k) {
      s += sh_sum[k][lane];
      n += sh_count[k][lane];
      nr += sh_rows[k];
    }
    float term = 0.f;
    if (e < a.E) {
      prob_sums[int64_t(b) * a.E + e] = s;
      counts[int64_t(b) * a.E + e] = n;
      if (nr > 0) term = s * (float(n) * (float(a.E) / (float(a.k) * float(nr))) / float(nr));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xffffffffu, term, o);
    if (lane == 0) {
      if (g == 0) rows[b] = nr;
      // checked mode: cu_seqlens runs from 0 to N and never falls
      if (a.cu && g == 0) {
        const int64_t u = ld(a.cu + b), v = ld(a.cu + b + 1);
        if (u > v || (b == 0 && u != 0) || (b == a.B - 1 && v != a.N)) raise_device_error(a.err, SAO_DEVERR_CU_SEQLENS);
      }
      if (cluster) {
        my_term = term;
      } else {
        terms[blockIdx.x] = term;
        __threadfence();
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
      }
    }
  }
  if (cluster) {
    cluster_barrier();
    if (blockIdx.x == 0 && slice == 0) {
      float t = lane < cols ? *peer_shared(&my_term, lane) : 0.f;
#pragma unroll
      for (int o = kCluster / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
      if (lane == 0) loss[0] = t;
    }
    cluster_barrier();  // no CTA leaves while its shared memory may still be read
    return;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  float t = 0.f;
  int used = 0;
  for (int64_t i = threadIdx.x; i < gridDim.x; i += 32 * kSlices) t += __ldcg(terms + i);
  for (int i = threadIdx.x; i < a.B; i += 32 * kSlices) used += __ldcg(rows + i) > 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  used = __reduce_add_sync(0xffffffffu, used);
  if (lane == 0) {
    sh_term[slice] = t;
    sh_used[slice] = used;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    t = 0.f;
    used = 0;
    for (int k = 0; k < kSlices; ++k) {
      t += sh_term[k];
      used += sh_used[k];
    }
    loss[0] = used ? t / float(used) : 0.f;
  }
}

// A group of `lanes` lanes per row, as in the forward; the segment's weights of its columns
// stay in registers until the segment ends. One pass, bound by reading the logits and
// writing their gradient: 2^20 x 160 bf16 108-115 us, 5.1-5.4 TB/s; 2^20 x 128 fp32 174 us,
// 6.2 TB/s.
template <class T, int kVec, int kC, bool kSigmoid>
__global__ void __launch_bounds__(kThreads<T, kVec, kC>)
    balance_grad_kernel(const BalanceArgs a, int lanes, const int64_t *counts, const int64_t *rows,
                        const float *grad_loss, T *dx) {
  const int block = blockDim.x, warps = block >> 5;
  __shared__ int sh_used[32];
  grid_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  extern __shared__ uint4 smem[];  // the stream's slots
  const int groups = 32 / lanes, l = lane & (lanes - 1);
  const int64_t r0 = int64_t(blockIdx.x) * a.chunk, r1 = r0 + a.chunk < a.N ? r0 + a.chunk : a.N;
  const Rows own = a.cu ? cta_rows(r0, r1, warp, warps, groups) : grid_rows(a, warp, warps, groups);
  Stream<T, kVec, kC> x(a, own, l, lanes, nullptr, smem, smem);
  const float g = ld(grad_loss);
  int used = 1;  // segments with a counted row
  if (a.B > 1) {
    used = 0;
    for (int i = threadIdx.x; i < a.B; i += block) used += ld(rows + i) > 0;
    used = __reduce_add_sync(0xffffffffu, used);
    if (lane == 0) sh_used[warp] = used;
    __syncthreads();
    used = 0;
    for (int i = 0; i < warps; ++i) used += sh_used[i];
  }
  int b = seg_of(a, own.first < a.N ? own.first : a.N - 1);
  int64_t seg_end = -1;  // from this row on the weights are another segment's
  float w[kC];
#pragma unroll
  for (int j = 0; j < kC; ++j) w[j] = 0.f;
  const int64_t first = own.first + lane / lanes;
  T *out = dx + first * a.E;
  const int64_t out_step = int64_t(own.step) * a.E;
  for (int64_t r = first; x.left > 0; r += own.step) {
    const bool on = x.on();
    if (on && r >= seg_end) {
      while (b + 1 < a.B && seg_at(a, b + 1) <= r) ++b;
      seg_end = b + 1 < a.B ? seg_at(a, b + 1) : a.N;
      // weights from the even load on: a constant in all of them has no gradient, and takes digits
      const int64_t counted = ld(rows + b), even = counted * a.k / a.E;
      const float n = float(counted);
      const float f = n > 0.f ? g * float(a.E) / (float(a.k) * n * n * float(used)) : 0.f;
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        const int c = Row<T, kVec, kC>::column(j, l, lanes);
        w[j] = c < a.E ? f * float(ld(counts + int64_t(b) * a.E + c) - even) : 0.f;
      }
    }
    x.wait();
    __syncwarp();
    float q[kC];
    if (__any_sync(0xffffffffu, on)) {
      float dot;  // sum q w
      const float inv = row_scores<kSigmoid>(x, q, w, &dot);
      if constexpr (!kSigmoid) {  // (inside scores() too: 2^20 x 160 bf16 115 -> 126 us)
        float d4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kC; ++j) d4[j & 3] = fmaf(q[j], w[j], d4[j & 3]);
        dot = lanes_sum((d4[0] + d4[1]) + (d4[2] + d4[3]), lanes);
      }
      // q inv (w - d), d = dot inv, with the two factors of the row taken into one multiply-add
      const float nd = -(dot * inv) * inv;
#pragma unroll
      for (int j = 0; j < kC; ++j) q[j] *= fmaf(w[j], inv, nd);
    }
    if (!on) {
#pragma unroll
      for (int j = 0; j < kC; ++j) q[j] = 0.f;
    }
    if (r < own.end) Row<T, kVec, kC>::store(out, q, a.E, l, lanes);
    x.advance();
    out += out_step;
  }
}

// The layout of a row of E: kC columns a lane and the lanes that take it.
struct Layout {
  int columns, lanes;
  bool vec;
};
// Vector loads where every row starts on 16 bytes. Of the layouts the one with the
// fewest instructions: about 5 for each of a lane's columns, 130 for all else that a
// row takes, times the lanes; of 8 to 24 columns (32 or 40, with fewer warps to hide latencies,
// were no faster for 128 to 256 experts) unless only 32 fit, and for single columns,
// whose words stay in registers, of 8 (98,301 x 63 bf16: 44 us against 51 with 16).
Layout layout(const void *x, const void *dx, sao_dtype dt, int E) {
  const int size = dt == SAO_BF16 ? 2 : 4, per = 16 / size;
  Layout best{0, 0, E % per == 0 && aligned16(x) && aligned16(dx)};
  const int vec = best.vec ? per : 1, most = best.vec ? 24 : 8;
  int least = 0;
  for (int c = 8; c <= 32; c += 8) {
    const int loads = c / vec, units = E / vec;
    int lanes = 1;
    while (lanes * loads < units) lanes <<= 1;
    if (lanes > 32) continue;
    const int cost = lanes * (5 * c + 130);
    if (best.columns == 0 || (c <= most && cost < least)) {
      best.columns = c;
      best.lanes = lanes;
      least = cost;
    }
  }
  return best;
}

// f(type, loads, columns, score) with the layout's values as types.
template <int kValue>
using Int = std::integral_constant<int, kValue>;
template <class T, class F>
void with_layout(const Layout &l, int score, F f) {
  auto columns = [&](auto vec, auto sig) {
    switch (l.columns) {
      case 8: return f(T{}, vec, Int<8>{}, sig);
      case 16: return f(T{}, vec, Int<16>{}, sig);
      case 24: return f(T{}, vec, Int<24>{}, sig);
      default: return f(T{}, vec, Int<32>{}, sig);
    }
  };
  auto loads = [&](auto sig) { l.vec ? columns(Int<int(16 / sizeof(T))>{}, sig) : columns(Int<1>{}, sig); };
  score == SAO_SCORE_SIGMOID ? loads(std::true_type{}) : loads(std::false_type{});
}

// CTAs on each of 152 SMs. One for a batch, whose rows they share evenly. Four, of a quarter of the
// threads, where trajectories are balanced by themselves: a CTA that meets the end of
// one adds up its sums twice, and the others of its SM work on (65,536 x 256 in 16
// trajectories 47 -> 42 us, 98,301 x 63 in 96 42 -> 37; a batch of 65,536 x 128 30 -> 37).
int ctas_of(bool segments) { return segments ? 4 : 1; }
// Rows per CTA, at least 64. From N alone: the sums' order does not depend on the device.
constexpr int64_t kLeastChunk = 64;
int chunk_rows(int64_t N, bool segments) {
  const int64_t ctas = 152 * ctas_of(segments), c = (N + ctas - 1) / ctas;
  return int(c < kLeastChunk ? kLeastChunk : c);
}
BalanceArgs make_args(const void *x, const int32_t *ids, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                      int32_t E, int32_t k, unsigned int *err) {
  BalanceArgs a{x, ids, mask, cu, cu ? B : 1, N, E, k, chunk_rows(N, cu != nullptr), 0, err};
  a.chunks = int((N + a.chunk - 1) / a.chunk);
  return a;
}

// Threads of a launch: no more warps than a CTA has rows for. (All of them, and their slots' shared
// memory, made a launch of a few rows 4 us longer.)
int block_of(int most, int chunk, int lanes, bool segments) {
  most = most / ctas_of(segments) / 32 * 32;
  const int groups = 32 / lanes, warps = (chunk + groups - 1) / groups;
  return warps * 32 < most ? warps * 32 : most;
}
constexpr size_t kPlainSmem = 40u << 10;  // dynamic shared memory that any kernel may have

// Small batches by one cluster, in one launch: up to 512 rows, and on to 3,072 while the rows, at the
// cost of 16 columns and their own, are few. Chosen for the GPU alone, as in a captured graph (us, fp32,
// cluster / two launches): 512 x 60 5.3 / 6.9, 512 x 256 8.2 / 8.6, 512 x 1,024 13.3 / 14.2, 640 x 1,024
// 14.6 / 14.2; 3,072 x 8 7.3 / 7.5, 4,096 x 8 8.4 / 8.0; 1,536 x 32 6.8 / 6.7, 2,048 x 32 8.1 / 6.9;
// 1,024 x 60 7.0 / 7.1, 4,096 x 60 10.6 / 7.6; 1,024 x 128 8.2 / 7.5. Called one by one, where another launch is
// 2 us of the host's time, it wins there too (2,304 x 8 7.5 / 9.2), and somewhat beyond (1,024 x 128 8.8 / 9.3).
bool one_cluster(int64_t N, int32_t E) { return N <= 512 || (N <= 3072 && N * (E + 16) <= 72 << 10); }

// Lets the kernel have an SM's shared memory (once per device).
template <auto kKernel>
sao_status allow_smem() {
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  static PerDevice<cudaError_t> set_up;
  const cudaError_t e = set_up.get(
      di.device, [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 << 10); });
  if (e != cudaSuccess) return fail(SAO_ERR_CUDA, "kernel set-up: %s", cudaGetErrorString(e));
  return SAO_OK;
}

// A grid of one cluster, as a programmatic dependent launch.
template <class K, class... A>
void launch_cluster(K kern, int ctas, int block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = unsigned(ctas);
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ctas));
  cfg.blockDim = dim3(unsigned(block));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  cudaLaunchKernelEx(&cfg, kern, args...);
}

struct Scratch {
  float *psum;
  int *pcount, *prows;
  float *terms;
  unsigned int *ticket;
};
Scratch take(Carver &c, int64_t N, int32_t E, int32_t B) {
  // the most chunks that up to N rows make (a batch fewer), so that a call of fewer rows fits too
  const int64_t most = 152 * ctas_of(true), chunks = (N + kLeastChunk - 1) / kLeastChunk;
  const size_t slots = size_t(chunks < most ? chunks : most) + size_t(B);
  Scratch s;
  s.psum = c.take<float>(slots * size_t(E));
  s.pcount = c.take<int>(slots * size_t(E));
  s.prows = c.take<int>(slots);
  s.terms = c.take<float>(size_t(B) * size_t((E + 31) / 32));
  s.ticket = c.take<unsigned int>(1);
  return s;
}

}  // namespace

size_t balance_ws_bytes(int64_t N, int32_t E, int32_t B) {
  Carver c(nullptr, ~size_t(0));
  take(c, N, E, B);
  return c.off;
}

sao_status balance_fwd_launch(const void *x, sao_dtype dt, const int32_t *ids, const uint8_t *mask, const int32_t *cu,
                              int32_t B, int64_t N, int32_t E, int32_t k, int score, float *loss, int64_t *counts,
                              float *prob_sums, int64_t *rows, unsigned int *err, void *ws, size_t ws_bytes,
                              cudaStream_t s) {
  const BalanceArgs a = make_args(x, ids, mask, cu, B, N, E, k, err);
  Carver c(ws, ws_bytes);
  const Scratch w = take(c, N, E, a.B);
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the balance loss");
  const Layout lay = layout(x, x, dt, E);
  const bool one = cu == nullptr && one_cluster(N, E);
  const BalanceOut out = one ? BalanceOut{loss, prob_sums, counts, rows} : BalanceOut{};
  int slot = launch_begin(one ? "balance_cluster" : "balance_partial", s);
  sao_status st = SAO_OK;
  auto partial = [&](auto t, auto vec, auto columns, auto sig) {
    using T = decltype(t);
    auto kern = balance_partial_kernel<T, vec.value, columns.value, sig.value>;
    const int block =
        block_of(kThreads<T, vec.value, columns.value>, one ? int((N + kCluster - 1) / kCluster) : a.chunk, lay.lanes,
                 a.cu != nullptr);
    const size_t smem = size_t(block) * (kRing<T, vec.value, columns.value> + kIdRing<T, vec.value, columns.value>) +
                        size_t(E) * (block / 32 + 1) * sizeof(float);
    if (smem > kPlainSmem) st = allow_smem<balance_partial_kernel<T, vec.value, columns.value, sig.value>>();
    if (st != SAO_OK) return;
    if (one) {
      launch_cluster(kern, kCluster, block, smem, s, a, lay.lanes, out, w.psum, w.pcount, w.prows, w.ticket);
    } else {
      pdl(kern, unsigned(a.chunks), block, smem, s)(a, lay.lanes, out, w.psum, w.pcount, w.prows, w.ticket);
    }
  };
  dt == SAO_BF16 ? with_layout<__nv_bfloat16>(lay, score, partial) : with_layout<float>(lay, score, partial);
  SAO_TRY(st);
  SAO_TRY(launch_end(slot, s));
  if (one) return SAO_OK;
  // a batch's partials, up to 152 in few CTAs: 16 warps to each; many trajectories: 8
  int cols = (E + 31) / 32;
  const bool cluster = cu == nullptr && cols <= kCluster;
  if (cluster)  // a power of two of CTAs: 1, 2, 4 or 8
    while (cols & (cols - 1)) ++cols;
  const unsigned grid = unsigned(a.B) * unsigned(cols);
  slot = launch_begin("balance_reduce", s);
  auto reduce = grid <= 152 ? balance_reduce_kernel<16> : balance_reduce_kernel<8>;
  if (cluster)
    launch_cluster(reduce, cols, 512, 0, s, a, cols, true, w.psum, w.pcount, w.prows, loss, counts, prob_sums, rows,
                   w.terms, w.ticket);
  else
    pdl(reduce, grid, grid <= 152 ? 512 : 256, 0, s)(a, cols, false, w.psum, w.pcount, w.prows, loss, counts, prob_sums,
                                                      rows, w.terms, w.ticket);
  return launch_end(slot, s);
}

sao_status balance_bwd_launch(const void *x, sao_dtype dt, const uint8_t *mask, const int32_t *cu, int32_t B, int64_t N,
                              int32_t E, int32_t k, int score, const int64_t *counts, const int64_t *rows,
                              const float *grad_loss, void *dx, unsigned int *err, cudaStream_t s) {
  const BalanceArgs a = make_args(x, nullptr, mask, cu, B, N, E, k, err);
  const Layout lay = layout(x, dx, dt, E);
  int slot = launch_begin("balance_grad", s);
  sao_status st = SAO_OK;
  auto grad = [&](auto t, auto vec, auto columns, auto sig) {
    using T = decltype(t);
    auto kern = balance_grad_kernel<T, vec.value, columns.value, sig.value>;
    const int block = block_of(kThreads<T, vec.value, columns.value>, a.chunk, lay.lanes, a.cu != nullptr);
    const size_t smem = size_t(block) * kRing<T, vec.value, columns.value>;
    if (smem > kPlainSmem) st = allow_smem<balance_grad_kernel<T, vec.value, columns.value, sig.value>>();
    if (st == SAO_OK)
      pdl(kern, unsigned(a.chunks), block, smem, s)(a, lay.lanes, counts, rows, grad_loss, static_cast<T *>(dx));
  };
  dt == SAO_BF16 ? with_layout<__nv_bfloat16>(lay, score, grad) : with_layout<float>(lay, score, grad);
  SAO_TRY(st);
  return launch_end(slot, s);
}

}  // namespace sao
