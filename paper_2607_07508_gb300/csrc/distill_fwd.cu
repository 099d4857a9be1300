// bf16 forward of the distillation from a teacher's top logits: Z = H W^T / T tile by
// tile on the tensor cores, each tile reduced to (max, sum-exp) over the columns outside
// the row's entries, the entries' logits kept.
//
// The tensor core truncates as it adds to its accumulator. Over a contraction of 2,048
// that moved a logit of 12 by 2.6e-5, always towards zero, and the losses by 2.7e-6 of
// themselves (7.2e-6 at h = 6,144), three to five times what fp32 FMAs lose. So the
// accumulator is emptied every 512 elements of the contraction (up to 128 rows: 128) and the parts are added
// in fp32 registers: a part's accumulator is smaller by the number of parts, and so is
// what truncation takes. Sixteen warps hold a 128x256 tile as 64 sums a thread. Losses
// off by (h = 2,048) and time of 12,288 rows on the moe head, with warps that still polled:
// parts of 256 3.6e-7, 5.83 ms; 512 6.7e-7, 5.68; 1,024 1.3e-6, 5.35; one part 2.7e-6, 5.41
// (fp32 FMAs 9.2e-7).
//
// A row's entries are sorted by id, and off[] counts them by tile, so a thread finds
// those of its 64 columns while the tile's products run. Per tile 128 x 256 x h
// multiply-adds against 128 x 256 exponentials: bound by the tensor cores, and those by
// the power cap: 12,288 rows, K = 1 4.66 ms, 1.64 PFLOP/s (of 1.89 in a burst, 1.69
// sustained); K = 128 5.13 ms, the entries' columns taken out of two thirds of the
// 16-column pieces. 388 rows 202 us, 24,576 rows of h = 1,024, V = 32,000 1.02 ms.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cudaTypedefs.h>
#include <math.h>
#include <stdint.h>

#include "distill.cuh"
#include "logprobs_common.cuh"
#include "per_device.h"
#include "rows.cuh"
#include "sao_common.cuh"
#include "sao_internal.h"
#include "tc_ptx.cuh"

namespace sao {
namespace {

using namespace tc;

constexpr int TM = 128, TN = 256, KB = 64;
static_assert(TN == kTopTile, "offsets count entries by tile");
// Contraction elements between two read-outs of an accumulator. One tile of rows waits for the bytes of
// W, so it is emptied four times as often: 3 to 64 rows of the moe head in the same 113-135
// us, the losses off by 2e-7 instead of 5e-7 to 1e-6. (With two tiles 130 -> 145 us.)
constexpr int kPart = 512, kFewPart = 128;
constexpr int64_t kFewPartRows = 128;
constexpr uint32_t A_BYTES = TM * KB * 2, B_BYTES = TN * KB * 2;
constexpr uint32_t RING_BYTES = 4 * (A_BYTES + B_BYTES);  // 4 stages, or 6 of half a B tile
constexpr int kMaxStages = 6;
constexpr int ACCS = 2;
constexpr uint32_t TMEM_COLS = ACCS * TN;
constexpr int NUM_THREADS = 640;             // warp 0 TMA, warp 1 MMA, warps 4-19 add the parts and finish
constexpr int HN = TN / 4;                   // columns per adding warp: four warps (128 rows) per quarter
constexpr int LAUNCH_REGS = 96, ISSUE_REGS = 40, SUM_REGS = 104;
static_assert(128 * ISSUE_REGS + 512 * SUM_REGS <= NUM_THREADS * LAUNCH_REGS, "split within the launch's registers");
constexpr float kLog2e = 1.4426950408889634f;

struct __align__(8) SmemCtl {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full[ACCS], acc_empty[ACCS];
  uint32_t tmem_base;
  int abort;
  float2 quarter[2][4][TM];  // (max, sum) of each quarter tile's rows, two tiles in turn
};
constexpr size_t SMEM_BYTES = 1024 + RING_BYTES + sizeof(SmemCtl);
static_assert(SMEM_BYTES <= 232448, "shared memory of an SM");

struct FwdParams {
  int nM, nN, nK;      // tiles along M and N, 64-wide K blocks
  int part_blocks;     // K blocks between two read-outs of an accumulator, a power of two
  int group_m;         // tile raster: group_m M tiles per group, M fastest inside
  int64_t rows;        // rows of H, and the stride of part
  int vocab;
  float2 *part;        // [nN][rows]
  const int *m_count;  // compacted rows (null: rows) ...
  const int *row_idx;  // ... and the row each one is
  TopRef top;
  unsigned int *err;
};

__device__ __forceinline__ void tile_of(int L, const FwdParams &p, int nM, int &m, int &n) {
  const int per_group = p.group_m * p.nN;
  const int g = L / per_group;
  const int within = L - g * per_group;
  const int m0 = g * p.group_m;
  const int gm = min(p.group_m, nM - m0);
  m = m0 + within % gm;
  n = within / gm;
}

// kCG = 2: CTA pairs, as in the backward's products (tc_gemm_kernel): every MMA is one of
// M = 256 over the pair, each CTA loads its own 128 rows of H and half of the tile of W,
// and keeps its own 128 rows' sums.
template <int kCG>
__global__ void __launch_bounds__(NUM_THREADS, 1)
    distill_logits_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                          const FwdParams p) {
  constexpr uint32_t kStageBytes = A_BYTES + B_BYTES / kCG;
  constexpr int kStages = int(RING_BYTES / kStageBytes);
  static_assert(kStages <= kMaxStages, "barrier arrays");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  SmemCtl *ctl = reinterpret_cast<SmemCtl *>(smem_raw + (base - raw) + RING_BYTES);
  volatile int *abort = &ctl->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = kCG == 2 ? cluster_ctarank() : 0u;
  const int cl = int(blockIdx.x) / kCG, ncl = int(gridDim.x) / kCG;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int a = 0; a < ACCS; ++a) {
      mbar_init(smem_u32(&ctl->acc_full[a]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[a]), 16 * kCG);
    }
    ctl->abort = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    if constexpr (kCG == 2) {
      tmem_alloc_pair(smem_u32(&ctl->tmem_base), TMEM_COLS);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(&ctl->tmem_base), TMEM_COLS);
      tmem_relinquish();
    }
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
  }
  fence_before_sync();
  __syncthreads();
  // both CTAs' barriers exist before either CTA's copies, commits or arrivals reach them
  if constexpr (kCG == 2) cluster_sync();
  fence_after_sync();
  const uint32_t tmem_base = ctl->tmem_base;
  grid_wait_long();
  int nM = p.nM;
  int64_t rows = p.rows;
  if (p.m_count) {
    rows = *p.m_count;
    nM = int((rows + TM * kCG - 1) / (TM * kCG));
  }
  const int tiles = nM * p.nN;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ISSUE_REGS));
    if (warp == 0 && lane == 0) {
      // ---------------------------------------------------------- TMA producer
      int stage = 0;
      uint32_t phase = 0, issued = 0, issued_phase = 0;
      bool ok = true;
      for (int L = cl; L < tiles && ok; L += ncl) {
        int m, n;
        tile_of(L, p, nM, m, n);
        for (int kb = 0; kb < p.nK; ++kb) {
          if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort, p.err)) {
            ok = false;
            break;
          }
          // a pair's bytes are all counted on the even CTA's barrier
          const uint32_t own = smem_u32(&ctl->full[stage]);
          issued |= 1u << stage;
          issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
          if (rank == 0u) mbar_arrive_expect_tx(own, kStageBytes * kCG);
          const uint32_t sa = base + uint32_t(stage) * kStageBytes;
          if constexpr (kCG == 2) {
            const uint32_t fb = mapa_shared(own, 0u);
            tma_load_2d_pair(sa, &map_a, fb, kb * KB, (m * kCG + int(rank)) * TM);
            tma_load_2d_pair(sa + A_BYTES, &map_b, fb, kb * KB, n * TN + int(rank) * (TN / kCG));
          } else {
            tma_load_2d(sa, &map_a, own, kb * KB, m * TM);
            tma_load_2d(sa + A_BYTES, &map_b, own, kb * KB, n * TN);
          }
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (!ok && rank == 0u) {
        // let the copies already in flight land before the CTA can exit
        for (int s = 0; s < kStages; ++s) {
          if (!((issued >> s) & 1u)) continue;
          const uint32_t par = (issued_phase >> s) & 1u;
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(smem_u32(&ctl->full[s]), par) && globaltimer_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
    }
    if (warp == 1 && lane == 0 && rank == 0u) {
      // ---------------------------------------------------------- MMA issuer (a pair's: the even CTA)
      constexpr uint32_t idesc = idesc_bf16(TM * kCG, TN, false, false);
      auto commit = [&](uint64_t *bar) {
        if constexpr (kCG == 2)
          mma_commit_pair(smem_u32(bar), uint16_t(0x3));
        else
          mma_commit(smem_u32(bar));
      };
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int L = cl; L < tiles && ok; L += ncl) {
        for (int kb = 0; kb < p.nK; ++kb) {
          const int in_part = kb & (p.part_blocks - 1);
          if ((in_part == 0 && !mbar_wait(smem_u32(&ctl->acc_empty[acc]), acc_phase ^ 1u, abort, p.err)) ||
              !mbar_wait(smem_u32(&ctl->full[stage]), phase, abort, p.err)) {
            ok = false;
            break;
          }
          fence_after_sync();
          const uint32_t sa = base + uint32_t(stage) * kStageBytes, sb = sa + A_BYTES;
          const uint32_t d = tmem_base + uint32_t(acc) * TN;
#pragma unroll
          for (int kk = 0; kk < KB / 16; ++kk) {
            const uint64_t ad = sdesc_sw128(sa + kk * 32u, 16u, 1024u), bd = sdesc_sw128(sb + kk * 32u, 16u, 1024u);
            const uint32_t accum = (in_part | kk) != 0 ? 1u : 0u;
            if constexpr (kCG == 2)
              mma_bf16_pair(d, ad, bd, idesc, accum);
            else
              mma_bf16(d, ad, bd, idesc, accum);
          }
          commit(&ctl->empty[stage]);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
          if (in_part == p.part_blocks - 1 || kb == p.nK - 1) {
            commit(&ctl->acc_full[acc]);
            if (++acc == ACCS) {
              acc = 0;
              acc_phase ^= 1u;
            }
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SUM_REGS));
    // ------------------------------------------------------------ add the parts and finish
    const int quad = warp & 3;  // TMEM lane quadrant this warp may access
    const int quarter = (warp - 4) >> 2;
    const int r = quad * 32 + lane;
    const int parts = (p.nK + p.part_blocks - 1) / p.part_blocks;
    const float scale = p.top.inv_t * kLog2e;
    int a = 0, local = 0;
    uint32_t a_phase = 0;
    for (int L = cl; L < tiles; L += ncl, ++local) {
      int m, n;
      tile_of(L, p, nM, m, n);
      const int64_t row = (int64_t(m) * kCG + int(rank)) * TM + r;
      const bool row_ok = row < rows;
      const int col0 = n * TN + quarter * HN;
      // this thread's entries: a bit per column, and where its first one stands in the row's list
      const int64_t t = (row_ok && p.row_idx) ? int64_t(ld(p.row_idx + row)) : row;
      uint32_t bits[2] = {0u, 0u};
      int first = 0;
      if (row_ok) {
        const uint16_t *off = p.top.off + t * (p.top.tiles + 1) + n;
        const int32_t *id = p.top.id + t * p.top.K;
        first = ld(off);
        const int end = ld(off + 1);
        constexpr int kU = 4;  // loads in flight
        for (int q = first; q < end; q += kU) {
          int c[kU];
#pragma unroll
          for (int u = 0; u < kU; ++u) c[u] = q + u < end ? ld(id + q + u) - col0 : HN;
#pragma unroll
          for (int u = 0; u < kU; ++u) {
            first += c[u] < 0;
            if (unsigned(c[u]) < 32u) bits[0] |= 1u << c[u];
            if (unsigned(c[u] - 32) < 32u) bits[1] |= 1u << (c[u] - 32);
          }
        }
      }
      float z[HN];
      bool ok = true;
#pragma unroll 1
      for (int part = 0; part < parts; ++part) {
        if (!mbar_wait(smem_u32(&ctl->acc_full[a]), a_phase, abort, p.err)) {
          ok = false;
          break;
        }
        fence_after_sync();
        const uint32_t taddr = tmem_base + (uint32_t(quad * 32) << 16) + uint32_t(a) * TN + uint32_t(quarter * HN);
#pragma unroll
        for (int c = 0; c < HN; c += 16) {
          uint32_t u[16];
          tmem_ld16(taddr + c, u);
          tmem_wait_ld();
          if (part == 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) z[c + j] = __uint_as_float(u[j]);
          } else {
#pragma unroll
            for (int j = 0; j < 16; j += 2)
              unpack_f32x2(add_f32x2(pack_f32x2(z[c + j], z[c + j + 1]),
                                     pack_f32x2(__uint_as_float(u[j]), __uint_as_float(u[j + 1]))),
                           z[c + j], z[c + j + 1]);
          }
        }
        // one arrival a warp: 512 of them a part, serialised in shared memory, held up the operands' reads
        fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          const uint32_t bar = smem_u32(&ctl->acc_empty[a]);
          if (kCG == 2 && rank != 0u)
            mbar_arrive_cluster(mapa_shared(bar, 0u));
          else
            mbar_arrive(bar);
        }
        if (++a == ACCS) {
          a = 0;
          a_phase ^= 1u;
        }
      }
      // the four warps of a row exchange their quarters below: they go on together or not at all
      if (!named_barrier_and(1 + quad, 128, ok)) break;
      float *dst = p.top.z + t * p.top.K + first;
#pragma unroll
      for (int c = 0; c < HN; c += 16) {
        const uint32_t some = bits[c / 32] >> (c % 32) & 0xffffu;
        if (!__any_sync(0xffffffffu, some != 0u)) continue;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if ((some >> j) & 1u) {
            *dst++ = z[c + j] * p.top.inv_t;
            z[c + j] = -INFINITY;
          }
      }
      const int valid = p.vocab - col0;  // <= 0: no column of a ragged last tile
      if (valid < HN) {
#pragma unroll
        for (int j = 0; j < HN; ++j) z[j] = j < valid ? z[j] : -INFINITY;
      }
      float m4[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
      for (int j = 4; j < HN; ++j) m4[j & 3] = fmaxf(m4[j & 3], z[j]);
      const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
      float s = 0.f;
      if (mx != -INFINITY) {
        // the difference first: as fma(z, scale, -mx scale) its rounding is that of the larger product
        const f32x2 neg = pack_f32x2(-mx, -mx), scale2 = pack_f32x2(scale, scale);
        f32x2 s2[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < HN; j += 2) {
          float t0, t1;
          unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(z[j], z[j + 1]), neg), scale2), t0, t1);
          s2[(j >> 1) & 1] = add_f32x2(s2[(j >> 1) & 1], pack_f32x2(ex2_approx(t0), ex2_approx(t1)));
        }
        float s1;
        unpack_f32x2(add_f32x2(s2[0], s2[1]), s, s1);
        s += s1;
      }
      float2(*sh)[TM] = ctl->quarter[local & 1];
      sh[quarter][r] = make_float2(mx, s);
      named_barrier(1 + quad, 128);
      if (quarter == (local & 3) && row_ok) {
        float2 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = sh[k][r];
        const float mm = fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x));
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (v[k].x != -INFINITY) ss = fmaf(v[k].y, ex2_approx((v[k].x - mm) * scale), ss);
        p.part[int64_t(n) * p.rows + row] = make_float2(mm * p.top.inv_t, ss);
      }
    }
  }

  fence_before_sync();
  __syncthreads();
  // neither CTA of a pair frees its TMEM or exits while the other may still reach its shared memory
  if constexpr (kCG == 2) cluster_sync();
  if (warp == 1) {
    fence_after_sync();
    if constexpr (kCG == 2)
      tmem_dealloc_pair(tmem_base, TMEM_COLS);
    else
      tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

template <int kCG>
sao_status launch_logits(const CUtensorMap &ma, const CUtensorMap &mb, const FwdParams &p, cudaStream_t s) {
  auto kern = distill_logits_kernel<kCG>;
  struct SetUp {
    cudaError_t err;
    int workers;  // CTAs, or CTA pairs, that fit on the device at once
  };
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(NUM_THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  static PerDevice<SetUp> set_up;
  const SetUp up = set_up.get(di.device, [&] {
    SetUp u{cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_BYTES)), di.sm_count};
    if (u.err == cudaSuccess && kCG == 2) u.err = cudaOccupancyMaxActiveClusters(&u.workers, kern, &cfg);
    return u;
  });
  if (up.err != cudaSuccess) return fail(SAO_ERR_CUDA, "kernel set-up: %s", cudaGetErrorString(up.err));
  if (up.workers < 1) return fail(SAO_ERR_UNSUPPORTED, "no CTA pair of the logits kernel fits on this device");
  const int64_t tiles = int64_t(p.nM) * p.nN;
  const int grid = tiles < up.workers ? int(tiles) : up.workers;
  int slot = launch_begin("distill_logits", s);
  if constexpr (kCG == 2) {
    cfg.gridDim = dim3(unsigned(2 * grid));
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, ma, mb, p);
    if (e != cudaSuccess) return fail(SAO_ERR_CUDA, "cudaLaunchKernelEx (distill_logits): %s", cudaGetErrorString(e));
  } else {
    pdl(kern, grid, NUM_THREADS, SMEM_BYTES, s)(ma, mb, p);
  }
  return launch_end(slot, s);
}

}  // namespace

size_t tc_distill_fwd_bytes(int64_t N, int32_t h, int32_t V) {
  const int64_t nvt = (int64_t(V) + TN - 1) / TN;
  return compact_ws_bytes(N, h) + round256(sizeof(float2) * size_t(nvt) * size_t(N));
}

sao_status tc_distill_fwd(const void *H, const void *W, const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                          const TopRef &top, const TopFinish &f, unsigned int *err, Carver &c, cudaStream_t s) {
  const int nvt = (V + TN - 1) / TN;
  CompactRows cr{};
  if (row_mask) SAO_TRY(compact_rows(row_mask, nullptr, N, static_cast<const __nv_bfloat16 *>(H), h, &cr, c, s));
  float2 *part = c.take<float2>(size_t(nvt) * size_t(N));
  if (!c.ok()) return fail(SAO_ERR_WORKSPACE, "workspace too small for the distillation forward");
  const int cg = cta_group();
  CUtensorMap ma, mb;
  SAO_TRY(make_map(&ma, row_mask ? cr.Hc : H, uint64_t(h), uint64_t(row_mask ? cr.cap : N), uint64_t(h), KB, TM));
  SAO_TRY(make_map(&mb, W, uint64_t(h), uint64_t(V), uint64_t(h), KB, TN / cg));
  FwdParams p{};
  p.nM = int((N + TM * cg - 1) / (TM * cg));
  p.nN = nvt;
  p.nK = (h + KB - 1) / KB;
  p.part_blocks = (N <= kFewPartRows ? kFewPart : kPart) / KB;
  p.group_m = 64;  // as the log-prob forward: 32 MB of H stay in L2 while W streams
  p.rows = N;
  p.vocab = V;
  p.part = part;
  p.top = top;
  p.err = err;
  if (row_mask) {
    p.m_count = cr.count;
    p.row_idx = cr.idx;
  }
  SAO_TRY(cg == 2 ? launch_logits<2>(ma, mb, p, s) : launch_logits<1>(ma, mb, p, s));
  return distill_finish(top, f, part, nvt, row_mask ? cr.pos : nullptr, N, s);
}

}  // namespace sao
