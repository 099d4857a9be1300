// bf16 forward of the distillation from a teacher's top logits: Z = H W^T / T tile by
// tile on the tensor cores, each tile reduced to (max, sum-exp) over the columns outside
// the row's entries, the entries' logits kept.
//
// The tensor core truncates as it adds to its accumulator. Over a contraction of 2,048
// that moved a logit of 12 by 2.6e-5, always towards zero, and the loss by 1e-5 of
// itself, some ten times what fp32 FMAs lose. So the accumulator is emptied every
// kPart elements of the contraction and the parts are added in fp32 registers: a part's
// accumulator is smaller by the number of parts, and so is what truncation takes.
// Sixteen warps hold a 128x256 tile as 64 sums a thread.
//
// A row's entries are sorted by id, and off[] counts them by tile, so a thread finds
// those of its 64 columns while the tile's products run. Per tile 128 x 256 x h
// multiply-adds against 128 x 256 exponentials: bound by the tensor cores from h = 512 on.
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

constexpr int TM = 128, TN = 256, KB = 64, STAGES = 4;
static_assert(TN == kTopTile, "offsets count entries by tile");
#ifndef KPART
#define KPART 512
#endif
constexpr int kPart = KPART;                   // contraction elements between two read-outs of an accumulator
constexpr int kPartBlocks = kPart / KB;
constexpr uint32_t A_BYTES = TM * KB * 2, B_BYTES = TN * KB * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int ACCS = 2;
constexpr uint32_t TMEM_COLS = ACCS * TN;
constexpr int NUM_THREADS = 640;             // warp 0 TMA, warp 1 MMA, warps 4-19 add the parts and finish
constexpr int HN = TN / 4;                   // columns per adding warp: four warps (128 rows) per quarter
constexpr int LAUNCH_REGS = 96, ISSUE_REGS = 40, SUM_REGS = 104;
static_assert(128 * ISSUE_REGS + 512 * SUM_REGS <= NUM_THREADS * LAUNCH_REGS, "split within the launch's registers");
constexpr float kLog2e = 1.4426950408889634f;

struct __align__(8) SmemCtl {
  uint64_t full[STAGES], empty[STAGES], acc_full[ACCS], acc_empty[ACCS];
  uint32_t tmem_base;
  int abort;
  float2 quarter[2][4][TM];  // (max, sum) of each quarter tile's rows, two tiles in turn
};
constexpr size_t SMEM_BYTES = 1024 + size_t(STAGES) * STAGE_BYTES + sizeof(SmemCtl);
static_assert(SMEM_BYTES <= 232448, "shared memory of an SM");

struct FwdParams {
  int nM, nN, nK;      // tiles along M and N, 64-wide K blocks
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

__global__ void __launch_bounds__(NUM_THREADS, 1)
    distill_logits_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                          const FwdParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  SmemCtl *ctl = reinterpret_cast<SmemCtl *>(smem_raw + (base - raw) + size_t(STAGES) * STAGE_BYTES);
  volatile int *abort = &ctl->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int a = 0; a < ACCS; ++a) {
      mbar_init(smem_u32(&ctl->acc_full[a]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[a]), 512);
    }
    ctl->abort = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem_base), TMEM_COLS);
    tmem_relinquish();
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_map(&map_a);
    tma_prefetch_map(&map_b);
  }
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem_base = ctl->tmem_base;
  grid_wait_long();
  int nM = p.nM;
  int64_t rows = p.rows;
  if (p.m_count) {
    rows = *p.m_count;
    nM = int((rows + TM - 1) / TM);
  }
  const int tiles = nM * p.nN;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ISSUE_REGS));
    if (warp == 0 && lane == 0) {
      // ---------------------------------------------------------- TMA producer
      int stage = 0;
      uint32_t phase = 0, issued = 0, issued_phase = 0;
      bool ok = true;
      for (int L = blockIdx.x; L < tiles && ok; L += gridDim.x) {
        int m, n;
        tile_of(L, p, nM, m, n);
        for (int kb = 0; kb < p.nK; ++kb) {
          if (!mbar_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort, p.err)) {
            ok = false;
            break;
          }
          const uint32_t fb = smem_u32(&ctl->full[stage]);
          issued |= 1u << stage;
          issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
          mbar_arrive_expect_tx(fb, STAGE_BYTES);
          const uint32_t sa = base + uint32_t(stage) * STAGE_BYTES;
          tma_load_2d(sa, &map_a, fb, kb * KB, m * TM);
          tma_load_2d(sa + A_BYTES, &map_b, fb, kb * KB, n * TN);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (!ok) {
        // let the copies already in flight land before the CTA can exit
        for (int s = 0; s < STAGES; ++s) {
          if (!((issued >> s) & 1u)) continue;
          const uint32_t par = (issued_phase >> s) & 1u;
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(smem_u32(&ctl->full[s]), par) && globaltimer_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
    }
    if (warp == 1 && lane == 0) {
      // ---------------------------------------------------------- MMA issuer
      constexpr uint32_t idesc = idesc_bf16(TM, TN, false, false);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int L = blockIdx.x; L < tiles && ok; L += gridDim.x) {
        for (int kb = 0; kb < p.nK; ++kb) {
          const int in_part = kb % kPartBlocks;
          if ((in_part == 0 && !mbar_wait(smem_u32(&ctl->acc_empty[acc]), acc_phase ^ 1u, abort, p.err)) ||
              !mbar_wait(smem_u32(&ctl->full[stage]), phase, abort, p.err)) {
            ok = false;
            break;
          }
          fence_after_sync();
          const uint32_t sa = base + uint32_t(stage) * STAGE_BYTES, sb = sa + A_BYTES;
          const uint32_t d = tmem_base + uint32_t(acc) * TN;
#pragma unroll
          for (int kk = 0; kk < KB / 16; ++kk)
            mma_bf16(d, sdesc_sw128(sa + kk * 32u, 16u, 1024u), sdesc_sw128(sb + kk * 32u, 16u, 1024u), idesc,
                     (in_part | kk) != 0 ? 1u : 0u);
          mma_commit(smem_u32(&ctl->empty[stage]));
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
          if (in_part == kPartBlocks - 1 || kb == p.nK - 1) {
            mma_commit(smem_u32(&ctl->acc_full[acc]));
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
    const int parts = (p.nK + kPartBlocks - 1) / kPartBlocks;
    int a = 0, local = 0;
    uint32_t a_phase = 0;
    for (int L = blockIdx.x; L < tiles; L += gridDim.x, ++local) {
      int m, n;
      tile_of(L, p, nM, m, n);
      const int64_t row = int64_t(m) * TM + r;
      const bool row_ok = row < rows;
      const int col0 = n * TN + quarter * HN;
      // this thread's entries: a bit per column, and where its first one stands in the row's list
      const int64_t t = (row_ok && p.row_idx) ? int64_t(ld(p.row_idx + row)) : row;
      uint32_t bits[2] = {0u, 0u};
      int first = 0;
      if (row_ok) {
        const uint16_t *off = p.top.off + t * (p.top.tiles + 1) + n;
        first = ld(off);
        const int end = ld(off + 1);
        for (int q = first; q < end; ++q) {
          const int c = ld(p.top.id + t * p.top.K + q) - col0;
          if (c < 0) {
            first = q + 1;
          } else if (c < HN) {
            if (c < 32)
              bits[0] |= 1u << c;
            else
              bits[1] |= 1u << (c - 32);
          } else {
            break;
          }
        }
      }
      float z[HN];
#pragma unroll
      for (int j = 0; j < HN; ++j) z[j] = 0.f;
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
#pragma unroll
          for (int j = 0; j < 16; ++j) z[c + j] += __uint_as_float(u[j]);
        }
        fence_before_sync();
        mbar_arrive(smem_u32(&ctl->acc_empty[a]));
        if (++a == ACCS) {
          a = 0;
          a_phase ^= 1u;
        }
      }
      // the four warps of a row exchange their quarters below: they go on together or not at all
      if (!named_barrier_and(1 + quad, 128, ok)) break;
      const int valid = p.vocab - col0;  // <= 0: no column of a ragged last tile
#pragma unroll
      for (int j = 0; j < HN; ++j) z[j] *= p.top.inv_t;
      if (__any_sync(0xffffffffu, (bits[0] | bits[1]) != 0u)) {
        float *dst = p.top.z + t * p.top.K + first;
#pragma unroll
        for (int j = 0; j < HN; ++j)
          if ((bits[j / 32] >> (j % 32)) & 1u) {
            *dst++ = z[j];
            z[j] = -INFINITY;
          }
      }
      if (valid < HN) {
#pragma unroll
        for (int j = 0; j < HN; ++j) z[j] = j < valid ? z[j] : -INFINITY;
      }
      float mx = z[0];
#pragma unroll
      for (int j = 1; j < HN; ++j) mx = fmaxf(mx, z[j]);
      float s = 0.f;
      if (mx != -INFINITY) {
        // the difference first: as fma(z, log2e, -mx log2e) its rounding is that of the larger product
        float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < HN; ++j) s4[j & 3] += ex2_approx((z[j] - mx) * kLog2e);
        s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
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
          if (v[k].x != -INFINITY) ss = fmaf(v[k].y, ex2_approx((v[k].x - mm) * kLog2e), ss);
        p.part[int64_t(n) * p.rows + row] = make_float2(mm, ss);
      }
    }
  }

  fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    fence_after_sync();
    tmem_dealloc(tmem_base, TMEM_COLS);
  }
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
  CUtensorMap ma, mb;
  SAO_TRY(make_map(&ma, row_mask ? cr.Hc : H, uint64_t(h), uint64_t(row_mask ? cr.cap : N), uint64_t(h), KB, TM));
  SAO_TRY(make_map(&mb, W, uint64_t(h), uint64_t(V), uint64_t(h), KB, TN));
  FwdParams p{};
  p.nM = int((N + TM - 1) / TM);
  p.nN = nvt;
  p.nK = (h + KB - 1) / KB;
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
  DeviceInfo di;
  SAO_TRY(device_info(&di));
  static PerDevice<cudaError_t> set_up;
  const cudaError_t e = set_up.get(di.device, [] {
    return cudaFuncSetAttribute(distill_logits_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_BYTES));
  });
  if (e != cudaSuccess) return fail(SAO_ERR_CUDA, "kernel set-up: %s", cudaGetErrorString(e));
  const int64_t tiles = int64_t(p.nM) * p.nN;
  const int grid = tiles < di.sm_count ? int(tiles) : di.sm_count;
  int slot = launch_begin("distill_logits", s);
  pdl(distill_logits_kernel, grid, NUM_THREADS, SMEM_BYTES, s)(ma, mb, p);
  SAO_TRY(launch_end(slot, s));
  return distill_finish(top, f, part, nvt, row_mask ? cr.pos : nullptr, N, s);
}

}  // namespace sao
