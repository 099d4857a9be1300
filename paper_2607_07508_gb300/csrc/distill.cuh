// Distillation from a teacher's top logits: what the row kernels (distill.cu) and the
// logit kernels of the two head types (logprobs_tc.cu, logprobs_f32.cu) share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sao.h"
#include "logprobs_common.cuh"
#include "rows.cuh"
#include "sao_common.cuh"

namespace sao {

constexpr int kTopTile = 256;  // vocabulary columns that an offset of TopRef counts by

// The teacher's entries of each row, sorted by token id, for the forward's epilogues:
// they keep the student's logit of each entry and leave it out of their tile's
// (max, sum). Row t has entries off[t][tiles], of which off[t][j] have ids below
// 256 j.
struct TopRef {
  const int32_t *id;    // [N][K] ascending
  const uint16_t *off;  // [N][tiles + 1]
  float *z;             // [N][K] out, in the order of id
  int K, tiles;
  float inv_t;          // 1 / temperature
  unsigned int *range;  // fp32 heads: classes of the operands, cleared
};

// The backward's view of the rows: dZ[t, v] = g[t] exp(z[t, v] / T - rest[t]) on the
// columns outside the entries, dz_top[t][k] / T at id ids[t][k].
struct TopGrad {
  const uint8_t *mask;   // [N] rows with a gradient
  const float *g, *rest; // [N]
  const float *dz_top;   // [N][K]
  const int32_t *ids;    // [N][K], the caller's order; < 0: no entry
  int K;
  float inv_t;
  unsigned int *range;   // fp32 heads: classes of the operands, cleared
  const int *extra;      // [kExtraRows] tokens with second pieces (-1: none), as rows tokens, tokens + 1, ...; or null
  int64_t tokens;        // with g, rest and mask for those rows too: 0, 0 and 1
};
constexpr int kRangeWords = 3;

// A bf16 head of up to this many rows keeps its dZ as two bf16 pieces, the second one's
// rows kFewRows after the first's in the same 128-row tile, with a copy of H's row, so
// that both products take in 16 bits of dZ at no cost. With many rows the rounding of
// dZ's elements averages out in dH and dW (1.4 times the error of rounding the outputs
// alone); with one row a single entry may be most of dZ, and its rounding, up to 2^-9,
// all of dW's error.
constexpr int kFewRows = 64;
// From there to kExtraMost rows, the kExtraRows rows whose entries lose most get a second row of
// dZ, with what their entries' rounding left, and of H. Where a row has few entries the
// error of dH and dW is that of a few of them, and a rounding is 1 to 3 times its mean. Against the error
// of rounding the outputs alone, 130 to 1,500 rows with one entry: 1.3 to 1.4 times on average, up to
// 2.0; with 32 such rows 1.0 to 1.1, up to 1.2; with five entries 1.4 and 1.7, 1.1 and 1.4.
// What that costs a backward of the moe head (us, with / without; one entry a row, error of an fp32 dW):
// where the padding to 128 rows has room 96 rows 470 / 446 (0.0007 / 0.0014), 224 524 / 508, 480 785 / 766;
// where it opens a tile 128 509 / 457 (0.0009 / 0.0016), 256 606 / 515 (0.0013 / 0.0017), 512 933 / 773
// (0.0014 / 0.0017); 1,024 1,390 / 1,396 (0.0016 / 0.0017), 4,096 5,010 / 4,970 (0.0016 both).
constexpr int kExtraRows = 32;
constexpr int64_t kExtraMost = 8192;
inline bool extra_rows(int64_t N) { return N > kFewRows && N <= kExtraMost; }

// The rows with mask != 0 of up to kFewRows: rows p and kFewRows + p of Hc are that
// token's, idx = -1 (and zeros) past the last one; count: rows of the products (0 or
// kFewRows + the active ones).
sao_status distill_few_rows(const uint8_t *mask, int64_t N, const __nv_bfloat16 *H, int32_t h, CompactRows *out,
                            Carver &c, cudaStream_t s);
// dH[t] = bf16(the sum of rows pos[t] and kFewRows + pos[t] over the parts), 0 where pos < 0.
sao_status distill_few_dH(const float *acc, const DhParts &parts, int32_t h, const int *pos, const int *count,
                          int64_t N, __nv_bfloat16 *dH, cudaStream_t s);

// Adds the fp32 dH of the extra rows to their tokens', in every part.
sao_status distill_fold_extra(const TopGrad &t, float *acc, const DhParts &parts, int32_t h, const int *pos,
                              const int *count, cudaStream_t s);

// Writes dz_top into a chunk of dZ (vocabulary [v0, v0 + vc), rows in the order of
// `idx`): one bf16 plane (`few`: the second pieces in the rows from kFewRows on), or the
// three planes of the fp32 path, whose class word `range` then takes the magnitudes.
sao_status patch_top_bf16(const TopGrad &t, const int *idx, const int *count, int64_t rows, bool few, int v0, int vc,
                          __nv_bfloat16 *dz, int64_t ldz, cudaStream_t s);
sao_status patch_top_f32(const TopGrad &t, const int *idx, const int *count, int64_t rows, int v0, int vc,
                         __nv_bfloat16 *dz, int64_t ldz, int64_t plane, unsigned int *range, cudaStream_t s);

// Merges the partials of the columns outside the entries and forms each row's loss.
struct TopFinish {
  const void *a;               // teacher logits [N][K]
  sao_dtype adt;
  const float *teacher_lse;    // [N] or null
  const uint16_t *slot;        // [N][K] sorted position -> the caller's
  const int32_t *entries;      // [N] entries, or -1 (an id out of range or there twice)
  const uint8_t *row_mask;     // [N] or null
  float *loss, *lse, *lse_rest, *z_top;
  int V;
};
sao_status distill_finish(const TopRef &top, const TopFinish &f, const float2 *part, int nvt, const int *pos,
                          int64_t N, cudaStream_t s);

// logprobs_tc.cu / logprobs_f32.cu: the logits of a call and its backward, each on what
// is left of the call's workspace.
size_t tc_distill_fwd_bytes(int64_t N, int32_t h, int32_t V);
size_t tc_distill_bwd_bytes(int64_t N, int32_t h, int32_t V);
size_t tc_distill_bwd_most(int64_t N, int32_t h, int32_t V);
sao_status tc_distill_fwd(const void *H, const void *W, const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                          const TopRef &top, const TopFinish &f, unsigned int *err, Carver &c, cudaStream_t s);
sao_status tc_distill_bwd(const void *H, const void *W, const TopGrad &t, int64_t N, int32_t h, int32_t V, void *dH,
                          void *dW, sao_dtype dw_dt, int accumulate, unsigned int *err, Carver &c, cudaStream_t s);
sao_status f32_distill_fwd(const float *H, const float *W, const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                           const TopRef &top, const TopFinish &f, unsigned int *err, Carver &c, cudaStream_t s);
sao_status f32_distill_bwd(const float *H, const float *W, const TopGrad &t, int64_t N, int32_t h, int32_t V,
                           float *dH, float *dW, int accumulate, unsigned int *err, Carver &c, cudaStream_t s);

// distill_rows.cu: a few rows on the fp32 units, W read once by each direction.
bool gemv_takes(int64_t N, int32_t h, sao_dtype dt);
int64_t gemv_rows(int32_t h, sao_dtype dt);  // the most rows that it takes
size_t gemv_fwd_bytes(int64_t N, int32_t V);
size_t gemv_bwd_bytes(int64_t N, int32_t h, int32_t V);
sao_status gemv_distill_fwd(const void *H, const void *W, sao_dtype dt, const uint8_t *row_mask, int64_t N, int32_t h,
                            int32_t V, const TopRef &top, const TopFinish &f, Carver &c, cudaStream_t s);
sao_status gemv_distill_bwd(const void *H, const void *W, sao_dtype dt, const TopGrad &t, int64_t N, int32_t h,
                            int32_t V, void *dH, void *dW, sao_dtype dw_dt, int accumulate, Carver &c, cudaStream_t s);

// distill.cu, called by the C entry points. _bytes: what a call of N rows needs; _most: of up
// to N rows (the paths for different N need different scratch, and more rows often less).
size_t distill_ws_bytes(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt);
size_t distill_ws_most(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt);
sao_status distill_fwd_launch(const void *H, const void *W, sao_dtype dt, const int32_t *ids, const void *a,
                              sao_dtype adt, const float *teacher_lse, const uint8_t *row_mask, int64_t N, int32_t h,
                              int32_t V, int32_t K, float temperature, float *loss, float *lse, float *lse_rest,
                              float *z_top, unsigned int *err, void *ws, size_t ws_bytes, cudaStream_t s);
sao_status distill_bwd_launch(const void *H, const void *W, sao_dtype dt, const int32_t *ids, const void *a,
                              sao_dtype adt, const float *teacher_lse, const float *lse, const float *lse_rest,
                              const float *z_top, const float *grad, int64_t N, int32_t h, int32_t V, int32_t K,
                              float temperature, void *dH, void *dW, sao_dtype dw_dt, int accumulate,
                              unsigned int *err, void *ws, size_t ws_bytes, cudaStream_t s);

}  // namespace sao
