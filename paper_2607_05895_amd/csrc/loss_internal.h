// Descriptors and launchers of the losses over a vocabulary (loss_host.cpp, kernels_loss.hip).
//
// For n tokens with hidden states x (n x h) and a head w (v x h), in chunks of rows of x:
//   z = x w^T / T            logits     P = x,   Q = w,    K = h
//   dx = dz w                           P = dz,  Q = w^T,  K = v
//   dw = dz^T x                         P = dz^T, Q = x^T, K = the chunk's rows
// Every operand is bf16, panel blocked (blk_index), zero padded: rows to the tile, K to a whole number of steps. An fp32
// tensor is held in three bf16 parts, and a product runs over six pairs of parts, one K segment each.
//
// Between the logits and their gradient a chunk of bf16 inputs holds each logit in 16 bits: the distance
// from the largest of its row in its 64 columns, in steps of 2^-10 of a factor of two. That is a relative error of p of
// at most 2^-11 ln 2 = 3.4e-4, a sixth of the rounding of dz to bf16 that follows, at half the bytes of fp32, and
// the bf16 dz then takes the codes' place. (Below 2^-64 of that largest one p is taken as 0.) What p - q loses where they
// are near is not lost here: the logits of the targets are kept in fp32. For fp32 inputs the logits are kept in fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfsdp_internal.h"

namespace mfsdp {

constexpr int kLossTile = 256;       // output tile of the products (kLossTileSmall for launches with few tiles)
constexpr int kLossTileSmall = 128;
constexpr int kLossGroup = 64;       // columns of one softmax partial
constexpr int kLossMaxSeg = 6;
constexpr int kLossMaxTop = 256;     // most teacher logits a token
constexpr float kLossCodeStep = 1024.0f;  // codes per factor of two

// One NT product over panel-blocked operands: tiles of P Q^T, K in nseg segments (part pairs) of nk steps of 32, cut
// into `splits` ranges of kper steps.
struct LossGemm {
  const uint16_t *P, *Q;
  int64_t ldp, ldq;                                // K columns of the buffers
  int64_t pseg[kLossMaxSeg], qseg[kLossMaxSeg];    // element offsets of each segment's parts
  int32_t nseg, nk, splits, kper;
  int32_t tm, tn;                                  // tiles
  int32_t rows, cols;                              // real rows and columns of the result
  // logits: softmax partials per row and 64 columns, the targets' logits, and the logits themselves (or none of them)
  float inv_t;
  float *gm, *gs;                                  // [group][ldr]: largest logit; sum of the others' exp relative to it
  int64_t ldr;
  const int32_t* ids;                              // rows x k columns (negative: none)
  float* zt;                                       // rows x k logits of those
  int32_t k;
  uint16_t* codes;                                 // 16-bit logits, panel blocked with ldc columns, or null
  float* logits;                                   // fp32 logits, row-major with ldc columns, or null
  int64_t ldc;
  // gradients: the result, row-major with ldo columns, or fp32 tiles in accumulator order (part); prev: such tiles to add
  void* out;
  int64_t ldo;
  int32_t out_bf16;
  float* part;
  const float* prev;
  float alpha;                                     // result = alpha / denom[0] (denom null: 1) P Q^T (part: P Q^T)
  const float* denom;
};

// Panel-blocked bf16 copies of a row-major R x C matrix: as it is (dst, ldn columns) and transposed (dst_t, ldt columns),
// in `parts` parts (1: bf16 source; 3: fp32 source) that lie dst_part (dst_t_part) elements apart.
struct LossPack {
  const void* src;
  int64_t R, C;
  uint16_t *dst, *dst_t;
  int64_t ldn, ldt, dst_part, dst_t_part;
  int64_t rows, cols;          // padded extent to write (multiples of 32 and of 256)
  const float* row_on;         // rows whose entry is 0 are written as zeros (whatever they hold); null: all
  int32_t blocks_begin, bf16;  // first workgroup
};
struct LossPack2 {
  LossPack d[2];
  int32_t count;
};

// Targets in one form: per token k ids with weights q that add up to 1 (0 and -1: none), the sum of q log q, and whether
// the token counts (on: 1, 0, or NaN for an id outside the vocabulary).
struct LossTargets {
  const void *ids, *logits;    // n x k; logits: the teacher's (null: hard labels)
  int32_t id64, logits_bf16, k;
  int64_t n, n_pad, v, ignore;
  float inv_t;
  int32_t* id;
  float *q, *ent, *on;
};

// Per row of a chunk: the row's softmax (largest logit M, sum s of the others' exp relative to it), its loss and its weight
// in the gradient.
struct LossRows {
  const float *gm, *gs;
  int64_t ldr;
  int32_t groups, rows, rows_pad, k;
  const int32_t* id;
  const float *q, *ent, *on, *weight, *zt;
  float z_loss;
  float4* row;                 // {M, s, weight, 2 z_loss lse}
  float *token_loss, *lse;     // optional
  float* weighted;             // weight x loss
};

// dz of a chunk, without the factor scale / (T D) common to all tokens (which the products apply: rounded with it, the
// -1 of every label would be off by the same share of a bf16 step): codes -> bf16 in place and transposed, or fp32 logits -> three bf16 parts and their transposes.
struct LossGrad {
  uint16_t* codes;
  const float* logits;
  int64_t ldc;
  uint16_t *dz, *dz_t;         // (codes: dz = codes)
  int64_t dz_part, dz_t_part, ldt;
  const float* gm;
  int64_t ldr;
  const float4* row;
  const int32_t* id;
  const float *q, *zt;
  int32_t k, rows, rows_pad, v, v_pad;
};

struct LossJoin {
  const float* part;
  int32_t splits, tiles, tm, tn, rows, cols, out_bf16;
  void* out;
  int64_t ldo;
  float alpha;
  const float* denom;
};

enum { kLossLogits = 0, kLossOut = 1 };
hipError_t launch_loss_gemm(const LossGemm& a, int kind, int tile, hipStream_t st);
hipError_t launch_loss_pack(const LossPack2& a, int blocks, hipStream_t st);
hipError_t launch_loss_targets(const LossTargets& a, hipStream_t st);
// out[0] = f(sum of a (times b where given) over n values), in a fixed order: mode 0 the sum times scale, 1 that over denom[0] (0
// where denom is 0)
hipError_t launch_loss_sum(const float* a, const float* b, int64_t n, float scale, const float* denom, float* out,
                           hipStream_t st);
hipError_t launch_loss_rows(const LossRows& a, hipStream_t st);
hipError_t launch_loss_grad(const LossGrad& a, hipStream_t st);
hipError_t launch_loss_join(const LossJoin& a, int tile, hipStream_t st);
hipError_t launch_loss_zero(void* p, int64_t bytes, hipStream_t st);

}  // namespace mfsdp
