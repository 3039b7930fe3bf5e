// Descriptors and launchers of the losses over a vocabulary (loss_host.cpp, kernels_loss.hip).
//
// For n tokens with hidden states x (n x h) and a head w (v x h), in chunks of rows of x:
//   z = x w^T / T    logits       dx = dz w       dw = dz^T x
// x and dz are 16-bit, panel blocked (blk_index), zero padded (rows to the tile, columns to 256); w is read as it lies,
// row-major, or, where it is fp32 or its rows are no multiple of 16 bytes, from a row-major copy.
//
// An fp32 tensor is held in two fp16 parts, the value and what is left of it, after scaling by a power of two that brings the
// largest value to [2^14, 2^15): 22 bits and the second part's sign, so a value is off by at most 2^-24 of itself, as in
// fp32, down to 2^-16 of the largest, and by 2^-40 of the largest below that. A product runs over three pairs of parts, one K
// segment each; the fourth would add at most 2^-24 of each product. (Three bf16 parts need no scale, and six pairs: 1024
// tokens on a 50257 x 768 head, both gradients, 1490 us; so 926.) The scale is one for all of w, and one per row of x and of
// dz, so that no token's digits depend on another token. For dw, which sums over the tokens, x is split a second time, its
// rows divided by dz's scales. Values that are not finite are left out of the scales.
//
// dz of bf16 inputs is rounded to bf16. Up to 128 tokens it is held in two bf16 parts instead (its products run over both,
// one K segment each): there one rounding of a target's dz is a share of a whole row of dx and dw that no other token evens
// out (up to 2^-8, beside the results' own rounding), and the second part costs next to nothing where reading w and writing
// dw take the time (48 tokens, 128256 x 4096, before dw's stores went past the caches: 722 us in one part, 727 in two).
//
// Between the logits and their gradient a chunk of bf16 inputs holds each logit in 16 bits: the distance
// from the largest of its row in its 64 columns, in steps of 64 / 65535 of a factor of two. That is a relative error of p of
// at most half a step times ln 2 = 3.4e-4, a sixth of the rounding of dz to bf16 that follows, at half the bytes of fp32, and
// the bf16 dz then takes the codes' place. (Below 2^-64 of that largest one p is taken as 0.) What p - q loses where they
// are near is not lost here: the logits of the targets are kept in fp32. For fp32 inputs the logits are kept in fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mfsdp_internal.h"

namespace mfsdp {

constexpr int kLossTile = 256;       // output tile of the products (kLossTileSmall for launches with few tiles)
constexpr int kLossTileSmall = 128;
constexpr int kLossGroup = 64;       // columns of one softmax partial (of the products for a few tokens: 32)
constexpr int kLossMaxSeg = 3;       // K segments of an fp32 product
constexpr int kLossMaxima = 256;     // workgroups, at most, that look for a tensor's largest value
constexpr int kLossQueues = 3;       // launches of products per chunk that take their tiles from counters
constexpr int kLossMaxTop = 256;     // most teacher logits a token
constexpr float kLossOctaves = 64.0f;  // factors of two that the 16-bit codes of the logits span

// One product: tiles of P Q^T, K in nseg segments (pairs of parts) of nk steps of 32, cut into `splits` ranges of kper steps.
// P is panel blocked, and so is dw's Q (x); the others' Q is w, row-major with qrows rows.
enum { kLossDx = 0, kLossDw = 1 };
struct LossGemm {
  const uint16_t *P, *Q;
  int64_t ldp, ldq, qrows;
  int64_t ppart, qpart;                            // elements between the parts
  const float *row_most, *unscale;                 // fp32: what the scales of P's rows come from (null: no scale), 1 / the scale of Q
  int32_t nseg, nk, splits, kper;                  // nseg: 1; 2: P in two bf16 parts; 3: both in two fp16 parts
  int32_t tm, tn;                                  // tiles
  int32_t rows, cols;                              // real rows and columns of the result
  int32_t op;                                      // kLossDx, kLossDw (gradients)
  // logits: softmax partials per row and 64 columns, the targets' logits, and the logits themselves (or none of them)
  float inv_t;
  float *gm, *gs;                                  // (group, row): largest logit; sum of the others' exp relative to it
  int64_t gstep, rstep;                            // elements from a group, from a row to the next
  const int32_t* ids;                              // rows x k columns (negative: none)
  float* zt;                                       // rows x k logits of those
  int32_t k;
  uint16_t* codes;                                 // 16-bit logits, panel blocked with ldc columns, or null
  float* logits;                                   // fp32 logits, row-major with ldc columns, or null
  int64_t ldc;
  // gradients: the result, row-major with ldo columns, or fp32 tiles in accumulator order (part); prev: such tiles to add.
  // logits: part: the sums of a K range, in such tiles, and nothing else; prev: tiles with the sum over the ranges, `splits`
  // tiles apart, instead of a product
  void* out;
  int64_t ldo;
  int32_t out_bf16;
  float* part;
  const float* prev;
  float alpha;                                     // result = alpha / denom[0] (denom null: 1) P Q^T (part: P Q^T)
  const float* denom;
};

// Up to two products of one launch (the second one's tiles follow the first one's).
struct LossGemm2 {
  LossGemm g[2];
  int32_t count;
  int32_t* queue;  // kGemmXcds counters, 0 before the launch
};

// Products for a few tokens (at most 32 MI), where reading w counts: w is read as it lies, once, with no packed copy.
//   logits: tiles of stream_rows(MI) ids, K = h in steps of 16384 / stream_rows;  dx: tiles of 256 columns of h, K = v in steps of
//   stream_step(MI), cut into `splits` ranges of kper steps, whose fp32 results lie row-major (32 MI x ldo) one after another in part.
__host__ __device__ constexpr int stream_rows(int mi) { return mi <= 2 ? 128 : 256; }
__host__ __device__ constexpr int stream_step(int mi) { return mi <= 2 ? 64 : 32; }
struct LossStream {
  const uint16_t *P, *w;     // P: x, or dz (two parts, ppart elements apart); panel blocked with ldp columns
  int64_t ppart;
  int64_t ldp, v, h;
  int32_t nk, tiles, splits, kper;
  float inv_t;
  float *gm, *gs;            // per row and 32 columns
  int64_t gstep, rstep;
  const int32_t* ids;
  float* zt;
  int32_t k;
  uint16_t* codes;
  int64_t ldc;
  float* part;
  int64_t ldo;
};

// Labels as the caller has them: n x k ids; logits: the teacher's (null: hard labels, of which `ignore` marks none).
struct LossLabels {
  const void *ids, *logits;
  int32_t id64, logits_bf16, k;
  int64_t n, v, ignore;
  float inv_t;
};

// A copy of a row-major R x C matrix, in bf16 or (fp32 source) in two scaled fp16 parts that lie dst_part elements
// apart: panel blocked with ld columns, padded with zeros to the launch's rows and ld, or row-major with ld columns.
struct LossPack {
  const void* src;
  int64_t R, C;
  uint16_t* dst;
  int64_t ld, dst_part;
  int64_t cols;                // columns that the launch covers (a multiple of 256)
  int64_t label_row;           // the label of row 0 (rows whose token does not count are written as zeros), or -1: all rows
  int32_t blocks_begin, bf16;  // first workgroup
  int32_t blocked;
  // fp32. w: the largest of `count` values of most sets the scale. x: row r's scale comes from row_most[r]; and for dw, row
  // r is divided by the scale that comes from row_most[r], and the largest of most sets the scale. 1 / the scale of all goes
  // to inv.
  const float *row_most, *most;
  int32_t count;
  float* inv;
};

// fp32: the largest finite magnitude of each row of x (of those that do not count and of the rows up to n_pad: 0), and of w,
// one per workgroup.
struct LossMaxima {
  LossLabels l;
  const float *x, *w;
  int64_t h, n_pad;
  int32_t xblocks, wblocks;
  float *xmax, *wmax;
};

// The first launch: the labels in one form (per token k different ids with weights q that add up to 1, -1 and 0 for none; the
// sum of q log q; on: whether the token counts, 1, 0, or NaN for an id outside the vocabulary or a teacher logit of +inf or
// NaN), the packed operands, and the counters of the chunk's products set to 0.
struct LossPrep {
  LossLabels l;
  int64_t n_pad;
  int32_t label_blocks;        // workgroups of four tokens each; the packs' workgroups follow
  int32_t *id, *queues;
  float *q, *ent, *on;
  LossPack d[2];
  int32_t packs;
};

// The loss of all tokens: scale / denom[0] (denom null: 1; 0: loss 0) times the sum of their weighted losses.
struct LossTotal {
  const float *weighted, *denom;
  int64_t n;
  float scale;
  float* loss;
};

// Per row of a chunk: the row's softmax (largest logit M, sum s of the others' exp relative to it), its loss and its weight
// in the gradient. The first chunk's launch may have one more workgroup, for denom (the sum of the weights of the tokens that
// count).
struct LossRows {
  const float *gm, *gs;
  int64_t gstep, rstep;        // (gstep 1: one row per workgroup)
  int32_t groups, rows, rows_pad, k;
  const int32_t* id;
  const float *q, *ent, *on, *weight, *zt;
  float z_loss;
  float4* row;                 // {M, s, weight, 2 z_loss lse}
  // fp32 gradients (else null): per row a bound on |dz| (0 where it is not finite); per workgroup the largest x_most / its
  // scale
  float *row_most, *most;
  const float* x_most;
  float *token_loss, *lse;     // optional
  float* weighted;             // weight x loss
  int64_t n;                   // for denom: all tokens
  const float *all_on, *all_weight;
  float* denom;                // null: no such workgroup
};

// dz of a chunk, without the factor scale / (T D) common to all tokens (which the products apply: rounded with it, the
// -1 of every label would be off by the same share of a bf16 step): codes -> bf16 in place (and a second part elsewhere), or
// fp32 logits -> two fp16 parts, each row scaled.
struct LossGrad {
  uint16_t* codes;
  const float* logits;
  int64_t ldc;
  uint16_t* dz;                // (codes: dz = codes)
  int64_t dz_part;
  int32_t parts;               // of dz
  const float* gm;
  int64_t gstep, rstep;
  const float4* row;
  const int32_t* id;
  const float *q, *zt;
  int32_t k, rows, rows_pad, v, v_pad;
  int32_t group_shift;         // log2 of the columns of one softmax partial
  const float* row_most;       // fp32
  LossPack x;                  // fp32: x split for dw, by the last workgroups (x.src null: dw is not asked for)
  LossTotal total;             // loss not null: summed by one more workgroup
};

// out = alpha / denom times the sum of the K ranges' results in their order: tiles in accumulator order (tile > 0), or
// row-major ones of `stride` elements (tile 0).
struct LossJoin {
  const float* part;
  int32_t splits, tiles, tm, tn, rows, cols, out_bf16;
  int64_t stride, ldp;
  void* out;
  int64_t ldo;
  float alpha;
  const float* denom;
};

enum { kLossLogits = 0, kLossOut = 1 };
hipError_t launch_loss_gemm(const LossGemm2& a, int kind, int tile, hipStream_t st);
// dw of `steps` (1, 2 or 4) times 32 tokens at most, bf16
hipError_t launch_loss_dw(const LossGemm& a, int steps, hipStream_t st);
hipError_t launch_loss_stream(const LossStream& a, int mi, int kind, hipStream_t st);
hipError_t launch_loss_maxima(const LossMaxima& a, hipStream_t st);
hipError_t launch_loss_prep(const LossPrep& a, int blocks, hipStream_t st);
hipError_t launch_loss_rows(const LossRows& a, hipStream_t st);
// workgroups of that launch with rows
inline int loss_row_blocks(const LossRows& a) { return a.gstep == 1 ? a.rows_pad : a.rows_pad / 32; }
hipError_t launch_loss_total(const LossTotal& a, hipStream_t st);
hipError_t launch_loss_grad(const LossGrad& a, hipStream_t st);
hipError_t launch_loss_join(const LossJoin& a, int tile, hipStream_t st);
// logits in K ranges: the ranges of each tile added in order, into the first one's place
hipError_t launch_loss_sum(float* part, int64_t tiles, int tile, int splits, hipStream_t st);
hipError_t launch_loss_zero(void* p, int64_t bytes, hipStream_t st);
hipError_t launch_scale_grad(void* p, int64_t n, int bf16, const float* factor, hipStream_t st);

}  // namespace mfsdp
