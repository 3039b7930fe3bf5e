// Host side of the losses over a vocabulary: argument checks, workspace plan and launch sequence (all on the caller's
// stream, descriptors as kernel arguments).
//
//   fp32: maxima  the largest values of x's rows and of w, for their scales
//   per chunk of rows of x (usually one):
//     prep    the labels in one form (first chunk); x's rows panel blocked; a copy of w where it cannot be read as
//             it lies (first chunk)
//     logits  z = x w^T: per row and 64 columns the softmax partials, the targets' logits and (for gradients) the logits
//             (few tiles of a long K: the K ranges' sums, their total, and from it the rest: three launches)
//     rows    the partials joined: the tokens' losses, and the weights of their gradients; with MEAN (first chunk) the weights'
//             sum
//     grad    dz in the logits' place; (last chunk) the loss
//     dx      dz w            (K ranges and their join where there are few tiles)
//     dw      dz^T x          (added to the earlier chunks' sum, held in fp32; in one launch with dx where both are small)
// For a few tokens the logits and dx run on kernels that read w once at HBM's rate.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/mfsdp.h"
#include "loss_internal.h"

using namespace mfsdp;

namespace mfsdp {
int set_last_error(int status, const std::string& msg);
}

namespace {

static_assert(MFSDP_MAX_TOP_LOGITS == kLossMaxTop, "teacher logits of the ABI and the kernel");

constexpr int64_t kMaxTokens = int64_t(1) << 25;  // (a launch holds fewer than 2^32 threads, the labels take 64 a token)
constexpr int64_t kMaxSide = int64_t(1) << 20;
constexpr int64_t kMaxChunk = 65536;
constexpr int64_t kLogitBytes = int64_t(1) << 31;  // of a chunk's logits, at 16 bits each

int fail(int status, const std::string& msg) { return set_last_error(status, msg); }
int hip_fail(hipError_t e, const char* what) {
  return fail(MFSDP_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}
int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Gemm {
  int tile = 0, tm = 0, tn = 0, splits = 1, kper = 0, nk = 0;
  int64_t items() const { return int64_t(tm) * tn * splits; }
};

struct Plan {
  bool f32 = false, grads = false;
  bool copy = false;            // w is read from a bf16 copy
  int stream = 0;               // rows / 32 of the products for a few tokens, or 0
  int parts = 1, dz_parts = 1;  // of x and w, of dz
  int nseg = 1, out_nseg = 1;   // pairs of parts: of the logits, of dx and dw
  int64_t n = 0, v = 0, h = 0, k = 1;
  int64_t chunk = 0, n_pad = 0, vp = 0, hk = 0, hp = 0, ldw = 0;
  int group = kLossGroup;       // columns of a softmax partial
  int64_t gstep = 0, rstep = 0; // elements from a group's, from a row's partial to the next one
  Gemm logits, dx, dw;
  // offsets
  size_t id = 0, q = 0, ent = 0, on = 0, weighted = 0, denom = 0, queues = 0, row = 0, zt = 0, gm = 0, gs = 0;
  size_t inv = 0, xmax = 0, wmax = 0, row_most = 0, most = 0;  // fp32: 1 / the scales of x (for dw) and w; what scales come from
  size_t xb = 0, wb = 0, codes = 0, z32 = 0, part = 0, acc = 0;
  size_t bytes = 0;
};

// The products for a few tokens: at most kStreamTokens, on at least stream_ids(tokens) ids. Measured in us, tiles' kernels
// against these, loss alone and with both gradients:
//   1 token    4096 x 768: 22, 21 and 44, 36      16384 x 2048: 39, 31 and 109, 73      128256 x 4096: 242, 230 and 1034, 615
//   64 tokens  4096 x 768: 23, 21 and 47, 44      16384 x 2048: 41, 36 and 118, 86      128256 x 4096: 244, 241 and 1053, 654
//   128        8192 x 768: 23, 29 and 60, 62      16384 x 2048: 41, 51 and 126, 119     128256 x 4096: 246, 285 and 1257, 963
//              4096 x 4096: 38, 77 and 100, 121   32768 x 4096: 78, 95 and 343, 268     50257 x 768: 41, 37 and 152, 125
// (512 to 2048 ids: the same time up to 32 tokens. 4096 x 8192 is too short a head: 1 token 44, 59 and 110, 94. Beyond 64 tokens
// a wave multiplies twice as much per byte of w, which a loss alone has nothing to make up for: it is up to 1.5 times slower
// below some 40000 ids.)
constexpr int64_t kStreamTokens = 128;
constexpr int64_t stream_ids(int64_t tokens) { return tokens <= 64 ? 4096 : 12288; }

constexpr int64_t kMinRange = 16, kMaxRanges = 64;        // K steps of a range at least; ranges of dx at most
constexpr int64_t kMaxItems = 512;                        // tiles of the logits in K ranges at most
constexpr int64_t kRangeBytes = int64_t(256) << 20;       // room for dx's ranges (see range_room)

// A launch's time in us on `tile` x `tile` tiles, items[i] of steps[i] K steps each: what the chip's workgroups share, or the
// longest item if that is more, and half of the shortest kind for the uneven end. Measured: a step of 32 takes 0.74 us on a
// 256 x 256 tile (1.45 PFLOP/s over 256 CUs) and a tile's start and epilogue 8 us; on 128 x 128 tiles 0.3 and 5 us with a CU
// of their own, 0.55 and 13 us on two that share one (4096 tokens, 20000 x 4096 head, dx and dw: 1064 us on 256 x 256 tiles,
// 1433 on 128 x 128; 200 tokens, 2000 x 2048: 30 and 23 us).
double launch_us(int tile, int kinds, const int64_t* items, const int64_t* steps) {
  int64_t count = 0;
  for (int i = 0; i < kinds; ++i) count += items[i];
  const bool large = tile == kLossTile, alone = count <= 256;
  const double per_step = large ? 0.74 : alone ? 0.3 : 0.55, ends = large ? 8.0 : alone ? 5.0 : 13.0;
  const int64_t slots = std::min<int64_t>(large ? 256 : 512, count);
  double work = 0.0, longest = 0.0, shortest = 1e30;
  for (int i = 0; i < kinds; ++i) {
    if (items[i] == 0) continue;
    const double us = per_step * double(steps[i]) + ends;
    work += double(items[i]) * us;
    longest = std::max(longest, us);
    shortest = std::min(shortest, us);
  }
  return std::max(work / double(std::max<int64_t>(slots, 1)), longest) + (count > slots ? 0.5 * shortest : 0.0);
}
Gemm grid_of(int tile, int64_t M, int64_t N) {
  Gemm g;
  g.tile = tile;
  g.tm = int(up(M, tile) / tile);
  g.tn = int(up(N, tile) / tile);
  return g;
}
// The tile of a product that runs alone; its K ranges if it may have them (the logits: on 128 x 128 tiles, in one round and
// of an even number of steps, at least kMinRange, each; their sum and the epilogue, launches of their own, taken as 14 us and the
// sum's traffic. 553 tokens, 722 ids, 1088 wide, fp32: 35 us, 43 in one range; 300 tokens, 400 ids, 4000 wide: 28 and 117
// us).
Gemm choose(int64_t M, int64_t N, int64_t steps, bool ranges) {
  Gemm best;
  double us = 0.0;
  for (int tile : {kLossTile, kLossTileSmall}) {
    Gemm g = grid_of(tile, M, N);
    const int64_t tiles = g.items();
    const int64_t most = ranges && tile == kLossTileSmall ? std::min(kMaxItems / tiles, steps / kMinRange) : 1;
    for (int64_t s = 1; s == 1 || s <= most; ++s) {
      const int64_t kper = s == 1 ? steps : up((steps + s - 1) / s, 2), items = tiles * s;
      if (s > 1 && (steps + kper - 1) / kper != s) continue;
      double t = launch_us(tile, 1, &items, &kper);
      if (s > 1) t += 14.0 + double(items) * tile * tile * 8.0 / 4.9e6;
      if (best.tile == 0 || t < us) {
        us = t;
        best = g;
        best.splits = int(s);
        best.kper = int(kper);
      }
    }
  }
  return best;
}
// The tile of dx (n x h, xsteps of K) and dw (v x h, wsteps of K; 0: not asked for) in one launch, and the K ranges of dx:
// at most kMaxRanges of at least kMinRange steps, whose results fit `room` bytes; their join is taken as its traffic and a
// launch.
void choose_grads(int64_t n, int64_t v, int64_t h, int64_t xsteps, int64_t wsteps, int64_t room, Gemm& dx, Gemm& dw) {
  double best = 0.0;
  dx.tile = 0;
  for (int tile : {kLossTile, kLossTileSmall}) {
    const Gemm x = grid_of(tile, n, h), w = grid_of(tile, v, h);
    for (int s = 1; s <= kMaxRanges && (s == 1 || xsteps / s >= kMinRange); ++s) {
      const int64_t kper = (xsteps + s - 1) / s;
      if ((xsteps + kper - 1) / kper != s || (s > 1 && x.items() * s * tile * tile * 4 > room)) continue;
      const int64_t items[2] = {x.items() * s, wsteps ? w.items() : 0}, steps[2] = {kper, wsteps};
      double us = launch_us(tile, 2, items, steps);
      if (s > 1) us += 6.0 + double(items[0]) * tile * tile * 8.0 / 4.9e6;
      if (dx.tile == 0 || us < best) {
        best = us;
        dx = x;
        dw = w;
        dx.splits = s;
        dx.kper = int(kper);
      }
    }
  }
}

int check(const mfsdp_head_loss* a, int64_t k, bool pointers) {
  if (!a) return fail(MFSDP_E_INVALID, "arguments are NULL");
  if (a->n < 0 || a->n > kMaxTokens) return fail(MFSDP_E_INVALID, "n must be in [0, 2^25]");
  if (a->v < 1 || a->v > kMaxSide) return fail(MFSDP_E_INVALID, "v must be in [1, 2^20]");
  if (a->h < 1 || a->h > kMaxSide) return fail(MFSDP_E_INVALID, "h must be in [1, 2^20]");
  if (k < 1 || k > kLossMaxTop) return fail(MFSDP_E_INVALID, "k must be in [1, MFSDP_MAX_TOP_LOGITS]");
  if (a->dtype != MFSDP_F32 && a->dtype != MFSDP_BF16) return fail(MFSDP_E_INVALID, "unsupported dtype");
  if (a->reduction != MFSDP_SUM && a->reduction != MFSDP_MEAN) return fail(MFSDP_E_INVALID, "unknown reduction");
  if (!std::isfinite(float(a->scale))) return fail(MFSDP_E_INVALID, "scale must be finite in fp32");
  if (a->chunk_rows < 0) return fail(MFSDP_E_INVALID, "chunk_rows must be >= 0");
  if (!pointers) return MFSDP_OK;
  if (!a->w || (a->n > 0 && !a->x)) return fail(MFSDP_E_INVALID, "x or w is NULL");
  if (a->n > 0 && !a->loss && !a->token_loss && !a->lse && !a->dx && !a->dw)
    return fail(MFSDP_E_INVALID, "every output is NULL");
  for (const void* p : {a->x, a->w, (const void*)a->token_weight, (const void*)a->loss, (const void*)a->token_loss,
                        (const void*)a->lse, (const void*)a->dx, (const void*)a->dw})
    if (!aligned16(p)) return fail(MFSDP_E_INVALID, "pointers must be 16-byte aligned");
  return MFSDP_OK;
}

// Room for K ranges: a bound over what the choices above may take, not what this call takes. A call over fewer rows may want
// more ranges than one over many, and a workspace that is enough for many rows has to be enough for fewer; so each bound
// grows with the call's rows alone.
//   dx: kRangeBytes or a quarter of a pass's rows (pass_bytes), whichever is more. Of 38000 calls drawn over all sizes 54
//   would be more than 1 % faster with ranges beyond that by launch_us, and none more than 5 %.
int64_t range_room(const Plan& p, int64_t pass_bytes) {
  const int64_t steps = (p.f32 ? kLossMaxSeg : 2) * (up(p.v, 32) / 32), most = std::min(kMaxRanges, steps / kMinRange);
  return most < 2 ? 0 : std::min(std::max(kRangeBytes, pass_bytes / 4), p.n_pad * p.hp * 4 * most);
}
int64_t logit_range_room(const Plan& p) {
  constexpr int64_t T = kLossTileSmall;
  const int64_t steps = p.nseg * p.hk / 32, tn = up(p.v, T) / T;
  if (steps / kMinRange < 2 || tn > kMaxItems / 2) return 0;
  return std::min(kMaxItems, p.n_pad / T * tn * (steps / kMinRange)) * T * T * 4;
}
// dx of a few tokens: a workgroup per CU, in ranges of at least eight steps.
int64_t stream_ranges(const Plan& p, int stream) {
  const int64_t kt = stream_step(stream), steps = up(p.v, kt) / kt, tiles = p.hp / 256;
  return std::max<int64_t>(1, std::min(steps / 8, (256 + tiles - 1) / tiles));
}

// The workspace grows, or stays, with the rows, the outputs and k.
Plan make_plan(const mfsdp_head_loss* a, int64_t k) {
  Plan p;
  p.f32 = a->dtype == MFSDP_F32;
  p.grads = a->dx || a->dw;
  p.parts = p.f32 ? 2 : 1;
  p.dz_parts = p.f32 || a->n <= kStreamTokens ? 2 : 1;
  p.nseg = p.f32 ? kLossMaxSeg : 1;
  p.out_nseg = p.f32 ? kLossMaxSeg : p.dz_parts;
  p.n = a->n;
  p.v = a->v;
  p.h = a->h;
  p.k = k;
  p.vp = up(p.v, 256);
  p.hk = up(p.h, 64);
  p.hp = up(p.h, 256);
  p.copy = p.f32 || p.h % 8 != 0;
  p.ldw = p.copy ? p.hk : p.h;
  const int64_t es = 2 * p.parts, vsteps = up(p.v, 32) / 32;
  // bytes of a row of x in a pass over many tokens, with gradients and without
  const int64_t loss_row = p.hp * es + p.vp / kLossGroup * 8 + k * 4 + 16;
  const int64_t grad_row = loss_row + p.vp * 2 * (p.f32 ? 2 : 1) + (p.f32 ? p.vp * 4 + 5 : 0);
  int64_t with_grads = 0;  // rows of a pass
  auto streams = [&](int64_t tokens) { return !p.copy && p.v >= stream_ids(tokens); };
  if (p.n > 0 && p.n <= kStreamTokens && streams(p.n)) {
    p.stream = p.n <= 32 ? 1 : p.n <= 64 ? 2 : 4;
    p.group = 32;
    p.chunk = p.n_pad = 32 * p.stream;
  } else {
    p.n_pad = up(std::max<int64_t>(p.n, 1), 256);
    const int64_t asked = a->chunk_rows > 0 ? std::min(kMaxChunk, up(a->chunk_rows, 256)) : kMaxChunk;
    with_grads = std::min({p.n_pad, asked, std::max<int64_t>(256, kLogitBytes / (2 * p.vp) / 256 * 256)});
    p.chunk = with_grads;
    const int64_t slots = (kLossMaxTop - k) * 4, without = with_grads * (grad_row + slots) / (loss_row + slots) / 256 * 256;
    if (!p.grads)  // as many rows as take the bytes of those with gradients, with the most slots a row (the same for any k)
      p.chunk = std::min({p.n_pad, asked, std::max(with_grads, without)});
    else if (a->dw && a->chunk_rows == 0 && p.n_pad <= kMaxChunk &&
             p.n_pad * grad_row <= with_grads * grad_row + p.vp * p.hp * 4)
      p.chunk = p.n_pad;  // one pass where the rows beyond with_grads take no more than the sum of dw over two
  }
  const int64_t groups = (p.vp + p.group - 1) / p.group;
  // many tokens: the logits' lanes (rows) store whole lines; few: a row's partials are read in one piece
  p.gstep = p.chunk > 256 ? p.chunk : 1;
  p.rstep = p.chunk > 256 ? 1 : groups;
  const int64_t rows = std::min(p.chunk, std::max<int64_t>(p.n, 1)), wsteps = p.out_nseg * up(rows, 32) / 32;
  int64_t part = 0;
  if (p.stream) {
    if (a->dx) {
      const int64_t kt = stream_step(p.stream), steps = up(p.v, kt) / kt, splits = stream_ranges(p, p.stream);
      p.dx.nk = int(steps);
      p.dx.tn = int(p.hp / 256);
      p.dx.kper = int((steps + splits - 1) / splits);
      p.dx.splits = int((steps + p.dx.kper - 1) / p.dx.kper);
      part = splits * p.chunk * p.hp * 4;
    }
  } else {
    p.logits = choose(rows, p.v, p.nseg * p.hk / 32, true);
    p.logits.nk = int(p.hk / 32);
    part = logit_range_room(p);
    if (a->dx) {
      const int64_t room = range_room(p, with_grads * grad_row);
      choose_grads(rows, p.v, p.h, p.out_nseg * vsteps, a->dw ? wsteps : 0, room, p.dx, p.dw);
      p.dx.nk = int(vsteps);
      part = std::max(part, room);
      if (streams(1)) part = std::max(part, stream_ranges(p, 4) * kStreamTokens * p.hp * 4);  // a call over few tokens
    }
  }
  if (a->dw && (p.stream || !a->dx)) p.dw = choose(p.v, p.h, wsteps, false);
  size_t o = 0;
  auto take = [&](int64_t bytes) {
    const size_t at = o;
    o += size_t(up(bytes, 256));
    return at;
  };
  p.id = take(p.n_pad * k * 4);
  p.q = take(p.n_pad * k * 4);
  p.ent = take(p.n_pad * 4);
  p.on = take(p.n_pad * 4);
  p.weighted = take(p.n_pad * 4);
  p.denom = take(4);
  p.queues = take(kLossQueues * kGemmXcds * 4);
  p.row = take(p.chunk * 16);
  p.zt = take(p.chunk * k * 4);
  p.gm = take(groups * p.chunk * 4);
  p.gs = take(groups * p.chunk * 4);
  if (p.f32) {
    p.inv = take(2 * 4);
    p.xmax = take(p.n_pad * 4);
    p.wmax = take(kLossMaxima * 4);
  }
  p.xb = take(p.chunk * p.hp * es);
  if (p.copy) p.wb = take(p.v * p.ldw * es);
  if (p.grads) {
    // (up to 128 tokens on the tiles' kernels: two parts of 256 rows, which 129 tokens keep room for)
    p.codes = take(std::max(p.chunk * p.dz_parts, streams(kStreamTokens) || p.f32 ? 0 : int64_t(512)) * p.vp * 2);
    if (p.f32) {
      p.z32 = take(p.chunk * p.vp * 4);
      p.row_most = take(p.chunk * 4);
      p.most = take(std::max<int64_t>(256, p.chunk / 32) * 4);
    }
  }
  p.part = take(part);
  if (a->dw && p.chunk < p.n) p.acc = take(p.vp * p.hp * 4);
  p.bytes = o;
  return p;
}

struct Labels {
  const void *ids, *logits;
  int32_t id_bytes, logit_dtype;
  int64_t ignore;
  double temperature, z_loss;
};

int run(const mfsdp_head_loss* a, int64_t k, const Labels& l, void* workspace, size_t workspace_bytes, void* stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int es = a->dtype == MFSDP_F32 ? 4 : 2;
  const Plan p = make_plan(a, k);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return fail(MFSDP_E_WORKSPACE, "workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < p.bytes)
    return fail(MFSDP_E_WORKSPACE, "workspace too small: " + std::to_string(workspace_bytes) + " bytes, " +
                                       std::to_string(p.bytes) + " needed");
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  auto f32p = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  auto u16p = [&](size_t off) { return reinterpret_cast<uint16_t*>(ws + off); };
  hipError_t e;
#define LOSS_TRY(call, what) \
  if ((e = (call)) != hipSuccess) return hip_fail(e, what)

  if (p.n == 0) {  // no token: loss 0, dw 0
    if (a->loss) LOSS_TRY(launch_loss_zero(a->loss, 4, st), "zero launch");
    if (a->dw) LOSS_TRY(launch_loss_zero(a->dw, p.v * p.h * es, st), "zero launch");
    return MFSDP_OK;
  }
  const float inv_t = float(1.0 / l.temperature), factor = float(a->scale / l.temperature);
  float* const denom = a->reduction == MFSDP_MEAN ? f32p(p.denom) : nullptr;
  LossPrep prep{};
  prep.l = LossLabels{l.ids, l.logits, l.id_bytes == 8, l.logit_dtype == MFSDP_BF16, int32_t(k), p.n, p.v, l.ignore, inv_t};
  prep.n_pad = p.n_pad;
  prep.id = reinterpret_cast<int32_t*>(ws + p.id);
  prep.queues = reinterpret_cast<int32_t*>(ws + p.queues);
  prep.q = f32p(p.q);
  prep.ent = f32p(p.ent);
  prep.on = f32p(p.on);

  const int64_t xpart = p.chunk * p.hp, wpart = p.v * p.ldw, dzpart = p.chunk * p.vp;
  const uint16_t* const w = p.copy ? u16p(p.wb) : static_cast<const uint16_t*>(a->w);
  // P Q^T with Q = w (row-major) or x (panel blocked)
  auto product = [&](const Gemm& g, size_t P, int64_t ldp, int64_t ppart, int nseg, bool of_w, int nk) {
    LossGemm m{};
    m.P = u16p(P);
    m.ldp = ldp;
    m.ppart = ppart;
    m.Q = of_w ? w : u16p(p.xb);
    m.ldq = of_w ? p.ldw : p.hp;
    m.qrows = p.v;
    m.qpart = of_w ? wpart : xpart;
    m.unscale = f32p(p.inv) + (of_w ? 1 : 0);
    m.nseg = nseg;
    m.nk = nk;
    m.kper = g.splits > 1 ? g.kper : nseg * nk;
    m.splits = (nseg * nk + m.kper - 1) / m.kper;
    m.tm = g.tm;
    m.tn = g.tn;
    return m;
  };
  LossMaxima mm{};
  if (p.f32) {
    mm.l = prep.l;
    mm.x = static_cast<const float*>(a->x);
    mm.w = static_cast<const float*>(a->w);
    mm.h = p.h;
    mm.n_pad = p.n_pad;
    mm.xblocks = int(std::min<int64_t>(kLossMaxima, p.n_pad / 16));
    mm.wblocks = int(std::min<int64_t>(kLossMaxima, up(p.v * p.h, 16384) / 16384));
    mm.xmax = f32p(p.xmax);
    mm.wmax = f32p(p.wmax);
    LOSS_TRY(launch_loss_maxima(mm, st), "maxima launch");
  }
  for (int64_t r0 = 0; r0 < p.n; r0 += p.chunk) {
    const int64_t rows = std::min(p.chunk, p.n - r0), rows_pad = up(rows, p.stream ? p.chunk : 256);
    const bool first = r0 == 0, last = r0 + p.chunk >= p.n;
    const int32_t* ids = prep.id + r0 * k;
    const float* q = prep.q + r0 * k;

    prep.label_blocks = first ? int((p.n_pad + 3) / 4) : 0;
    prep.packs = 0;
    int blocks = prep.label_blocks;
    auto pack = [&](const void* src, int64_t R, int64_t rpad, size_t dst, int64_t ld, int64_t part, int64_t label_row) {
      LossPack& d = prep.d[prep.packs++];
      d.src = src;
      d.R = R;
      d.C = p.h;
      d.dst = u16p(dst);
      d.ld = ld;
      d.dst_part = part;
      d.cols = p.hp;
      d.label_row = label_row;
      d.blocks_begin = blocks;
      d.bf16 = !p.f32;
      d.blocked = label_row >= 0;
      d.row_most = d.blocked ? f32p(p.xmax) + r0 : nullptr;
      d.most = d.blocked ? nullptr : mm.wmax;
      d.count = mm.wblocks;
      d.inv = f32p(p.inv) + 1;
      blocks += int(rpad / 32 * (p.hp / 256));
    };
    pack(static_cast<const uint8_t*>(a->x) + r0 * p.h * es, rows, rows_pad, p.xb, p.hp, xpart, r0);
    if (first && p.copy) pack(a->w, p.v, up(p.v, 32), p.wb, p.ldw, wpart, -1);
    LOSS_TRY(launch_loss_prep(prep, blocks, st), "prep launch");

    if (p.stream) {
      LossStream z{};
      z.P = u16p(p.xb);
      z.w = w;
      z.ldp = p.hp;
      z.v = p.v;
      z.h = p.h;
      const int qrows = stream_rows(p.stream), kt = 16384 / qrows;
      z.nk = int(up(p.h, kt) / kt);
      z.tiles = int(up(p.v, qrows) / qrows);
      z.splits = 1;
      z.kper = z.nk;
      z.inv_t = inv_t;
      z.gm = f32p(p.gm);
      z.gs = f32p(p.gs);
      z.gstep = p.gstep;
      z.rstep = p.rstep;
      z.ids = ids;
      z.zt = f32p(p.zt);
      z.k = int32_t(k);
      z.codes = p.grads ? u16p(p.codes) : nullptr;
      z.ldc = p.vp;
      LOSS_TRY(launch_loss_stream(z, p.stream, kLossLogits, st), "logits launch");
    } else {
      LossGemm2 zz{};
      LossGemm& z = zz.g[0];
      z = product(p.logits, p.xb, p.hp, xpart, p.nseg, true, p.logits.nk);
      zz.count = 1;
      zz.queue = prep.queues;
      z.tm = int(up(rows, p.logits.tile) / p.logits.tile);
      z.row_most = f32p(p.xmax) + r0;
      z.rows = int(rows);
      z.cols = int(p.v);
      z.inv_t = inv_t;
      z.gm = f32p(p.gm);
      z.gs = f32p(p.gs);
      z.gstep = p.gstep;
      z.rstep = p.rstep;
      z.ids = ids;
      z.zt = f32p(p.zt);
      z.k = int32_t(k);
      z.ldc = p.vp;
      if (p.grads && p.f32) z.logits = f32p(p.z32);
      if (p.grads && !p.f32) z.codes = u16p(p.codes);
      if (z.splits > 1) z.part = f32p(p.part);
      LOSS_TRY(launch_loss_gemm(zz, kLossLogits, p.logits.tile, st), "logits launch");
      if (z.splits > 1) {
        LOSS_TRY(launch_loss_sum(z.part, int64_t(z.tm) * z.tn, p.logits.tile, z.splits, st), "logits sum launch");
        z.prev = z.part;
        z.part = nullptr;
        LOSS_TRY(launch_loss_gemm(zz, kLossLogits, p.logits.tile, st), "logits epilogue launch");
      }
    }

    LossRows rw{};
    rw.gm = f32p(p.gm);
    rw.gs = f32p(p.gs);
    rw.gstep = p.gstep;
    rw.rstep = p.rstep;
    rw.groups = int((p.v + p.group - 1) / p.group);
    rw.rows = int(rows);
    rw.rows_pad = int(rows_pad);
    rw.k = int32_t(k);
    rw.id = ids;
    rw.q = q;
    rw.ent = prep.ent + r0;
    rw.on = prep.on + r0;
    rw.weight = a->token_weight ? a->token_weight + r0 : nullptr;
    rw.zt = f32p(p.zt);
    rw.z_loss = float(l.z_loss);
    rw.row = reinterpret_cast<float4*>(ws + p.row);
    rw.token_loss = a->token_loss ? a->token_loss + r0 : nullptr;
    rw.lse = a->lse ? a->lse + r0 : nullptr;
    if (p.f32 && p.grads) {
      rw.row_most = f32p(p.row_most);
      rw.most = f32p(p.most);
      rw.x_most = f32p(p.xmax) + r0;
    }
    rw.weighted = f32p(p.weighted) + r0;
    rw.n = p.n;
    rw.all_on = prep.on;
    rw.all_weight = a->token_weight;
    rw.denom = first ? denom : nullptr;
    LOSS_TRY(launch_loss_rows(rw, st), "rows launch");
    const LossTotal total{f32p(p.weighted), denom, p.n, float(a->scale), last ? a->loss : nullptr};
    if (!p.grads) {
      if (total.loss) LOSS_TRY(launch_loss_total(total, st), "loss sum launch");
      continue;
    }

    LossGrad gr{};
    gr.codes = p.f32 ? nullptr : u16p(p.codes);
    gr.logits = p.f32 ? f32p(p.z32) : nullptr;
    gr.ldc = p.vp;
    gr.dz = u16p(p.codes);
    gr.dz_part = dzpart;
    gr.parts = p.dz_parts;
    gr.gm = rw.gm;
    gr.gstep = p.gstep;
    gr.rstep = p.rstep;
    gr.row = rw.row;
    gr.id = ids;
    gr.q = q;
    gr.zt = rw.zt;
    gr.k = int32_t(k);
    gr.rows = int(rows);
    gr.rows_pad = int(rows_pad);
    gr.v = int(p.v);
    gr.v_pad = int(p.vp);
    gr.group_shift = p.group == 32 ? 5 : 6;
    gr.row_most = rw.row_most;
    if (p.f32 && a->dw) {
      gr.x = prep.d[0];
      gr.x.label_row = -1;
      gr.x.row_most = rw.row_most;
      gr.x.most = rw.most;
      gr.x.count = loss_row_blocks(rw);
      gr.x.inv = f32p(p.inv);
    }
    gr.total = total;
    LOSS_TRY(launch_loss_grad(gr, st), "gradient launch");

    LossGemm mx{}, mw{};
    if (a->dx && !p.stream) {
      mx = product(p.dx, p.codes, p.vp, dzpart, p.out_nseg, true, p.dx.nk);
      mx.op = kLossDx;
      mx.row_most = rw.row_most;
      mx.tm = int(up(rows, p.dx.tile) / p.dx.tile);
      mx.rows = int(rows);
      mx.cols = int(p.h);
      mx.out = static_cast<uint8_t*>(a->dx) + r0 * p.h * es;
      mx.ldo = p.h;
      mx.out_bf16 = !p.f32;
      mx.alpha = factor;
      mx.denom = denom;
      if (mx.splits > 1) mx.part = f32p(p.part);
    }
    if (a->dw) {
      mw = product(p.dw, p.codes, p.vp, dzpart, p.out_nseg, false, int(up(rows, 32) / 32));
      mw.op = kLossDw;
      mw.rows = int(p.v);
      mw.cols = int(p.h);
      mw.out = a->dw;
      mw.ldo = p.h;
      mw.out_bf16 = !p.f32;
      mw.alpha = factor;
      mw.denom = denom;
      if (!first) mw.prev = f32p(p.acc);
      if (!last) mw.part = f32p(p.acc);
    }
    LossGemm2 both{};
    // dw of a few tokens on a kernel of its own (128256 x 4096, the whole call with dx and dw: 48 tokens 654 us, 865 with dw on
    // the tiles' kernel, 100 tokens 931 and 1073), unless its tiles go into dx's launch in one round (64 tokens, 1000 x 64, dx
    // and dw: 13 us in one launch, 20 in two)
    const bool short_dw = !p.f32 && first && last && rows <= kStreamTokens && (p.stream || !a->dx || p.dw.items() > 256);
    // otherwise one launch where both use the same tile, the longer tiles first
    const bool together = a->dx && a->dw && !p.stream && !short_dw && p.dx.tile == p.dw.tile;
    both.queue = prep.queues + kGemmXcds;
    if (a->dx && p.stream) {
      LossStream s{};
      s.P = u16p(p.codes);
      s.w = w;
      s.ldp = p.vp;
      s.ppart = dzpart;
      s.v = p.v;
      s.h = p.h;
      s.nk = p.dx.nk;
      s.tiles = p.dx.tn;
      s.splits = p.dx.splits;
      s.kper = p.dx.kper;
      s.part = f32p(p.part);
      s.ldo = p.hp;
      LOSS_TRY(launch_loss_stream(s, p.stream, kLossOut, st), "dx launch");
    } else if (a->dx) {
      const bool swap = together && mw.kper > mx.kper;
      both.g[swap ? 1 : 0] = mx;
      both.g[swap ? 0 : 1] = mw;
      both.count = together ? 2 : 1;
      LOSS_TRY(launch_loss_gemm(both, kLossOut, p.dx.tile, st), "dx launch");
    }
    if (a->dw && short_dw) {
      LOSS_TRY(launch_loss_dw(mw, rows <= 32 ? 1 : rows <= 64 ? 2 : 4, st), "dw launch");
    } else if (a->dw && !together) {
      both.g[0] = mw;
      both.count = 1;
      both.queue = prep.queues + 2 * kGemmXcds;
      LOSS_TRY(launch_loss_gemm(both, kLossOut, p.dw.tile, st), "dw launch");
    }
    if (a->dx && (p.stream || mx.splits > 1)) {
      LossJoin j{};
      j.part = f32p(p.part);
      j.splits = p.stream ? p.dx.splits : mx.splits;
      j.tiles = mx.tm * mx.tn;
      j.tm = mx.tm;
      j.tn = mx.tn;
      j.rows = int(rows);
      j.cols = int(p.h);
      j.out_bf16 = !p.f32;
      j.stride = p.chunk * p.hp;
      j.ldp = p.hp;
      j.out = static_cast<uint8_t*>(a->dx) + r0 * p.h * es;
      j.ldo = p.h;
      j.alpha = factor;
      j.denom = denom;
      LOSS_TRY(launch_loss_join(j, p.stream ? 0 : p.dx.tile, st), "dx join launch");
    }
  }
#undef LOSS_TRY
  return MFSDP_OK;
}

}  // namespace

extern "C" {

size_t mfsdp_head_loss_workspace_size(const mfsdp_head_loss* args, int32_t k) {
  if (check(args, k, false)) return 0;
  return std::max<size_t>(make_plan(args, k).bytes, 256);
}

int mfsdp_linear_xent(const mfsdp_head_loss* args, const void* targets, int32_t target_bytes, int64_t ignore_index,
                      double z_loss, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check(args, 1, true)) return rc;
  if (!targets && args->n > 0) return fail(MFSDP_E_INVALID, "targets is NULL");
  if (target_bytes != 4 && target_bytes != 8) return fail(MFSDP_E_INVALID, "target_bytes must be 4 or 8");
  if (!aligned16(targets)) return fail(MFSDP_E_INVALID, "pointers must be 16-byte aligned");
  if (!std::isfinite(float(z_loss)) || z_loss < 0.0) return fail(MFSDP_E_INVALID, "z_loss must be >= 0 and finite in fp32");
  return run(args, 1, Labels{targets, nullptr, target_bytes, 0, ignore_index, 1.0, z_loss}, workspace, workspace_bytes, stream);
}

int mfsdp_linear_distill(const mfsdp_head_loss* args, const void* ids, int32_t id_bytes, const void* logits,
                         int32_t logit_dtype, int32_t k, double temperature, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (const int rc = check(args, k, true)) return rc;
  if ((!ids || !logits) && args->n > 0) return fail(MFSDP_E_INVALID, "ids or logits is NULL");
  if (id_bytes != 4 && id_bytes != 8) return fail(MFSDP_E_INVALID, "id_bytes must be 4 or 8");
  if (logit_dtype != MFSDP_F32 && logit_dtype != MFSDP_BF16) return fail(MFSDP_E_INVALID, "unsupported logit dtype");
  if (!aligned16(ids) || !aligned16(logits)) return fail(MFSDP_E_INVALID, "pointers must be 16-byte aligned");
  // (the kernels multiply by its inverse)
  if (!(temperature > 0.0) || !std::isnormal(float(1.0 / temperature)) || !std::isfinite(float(args->scale / temperature)))
    return fail(MFSDP_E_INVALID, "temperature must be > 0, 1 / temperature normal and scale / temperature finite in fp32");
  return run(args, k, Labels{ids, logits, id_bytes, logit_dtype, 0, temperature, 0.0}, workspace, workspace_bytes, stream);
}

int mfsdp_scale_grad(void* grad, int64_t numel, int32_t dtype, const float* factor, void* stream) {
  if (numel < 0) return fail(MFSDP_E_INVALID, "numel must be >= 0");
  if (dtype != MFSDP_F32 && dtype != MFSDP_BF16) return fail(MFSDP_E_INVALID, "unsupported dtype");
  if (!factor || (numel > 0 && !grad)) return fail(MFSDP_E_INVALID, "NULL pointer");
  if (!aligned16(grad)) return fail(MFSDP_E_INVALID, "pointers must be 16-byte aligned");
  const hipError_t e = launch_scale_grad(grad, numel, dtype == MFSDP_BF16, factor, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? MFSDP_OK : hip_fail(e, "scale launch");
}

}  // extern "C"
