// Losses over a vocabulary from hidden states and an output head, with both gradients, without the n x v logits
// (loss_internal.h says what is held where).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "loss_internal.h"

namespace mfsdp {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// row-major tensors of any width: vectors at their elements' alignment
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
using gptr = __attribute__((address_space(1))) T*;
template <typename T>
using lptr = __attribute__((address_space(3))) T*;
typedef __attribute__((address_space(3))) uint8_t lds_byte;

template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kBKE = 32;          // K elements per stage
constexpr int kRowB = kBKE * 2;   // bytes per staged row
constexpr int kStages = 5;

// Slot of 16-byte chunk c of row r in LDS: c ^ swz(r) (bank-conflict-free fragment reads).
__device__ __forceinline__ int swz(int r) { return ((r >> 1 ^ r >> 3) & 1) | (((r >> 2) & 1) << 1); }
#define LOSS_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 0xF) | (((n) >> 4) << 14) | (7 << 4) | (0xF << 8))
#define LOSS_WAIT_LGKM0() __builtin_amdgcn_s_waitcnt(0xF | (7 << 4) | (0 << 8) | (3 << 14))

// A transposing read (four rows by one column per lane and 16 lanes). Through a restrict pointer: without alias information
// of their own the compiler takes these reads to depend on every load into LDS in flight and waits for all of them (8192 x
// 4096 x 128256: 0.99 PFLOP/s so, 1.47 without those waits, as with plain reads of a transposed copy).
__device__ __forceinline__ bf16x4_t read_tr(lptr<bf16x4_t> __restrict p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(p);
}
__device__ __forceinline__ bf16x8_t join_tr(bf16x4_t lo, bf16x4_t hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// NW waves, 2 x NW/2, on a TB x TB tile; a wave's part is MI x 2 blocks of 32 x 32.
template <int NW, int TB>
struct Grid {
  static constexpr int WN = NW / 2;
  static constexpr int MI = TB / 64, NI = 2;
  static_assert(WN * 64 == TB, "64 columns a wave");
  static constexpr int HALF = TB * kRowB;                 // bytes of one operand's step of 32
  static constexpr int STAGE = 2 * HALF;
  static constexpr int DW = NW == 8 ? 4 : NW;             // waves that issue the loads
  static constexpr int PL = TB / kBlkRows / DW;           // loads of P (and of Q) per issuing wave and step
  static constexpr int DLOADS = 2 * PL;
  static constexpr int SLOTS = (TB == kLossTile ? 1 : 2) * kGemmSlots;  // workgroups per XCD
  static constexpr int BAND = TB == kLossTile ? 4 : 8;    // block rows of a locality band
};

// alpha / denom, 0 where denom is 0
__device__ __forceinline__ float out_factor(float alpha, const float* denom) {
  if (!denom) return alpha;
  const float d = *denom;
  return d != 0.0f ? alpha / d : 0.0f;
}

// two logits' 16-bit codes from their distances in [0, 1]
__device__ __forceinline__ uint32_t code2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pknorm_u16(a, b));
}

// a lane's value joined with the other half wave's
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The scale that brings values of at most `most` to at most 2^15, and its inverse; both normal numbers.
__device__ __forceinline__ float scale_for(float most, float& inv) {
  int e = int(__float_as_uint(most) >> 23) - 126;  // most < 2^e
  e = most > 0.0f ? max(e, -100) : 15;
  inv = __uint_as_float(uint32_t(127 + e - 15) << 23);
  return __uint_as_float(uint32_t(127 + 15 - e) << 23);
}
// the magnitude of a finite value, 0 for others
__device__ __forceinline__ float finite_mag(float x) { return fabsf(x) < __builtin_inff() ? fabsf(x) : 0.0f; }

struct Item {
  int p, bi, bj, k0, nk;  // problem, tile, K steps
};

// Tiles of P Q^T on a persistent grid, all operands as they lie:
//   logits  P = x (panel blocked),  Q = w, rows of K;             K = h
//   dx      P = dz (panel blocked), Q = w, read transposed;       K = v
//   dw      P = dz, Q = x (panel blocked), both read transposed;  K = tokens
// LDS is filled by direct loads, from one wave of each SIMD, of whole 1 KiB blocks of a panel-blocked operand (16 rows by 32
// columns) or of whole 128-byte lines of w. One barrier per K step of 32 inside its second 16-wide slice; the next step's
// fragments are read while the rest of that slice multiplies, and the next tile's first loads are issued before this
// tile's epilogue. dx, dw: a ring of five steps, filled four steps ahead. logits: w's lines span two steps, so w has a ring
// of three pairs of steps and x one of four steps (three ahead).
// The order in the loops is the instruction order: left to itself the compiler gathers the loads (which write LDS) between
// the LDS reads, and the MFMAs wait behind them (8192 x 4096 x 128256: 1.19 PFLOP/s so, 1.50 in this order).
// Tiles are dealt to the XCDs in groups that share operand panels in L2 (bands of BAND block rows, column by
// column) and taken from counters, so that long and short tiles (the K ranges of dx, the tiles of dw) share the chip evenly.
template <int NW, int TB, int NSEG, int KIND>
__global__ __launch_bounds__(NW * 64, TB == kLossTile ? 1 : 2) void loss_gemm_kernel(const LossGemm2 b) {
  using G = Grid<NW, TB>;
  constexpr int MI = G::MI, NI = G::NI, HALF = G::HALF, STAGE = G::STAGE, DW = G::DW, PL = G::PL, DLOADS = G::DLOADS;
  constexpr bool F16 = NSEG == kLossMaxSeg;
  constexpr int kSlabAt = (kStages - 1) * STAGE;  // the part of LDS that no tile's first loads touch
  constexpr int kQAt = 4 * HALF;                  // logits: w's pairs of steps behind x's four steps
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * STAGE];

  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = w / G::WN, wn = w % G::WN;
  // (a launch that goes on from the sum over K ranges has one item per tile)
  const int first = b.g[0].tm * b.g[0].tn * (KIND == kLossLogits && b.g[0].prev ? 1 : b.g[0].splits);
  const int total = first + (KIND == kLossOut && b.count > 1 ? b.g[1].tm * b.g[1].tn * b.g[1].splits : 0);
  const int per = min(G::SLOTS, (total + kGemmXcds - 1) / kGemmXcds);  // items of one group
  const int groups = (total + per - 1) / per;

  // Items are dealt in groups that run together on one XCD: group g belongs to XCD g % 8. A workgroup's first item is its
  // place in its XCD's first group; the next ones come from a counter of its XCD or, once that has run out, of the XCD with
  // the most items left. (One lane asks; -1: none left.)
  const int home = blockIdx.x % kGemmXcds, place = blockIdx.x / kGemmXcds;
  if (place >= per) return;
  auto left_in = [&](int x, int taken) {  // XCD x's items beyond its first group that are not taken yet
    const int ng = (groups - x + kGemmXcds - 1) / kGemmXcds;
    return (ng - 1) * per - ((groups - 1) % kGemmXcds == x ? groups * per - total : 0) - taken;
  };
  bool home_out = false;
  gptr<int> q = (gptr<int>)b.queue;
  auto ask = [&](int x) { return __hip_atomic_fetch_add(q + x, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  auto item_of = [&](int x, int i) { return ((i / per + 1) * kGemmXcds + x) * per + i % per; };
  auto take = [&](int i) -> int {  // i: what home's counter gave, if it was asked
    for (int x = home;;) {
      if (home_out) {
        int most = 0;
#pragma unroll
        for (int y = 0; y < kGemmXcds; ++y) {
          const int n = left_in(y, __hip_atomic_load(q + y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
          if (n > most) {
            most = n;
            x = y;
          }
        }
        if (most == 0) return -1;
        i = ask(x);
      }
      if (left_in(x, i) > 0) return item_of(x, i);
      home_out = true;
    }
  };
  auto item_at = [&](int i, Item& it) -> bool {
    if (i < 0 || i >= total) return false;
    it.p = KIND == kLossOut && i >= first ? 1 : 0;
    const LossGemm& a = b.g[it.p];
    if (it.p) i -= first;
    const int tiles = a.tm * a.tn, steps = NSEG * a.nk;
    const int s = i / tiles, j = i - s * tiles;
    const int band = j / (G::BAND * a.tn), r0 = band * G::BAND, hb = min(G::BAND, a.tm - r0);
    const int jj = j - r0 * a.tn;
    it.bj = jj / hb;
    it.bi = r0 + jj - it.bj * hb;
    it.k0 = s * a.kper;
    it.nk = min(a.kper, steps - it.k0);
    return true;
  };

  const bool issuer = w < DW;
  // Lane offsets (bytes) of a load: a 1 KiB block (lane l: row l / 4, 16-byte chunk (l % 4) ^ swz(row), so that the plain
  // fragment reads are conflict-free); eight 128-byte lines of w (row l / 8, chunk (l % 8) ^ (row / 2) % 8); 64 lanes along
  // TB columns of w's rows (chunk ^ 4 (row % 4)). Loads past w's last 16 bytes are held there: what they bring meets zeros of
  // x or dz, or belongs to columns that are not stored.
  const uint32_t loff = (lane >> 2) * kRowB + ((lane & 3) ^ swz(lane >> 2)) * 16;
  constexpr int RPL = 512 / TB;  // rows of w per load of TB columns
  // of the tile whose loads are being issued
  uint32_t qlane = 0, prow32 = 0, qrow2 = 0, qrow32 = 0;
  const char *pbase = nullptr, *qbase = nullptr;
  int64_t wleft = 0, ppart = 0, qpart = 0, pstep = 0, qstep = 0;  // bytes: of w from qbase; between parts; of one step
  int seg_steps = 1;
  bool dw = false;
  auto aim = [&](const Item& it) {
    const LossGemm& a = b.g[it.p];
    dw = KIND == kLossOut && a.op == kLossDw;
    prow32 = uint32_t(a.ldp * 32);   // a 16-row panel
    qrow2 = uint32_t(a.ldq * 2);
    qrow32 = uint32_t(a.ldq * 32);
    ppart = a.ppart * 2;
    qpart = a.qpart * 2;
    seg_steps = a.nk;
    if (dw) {
      pbase = (const char*)(a.P + int64_t(it.bi) * (TB * kBlkRows));
      qbase = (const char*)(a.Q + int64_t(it.bj) * (TB * kBlkRows));
      pstep = a.ldp * 64;
      qstep = a.ldq * 64;
    } else {
      pbase = (const char*)(a.P + (int64_t(it.bi) * TB + w * kBlkRows) * a.ldp);
      pstep = 1024;
      const int64_t row = a.ldq * 2, at = KIND == kLossLogits ? int64_t(it.bj) * TB * row : int64_t(it.bj) * TB * 2;
      qbase = (const char*)a.Q + at;
      qstep = row * 32;
      wleft = a.qrows * row - at;
      if constexpr (KIND == kLossLogits)
        qlane = uint32_t((w * 8 + (lane >> 3)) * row) + ((lane & 7) ^ (((w & 1) * 4 + (lane >> 4)) & 7)) * 16;
      else
        qlane = uint32_t((w * RPL + lane / (TB / 8)) * row) +
                ((lane % (TB / 8)) ^ (((w * RPL + lane / (TB / 8)) & 3) << 2)) * 16;
    }
  };
  auto load = [&](const char* base, uint32_t voff, uint32_t soff, int at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffffu, 0x00020000),
                                             (lds_byte*)(smem + at), 16, voff, soff, 0, 0);
  };
  // Step k of all segments: the step in its segment, and the bytes to its parts of P and Q. fp32 operands lie in two fp16
  // parts (F16), few tokens' dz in two bf16 parts; the pairs (1, 0), (0, 1) (F16), (0, 0): the small products first, while
  // the sum is small.
  auto in_segment = [&](int k, int64_t& po, int64_t& qo) {
    po = qo = 0;
    if constexpr (NSEG > 1) {
      const int sg = k / seg_steps;
      po = sg == 0 ? ppart : 0;
      qo = F16 && sg == 1 ? qpart : 0;
      k -= sg * seg_steps;
    }
    return k;
  };
  // load i (of PL) of step k of P, of Q, into `at`. A blocked operand's next step is one block further along each panel, or
  // (read transposed) two panels further down; load i moves block i DW + w of the step.
  auto issue_blocked = [&](const char* base, uint32_t row32, int i, int at, auto trans_c) {
    const int blk = i * DW + w;
    if constexpr (decltype(trans_c)::value)
      load(base, loff, uint32_t(blk / (TB / 32)) * row32 + (blk % (TB / 32)) * 1024, at + blk * 1024);
    else
      load(base, loff, uint32_t(i * DW) * row32, at + blk * 1024);
  };
  auto issue_p = [&](int i, int k, int at, auto trans_c) {
    int64_t po, qo;
    const int kk = in_segment(k, po, qo);
    issue_blocked(pbase + po + kk * pstep, prow32, i, at, trans_c);
  };
  auto issue_q = [&](int i, int k, int at, auto trans_c) {  // dx, dw
    int64_t po, qo;
    const int kk = in_segment(k, po, qo);
    const int64_t off = kk * qstep;
    if constexpr (decltype(trans_c)::value) {
      issue_blocked(qbase + qo + off, qrow32, i, at, trans_c);
    } else {  // rows (i DW + w) RPL .. of the 32
      const int64_t left = wleft - off;
      const uint32_t most = uint32_t(left < 0x7ffffff0 ? left : 0x7ffffff0) - 16, v = qlane + uint32_t(i * DW * RPL) * qrow2;
      load(qbase + qo + off, v < most ? v : most, 0, at + (i * DW + w) * 1024);
    }
  };
  auto issue_w = [&](int i, int u, int at) {  // logits: load i (of 2 PL) of pair u of steps
    int64_t po, qo;
    const int kk = in_segment(u * 2, po, qo);
    const uint32_t most = uint32_t(wleft < 0x7ffffff0 ? wleft : 0x7ffffff0) - 16;
    const uint32_t v = qlane + uint32_t(i * DW * 8) * qrow2 + uint32_t(kk) * 64;
    load(qbase + qo, v < most ? v : most, 0, at + (i * DW + w) * 1024);
  };
  // the first steps of a tile (past its end: its last step again, into places nobody reads)
  auto prologue = [&](const Item& it) {
    aim(it);
    if constexpr (KIND == kLossLogits) {
      const int units = it.nk / 2, u0 = it.k0 / 2;
#pragma unroll
      for (int i = 0; i < 2 * PL; ++i) issue_w(i, u0, kQAt);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < PL; ++i) issue_p(i, it.k0 + s, s * HALF, std::false_type{});
#pragma unroll
      for (int i = 0; i < 2 * PL; ++i) issue_w(i, u0 + min(1, units - 1), kQAt + 2 * HALF);
#pragma unroll
      for (int i = 0; i < PL; ++i) issue_p(i, it.k0 + min(2, it.nk - 1), 2 * HALF, std::false_type{});
    } else {
      auto steps = [&](auto trans_c) {
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) {
          const int k = it.k0 + min(s, it.nk - 1);
#pragma unroll
          for (int i = 0; i < PL; ++i) issue_p(i, k, s * STAGE, trans_c);
#pragma unroll
          for (int i = 0; i < PL; ++i) issue_q(i, k, s * STAGE + HALF, trans_c);
        }
      };
      if (dw) steps(std::true_type{});
      else steps(std::false_type{});
    }
  };

  // Fragment addresses: plain (row lane % 32 of a block of 32, chunk 2 slice + lane / 32) and transposed (lane: rows lane / 4
  // % 4 (+ 4) + 8 (lane / 32), columns 4 (lane % 4) + 16 (lane / 16 % 2) of 32).
  const int frow = lane & 31, fhalf = lane >> 5;
  const int prow = (wm * (MI * 32) + frow) * kRowB, slot0 = ((0 + fhalf) ^ swz(frow)) * 16, slot1 = ((2 + fhalf) ^ swz(frow)) * 16;
  const int trow = (lane >> 5) * 8 + ((lane >> 2) & 3), tchunk = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1), tbyte = (lane & 1) * 8;
  const int tlo = trow * kRowB + ((tchunk ^ swz(trow)) << 4) + tbyte;            // in a 1 KiB block
  const int thi = (trow + 4) * kRowB + ((tchunk ^ swz(trow + 4)) << 4) + tbyte;
  auto frag_blocked = [&](int at, int block) {
    lds_byte* q = (lds_byte*)(smem + at) + block * 1024;
    return join_tr(read_tr((lptr<bf16x4_t>)(q + tlo)), read_tr((lptr<bf16x4_t>)(q + thi)));
  };
  auto frag_p = [&](int at, int i, int sl, auto trans_c) -> bf16x8_t {
    if constexpr (decltype(trans_c)::value) return frag_blocked(at, sl * (TB / 32) + wm * MI + i);
    else return *reinterpret_cast<const bf16x8_t*>(smem + at + prow + (sl ? slot1 : slot0) + i * 32 * kRowB);
  };
  auto frag_q = [&](int at, int j, int sl, auto trans_c) -> bf16x8_t {  // dx, dw
    if constexpr (decltype(trans_c)::value) {
      return frag_blocked(at, sl * (TB / 32) + wn * NI + j);
    } else {  // w's rows of TB columns
      const int s16 = (wn * NI + j) * 4 + tchunk;
      lds_byte* q = (lds_byte*)(smem + at) + (sl * 16 + trow) * (TB * 2) + ((s16 ^ ((trow & 3) << 2)) << 4) + tbyte;
      return join_tr(read_tr((lptr<bf16x4_t>)q), read_tr((lptr<bf16x4_t>)(q + 4 * (TB * 2))));
    }
  };
  const int wrow = (wn * (NI * 32) + frow) * 128, wswz = (frow >> 1) & 7;
  auto frag_w = [&](int at, int j, int sl) {  // slice sl (of 4) of a pair of steps
    return *reinterpret_cast<const bf16x8_t*>(smem + at + wrow + (((sl * 2 + fhalf) ^ wswz) << 4) + j * 32 * 128);
  };
  constexpr int NMF = MI * NI, NRD = MI + NI;  // MFMAs and fragments per 16-wide slice
  static_assert(DLOADS == NMF && PL == NMF / 2, "half of the loads in each half");

  // logits in K ranges (small tiles only): the launch that goes on from their sum
  constexpr bool RANGES = KIND == kLossLogits && TB == kLossTileSmall;
  const bool summed = RANGES && b.g[0].prev;

  Item cur, nxt;
  if (!item_at(home * per + place, cur)) return;
  if (issuer && !summed) prologue(cur);
  // (the last part of LDS is free whenever items are taken; the last wave asks: of eight waves it issues no loads to wait
  // behind)
  int* mail = reinterpret_cast<int*>(smem + kSlabAt);
  const bool asks = threadIdx.x == (NW - 1) * 64, queued = groups > kGemmXcds;
  bool has_next = false;
  if (queued) {
    if (asks) mail[0] = take(ask(home));
    LOSS_WAIT_LGKM0();
    __builtin_amdgcn_s_barrier();
    has_next = item_at(__builtin_amdgcn_readfirstlane(mail[0]), nxt);
  }
  while (true) {
    f32x16_t acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    bf16x8_t pf[2][MI], qf[2][NI];  // fragments of the two slices
    auto mfma = [&](int m, int sl) {
      const int i = m / NI, j = (i & 1) ? NI - 1 - m % NI : m % NI;
      if constexpr (F16)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, qf[sl][j]),
                                                           __builtin_bit_cast(f16x8_t, pf[sl][i]), acc[i][j], 0, 0, 0);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[sl][j], pf[sl][i], acc[i][j], 0, 0, 0);
    };
    // One step: the first slice with the second one's reads and P's loads; half of the second slice with Q's loads; the
    // barrier; the rest with the next step's first reads. wait_c: loads that may still be in flight for the next step to have
    // landed.
    auto step = [&](auto iss_c, auto wait_c, auto read1, auto read0, auto load_p, auto load_q) {
      constexpr bool ISS = decltype(iss_c)::value;
      __builtin_amdgcn_sched_barrier(0);
      static_for<NMF>([&](auto tc) {
        constexpr int t = decltype(tc)::value;
        mfma(t, 0);
        if constexpr (t < NRD) read1(t);
        if constexpr (ISS && t % 2 == 1) load_p(t / 2);
        __builtin_amdgcn_sched_barrier(0);
      });
      static_for<NMF / 2>([&](auto tc) {
        constexpr int t = decltype(tc)::value;
        mfma(t, 1);
        if constexpr (ISS) load_q(t);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (ISS) LOSS_WAIT_VMCNT(decltype(wait_c)::value);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      static_for<NMF / 2>([&](auto tc) {
        constexpr int t = decltype(tc)::value, R0 = t * NRD / (NMF / 2), R1 = (t + 1) * NRD / (NMF / 2);
        mfma(NMF / 2 + t, 1);
#pragma unroll
        for (int r = R0; r < R1; ++r) read0(r);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // where this wave's part of a tile of sums lies: range 0 of the item's tile, in accumulator order
    auto part_at = [&](int splits) {
      return int64_t((cur.bj * b.g[cur.p].tm + cur.bi) * splits) * (TB * TB) + (w * MI * NI * 4 * 64 + lane) * 4;
    };
    auto load_sum = [&](const float* sum) {
#pragma unroll
      for (int q = 0; q < MI * NI * 4; ++q) {
        const f32x4_t v = *(gptr<const f32x4_t>)(sum + q * 256);
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[q / (NI * 4)][(q >> 2) & 1][4 * (q & 3) + t] = v[t];
      }
    };
    auto store_part = [&](float* part) {
#pragma unroll
      for (int q = 0; q < MI * NI * 4; ++q) {
        const f32x16_t& c = acc[q / (NI * 4)][(q >> 2) & 1];
        *(gptr<f32x4_t>)(part + q * 256) = f32x4_t{c[4 * (q & 3)], c[4 * (q & 3) + 1], c[4 * (q & 3) + 2], c[4 * (q & 3) + 3]};
      }
    };
    if constexpr (KIND == kLossLogits) {
      auto main_loop = [&](auto iss_c) {
        using Wait = std::integral_constant<int, 2 * DLOADS>;  // the loads of this step and the last one
        const int nk = cur.nk, units = nk / 2, k0 = cur.k0;
        if constexpr (decltype(iss_c)::value) LOSS_WAIT_VMCNT(4 * PL);
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int r = 0; r < NRD; ++r) {
          if (r < MI) pf[0][r] = frag_p(0, r, 0, std::false_type{});
          else qf[0][r - MI] = frag_w(kQAt, r - MI, 0);
        }
        int qs = 0;  // this pair's place of w
        for (int u = 0; u < units; ++u) {
          const int qn = qs == 2 ? 0 : qs + 1, qfar = qs == 0 ? 2 : qs - 1;
          static_for<2>([&](auto hc) {
            constexpr int h = decltype(hc)::value;
            const int k = u * 2 + h, at = (k & 3) * HALF, an = ((k + 1) & 3) * HALF, af = ((k + 3) & 3) * HALF;
            const int w1 = kQAt + qs * (2 * HALF), w0 = kQAt + (h ? qn : qs) * (2 * HALF);
            step(iss_c, Wait{},
                 [&](int r) {
                   if (r < MI) pf[1][r] = frag_p(at, r, 1, std::false_type{});
                   else qf[1][r - MI] = frag_w(w1, r - MI, h * 2 + 1);
                 },
                 [&](int r) {
                   if (r < MI) pf[0][r] = frag_p(an, r, 0, std::false_type{});
                   else qf[0][r - MI] = frag_w(w0, r - MI, h ? 0 : 2);
                 },
                 [&](int i) { issue_p(i, k0 + min(k + 3, nk - 1), af, std::false_type{}); },
                 [&](int i) { issue_w(h * PL + i, k0 / 2 + min(u + 2, units - 1), kQAt + qfar * (2 * HALF)); });
          });
          qs = qn;
        }
      };
      if (summed) load_sum(b.g[0].prev + part_at(b.g[0].splits));
      else if (issuer) main_loop(std::true_type{});
      else main_loop(std::false_type{});
    } else {
      auto main_loop = [&](auto iss_c, auto trans_c) {
        using Wait = std::integral_constant<int, (kStages - 2) * DLOADS>;
        const int nk = cur.nk, last = cur.k0 + nk - 1;
        if constexpr (decltype(iss_c)::value) LOSS_WAIT_VMCNT((kStages - 2) * DLOADS);
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int r = 0; r < NRD; ++r) {
          if (r < MI) pf[0][r] = frag_p(0, r, 0, trans_c);
          else qf[0][r - MI] = frag_q(HALF, r - MI, 0, trans_c);
        }
        int cs = 0, ns = 1, fs = kStages - 1;  // stages of steps kt, kt + 1, kt + kStages - 1
        for (int kt = 0; kt < nk; ++kt) {
          const int kl = min(cur.k0 + kt + kStages - 1, last);
          const int at = cs * STAGE, an = ns * STAGE, af = fs * STAGE;
          step(iss_c, Wait{},
               [&](int r) {
                 if (r < MI) pf[1][r] = frag_p(at, r, 1, trans_c);
                 else qf[1][r - MI] = frag_q(at + HALF, r - MI, 1, trans_c);
               },
               [&](int r) {
                 if (r < MI) pf[0][r] = frag_p(an, r, 0, trans_c);
                 else qf[0][r - MI] = frag_q(an + HALF, r - MI, 0, trans_c);
               },
               [&](int i) { issue_p(i, kl, af, trans_c); }, [&](int i) { issue_q(i, kl, af + HALF, trans_c); });
          cs = ns;
          ns = (ns + 1 == kStages) ? 0 : ns + 1;
          fs = (fs + 1 == kStages) ? 0 : fs + 1;
        }
      };
      auto by_op = [&](auto iss_c) {
        if (b.g[cur.p].op == kLossDw) main_loop(iss_c, std::true_type{});
        else main_loop(iss_c, std::false_type{});
      };
      if (issuer) by_op(std::true_type{});
      else by_op(std::false_type{});
    }
    // this tile's last loads have landed and its fragments are read before the next tile's loads reuse the stages
    LOSS_WAIT_VMCNT(0);
    __builtin_amdgcn_s_barrier();
    if (has_next && issuer) prologue(nxt);  // (leaves the last part of LDS to the epilogue)
    int after = 0;  // the item after that: home's counter is asked here and looked at behind the epilogue
    if (has_next && asks && !home_out) after = ask(home);

    // acc[mi][ni][4 gg + t] of a lane is element (row, column) of the wave's part with row = 32 mi + lane % 32,
    // column = 32 ni + 8 gg + 4 (lane / 32) + t.
    lds_byte* slab = (lds_byte*)(smem + kSlabAt);
    int ln = lane;
    asm volatile("" : "+v"(ln));  // lane-dependent offsets are formed here, not kept through the main loop
    const int er = ln & 31, eh = ln >> 5;
    const LossGemm& a = b.g[cur.p];
    // fp32: 1 / (the scales of row r of P and of Q)
    const float q_inv = F16 ? *a.unscale : 1.0f;
    auto unscale = [&](int r) {
      float inv = 1.0f;
      if (a.row_most) scale_for(a.row_most[r], inv);
      return inv * q_inv;
    };
    if (RANGES && a.part) {
      store_part(a.part + part_at(a.splits) + cur.k0 / a.kper * (TB * TB));
    } else if constexpr (KIND == kLossLogits) {
      const int c0 = cur.bj * TB + wn * 64;       // the wave's first column
      const int left = a.cols - c0;               // real columns from there
      const int wsw = swz((wm * 32 + er) & 15);
      auto slab_off = [](int sr, int c) -> int {
        return (((sr >> 4) * (TB / 32) + (c >> 5)) << 10) + ((sr & 15) << 6) + ((((c & 31) >> 3) ^ swz(sr & 15)) << 4) +
               ((c & 7) << 1);
      };
      const int wr_base = slab_off(wm * 32 + er, wn * 64 + eh * 4);
      const int row0 = cur.bi * TB + wm * (MI * 32) + er;
      // the rows' first targets, all asked for before any is needed
      int id0[MI];
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) id0[mi] = *(gptr<const int32_t>)(a.ids + int64_t(row0 + mi * 32) * a.k);
      float inv_ts[MI];
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) inv_ts[mi] = F16 ? a.inv_t * unscale(row0 + mi * 32) : a.inv_t;
      if (left < 64) {  // columns past the vocabulary
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if ((e >> 4) * 32 + ((e & 15) >> 2) * 8 + eh * 4 + (e & 3) >= left) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) acc[mi][e >> 4][e & 15] = -__builtin_inff();
          }
      }
      float top[MI];
      static_for<MI>([&](auto mi_c) {
        constexpr int mi = decltype(mi_c)::value;
        const int row = row0 + mi * 32;
        const float inv_t = inv_ts[mi], L = kLog2e * inv_t;
        // the row's first 16 targets, on their way during the softmax (past the last one lie the next row's, or the
        // workspace's next array)
        i32x4 at[4] = {};
        auto load_ids = [&](int j0) {
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (j0 + v * 4 < a.k) at[v] = *(gptr<const i32x4_a4>)(a.ids + int64_t(row) * a.k + j0 + v * 4);
        };
        if (a.k > 1) load_ids(0);
        else at[0][0] = id0[mi];
        float u[32];  // logits before the temperature
#pragma unroll
        for (int e = 0; e < 32; ++e) u[e] = acc[mi][e >> 4][e & 15];
        float m = u[0];
#pragma unroll
        for (int e = 1; e < 32; ++e) m = fmaxf(m, u[e]);
        m = half_max(m);
        const float ref = top[mi] = fmaxf(m, -3.4e38f);  // (64 logits of -inf: terms of 0)
        // Sum of the others' exp: the largest term itself is 1, and what is far below it must not vanish in that 1. A
        // term's fraction is the term, but 0 for a 1; how many ones there are (equal logits) is what the two sums differ by.
        float s = 0.0f, all = 0.0f;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const float x = __builtin_amdgcn_exp2f((u[e] - ref) * L);
          s += __builtin_amdgcn_fractf(x);
          all += x;
        }
        const float ones = half_sum(__builtin_rintf(all - s));
        s = half_sum(s);
        if (left > 0 && eh == 0) {
          const int64_t at = int64_t(c0 >> 6) * a.gstep + row * a.rstep;
          a.gm[at] = m * inv_t;
          a.gs[at] = s + (ones - 1.0f);
        }
        // the row's targets among the wave's columns, 16 at a time, then one by one, in one place of the code (a small call
        // spends its time on fetching instructions)
        for (int j0 = 0; j0 < a.k; j0 += 16) {
          if (j0 > 0) load_ids(j0);
          uint32_t hits = 0;
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (v == 0 || j0 + v * 4 < a.k) {
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                at[v][t] -= c0;
                hits |= uint32_t(at[v][t]) < 64u ? 1u << (v * 4 + t) : 0u;
              }
            }
          if (a.k - j0 < 16) hits &= (1u << (a.k - j0)) - 1;
          while (hits) {
            const int i = __builtin_ctz(hits), j = j0 + i;
            hits &= hits - 1;
            int x = at[0][0];
#pragma unroll
            for (int f = 1; f < 16; ++f) x = i == f ? at[f >> 2][f & 3] : x;
            if (((x >> 2) & 1) != eh) continue;  // (the other half wave's column)
            const int e = (x >> 5) * 16 + ((x >> 3) & 3) * 4 + (x & 3);
            float z = 0.0f;
#pragma unroll
            for (int f = 0; f < 32; ++f) z = e == f ? u[f] : z;
            a.zt[int64_t(row) * a.k + j] = z * inv_t;
          }
        }
        if (F16 && a.logits) {
          float* dst = a.logits + int64_t(row) * a.ldc + c0;
#pragma unroll
          for (int p = 0; p < 8; ++p)
            *(gptr<f32x4_t>)(dst + (p >> 2) * 32 + (p & 3) * 8 + eh * 4) =
                f32x4_t{u[4 * p] * inv_t, u[4 * p + 1] * inv_t, u[4 * p + 2] * inv_t, u[4 * p + 3] * inv_t};
        }
      });
      if (!F16 && a.codes) {
        static_for<MI>([&](auto mi_c) {
          constexpr int mi = decltype(mi_c)::value;
          // round(65535 x) for x in [0, 1], clamped: x = 1 is kLossOctaves factors of two below the largest
          const float C = -kLog2e * a.inv_t * (1.0f / kLossOctaves), m = top[mi];
#pragma unroll
          for (int p = 0; p < 8; ++p) {
            const f32x16_t& u = acc[mi][p >> 2];
            const int o = 4 * (p & 3);
            *(lptr<u32x2>)(slab + wr_base + (p >> 2) * 1024 + ((((p & 3) ^ wsw) - wsw) << 4)) =
                u32x2{code2((u[o] - m) * C, (u[o + 1] - m) * C), code2((u[o + 2] - m) * C, (u[o + 3] - m) * C)};
          }
          // (the wave's own four blocks: its LDS writes and reads are in order, and no wave waits for another)
          const int rin = ln >> 2, ch = ln & 3;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int sp = wm * 2 + (b >> 1), cb = wn * 2 + (b & 1), blk = sp * (TB / 32) + cb;
            const u32x4 val = *(lptr<u32x4>)(slab + (blk << 10) + (rin << 6) + ((ch ^ swz(rin)) << 4));
            const int dr = (sp >> 1) * (MI * 32) + mi * 32 + (sp & 1) * 16 + rin;
            *(gptr<u32x4>)(a.codes + blk_index(int64_t(cur.bi) * TB + dr, int64_t(cur.bj) * TB + cb * 32 + ch * 8, a.ldc)) = val;
          }
        });
      }
    } else {
      const int i = (cur.bj * a.tm + cur.bi) * a.splits + cur.k0 / a.kper;  // tile and range
      const int64_t tile_at = int64_t(i) * (TB * TB) + (w * MI * NI * 4 * 64 + ln) * 4;
      if constexpr (F16) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const float f = unscale(cur.bi * TB + wm * (MI * 32) + i * 32 + er);
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] *= f;
        }
      }
      if (a.prev) {
#pragma unroll
        for (int q = 0; q < MI * NI * 4; ++q) {
          const f32x4_t p = *(gptr<const f32x4_t>)(a.prev + tile_at + q * 256);
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[q / (NI * 4)][(q >> 2) & 1][4 * (q & 3) + t] += p[t];
        }
      }
      if (!a.part) {
        const float f = out_factor(a.alpha, a.denom);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] *= f;
      }
      if (a.part) {
        store_part(a.part + tile_at);
      } else if (!a.out_bf16) {
        static_for<MI>([&](auto mi_c) {
          constexpr int mi = decltype(mi_c)::value;
          const int row = cur.bi * TB + wm * (MI * 32) + mi * 32 + er;
          if (row < a.rows) {
            float* dst = (float*)a.out + int64_t(row) * a.ldo;
#pragma unroll
            for (int p = 0; p < 8; ++p) {
              const int c = cur.bj * TB + wn * 64 + (p >> 2) * 32 + (p & 3) * 8 + eh * 4;
              const f32x16_t& v = acc[mi][p >> 2];
              const int o = 4 * (p & 3);
              if (c + 4 <= a.cols) {
                *(gptr<f32x4_a4>)(dst + c) = f32x4_a4{v[o], v[o + 1], v[o + 2], v[o + 3]};
              } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                  if (c + t < a.cols) *(gptr<float>)(dst + c + t) = v[o + t];
              }
            }
          }
        });
      } else {
        // bf16, row-major, through the free stage: each wave its own 32 rows of 128 bytes at a time, whole lines per store,
        // and no wave waits for another; 16-byte slots XORed by the row
        const int slab_w = w * 4096;
        auto at = [](int r, int s) { return r * 128 + ((s ^ r) & 7) * 16; };
        static_for<MI>([&](auto mi_c) {
          constexpr int mi = decltype(mi_c)::value;
#pragma unroll
          for (int p = 0; p < 8; ++p) {
            const f32x16_t& v = acc[mi][p >> 2];
            const int o = 4 * (p & 3);
            *(lptr<u32x2>)(slab + slab_w + at(er, p) + eh * 8) = u32x2{pack_bf16x2(v[o], v[o + 1]), pack_bf16x2(v[o + 2], v[o + 3])};
          }
#pragma unroll
          for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + (ln >> 3), s = ln & 7;
            const u32x4 val = *(lptr<u32x4>)(slab + slab_w + at(r, s));
            const int row = cur.bi * TB + wm * (MI * 32) + mi * 32 + r, c = cur.bj * TB + wn * 64 + s * 8;
            if (row < a.rows) {
              uint16_t* dst = (uint16_t*)a.out + int64_t(row) * a.ldo + c;
              if (c + 8 <= a.cols) {
                *(gptr<u32x4_a2>)dst = val;
              } else {
#pragma unroll
                for (int t = 0; t < 8; ++t)
                  if (c + t < a.cols) *(gptr<uint16_t>)(dst + t) = uint16_t(val[t >> 1] >> (16 * (t & 1)));
              }
            }
          }
        });
      }
    }
    // (every wave has left the last part of LDS)
    LOSS_WAIT_LGKM0();
    __builtin_amdgcn_s_barrier();
    if (!has_next) break;
    cur = nxt;
    if (asks) mail[0] = take(after);
    LOSS_WAIT_LGKM0();
    __builtin_amdgcn_s_barrier();
    has_next = item_at(__builtin_amdgcn_readfirstlane(mail[0]), nxt);
  }
  LOSS_WAIT_VMCNT(0);
}

__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  u32x4 o;
#pragma unroll
  for (int t = 0; t < 4; ++t) o[t] = pack_bf16x2(x[2 * t], x[2 * t + 1]);
  return o;
}
// the next of two bf16 parts, of scaled fp32 values' two fp16 parts; what is left of the values stays in x
__device__ __forceinline__ u32x4 split8_bf16(float (&x)[8]) {
  const u32x4 o = pack8(x);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    x[2 * t] -= __uint_as_float(o[t] << 16);
    x[2 * t + 1] -= __uint_as_float(o[t] & 0xffff0000u);
  }
  return o;
}
__device__ __forceinline__ u32x4 split8(float (&x)[8]) {
  f16x8_t o;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    o[t] = _Float16(x[t]);
    x[t] -= float(o[t]);
  }
  return __builtin_bit_cast(u32x4, o);
}
// Label entry `at` (token times k plus slot): its id; its teacher logit; whether it makes its token count.
__device__ __forceinline__ int64_t label_id(const LossLabels& l, int64_t at) {
  return l.id64 ? ((const int64_t*)l.ids)[at] : int64_t(((const int32_t*)l.ids)[at]);
}
__device__ __forceinline__ float label_logit(const LossLabels& l, int64_t at) {
  return l.logits_bf16 ? __uint_as_float(uint32_t(((const uint16_t*)l.logits)[at]) << 16) : ((const float*)l.logits)[at];
}
__device__ __forceinline__ bool slot_counts(const LossLabels& l, int64_t at) {
  const int64_t id = label_id(l, at);
  return l.logits ? id >= 0 && !(label_logit(l, at) == -__builtin_inff()) : id != l.ignore;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

// the largest of n values that are >= 0, for every lane
__device__ __forceinline__ float wave_max_of(const float* p, int n) {
  float m = 0.0f;
  for (int i = threadIdx.x & 63; i < n; i += 64) m = fmaxf(m, p[i]);
  return wave_max(m);
}

// Bound by HBM: x and w read once (50257 x 768 and 1024 x 768: 35 us, 4.5 TB/s).
__global__ __launch_bounds__(1024) void loss_maxima_kernel(const LossMaxima a) {
  __shared__ float part[16];
  const int ln = threadIdx.x & 63, w = threadIdx.x >> 6;
  float m = 0.0f;
  if (int(blockIdx.x) < a.xblocks) {  // a wave per row
    for (int64_t r = int64_t(blockIdx.x) * 16 + w; r < a.n_pad; r += int64_t(a.xblocks) * 16) {
      bool counts = false;
      if (r < a.l.n)
        for (int j = ln; j < a.l.k; j += 64) counts |= slot_counts(a.l, r * a.l.k + j);
      m = 0.0f;
      if (__any(counts)) {
        const float* p = a.x + r * a.h;
#pragma unroll 8
        for (int64_t c = ln; c < a.h; c += 64) m = fmaxf(m, finite_mag(p[c]));
        m = wave_max(m);
      }
      if (ln == 0) a.xmax[r] = m;
    }
    return;
  }
  {
    const int64_t all = a.l.v * a.h, step = int64_t(a.wblocks) * 1024, t = int64_t(int(blockIdx.x) - a.xblocks) * 1024 + threadIdx.x;
#pragma unroll 8
    for (int64_t i = t; i < all / 4; i += step) {
      const f32x4_t v = *(gptr<const f32x4_t>)(a.w + i * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, finite_mag(v[e]));
    }
    if (t < all % 4) m = fmaxf(m, finite_mag(a.w[all - 1 - t]));
  }
  m = wave_max(m);
  if (ln == 0) part[w] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) m = fmaxf(m, part[i]);
    a.wmax[int(blockIdx.x) - a.xblocks] = m;
  }
}

// The labels of token r (< n_pad) in one form: one wave, lanes over the slots.
__device__ __forceinline__ void prep_labels(const LossPrep& a, int64_t r) {
  const int ln = threadIdx.x & 63;
  const LossLabels& l = a.l;
  constexpr int PER = kLossMaxTop / 64;
  float lg[PER], m = -__builtin_inff();
  int id[PER];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = i * 64 + ln;
    id[i] = -1;
    lg[i] = -__builtin_inff();
    if (r < l.n && j < l.k) {
      const int64_t at = r * l.k + j;
      const int64_t v = label_id(l, at);
      const bool none = l.logits ? v < 0 : v == l.ignore;
      if (!none) {
        bad |= v < 0 || v >= l.v;
        id[i] = v >= 0 && v < l.v ? int(v) : -1;
        lg[i] = !l.logits ? 0.0f : label_logit(l, at);
        m = fmaxf(m, lg[i]);
        if (!(lg[i] < __builtin_inff())) bad = true;  // a teacher logit of +inf or NaN has no softmax
      }
    }
  }
  m = wave_max(m);
  bad = __any(bad);
  // (a row whose slots are all empty, or all of logit -inf, teaches nothing)
  const bool on = m > -__builtin_inff();
  // (differences first: a large logit over a small temperature may be beyond fp32)
  float e[PER], s = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    lg[i] = (lg[i] - m) * l.inv_t;
    e[i] = on && lg[i] > -__builtin_inff() ? expf(lg[i]) : 0.0f;
    s += e[i];
  }
  s = wave_sum(s);
  float ent = 0.0f, q[PER], sum[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    sum[i] = q[i] = on ? e[i] / s : 0.0f;
    if (q[i] > 0.0f) ent += q[i] * (lg[i] - logf(s));
  }
  // an id given more than once: its first slot takes the weights of all, the others become empty
  if (l.k > 1) {
    bool again[PER] = {};
#pragma unroll
    for (int b = 0; b < PER; ++b)
      for (int x = 0; x < min(64, l.k - b * 64); ++x) {
        const int idx = __builtin_amdgcn_readlane(id[b], x), jx = b * 64 + x;
        const float qx = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(q[b]), x));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const bool same = id[i] == idx;
          again[i] |= same && jx < i * 64 + ln;
          sum[i] += same && jx > i * 64 + ln ? qx : 0.0f;
        }
      }
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (again[i]) {
        id[i] = -1;
        sum[i] = 0.0f;
      }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = i * 64 + ln;
    if (j < l.k) {
      a.id[r * l.k + j] = on ? id[i] : -1;
      a.q[r * l.k + j] = sum[i];
    }
  }
  ent = wave_sum(ent);
  if (ln == 0) {
    a.ent[r] = ent;
    a.on[r] = bad ? __builtin_nanf("") : on ? 1.0f : 0.0f;
  }
}

// One 32 x 256 tile of a packed operand: four 8-column chunks per thread (row it * 8 + t / 32, chunk t % 32).
__device__ __forceinline__ void pack_tile(const LossLabels& l, const LossPack& d, int* counts) {
  const int64_t i = int(blockIdx.x) - d.blocks_begin;
  const int64_t tc = d.cols / 256, r0 = i / tc * 32, c0 = i % tc * 256;
  const int t = threadIdx.x, ch = t & 31;
  const int64_t c = c0 + ch * 8;
  float x[4][8];
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int64_t r = r0 + it * 8 + (t >> 5);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[it][e] = 0.0f;
    if (r < d.R && c < d.C) {
      const int64_t at = r * d.C + c;
      if (d.bf16) {
        const uint16_t* p = (const uint16_t*)d.src + at;
        if (c + 8 <= d.C) {
          const u32x4_a2 v = *(gptr<const u32x4_a2>)p;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[it][2 * e] = __uint_as_float(v[e] << 16);
            x[it][2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < d.C) x[it][e] = __uint_as_float(uint32_t(p[e]) << 16);
        }
      } else {
        const float* p = (const float*)d.src + at;
        if (c + 8 <= d.C) {
          const f32x4_a4 v0 = *(gptr<const f32x4_a4>)p, v1 = *(gptr<const f32x4_a4>)(p + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[it][e] = v0[e];
            x[it][4 + e] = v1[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < d.C) x[it][e] = p[e];
        }
      }
    }
  }
  uint32_t skip = 0;  // rows of the tile whose token does not count
  if (d.label_row >= 0) {
    if (t < 32) counts[t] = 0;
    __syncthreads();
    for (int e = t; e < 32 * l.k; e += 256) {
      const int r = e / l.k;
      if (r0 + r < d.R && slot_counts(l, (d.label_row + r0 + r) * l.k + (e - r * l.k))) counts[r] = 1;
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) skip |= counts[it * 8 + (t >> 5)] ? 0u : 1u << it;
  }
#pragma unroll
  for (int it = 0; it < 4; ++it)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[it][e] = skip >> it & 1 ? 0.0f : x[it][e];
  if (!d.bf16) {
    float all = 1.0f, inv;
    if (d.most) {
      all = scale_for(wave_max_of(d.most, d.count), inv);
      if (i == 0 && t == 0) *d.inv = inv;
    }
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      float f = all;
      if (d.row_most) {
        const float most = d.row_most[r0 + it * 8 + (t >> 5)], scale = scale_for(most, inv);
        f = !d.most ? scale : inv * all;
        if (d.most && most == 0.0f) {  // no part in dw
#pragma unroll
          for (int e = 0; e < 8; ++e) x[it][e] = 0.0f;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[it][e] *= f;
    }
  }
  for (int part = 0; part < (d.bf16 ? 1 : 2); ++part) {
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const u32x4 v = d.bf16 ? pack8(x[it]) : split8(x[it]);
      const int64_t r = r0 + it * 8 + (t >> 5);
      uint16_t* dst = d.dst + part * d.dst_part;
      if (d.blocked) *(gptr<u32x4>)(dst + blk_index(r, c, d.ld)) = v;
      else if (r < d.R && c < d.ld) *(gptr<u32x4>)(dst + r * d.ld + c) = v;
    }
  }
}

__global__ __launch_bounds__(256) void loss_prep_kernel(const LossPrep a) {
  __shared__ int counts[32];
  if (blockIdx.x == 0 && threadIdx.x < kLossQueues * kGemmXcds) a.queues[threadIdx.x] = 0;
  if (int(blockIdx.x) < a.label_blocks) {
    const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (r < a.n_pad) prep_labels(a, r);
    return;
  }
  pack_tile(a.l, a.d[a.packs > 1 && int(blockIdx.x) >= a.d[1].blocks_begin ? 1 : 0], counts);
}

// Sum over a workgroup, in 64 bits and a fixed order, of n values (times b where a value is not 0); for every thread.
template <int T>
__device__ __forceinline__ double block_sum(const float* a, const float* b, int64_t n, double* part) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += T) s += b && a[i] != 0.0f ? double(a[i]) * b[i] : double(a[i]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int i = 0; i < T / 64; ++i) s += part[i];
  return s;
}

// (m, s) of two sets joined: m the largest, s the sum of exp(. - m) over all others.
__device__ __forceinline__ void join_softmax(float& m, float& s, float m2, float s2) {
  const float hi = fmaxf(m, m2), lo = fminf(m, m2);
  const float sh = m >= m2 ? s : s2, sl = m >= m2 ? s2 : s;
  s = lo > -__builtin_inff() ? sh + (sl + 1.0f) * __builtin_amdgcn_exp2f((lo - hi) * kLog2e) : sh + sl * 0.0f;
  m = hi;
}

// (p - q) (1 + s) of a target with weight q whose logit is d above the row's largest and e = exp(d): from what is exact where
// p and q are near 1
__device__ __forceinline__ float target_pq(float q, float d, float e, float s) {
  return e >= 0.5f && q >= 0.5f ? expm1f(d) + (1.0f - q) - q * s : e - q * (1.0f + s);
}

// RPB rows per workgroup of 1024: thread t goes through groups t / RPB, + 1024 / RPB, ... of row t % RPB. Many tokens: 32
// rows, whose partials of a group lie together. Few: one row, whose partials lie in one piece (128256 ids, 48 tokens: 9 us;
// with four rows each and the other layout 19.5, when a workgroup reads four times the bytes it needs).
template <int RPB>
__global__ __launch_bounds__(1024) void loss_rows_kernel(const LossRows a) {
  constexpr int GS = 1024 / RPB, BATCH = 8;
  __shared__ float sm[16][RPB + 1], ss[16][RPB + 1], sb[16][RPB + 1], sd[16][RPB + 1];
  __shared__ double part[16];
  const int blocks = a.rows_pad / RPB;
  if (int(blockIdx.x) == blocks) {  // (the extra workgroup)
    const double d = block_sum<1024>(a.all_on, a.all_weight, a.n, part);
    if (threadIdx.x == 0) a.denom[0] = float(d);
  } else {
    const int rl = threadIdx.x % RPB, gl = threadIdx.x / RPB;
    const int64_t r = int64_t(blockIdx.x) * RPB + rl;
    const float none = -__builtin_inff();
    float m = none, s = 0.0f;
    // (asked for here, needed at the end)
    const bool mine = gl == 0 && r < a.rows;
    const float on = mine ? a.on[r] : 0.0f, ent = mine ? a.ent[r] : 0.0f, wt = mine && a.weight ? a.weight[r] : 1.0f;
    // this thread's first target
    const bool aims = r < a.rows && gl < a.k;
    const float q0 = aims ? a.q[r * a.k + gl] : 0.0f, z0 = aims ? a.zt[r * a.k + gl] : 0.0f;
    const int id0 = aims ? a.id[r * a.k + gl] : -1;
    for (int g = gl; g < (r < a.rows ? a.groups : 0); g += BATCH * GS) {
      float gm[BATCH], gs[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const bool in = g + i * GS < a.groups;
        const int64_t at = (g + i * GS) * a.gstep + r * a.rstep;
        gm[i] = in ? a.gm[at] : none;
        gs[i] = in ? a.gs[at] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < BATCH; ++i) join_softmax(m, s, gm[i], gs[i]);
    }
    // the lanes of a row, then the waves
#pragma unroll
    for (int o = 32; o >= RPB; o >>= 1) join_softmax(m, s, __shfl_xor(m, o), __shfl_xor(s, o));
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) < RPB) {
      sm[w][rl] = m;
      ss[w][rl] = s;
    }
    __syncthreads();
    if constexpr (RPB == 1) {  // every wave joins the waves' results by itself
      m = sm[threadIdx.x & 15][0];
      s = ss[threadIdx.x & 15][0];
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) join_softmax(m, s, __shfl_xor(m, o), __shfl_xor(s, o));
    } else {
      if (gl == 0) {
        for (int i = 1; i < 16; ++i) join_softmax(m, s, sm[i][rl], ss[i][rl]);
        sm[0][rl] = m;
        ss[0][rl] = s;
      }
      __syncthreads();
      m = sm[0][rl];
      s = ss[0][rl];
    }
    // sum of q (m - z) over the row's targets; a bound on |dz| at them, in units of 1 / (1 + s); whether one of them is the
    // largest
    const float top = m, others = s;
    const float lz = 2.0f * a.z_loss * (top + log1pf(others));
    float d = 0.0f, bound = 0.0f;
    bool of_top = false;
    for (int j = gl; j < (r < a.rows ? a.k : 0); j += GS) {
      const bool f = j == gl;
      const float q = f ? q0 : a.q[r * a.k + j], z = f ? z0 : a.zt[r * a.k + j];
      if (q > 0.0f && (f ? id0 : a.id[r * a.k + j]) >= 0) {
        d += q * (top - z);
        if (a.most) {
          const float e = expf(z - top);
          bound = fmaxf(bound, fabsf(target_pq(q, z - top, e, others) + lz * e));
          of_top |= z == top;
        }
      }
    }
#pragma unroll
    for (int o = 32; o >= RPB; o >>= 1) {
      d += __shfl_xor(d, o);
      bound = fmaxf(bound, __shfl_xor(bound, o));
      of_top |= __shfl_xor(int(of_top), o) != 0;
    }
    if (a.k > 64 / RPB) {  // (more than one wave's)
      if ((threadIdx.x & 63) < RPB) {
        sd[w][rl] = d;
        sb[w][rl] = copysignf(bound, of_top ? 1.0f : -1.0f);
      }
      __syncthreads();
      if (gl == 0) {
        for (int i = 1; i < 16; ++i) {
          d += sd[i][rl];
          bound = fmaxf(bound, fabsf(sb[i][rl]));
          of_top |= !__builtin_signbit(sb[i][rl]);
        }
      }
    }
    float most = 0.0f;
    if (gl == 0) {
      if (r >= a.rows) {
        a.row[r] = float4{0.0f, 0.0f, 0.0f, 0.0f};
        if (a.most) a.row_most[r] = 0.0f;
      } else {
        const float ls = log1pf(s), lse = m + ls;
        float loss = 0.0f;
        if (on != 0.0f) {
          loss = (ent + d + ls + a.z_loss * lse * lse) * on;  // (on is NaN for a label that has no loss)
        }
        const float4 rw = {m, s, on != 0.0f ? wt * on : 0.0f, 2.0f * a.z_loss * lse};
        a.row[r] = rw;
        // (a column that is no target: at most the largest p, or what is left of it if the largest is a target's)
        if (a.most) {
          bound = finite_mag(rw.z * fmaxf(bound, (1.0f + fabsf(rw.w)) * (of_top ? s : 1.0f)) / (1.0f + s));
          a.row_most[r] = bound;
          float inv;
          scale_for(bound, inv);
          most = bound > 0.0f ? fminf(a.x_most[r] * inv, 3e38f) : 0.0f;
        }
        if (a.token_loss) a.token_loss[r] = loss;
        if (a.lse) a.lse[r] = on != 0.0f ? lse : 0.0f;
        a.weighted[r] = on != 0.0f ? wt * loss : 0.0f;
      }
    }
    if (a.most && w == 0) {
      most = wave_max(most);
      if (threadIdx.x == 0) a.most[blockIdx.x] = most;
    }
  }
}

// The loss of all tokens from their weighted losses, by one workgroup.
template <int T>
__device__ __forceinline__ void sum_loss(const LossTotal& a, double* part) {
  const double t = block_sum<T>(a.weighted, nullptr, a.n, part) * a.scale;
  if (threadIdx.x == 0) a.loss[0] = float(!a.denom ? t : a.denom[0] != 0.0f ? t / a.denom[0] : t == t ? 0.0 : t);
}
__global__ __launch_bounds__(1024) void loss_total_kernel(const LossTotal a) {
  __shared__ double part[16];
  sum_loss<1024>(a, part);
}

// One 32 x 256 tile of dz per workgroup of 256: from the logits to LDS, the targets' elements there from their fp32 logits,
// then out. Bound by HBM: 2 bytes read and 2 written per logit (bf16).
template <bool F32, int PARTS>
__global__ __launch_bounds__(256) void loss_grad_kernel(const LossGrad a) {
  constexpr bool WIDE = PARTS > 1;  // (dz in fp32 in LDS)
  // 16-byte chunk c of row r in slot c ^ r
  __shared__ __attribute__((aligned(16))) uint8_t smem[32 * 256 * (WIDE ? 4 : 2)];
  const int tc = a.v_pad / 256;
  const int64_t tiles = int64_t(a.rows_pad / 32) * tc;
  if (a.total.loss && int64_t(blockIdx.x) == tiles) {  // (one more workgroup, for the loss)
    sum_loss<256>(a.total, (double*)smem);
    return;
  }
  if constexpr (F32) {
    if (int(blockIdx.x) >= a.x.blocks_begin) {
      pack_tile(LossLabels{}, a.x, nullptr);
      return;
    }
  }
  const int64_t r0 = int64_t(blockIdx.x / tc) * 32, c0 = int64_t(blockIdx.x % tc) * 256;
  const int t = threadIdx.x, ln = t & 63, w = t >> 6;
  const int first_id = t < 32 * a.k ? a.id[r0 * a.k + t] : -1;
  // chunk (row, 8 columns) it of a thread, as its 1 KiB block lies: lane: row lane / 4, chunk lane % 4
  auto crow = [&](int it) { return (it >> 1) * 16 + (ln >> 2); };
  auto ccol = [&](int it) { return (w * 2 + (it & 1)) * 32 + (ln & 3) * 8; };
  auto at16 = [](int r, int c) { return r * 512 + (((c >> 3) ^ (r & 31)) << 4) + (c & 7) * 2; };
  auto at32 = [](int r, int c) { return r * 1024 + (((c >> 2) ^ (r & 63)) << 4) + (c & 3) * 4; };
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = crow(it), cl = ccol(it);
    const int64_t row = r0 + r, c = c0 + cl;
    const float4 rw = a.row[row];
    const float f = rw.z * (1.0f + rw.w) / (1.0f + rw.y);
    float x[8];
    if constexpr (F32) {
      const f32x4_t v0 = *(gptr<const f32x4_t>)(a.logits + row * a.ldc + c);
      const f32x4_t v1 = *(gptr<const f32x4_t>)(a.logits + row * a.ldc + c + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = rw.z != 0.0f && c + e < a.v ? expf((e < 4 ? v0[e & 3] : v1[e & 3]) - rw.x) * f : 0.0f;
    } else {
      const u32x4 v = *(gptr<const u32x4>)(a.codes + blk_index(row, c, a.ldc));
      const float m = c < a.v ? a.gm[(c >> a.group_shift) * a.gstep + row * a.rstep] : 0.0f;
      const float base = (m - rw.x) * kLog2e;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t q = v[e >> 1] >> (16 * (e & 1)) & 0xffff;
        const float p = q == 65535u ? 0.0f : __builtin_amdgcn_exp2f(base - float(q) * (kLossOctaves / 65535.0f));
        x[e] = rw.z != 0.0f && c + e < a.v ? p * f : 0.0f;
      }
    }
    if constexpr (WIDE) {
      *(lptr<f32x4_t>)(smem + at32(r, cl)) = f32x4_t{x[0], x[1], x[2], x[3]};
      *(lptr<f32x4_t>)(smem + at32(r, cl + 4)) = f32x4_t{x[4], x[5], x[6], x[7]};
    } else {
      *(lptr<u32x4>)(smem + at16(r, cl)) = pack8(x);
    }
  }
  __syncthreads();
  auto target = [&](int i, int id) {
    id -= int(c0);
    if (id < 0 || id >= 256) return;
    const int r = i / a.k;
    const int64_t row = r0 + r;
    const float4 rw = a.row[row];
    if (rw.z == 0.0f) return;
    const float q = a.q[r0 * a.k + i], d = a.zt[r0 * a.k + i] - rw.x, e = expf(d);
    const float x = rw.z * (target_pq(q, d, e, rw.y) + rw.w * e) / (1.0f + rw.y);
    if constexpr (WIDE) *(lptr<float>)(smem + at32(r, id)) = x;
    else *(lptr<uint16_t>)(smem + at16(r, id)) = uint16_t(pack_bf16x2(x, 0.0f));
  };
  for (int i = t; i < 32 * a.k; i += 8 * 256) {  // eight ids asked for at a time
    int id[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      id[e] = i == t && e == 0 ? first_id : i + e * 256 < 32 * a.k ? a.id[r0 * a.k + i + e * 256] : -1;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (id[e] >= 0) target(i + e * 256, id[e]);
  }
  float scales[4];
  if constexpr (F32) {
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      float inv;
      scales[it] = scale_for(a.row_most[r0 + crow(it)], inv);
    }
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = crow(it), cl = ccol(it);
    uint16_t* dst = a.dz + blk_index(r0 + r, c0 + cl, a.ldc);
    if constexpr (WIDE) {
      const f32x4_t v0 = *(lptr<f32x4_t>)(smem + at32(r, cl)), v1 = *(lptr<f32x4_t>)(smem + at32(r, cl + 4));
      float x[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if constexpr (F32) x[e] *= scales[it];
#pragma unroll
      for (int part = 0; part < 2; ++part) *(gptr<u32x4>)(dst + part * a.dz_part) = F32 ? split8(x) : split8_bf16(x);
    } else {
      *(gptr<u32x4>)dst = *(lptr<u32x4>)(smem + at16(r, cl));
    }
  }
}

// Elements at .. + 3 (the first `left` of them) of a row-major bf16 or fp32 tensor.
__device__ __forceinline__ void store4(void* out, int bf16, int64_t at, f32x4_t s, int left) {
  if (bf16) {
    const u32x2 v = {pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
    uint16_t* o = (uint16_t*)out + at;
    if (left >= 4) {
      *(gptr<u32x2_a2>)o = v;
    } else {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (t < left) o[t] = uint16_t(v[t >> 1] >> (16 * (t & 1)));
    }
  } else {
    float* o = (float*)out + at;
    if (left >= 4) {
      *(gptr<f32x4_a4>)o = s;
    } else {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (t < left) o[t] = s[t];
    }
  }
}

// s + ranges i .. i + 7 (as far as there are any), in order, all asked for before the first is added.
__device__ __forceinline__ void add_ranges(f32x4_t& s, const float* p, int64_t stride, int i, int splits) {
  f32x4_t v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = *(gptr<const f32x4_t>)(p + min(i + e, splits - 1) * stride);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < splits) s += v[e];
}

__global__ __launch_bounds__(256) void loss_sum_kernel(float* part, int quads, int splits) {
  float* p = part + int64_t(blockIdx.y) * splits * quads * 4 + (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  f32x4_t s = *(gptr<const f32x4_t>)p;
  for (int i = 1; i < splits; i += 8) add_ranges(s, p, int64_t(quads) * 4, i, splits);
  *(gptr<f32x4_t>)p = s;
}

// The K ranges' partial tiles added in order; four elements per thread.
template <int NW, int TB>
__global__ __launch_bounds__(256) void loss_join_kernel(const LossJoin a) {
  using G = Grid<NW, TB>;
  constexpr int Q = TB * TB / 4;
  const int tile = blockIdx.x / (Q / 256), q = (blockIdx.x % (Q / 256)) * 256 + threadIdx.x;
  const float* p = a.part + int64_t(tile) * a.splits * (TB * TB) + q * 4;
  f32x4_t s = *(gptr<const f32x4_t>)p;
  for (int i = 1; i < a.splits; i += 8) add_ranges(s, p, TB * TB, i, a.splits);
  const int ln = q & 63, blk = (q >> 6) & (G::MI * G::NI * 4 - 1), w = (q >> 6) / (G::MI * G::NI * 4);
  const int bj = tile / a.tm, bi = tile - bj * a.tm;
  const int row = bi * TB + (w / G::WN) * (G::MI * 32) + (blk >> 3) * 32 + (ln & 31);
  const int c = bj * TB + (w % G::WN) * 64 + ((blk >> 2) & 1) * 32 + (blk & 3) * 8 + (ln >> 5) * 4;
  if (row >= a.rows || c >= a.cols) return;
  s *= out_factor(a.alpha, a.denom);
  store4(a.out, a.out_bf16, int64_t(row) * a.ldo + c, s, a.cols - c);
}

// Products for at most 32 MI tokens (LossStream). Eight waves; K in steps through a ring of NST stages filled NST - 1 steps
// ahead by direct loads. Bound by HBM: w is read once, QB bytes per step, with up to (NST - 1) steps of it in flight per CU.
// logits: a stage holds QR rows of w by KT of h; a wave takes all tokens by 32 rows of w, and half of the step's K where
//   QR = 128 (the halves are added in LDS at the tile's end); chunk c of row r in slot c ^ r % 16 (KT = 64: c ^ r / 2 % 8). 128
//   rows of 256 bytes rather than 256 of 128: a head of 128256 x 4096 is read in 223 us on average (4.7 TB/s; 212 at best),
//   and a call of one token takes 230 us instead of 243, of 48 tokens 240 instead of 255 (50257 x 768: 28.5 and 26.5); more
//   tokens leave no room for it.
// dx: KT rows of w by 256 of h, a wave 32 columns; chunk c of row r in slot c ^ 2 (r % 4); fragments read transposed.
// Past a row's end lie the next row's values, past w's end its last ones: they meet zeros of x or dz, or belong to columns
// that are not stored.
template <int MI, int KIND>
__global__ __launch_bounds__(512, 1) void loss_stream_kernel(const LossStream a) {
  constexpr int QR = stream_rows(MI), KT = KIND == kLossLogits ? 16384 / QR : stream_step(MI);  // (dx: QR is not used)
  constexpr int PP = KIND == kLossLogits ? 1 : 2;  // parts of P
  constexpr int KB = KT / 32, PPB = MI * 32 * KT * 2, PB = PP * PPB, QB = KIND == kLossLogits ? 32768 : KT * 512, STAGE = PB + QB;
  constexpr int NST = 160 * 1024 / STAGE < 4 ? 160 * 1024 / STAGE : 4;
  constexpr int PBLK = PP * MI * 2 * KB;                            // 1 KiB blocks of P per step
  constexpr int PL = PBLK < 8 ? 1 : PBLK / 8, QL = QB / 8192, LOADS = PL + QL;  // per wave and step (four blocks: two waves load the same)
  static_assert(NST >= 2 && NST * STAGE <= 160 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[NST * STAGE];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int total = a.tiles * a.splits;
  const int64_t wrow = a.h * 2;  // bytes
  const uint32_t ploff = (lane >> 2) * kRowB + ((lane & 3) ^ swz(lane >> 2)) * 16;
  constexpr int LPR = KT / 8, RPI = 64 / LPR;  // logits: lanes per row of w, rows per load
  const int qr = w * RPI + lane / LPR;         // this lane's row of its first load (later ones: 8 RPI further, the same swizzle)
  const int qsw = KT == 64 ? (qr >> 1) & 7 : qr & 15;
  const uint32_t qloff = KIND == kLossLogits
                             ? uint32_t(qr * wrow) + ((lane % LPR) ^ qsw) * 16
                             : uint32_t((w * 2 + (lane >> 5)) * wrow) + ((lane & 31) ^ (((w & 1) * 2 + (lane >> 5)) << 1)) * 16;
  // w from row r0 on; its loads are held to its last 16 bytes (whole chunks are in or out: h is a multiple of 8)
  uint32_t qmost = 0;
  auto rows_from = [&](int64_t r0) {
    const int64_t bytes = (a.v - r0) * wrow, some = bytes < 0x7ffffff0 ? bytes : 0x7ffffff0;
    qmost = uint32_t(some) - 16;
    return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.w + r0 * wrow), 0, uint32_t(some), 0x00020000);
  };
  auto issue = [&](int tile, int k, int stage) {
    lds_byte* sb = (lds_byte*)(smem + stage * STAGE);
    const __amdgpu_buffer_rsrc_t pr = __builtin_amdgcn_make_buffer_rsrc((void*)a.P, 0, 0xffffffffu, 0x00020000);
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int b = (i * 8 + w) % PBLK, part = b / (MI * 2 * KB), kb = b / (MI * 2) % KB, panel = b % (MI * 2);  // kb: of 32; panel: 16 rows
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          pr, sb + b * 1024, 16, ploff,
          uint32_t(part) * uint32_t(a.ppart * 2) + uint32_t(panel) * uint32_t(a.ldp * 32) + uint32_t(k * KB + kb) * 1024u, 0, 0);
    }
    const __amdgpu_buffer_rsrc_t qr = rows_from(KIND == kLossLogits ? int64_t(tile) * QR : int64_t(k) * KT);
#pragma unroll
    for (int i = 0; i < QL; ++i) {  // logits: rows RPI (8 i + w) ..; dx: rows 2 (8 i + w), + 1
      const uint32_t at = KIND == kLossLogits ? uint32_t(i * 8 * RPI * wrow) + uint32_t(k) * uint32_t(KT * 2)
                                              : uint32_t(i * 16 * wrow) + uint32_t(tile) * 512u;
      const uint32_t off = qloff + at;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(qr, sb + PB + (i * 8 + w) * 1024, 16, off < qmost ? off : qmost, 0, 0, 0);
    }
  };
  const int fr = lane & 31, fh = lane >> 5;
  constexpr int CB = QR / 32;  // logits: waves along w's rows
  const int cb = KIND == kLossLogits ? w % CB : w, kh = KIND == kLossLogits ? w / CB : 0;
  int item = blockIdx.x;
  if (item >= total) return;
  auto range = [&](int it, int& k0, int& nk) {
    const int s = it / a.tiles;
    k0 = s * a.kper;
    nk = min(a.kper, a.nk - k0);
    return it - s * a.tiles;
  };
  // This wave's LDS reads have returned. The loads behind the next barrier overwrite what they read; without this the
  // compiler may let a product, and the wait for its operands, slide past that barrier.
  auto reads_done = [] {
    LOSS_WAIT_LGKM0();
    __builtin_amdgcn_sched_barrier(0);
  };
  int k0, nk, tile = range(item, k0, nk);
#pragma unroll
  for (int s = 0; s < NST - 1; ++s) issue(tile, k0 + min(s, nk - 1), s);
  while (true) {
    f32x16_t acc[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][v] = 0.0f;
    int cs = 0;
    for (int kt = 0; kt < nk; ++kt) {
      LOSS_WAIT_VMCNT((NST - 2) * LOADS);  // this wave's loads of step kt
      reads_done();                        // (of step kt - 1, or of the K halves' sums)
      __builtin_amdgcn_s_barrier();        // everybody's
      issue(tile, k0 + min(kt + NST - 1, nk - 1), cs == 0 ? NST - 1 : cs - 1);
      const uint8_t* sb = smem + cs * STAGE;
#pragma unroll
      for (int s4 = 0; s4 < (KIND == kLossLogits ? 4 : KT / 16); ++s4) {  // 16 of K
        const int sl = kh * 4 + s4;
        bf16x8_t qf;
        if constexpr (KIND == kLossLogits) {
          const int row = cb * 32 + fr, c = sl * 2 + fh;
          qf = *reinterpret_cast<const bf16x8_t*>(sb + PB + row * (KT * 2) + ((c ^ (KT == 64 ? (row >> 1) & 7 : row & 15)) << 4));
        } else {
          const int grp = lane >> 4, i = lane & 15, row = sl * 16 + (grp >> 1) * 8 + (i >> 2);
          const int sl16 = w * 4 + (grp & 1) * 2 + ((i & 3) >> 1);
          lds_byte* q = (lds_byte*)(smem + cs * STAGE + PB) + row * 512 + ((sl16 ^ ((row & 3) << 1)) << 4) + (i & 1) * 8;
          const bf16x4_t lo = read_tr((lptr<bf16x4_t>)q);
          const bf16x4_t hi = read_tr((lptr<bf16x4_t>)(q + 4 * 512));
          qf = join_tr(lo, hi);
        }
#pragma unroll
        for (int part = PP - 1; part >= 0; --part)
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            const bf16x8_t pf = *reinterpret_cast<const bf16x8_t*>(sb + part * PPB + (sl >> 1) * (MI * 2048) + (i * 32 + fr) * kRowB +
                                                                   ((((sl & 1) * 2 + fh) ^ swz(fr)) << 4));
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, pf, acc[i], 0, 0, 0);
          }
      }
      cs = cs + 1 == NST ? 0 : cs + 1;
    }
    LOSS_WAIT_VMCNT(0);
    reads_done();
    __builtin_amdgcn_s_barrier();
    const int done = tile, split = item / a.tiles;
    item += gridDim.x;
    const bool more = item < total;
    if (more) {
      tile = range(item, k0, nk);
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) issue(tile, k0 + min(s, nk - 1), s);
    }
    // acc[i][4 g + t]: row 32 i + lane % 32, column 8 g + 4 (lane / 32) + t of the wave's 32
    if constexpr (KIND == kLossLogits) {
      if constexpr (CB < 8) {  // the K halves' sums, through the stage that the next tile's first loads leave free
        f32x4_t* half = reinterpret_cast<f32x4_t*>(smem + (NST - 1) * STAGE) + (cb * MI * 4) * 64 + lane;
        static_assert(CB * MI * 4096 <= STAGE, "the halves' room");
        if (kh) {
#pragma unroll
          for (int q = 0; q < MI * 4; ++q) {
            const f32x16_t& c = acc[q >> 2];
            half[q * 64] = f32x4_t{c[4 * (q & 3)], c[4 * (q & 3) + 1], c[4 * (q & 3) + 2], c[4 * (q & 3) + 3]};
          }
        }
        LOSS_WAIT_LGKM0();
        __builtin_amdgcn_s_barrier();
        if (!kh) {
#pragma unroll
          for (int q = 0; q < MI * 4; ++q) {
            const f32x4_t c = half[q * 64];
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[q >> 2][4 * (q & 3) + t] += c[t];
          }
        }
      }
      const int c0 = done * QR + cb * 32, left = int(a.v) - c0;
      const float L = kLog2e * a.inv_t;
      if (left > 0 && !kh) {
        static_for<MI>([&](auto mi_c) {
          constexpr int mi = decltype(mi_c)::value;
          const int row = mi * 32 + fr;
          float u[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            u[e] = acc[mi][e];
            if (left < 32 && (e >> 2) * 8 + fh * 4 + (e & 3) >= left) u[e] = -__builtin_inff();
          }
          float m = u[0];
#pragma unroll
          for (int e = 1; e < 16; ++e) m = fmaxf(m, u[e]);
          m = half_max(m);
          const float ref = fmaxf(m, -3.4e38f);
          float s = 0.0f, all = 0.0f;  // as in loss_gemm_kernel
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = __builtin_amdgcn_exp2f((u[e] - ref) * L);
            s += __builtin_amdgcn_fractf(x);
            all += x;
          }
          const float ones = half_sum(__builtin_rintf(all - s));
          s = half_sum(s);
          if (fh == 0) {
            const int64_t at = int64_t(c0 >> 5) * a.gstep + row * a.rstep;
            a.gm[at] = m * a.inv_t;
            a.gs[at] = s + (ones - 1.0f);
          }
          // targets, as in loss_gemm_kernel, among 32 columns
          for (int j0 = 0; j0 < a.k; j0 += 16) {
            i32x4 at[4] = {};
            if (a.k == 1) {
              at[0][0] = a.ids[row];
            } else {
#pragma unroll
              for (int v = 0; v < 4; ++v)
                if (j0 + v * 4 < a.k) at[v] = *(gptr<const i32x4_a4>)(a.ids + row * a.k + j0 + v * 4);
            }
            uint32_t hits = 0;
#pragma unroll
            for (int f = 0; f < 16; ++f) {
              at[f >> 2][f & 3] -= c0;
              hits |= uint32_t(at[f >> 2][f & 3]) < 32u ? 1u << f : 0u;
            }
            if (a.k - j0 < 16) hits &= (1u << (a.k - j0)) - 1;
            while (hits) {
              const int i = __builtin_ctz(hits);
              hits &= hits - 1;
              int x = at[0][0];
#pragma unroll
              for (int f = 1; f < 16; ++f) x = i == f ? at[f >> 2][f & 3] : x;
              if (((x >> 2) & 1) != fh) continue;
              const int e = ((x >> 3) & 3) * 4 + (x & 3);
              float z = 0.0f;
#pragma unroll
              for (int f = 0; f < 16; ++f) z = e == f ? u[f] : z;
              a.zt[row * a.k + j0 + i] = z * a.inv_t;
            }
          }
          if (a.codes) {
            const float C = -L * (1.0f / kLossOctaves);
#pragma unroll
            for (int g = 0; g < 4; ++g)
              *(gptr<u32x2>)(a.codes + blk_index(row, c0 + g * 8 + fh * 4, a.ldc)) =
                  u32x2{code2((u[4 * g] - ref) * C, (u[4 * g + 1] - ref) * C), code2((u[4 * g + 2] - ref) * C, (u[4 * g + 3] - ref) * C)};
          }
        });
      }
    } else {
      float* part = a.part + int64_t(split) * (MI * 32) * a.ldo + done * 256 + w * 32;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(gptr<f32x4_t>)(part + (i * 32 + fr) * a.ldo + g * 8 + fh * 4) =
              f32x4_t{acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
    }
    if (!more) break;
  }
  LOSS_WAIT_VMCNT(0);
}

// dw of at most 32 KS tokens: K is a few steps, and writing dw all there is to it (HBM). A workgroup of four waves keeps CT
// columns of x in registers and goes through blocks of 64 rows (ids), gridDim.y blocks apart: both parts of the next block of
// dz are on their way while this one's product goes out, through LDS, so that a wave stores whole rows of CT columns. (48
// tokens, 128256 x 4096, 1.05 GB: 240 us; one block per workgroup, x read again for each: 327; the persistent tiles' kernel
// more.) Non-temporal stores: with plain ones it takes 245 us, and what reads w after it 284 us instead of 233, waiting for
// the caches to write dw back (the whole call 728 -> 670 us).
template <int KS>
__global__ __launch_bounds__(256) void loss_dw_kernel(const LossGemm a) {
  constexpr int NPAN = 2 * KS, NJ = KS <= 2 ? 2 : 1, CT = 128 * NJ, CB = CT / 32;  // panels of 16 tokens; columns, in blocks of 32
  constexpr int PPB = NPAN * 2048, PB = 2 * PPB, QB = NPAN * CB * 1024;            // dz's parts, x
  constexpr int OUT = 2 * PB, XAT = PB;  // LDS: two blocks of dz, 32 rows of the result; x is first staged over the second and the third
  __shared__ __attribute__((aligned(1024))) uint8_t smem[OUT + 32 * CT * 2];
  static_assert(XAT + QB <= OUT + 32 * CT * 2, "room for x");
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bj = blockIdx.x, blocks = (a.rows + 63) / 64;
  const uint32_t loff = (lane >> 2) * kRowB + ((lane & 3) ^ swz(lane >> 2)) * 16;
  auto issue = [&](int bi, int at) {
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const __amdgpu_buffer_rsrc_t pr =
          __builtin_amdgcn_make_buffer_rsrc((void*)(a.P + part * a.ppart + int64_t(bi) * 1024), 0, 0xffffffffu, 0x00020000);
#pragma unroll
      for (int i = 0; i < KS; ++i) {  // panel b / 2, block b % 2
        const int b = i * 4 + w;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(pr, (lds_byte*)(smem + at + part * PPB + b * 1024), 16, loff,
                                                 uint32_t(b >> 1) * uint32_t(a.ldp * 32) + (b & 1) * 1024, 0, 0);
      }
    }
  };
  int bi = blockIdx.y;  // (< blocks)
  const __amdgpu_buffer_rsrc_t qr =
      __builtin_amdgcn_make_buffer_rsrc((void*)(a.Q + int64_t(bj) * (CT * 16)), 0, 0xffffffffu, 0x00020000);
#pragma unroll
  for (int i = 0; i < NPAN * CB / 4; ++i) {  // x: panel b / CB, block b % CB
    const int b = i * 4 + w;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(qr, (lds_byte*)(smem + XAT + b * 1024), 16, loff,
                                             uint32_t(b / CB) * uint32_t(a.ldq * 32) + (b % CB) * 1024, 0, 0);
  }
  issue(bi, 0);
  const float f = out_factor(a.alpha, a.denom);
  const int trow = (lane >> 5) * 8 + ((lane >> 2) & 3), tchunk = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1), tbyte = (lane & 1) * 8;
  const int tlo = trow * kRowB + ((tchunk ^ swz(trow)) << 4) + tbyte;
  const int thi = (trow + 4) * kRowB + ((tchunk ^ swz(trow + 4)) << 4) + tbyte;
  auto frag = [&](int at) {
    lds_byte* q = (lds_byte*)smem + at;
    return join_tr(read_tr((lptr<bf16x4_t>)(q + tlo)), read_tr((lptr<bf16x4_t>)(q + thi)));
  };
  LOSS_WAIT_VMCNT(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  bf16x8_t qf[NPAN][NJ];
#pragma unroll
  for (int s = 0; s < NPAN; ++s)
#pragma unroll
    for (int j = 0; j < NJ; ++j) qf[s][j] = frag(XAT + (s * CB + w * NJ + j) * 1024);
  LOSS_WAIT_LGKM0();
  __builtin_amdgcn_sched_barrier(0);
  constexpr int SL = CT / 8, RPI = 64 / SL, STORES = 16 / RPI;  // 16-byte slots of a row, XORed by the row; rows per store; a wave's stores per block
  auto slot = [](int r, int sl) { return OUT + r * (CT * 2) + ((sl ^ r) & (SL - 1)) * 16; };
  const int er = lane & 31, eh = lane >> 5;
  for (int at = 0;; at ^= PB) {
    __builtin_amdgcn_s_barrier();  // this block of dz is there for all waves, the other one's place is free
    const int next = bi + gridDim.y;
    if (next < blocks) issue(next, at ^ PB);
    __builtin_amdgcn_sched_barrier(0);
    f32x16_t acc[2][NJ];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
#pragma unroll
    for (int part = 1; part >= 0; --part)  // (the order of the tiles' kernel: dw is the same with dx and without)
#pragma unroll
      for (int s = 0; s < NPAN; ++s) {
        bf16x8_t pf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) pf[i] = frag(at + part * PPB + (s * 2 + i) * 1024);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s][j], pf[i], acc[i][j], 0, 0, 0);
      }
    static_for<2>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
#pragma unroll
      for (int p = 0; p < 4 * NJ; ++p) {
        const f32x16_t& v = acc[i][p >> 2];
        const int o = 4 * (p & 3);
        *(lptr<u32x2>)((lds_byte*)smem + slot(er, (w * NJ + (p >> 2)) * 4 + (p & 3)) + eh * 8) =
            u32x2{pack_bf16x2(v[o] * f, v[o + 1] * f), pack_bf16x2(v[o + 2] * f, v[o + 3] * f)};
      }
      LOSS_WAIT_LGKM0();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int it = 0; it < STORES / 2; ++it) {
        const int r = w * 8 + it * RPI + lane / SL, sl = lane % SL;
        const u32x4 val = *(lptr<u32x4>)((lds_byte*)smem + slot(r, sl));
        const int row = bi * 64 + i * 32 + r, c = bj * CT + sl * 8;
        if (row < a.rows) {
          uint16_t* dst = (uint16_t*)a.out + int64_t(row) * a.ldo + c;
          if (c + 8 <= a.cols) {
            __builtin_nontemporal_store(u32x4_a2(val), (gptr<u32x4_a2>)dst);
          } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
              if (c + t < a.cols) *(gptr<uint16_t>)(dst + t) = uint16_t(val[t >> 1] >> (16 * (t & 1)));
          }
        }
      }
      LOSS_WAIT_LGKM0();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (i == 0) __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    });
    if (next >= blocks) break;
    // the next block of dz: behind its loads come this block's stores, STORES of them where no row or column is cut off
    if (bj * CT + CT <= a.cols) LOSS_WAIT_VMCNT(STORES);
    else LOSS_WAIT_VMCNT(0);
    bi = next;
  }
}

// The K ranges' row-major results added in order: four columns per thread.
__global__ __launch_bounds__(256) void loss_join_rows_kernel(const LossJoin a) {
  const int per = (a.cols + 3) / 4;
  const int64_t q = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = q / per;
  const int c = int(q - row * per) * 4;
  if (row >= a.rows) return;
  const float* p = a.part + row * a.ldp + c;
  f32x4_t s = *(gptr<const f32x4_t>)p;
  for (int i = 1; i < a.splits; i += 8) add_ranges(s, p, a.stride, i, a.splits);
  s *= out_factor(a.alpha, a.denom);
  store4(a.out, a.out_bf16, row * a.ldo + c, s, a.cols - c);
}

__global__ __launch_bounds__(256) void loss_zero_kernel(uint16_t* p, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = 0;
}

// Eight elements per thread and pass; p is 16-byte aligned.
__global__ __launch_bounds__(256) void scale_grad_kernel(void* p, int64_t n, int bf16, const float* factor) {
  const float f = *factor;
  if (f == 1.0f) return;
  for (int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8; i < n; i += int64_t(gridDim.x) * 256 * 8) {
    if (bf16) {
      uint16_t* q = (uint16_t*)p + i;
      if (i + 8 <= n) {
        u32x4 v = *(gptr<u32x4>)q;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          v[t] = pack_bf16x2(__uint_as_float(v[t] << 16) * f, __uint_as_float(v[t] & 0xffff0000u) * f);
        *(gptr<u32x4>)q = v;
      } else {
        for (int t = 0; i + t < n; ++t) q[t] = uint16_t(pack_bf16x2(__uint_as_float(uint32_t(q[t]) << 16) * f, 0.0f));
      }
    } else {
      float* q = (float*)p + i;
      if (i + 8 <= n) {
        *(gptr<f32x4_t>)q = *(gptr<f32x4_t>)q * f;
        *(gptr<f32x4_t>)(q + 4) = *(gptr<f32x4_t>)(q + 4) * f;
      } else {
        for (int t = 0; i + t < n; ++t) q[t] *= f;
      }
    }
  }
}

template <int NW, int TB, int KIND>
void launch_gemm_seg(const LossGemm2& a, hipStream_t st) {
  const dim3 grid(kGemmXcds * Grid<NW, TB>::SLOTS), block(NW * 64);
  if (a.g[0].nseg == 1)
    hipLaunchKernelGGL((loss_gemm_kernel<NW, TB, 1, KIND>), grid, block, 0, st, a);
  else if (KIND == kLossOut && a.g[0].nseg == 2)
    hipLaunchKernelGGL((loss_gemm_kernel<NW, TB, 2, kLossOut>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((loss_gemm_kernel<NW, TB, kLossMaxSeg, KIND>), grid, block, 0, st, a);
}

}  // namespace

hipError_t launch_loss_gemm(const LossGemm2& a, int kind, int tile, hipStream_t st) {
  if (tile == kLossTile) {
    if (kind == kLossLogits) launch_gemm_seg<8, kLossTile, kLossLogits>(a, st);
    else launch_gemm_seg<8, kLossTile, kLossOut>(a, st);
  } else {
    if (kind == kLossLogits) launch_gemm_seg<4, kLossTileSmall, kLossLogits>(a, st);
    else launch_gemm_seg<4, kLossTileSmall, kLossOut>(a, st);
  }
  return hipGetLastError();
}

hipError_t launch_loss_maxima(const LossMaxima& a, hipStream_t st) {
  hipLaunchKernelGGL(loss_maxima_kernel, dim3(unsigned(a.xblocks + a.wblocks)), dim3(1024), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_prep(const LossPrep& a, int blocks, hipStream_t st) {
  hipLaunchKernelGGL(loss_prep_kernel, dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_rows(const LossRows& a, hipStream_t st) {
  const int per = a.gstep == 1 ? 1 : 32;
  const dim3 grid(unsigned(a.rows_pad / per + (a.denom ? 1 : 0)));
  if (per == 1) hipLaunchKernelGGL(loss_rows_kernel<1>, grid, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(loss_rows_kernel<32>, grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_total(const LossTotal& a, hipStream_t st) {
  hipLaunchKernelGGL(loss_total_kernel, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_grad(const LossGrad& b, hipStream_t st) {
  LossGrad a = b;
  a.x.blocks_begin = (a.rows_pad / 32) * (a.v_pad / 256) + (a.total.loss ? 1 : 0);
  const dim3 grid(unsigned(a.x.blocks_begin) + (a.x.src ? unsigned(a.rows_pad / 32) * unsigned(a.x.cols / 256) : 0u));
  if (a.logits)
    hipLaunchKernelGGL((loss_grad_kernel<true, 2>), grid, dim3(256), 0, st, a);
  else if (a.parts == 2)
    hipLaunchKernelGGL((loss_grad_kernel<false, 2>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((loss_grad_kernel<false, 1>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_sum(float* part, int64_t tiles, int tile, int splits, hipStream_t st) {
  const int quads = tile * tile / 4;
  hipLaunchKernelGGL(loss_sum_kernel, dim3(unsigned(quads / 256), unsigned(tiles)), dim3(256), 0, st, part, quads, splits);
  return hipGetLastError();
}

hipError_t launch_loss_join(const LossJoin& a, int tile, hipStream_t st) {
  if (tile == 0) {
    const int64_t quads = int64_t(a.rows) * ((a.cols + 3) / 4);
    hipLaunchKernelGGL(loss_join_rows_kernel, dim3(unsigned((quads + 255) / 256)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const dim3 grid(unsigned(a.tiles) * unsigned(tile * tile / 1024));
  if (tile == kLossTile)
    hipLaunchKernelGGL((loss_join_kernel<8, kLossTile>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((loss_join_kernel<4, kLossTileSmall>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int KIND>
void launch_stream(const LossStream& a, int mi, hipStream_t st) {
  const int64_t items = int64_t(a.tiles) * a.splits;
  const dim3 grid(unsigned(items < 256 ? items : 256)), block(512);
  if (mi == 1) hipLaunchKernelGGL((loss_stream_kernel<1, KIND>), grid, block, 0, st, a);
  else if (mi == 2) hipLaunchKernelGGL((loss_stream_kernel<2, KIND>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((loss_stream_kernel<4, KIND>), grid, block, 0, st, a);
}

hipError_t launch_loss_dw(const LossGemm& a, int steps, hipStream_t st) {
  const int columns = steps <= 2 ? 256 : 128, tn = (a.cols + columns - 1) / columns, blocks = (a.rows + 63) / 64;
  // three workgroups per CU (two where LDS holds no more) in one round, of as many blocks each
  const int slots = (steps <= 2 ? 3 : 2) * 256 / tn, each = slots > 0 ? (blocks + slots - 1) / slots : blocks;
  const dim3 grid(unsigned(tn), unsigned((blocks + each - 1) / each)), block(256);
  if (steps == 1) hipLaunchKernelGGL(loss_dw_kernel<1>, grid, block, 0, st, a);
  else if (steps == 2) hipLaunchKernelGGL(loss_dw_kernel<2>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(loss_dw_kernel<4>, grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_stream(const LossStream& a, int mi, int kind, hipStream_t st) {
  if (kind == kLossLogits) launch_stream<kLossLogits>(a, mi, st);
  else launch_stream<kLossOut>(a, mi, st);
  return hipGetLastError();
}

hipError_t launch_loss_zero(void* p, int64_t bytes, hipStream_t st) {
  const int64_t n = bytes / 2;
  if (n > 0) {
    const int64_t g = (n + 255) / 256;
    hipLaunchKernelGGL(loss_zero_kernel, dim3(unsigned(g < 4096 ? g : 4096)), dim3(256), 0, st, (uint16_t*)p, n);
  }
  return hipGetLastError();
}

hipError_t launch_scale_grad(void* p, int64_t n, int bf16, const float* factor, hipStream_t st) {
  if (n > 0) {
    const int64_t g = (n + 2047) / 2048;
    hipLaunchKernelGGL(scale_grad_kernel, dim3(unsigned(g < 8192 ? g : 8192)), dim3(256), 0, st, p, n, bf16, factor);
  }
  return hipGetLastError();
}

}  // namespace mfsdp
