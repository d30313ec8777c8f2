// attn_core.h -- the parts that the attention kernels over the paged KV cache share
// (gfx950): the key step (scores, online softmax, PV product) on operands in
// registers, the layout of the LDS ring, and the arithmetic of the work split.
#pragma once

#include "dsv_internal.h"

#include <math.h>

namespace dsv {
namespace {

constexpr int kBlockKeys = kAttnBlockKeys;  // keys per inner step (two pages)
// Smallest stream-K share: with little work (short contexts, few requests)
// eight blocks per workgroup beat spreading it over every resident
// workgroup -- fewer cut segments, so less partial traffic and combine work,
// and a longer pipeline per workgroup.
constexpr int kMinShare = 8 * kBlockKeys;
// Stream-K lead-in: every segment with keys counts kLeadKeys more in the
// linear work space than it holds, the cost of starting a piece on it
// (metadata, page ids, query rows, the ring's first blocks), so that equal
// shares are equal in streaming plus piece starts.  A multiple of the block;
// six blocks measured best across shapes (two to eight were compared).
constexpr int kLeadKeys = kAttnLeadKeys;
// Wave priority.  At D = 128 the persistent grid holds two workgroups per CU
// (one at G = 16), and the one the dispatcher places second (grid index >= number
// of CUs) loses instruction arbitration to the older first one: with equal
// shares and no priorities the first ended at 66 us and the second at 91 (B=32,
// contexts up to 8K).  Its waves therefore run at raised priority until kBoostPct
// percent of its share is done, then at the default, and both end at about 90 us.
// Priority changes no arithmetic.  Drop points, B=32 contexts to 8K / eight
// query heads to a KV head and contexts to 16K, us a call: 50% 104.2 / 226.7,
// 65% 104.4 / 228.8, 80% 106.1 / 229.6, none 113 / 244.
// At D = 64, with two to four workgroups to a CU, all but the first are raised: 8 KV
// heads, B=32 contexts to 8K, groups of 1 / 4 / 8 / 16, us a call: 56.4 / 60.3 /
// 66.3 / 108.4, none raised 57.7 / 61.9 / 70.1 / 116.1, the last alone 56.5 / 60.7 /
// 68.3 / 108.9.
constexpr int kBoostPct = 50;

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) {
  return __builtin_bit_cast(bf16x8, v);
}

// Two bf16 -> one uint32 (low half first), round to nearest even: one
// v_cvt_pk_bf16_f32 (two scalar conversions compile to four instructions).
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

__device__ __forceinline__ int round_up_block(int x) {
  return (x + kBlockKeys - 1) / kBlockKeys * kBlockKeys;
}

// -------------------------------------------------------------------- steps
// The key loop works in steps of one 32-key block, a pair of pages whose tiles
// hold exactly the MFMA operands:
//  K: the 1 KiB chunk c of a page's K tile is the A operand of the score
//     MFMA over dims 32c .. 32c+31, lane l holding slot l & 15.
//  V: lane (kq, m) of d block u takes the 16 bytes of dim 16u+m that hold
//     slots 8*(kq>>1) .. +7 of page kq & 1.
constexpr int kSubKeys = 8192;              // keys whose page ids are staged at a time
constexpr int kSubPages = kSubKeys / kPage;

template <int D>
struct KRegs {
  u32x4 x[2][D / 32];  // [page][chunk]
};
template <int NE>
struct VRegs {
  u32x4 x[NE];  // [d block]
};

// Maximum / sum over the four lanes that hold one query row (lanes n, n+16,
// n+32, n+48), with the gfx950 row-swap permutes.
__device__ __forceinline__ float row_max4(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Sum over the same four lanes.  Each swap hands every lane the pair in the
// same order, so the four lanes end with bitwise equal sums.
__device__ __forceinline__ float row_sum4(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The running maximum is only raised when a block's maximum exceeds it by
// more than this (base-2 units): weights then stay below 2^8, and the
// accumulators are rescaled only on such a jump instead of every block.
// The maximum is kept an integer (the block maximum rounded up), so every
// rescale factor and every merge weight, in the workgroup and in the combine,
// is an exact power of two: where a segment is cut, or which rows share its
// tile, moves a row's weights and sums by powers of two only, and its result
// changes only through fp32 summation order.
constexpr float kRescaleSlack = 8.f;
// Running maximum of a row that has seen no key yet: finite, so that no
// difference of two of them is a NaN.
constexpr float kNoMax = -3.402823466e38f;

// Online-softmax state of one wave, for TW row tiles and NE d blocks.  A lane
// holds one query row (lane & 15) of each tile: its running maximum, its own
// lane's share of the sum of the weights (the row's four lanes are added at
// the end), and for each d block u the outputs of dims 16u + 4*(lane>>4) +
// [0..3] from the wave's first d block on.
template <int TW, int NE>
struct RowState {
  float m[TW];
  float l[TW];
  f32x4 o[TW][NE];
};

// Small batches.  When the even share falls to the minimum, each segment is
// instead cut into pieces of at most `cap` keys, as equal as whole blocks
// allow, one piece per workgroup: no workgroup then pays for a second piece
// (its metadata, page ids and pipeline refill), which at this size is a
// large part of the kernel.  The cap leaves at most one piece per CU -- a
// second workgroup on a CU shares its MFMA and LDS with the first and finishes
// last.  The smallest batches take the smallest cap that does so with at most
// kMaxMerge pieces to a segment, which the combine kernel loads in one round trip
// (one request, 716 keys, four layers: 63.1 -> 58.3 us with three blocks instead
// of eight; 16 pieces to a segment took 70.6 us); the others the smallest of 8 to
// 12 blocks that fits, else eight, if the pieces fit the grid.
//   A cut costs the combine's round trip and the partials, written and read, so
// cut_rule bounds the smallest caps by the elements of a segment's partial: the
// least blocks of a piece, the blocks up to which a segment stays whole, and the
// pieces, in sixteenths of the CUs.  us a call, D = 128, S segments of b blocks, r
// rows each: S=64, b=3, r=16 cut 10.4, whole 9.8; b=4 cut 10.2, whole 10.9; b=5, r=64
// in 192 pieces 14.4, in 128 12.5; S=96, b=4, r=256 in 192 pieces 31.7, whole 21.5.
// Of caps from two to twelve blocks, over 864 shapes, the rule's is 1.8% off the best
// in the mean and 27% at most; with the first line for all it was 4.7% and 68%.
// Piece q of n of a `seg`-key segment starts at piece_begin(seg, n, q).
constexpr int kNumPieceCaps = 5;
__device__ __forceinline__ int piece_cap(int c) { return (8 + c) * kBlockKeys; }  // 8..12 blocks
constexpr int kMaxMerge = 8;
struct CutRule {
  int min_blocks, whole_blocks, cu_sixteenths;
};
// Of `total` partial elements over `segs` segments (no division: this is on the way
// to the first load of every workgroup).
__device__ __forceinline__ CutRule cut_rule(float total, float segs) {
  if (total <= 2048.f * segs) return {2, 3, 16};
  if (total <= 4096.f * segs) return {3, 4, 12};
  if (total <= 8192.f * segs) return {3, 5, 10};
  return {3, 5, 5};
}
__device__ __forceinline__ int seg_pieces(int seg, int cap) { return (seg + cap - 1) / cap; }
__device__ __forceinline__ int piece_begin(int seg, int n, int q) {
  return (int)((long long)(seg / kBlockKeys) * q / n) * kBlockKeys;
}

// Stream-K shares alternate in size with the workgroup's grid index.  The
// dispatcher places workgroup b on XCD b mod 8, and with equal shares the
// workgroups on the odd XCDs finished 6-10 us after those on the even ones
// in every clocked launch of the Qwen3-8B shape at B=32, contexts up to 8K,
// while the shader clocks of all eight XCDs agreed within 2%.  Even
// workgroups therefore take kSkewPct percent more than the mean share and
// odd ones as much less (whole blocks).
constexpr int kSkewPct = 6;
__device__ __forceinline__ int share_skew(int share) {
  return (int)((long long)share * kSkewPct / 100) / kBlockKeys * kBlockKeys;
}
// First virtual key of workgroup b's share.
__device__ __forceinline__ int share_begin(int b, int share, int skew) {
  return b * share + (b & 1) * skew;
}
// The workgroup whose share holds virtual key pos.
__device__ __forceinline__ int share_owner(int pos, int share, int skew) {
  const int pair = pos / (2 * share);
  return 2 * pair + (pos - pair * 2 * share >= share + skew ? 1 : 0);
}

// Inclusive prefix sum over the 64 lanes of a wave with DPP row shifts and
// row broadcasts (lanes without a source add 0): six VALU steps, where a
// shuffle-based scan would take six LDS permutes.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ int dpp_src(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, kRowMask, 0xf, false);
}
__device__ __forceinline__ int wave_incl_scan(int v) {
  v += dpp_src<0x111, 0xf>(v);  // row_shr:1
  v += dpp_src<0x112, 0xf>(v);  // row_shr:2
  v += dpp_src<0x114, 0xf>(v);  // row_shr:4
  v += dpp_src<0x118, 0xf>(v);  // row_shr:8
  v += dpp_src<0x142, 0xa>(v);  // row_bcast:15
  v += dpp_src<0x143, 0xc>(v);  // row_bcast:31
  return v;
}

// Largest of the wave's values (not negative), in lane 63.
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, dpp_src<0x111, 0xf>(v));
  v = max(v, dpp_src<0x112, 0xf>(v));
  v = max(v, dpp_src<0x114, 0xf>(v));
  v = max(v, dpp_src<0x118, 0xf>(v));
  v = max(v, dpp_src<0x142, 0xa>(v));
  v = max(v, dpp_src<0x143, 0xc>(v));
  return v;
}

// Block-wide exclusive scan of one value per thread: the wave scan, then the
// wave totals through LDS (`tot` receives the block total).
template <int NW>
__device__ __forceinline__ int block_excl_scan(int v, int *lds_tot, int &tot) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int incl = wave_incl_scan(v);
  if (lane == kWave - 1) lds_tot[wave] = incl;
  __syncthreads();
  int before = 0;
  tot = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    before += w < wave ? lds_tot[w] : 0;
    tot += lds_tot[w];
  }
  return before + incl - v;
}

template <int TW, int NE>
__device__ __forceinline__ void clear_state(RowState<TW, NE> &st) {
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    st.m[t] = kNoMax;
    st.l[t] = 0.f;
#pragma unroll
    for (int u = 0; u < NE; ++u) st.o[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
}

// Scores of one step for the wave's tiles (raw: the scale is positive and
// applied inside the exponent).  Element (h, q) of a lane is key
// t0 + 16h + 4*(lane>>4) + q.
template <int TW>
struct Scores {
  f32x4 x[TW][2];
};
template <int D, int TW, typename QOps>
__device__ __forceinline__ void step_scores(const KRegs<D> &k, const QOps &qv, Scores<TW> &s) {
#pragma unroll
  for (int t = 0; t < TW; ++t) {
#pragma unroll
    for (int h = 0; h < 2; ++h) s.x[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        s.x[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            as_bf16x8(__builtin_bit_cast(uint4, k.x[h][c])), qv.r[t][c], s.x[t][h], 0, 0, 0);
    }
  }
}

// Online softmax and the PV product of one step.  A V whose rows have scales
// (`VScale::kOn`: x[h][q] of the lane's keys) takes them in the weights.
struct NoScale {
  static constexpr bool kOn = false;
  f32x4 x[2];
};
template <int TW, int NE, typename VScale = NoScale>
__device__ __forceinline__ void step_update(const Scores<TW> &s, const VRegs<NE> &v,
                                            float scale_log2, RowState<TW, NE> &st,
                                            const VScale &scale = VScale()) {
  // a lane's own keys decide whether any row's maximum moves; only then are
  // the row's four lanes brought together
  bool jump = false;
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        top = fmaxf(top, __builtin_fmaf(s.x[t][h][q], scale_log2, -st.m[t]));
    jump |= top > kRescaleSlack;
  }
  if (__builtin_amdgcn_ballot_w64(jump) != 0) {
#pragma unroll
    for (int t = 0; t < TW; ++t) {
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) top = fmaxf(top, s.x[t][h][q]);
      const float m_new = fmaxf(st.m[t], ceilf(row_max4(top) * scale_log2));
      // 0 on a row's first visible step, 1 for a row that still sees nothing
      const float alpha = __builtin_amdgcn_exp2f(st.m[t] - m_new);
      st.l[t] *= alpha;
#pragma unroll
      for (int u = 0; u < NE; ++u) st.o[t][u] *= alpha;
      st.m[t] = m_new;
    }
  }
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    // P enters the bf16 PV product as a pair: hi = P rounded to bf16 and
    // lo = the remainder rounded to bf16, so hi + lo carries P to about
    // 2^-17 of its value and the weights add no error next to the output's
    // own bf16 rounding.  The row sum adds the fp32 weights themselves.
    uint32_t hi[2][2], lo[2][2];
    float psum[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float pw[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        pw[q] = __builtin_amdgcn_exp2f(
            __builtin_fmaf(s.x[t][h][q], scale_log2, -st.m[t]));
      psum[h] = (pw[0] + pw[1]) + (pw[2] + pw[3]);
      if constexpr (VScale::kOn)
#pragma unroll
        for (int q = 0; q < 4; ++q) pw[q] *= scale.x[h][q];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t x = pack_bf16x2(pw[2 * w], pw[2 * w + 1]);
        hi[h][w] = x;
        lo[h][w] = pack_bf16x2(pw[2 * w] - __uint_as_float(x << 16),
                               pw[2 * w + 1] - __uint_as_float(x & 0xFFFF0000u));
      }
    }
    st.l[t] += psum[0] + psum[1];
    // lane (kq, n) holds slots 4kq .. +3 of both pages; trading odd rows of
    // page 0's against even rows of page 1's leaves it slots 8*(kq>>1) .. +7
    // of page kq & 1, the keys of its V operand
    const auto h0 = __builtin_amdgcn_permlane16_swap(hi[0][0], hi[1][0], false, false);
    const auto h1 = __builtin_amdgcn_permlane16_swap(hi[0][1], hi[1][1], false, false);
    const auto l0 = __builtin_amdgcn_permlane16_swap(lo[0][0], lo[1][0], false, false);
    const auto l1 = __builtin_amdgcn_permlane16_swap(lo[0][1], lo[1][1], false, false);
    const bf16x8 ph = as_bf16x8(make_uint4(h0[0], h1[0], h0[1], h1[1]));
    const bf16x8 pl = as_bf16x8(make_uint4(l0[0], l1[0], l0[1], l1[1]));
#pragma unroll
    for (int u = 0; u < NE; ++u)
      st.o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          as_bf16x8(__builtin_bit_cast(uint4, v.x[u])), ph, st.o[t][u], 0, 0, 0);
#pragma unroll
    for (int u = 0; u < NE; ++u)
      st.o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          as_bf16x8(__builtin_bit_cast(uint4, v.x[u])), pl, st.o[t][u], 0, 0, 0);
  }
}

// --------------------------------------------------------------------- ring
// K and V stream through an LDS ring of kStages stages, all of them in flight
// in registers: one step a stage with four waves, two with eight (a tile or
// more for every wave).  Each wave loads its tiles of a stage (a page's K or
// V, contiguous 1 KiB loads), writes them to the ring when the stage comes up,
// and after the barrier the waves read their operands from it.  With four
// waves, stages of two steps (two in flight, 128 KiB to a CU instead of 96)
// measured slower: B=32, contexts to 8K 104.4 -> 107-112 us, with eight query
// heads to a KV head and contexts to 16K 229 -> 238 us.
template <int D, int NW>
struct Ring {
  static constexpr int kSteps = NW / 4;
  static constexpr int kKeys = kSteps * kBlockKeys;
  static constexpr int kPages = kKeys / kPage;
  static constexpr int kTile = kPage * D * 2;          // bytes of a page's K or V
  static constexpr int kStage = 2 * kPages * kTile;    // K tiles, then V tiles (kSteps * 16 KiB)
  static constexpr int kStages = 3;
  static constexpr int kTiles = 2 * kPages / NW;       // tiles a wave loads per stage
  static constexpr int kBytes = kStages * kStage;
  // page and kind (0: K, 1: V) of a wave's q-th tile
  static __device__ __forceinline__ int page(int wave, int q) { return (wave * kTiles + q) >> 1; }
  static __device__ __forceinline__ int kind(int wave, int q) { return (wave * kTiles + q) & 1; }
};

// V tiles sit in the ring with their 16-byte units (dim, half of the slots)
// permuted inside each 1 KiB, so that the operand reads are free of bank
// conflicts: global unit u = 2*dim + half is LDS unit v_unit(u), and
// v_unit_inv is the inverse.  Aligned groups of four lanes still load aligned
// 64-byte pieces.
__device__ __forceinline__ int v_sel(int k) { return ((k >> 1) ^ (k >> 2)) & 1; }
__device__ __forceinline__ int v_unit(int u) {
  const int k = u >> 2, j = (u >> 1) & 1, b = u & 1;
  return 4 * k + 2 * (b ^ v_sel(k)) + j;
}
__device__ __forceinline__ int v_unit_inv(int l) {
  const int k = l >> 2, j = l & 1, b = ((l >> 1) & 1) ^ v_sel(k);
  return 4 * k + 2 * j + b;
}

// A wave's part of the work on a piece: its row tiles and its d blocks.
struct Role {
  int tile0, e_lo;
  bool active;
};

}  // namespace
}  // namespace dsv
