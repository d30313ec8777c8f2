// tree.hip -- attention of drafted trees over a paged GQA KV cache, bf16 or 8-bit
// (gfx950), and the masks that a tree's parents stand for.
//
// What it computes: row j of request i (node j of its tree) attends to the committed
// context, keys 0 .. ctx_i - 1, and to the nodes n whose bit is set in the row's mask,
// keys ctx_i + n (without masks: n <= j, the causal block).  A row that sees no key is 0.
//
// How.  The key loop, the LDS ring and the arithmetic of the work split are verify
// attention's (attn_core.h).  What differs:
//  * A tree of 64 nodes under 16 query heads has 1,024 rows to a KV head, more than a
//    workgroup's registers hold.  A request's rows are cut into row groups of up to
//    `group_rows` rows, and a segment of the work is (request, KV head, row group); the
//    groups of one KV head lie next to each other in the plan, so that the second one's
//    K and V come out of the cache.
//  * Masks only matter in the one to three blocks that hold nodes.  There each lane
//    takes its row's 64-bit mask, shifted so that bit b is key t0 + b; other blocks are
//    as in verify attention.
//  * Nodes that a row does not see may hold anything, also infinities and NaN: a
//    weight of 0 times such a V would be NaN in the matrix product.  V cells of node blocks
//    that are not finite are therefore left out on the way to the ring, as are cells past
//    the nodes, and noted; a piece that met one adds them, at its end and cell by cell, to
//    the rows that see them: a node's to those with its bit, one of the context, which
//    shares the block, to all.  (Telling the two apart on the way to the ring took one
//    request of 16 nodes from 12.9 to 13.4 us a call.)
//  * An 8-bit cache is half the bytes.  Codes become bf16 on the way from the load
//    registers to the LDS ring, which is exact, so the ring's layout and all after it are
//    the bf16 cache's, and each code is converted once for all waves.  A K tile's lane
//    holds dims of one slot, so K's scale goes into the conversion instruction; V's lane
//    holds the slots of one dim, so V's scales, through LDS, go into the fp32 weights.
//    Both are powers of two: exact.
//
// What bounds it, and what it measured (MI355X, split + combine kernels, us a call):
//   B=32, 32/8 heads, contexts to 8K, bf16 cache (0.6 GB): one node 103, 5.8 TB/s (HBM);
//     16 nodes (4 row tiles) 120; 32 nodes (8) 157; 64 nodes (16) 283: from five tiles on
//     the matrix products and the softmax of the waves, which share their barriers and
//     so their phases.
//   The same with the 8-bit cache (0.3 GB): 78, 97, 146, 270.  One to four tiles are bound
//     by instruction issue: four waves of which each does the softmax of its rows for its
//     own dims (with no products the loads and conversions take 62).
//   B=16, 64/8 heads, 32 to 64 nodes, contexts to 16K, bf16 (0.25 TFLOP): 440, 0.57 PFLOP/s
//     counting each product once (the weights' second half adds another half); the
//     vector units are busy 37% of the time and the matrix units 35%, hardly at once.
//   B=1, 16 nodes, context 700: 10.0 + 3.5, the chain from launch to the last block.
// Tried, and slower: each wave streaming blocks of its own straight into the operands'
// registers, no LDS and no barriers (64 nodes: 1,438; the four-tile form spills, and loads
// that land in accumulation registers are waited for at once; D = 64, which does not spill,
// 209 against 168); one wave per SIMD with four tiles (500); six stages in flight
// (8-bit, 24 nodes: 245 against 128, spills); the tiles of a request dealt evenly with a
// branch for each (10 tiles 228 against 239, 16 tiles 309 against 293: the branch keeps one
// tile's products from running under another's softmax); neighbouring shares on one
// XCD, and cached loads, for several row groups (490 either way).
#include "attn_core.h"

#include <atomic>

namespace dsv {
namespace {

// Combine kernel (one request of 16 nodes, context 700: 13.6 us a call, with 1,024 threads
// 15.2; the large batches alike).
constexpr int kCombThreads = 256;

// Request-level metadata after the device-side checks: seg is ctx + k rounded up to
// whole blocks, 0 for a request without rows or with metadata out of range; groups its
// row groups.
struct TreeMeta {
  int q0, k, ctx, len, seg, groups;
};

__device__ __forceinline__ TreeMeta tree_meta(const TreeParams &p, int q0, int q1, int ctx) {
  TreeMeta r;
  r.q0 = q0;
  r.ctx = ctx;
  r.k = q1 - q0;
  const bool ok = q0 >= 0 && q1 <= p.cap && r.k > 0 && r.k <= p.max_nodes && ctx >= 0 &&
                  ctx <= p.max_kv_len - r.k;
  r.len = ok ? ctx + r.k : 0;
  r.seg = round_up_block(r.len);
  r.groups = ok ? (p.group * r.k + p.group_rows - 1) >> __builtin_ctz(p.group_rows) : 0;
  return r;
}
__device__ __forceinline__ TreeMeta tree_meta(const TreeParams &p, int i) {
  return tree_meta(p, p.cu[i], p.cu[i + 1], p.ctx[i]);
}

// A workgroup's share of the work, [start, end) in keys over all segments laid end to
// end: request, then KV head, then row group.
struct TreeShare {
  int start, end;
  int i, sub, off;  // request, segment of the request, virtual offset where `start` falls
  int lead;         // keys of lead-in per segment: kLeadKeys (stream-K) or 0
  TreeMeta first;
};

// The plan of verify attention (plan_share in attn.hip: stream-K shares, or equal pieces
// of segments for small batches) over segments whose number differs by request.
// Workgroup 0 publishes the prefixes for the combine kernel.  LDS use: scan totals, the
// located share, the small-batch counts.
template <int D, int NW>
__device__ TreeShare tree_plan(const TreeParams &p, int *lds) {
  constexpr int kThreads = NW * kWave;
  const int B = p.num_reqs, tid = threadIdx.x;
  int live = p.cu[B];
  const int per = (B + kThreads - 1) / kThreads;
  const int lo = min(B, tid * per), hi = min(B, lo + per);
  TreeMeta mine = {};  // this thread's request where each has one
  int work = 0, segs = 0;
  for (int i = lo; i < hi; ++i) {
    mine = tree_meta(p, i);
    segs += mine.groups * p.hkv;
    work += mine.groups * p.hkv * mine.seg;
  }
  asm volatile("" : "+v"(live));  // its load is in flight with the others
  auto meta = [&](int i) { return per == 1 ? mine : tree_meta(p, i); };
  int total;
  const int excl = block_excl_scan<NW>(work, lds, total);
  int *loc = lds + 2 * NW;  // located share: i, sub, off, q0, q1, ctx, start, end
  int share = (total + (int)gridDim.x - 1) / (int)gridDim.x;
  share = max(kMinShare, round_up_block(share));
  int cap = 0;
  if (share == kMinShare) {
    // pieces under each cap and, last, segments: at most eight blocks for every
    // workgroup of the grid, so they fit 16 bits
    constexpr int kPacked = kNumPieceCaps / 2 + 1;
    uint32_t cnt[kPacked] = {};
    int longest = 0;
    for (int i = lo; i < hi; ++i) {
      const TreeMeta r = meta(i);
      const int m = r.groups * p.hkv;
#pragma unroll
      for (int c = 0; c < kNumPieceCaps; ++c)
        cnt[c / 2] += (uint32_t)(m * seg_pieces(r.seg, piece_cap(c))) << (16 * (c % 2));
      cnt[kPacked - 1] += (uint32_t)m << 16;
      longest = max(longest, r.seg);
    }
    uint32_t *red = reinterpret_cast<uint32_t *>(loc + 8);  // [kPacked + 1][NW]
    const int lane = tid % kWave, wave = tid / kWave;
#pragma unroll
    for (int c = 0; c <= kPacked; ++c) {
      const int v = c < kPacked ? wave_incl_scan((int)cnt[c < kPacked ? c : 0]) : wave_max(longest);
      if (lane == kWave - 1) red[c * NW + wave] = (uint32_t)v;
    }
    __syncthreads();
    const int one_per_cu = min(p.num_cu, (int)gridDim.x);
    longest = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) longest = max(longest, (int)red[kPacked * NW + w]);
    int pieces[kNumPieceCaps + 1];
#pragma unroll
    for (int c = 0; c <= kNumPieceCaps; ++c) {
      int t = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) t += (int)(red[c / 2 * NW + w] >> (16 * (c % 2)) & 0xFFFFu);
      pieces[c] = t;
    }
#pragma unroll
    for (int c = kNumPieceCaps - 1; c >= 0; --c)
      if (pieces[c] <= one_per_cu || (c == 0 && cap == 0 && pieces[c] <= (int)gridDim.x))
        cap = piece_cap(c);
    const int all = pieces[kNumPieceCaps];  // segments
    const CutRule rule = NW == 8 && D == 128
                             ? CutRule{3, 5, 5}
                             : cut_rule((float)live * (float)(p.group * p.hkv * D), (float)all);
    const int spare = min(p.num_cu * rule.cu_sixteenths / 16, (int)gridDim.x) - all;
    if (spare > 0 && longest > rule.whole_blocks * kBlockKeys) {
      const int blocks = max(rule.min_blocks, max((longest / kBlockKeys + kMaxMerge - 1) / kMaxMerge,
                                                  (total / kBlockKeys + spare - 1) / spare));
      if (blocks < 8) cap = blocks * kBlockKeys;
    }
  }
  const bool seg_mode = cap > 0;
  const int lead = seg_mode ? 0 : kLeadKeys;
  int my_pc = 0, total_pc = 0, excl_pc = 0;          // pieces (small batches)
  int my_v = work, total_v = total, excl_v = excl;  // keys with lead-ins (stream-K)
  if (seg_mode) {
    for (int i = lo; i < hi; ++i) {
      const TreeMeta r = meta(i);
      my_pc += r.groups * p.hkv * seg_pieces(r.seg, cap);
    }
    excl_pc = block_excl_scan<NW>(my_pc, lds + NW, total_pc);
  } else {
    my_v = work + lead * segs;
    excl_v = block_excl_scan<NW>(my_v, lds + NW, total_v);
    share = (total_v + (int)gridDim.x - 1) / (int)gridDim.x;
    share = max(kMinShare, round_up_block(share));
  }
  if (blockIdx.x == 0) {
    int acc = excl_v, acc_pc = excl_pc;
    for (int i = lo; i < hi; ++i) {
      const TreeMeta r = meta(i);
      const int m = r.groups * p.hkv;
      p.plan[i] = acc;
      p.plan[B + 2 + i] = acc_pc;
      acc += m * (r.seg + lead);
      if (seg_mode) acc_pc += m * seg_pieces(r.seg, cap);
    }
    if (tid == 0) {
      p.plan[B] = total_v;
      p.plan[B + 1] = seg_mode ? -cap : share;  // negative: the small-batch cap
      p.plan[2 * B + 2] = total_pc;
    }
  }
  const int b = (int)blockIdx.x;
  int start = total_v, end = total_v;
  if (!seg_mode) {
    const int skew = share_skew(share);
    start = min(total_v, share_begin(b, share, skew));
    end = min(total_v, share_begin(b + 1, share, skew));
  }
  // the thread whose requests contain this workgroup's share locates it
  const bool here = seg_mode ? excl_pc <= b && b < excl_pc + my_pc
                             : start < total_v && excl_v <= start && start < excl_v + my_v;
  if (here) {
    int acc = excl_v, acc_pc = excl_pc;
    for (int i = lo; i < hi; ++i) {
      const TreeMeta r = meta(i);
      const int m = r.groups * p.hkv, segv = r.seg + lead;
      const int n = seg_mode ? seg_pieces(r.seg, cap) : 0;
      int sub = -1, off = 0, s0 = 0, s1 = 0;
      if (seg_mode) {
        if (b < acc_pc + m * n) {
          const int rel = b - acc_pc;
          sub = rel / n;
          const int q = rel % n;
          off = piece_begin(r.seg, n, q);
          s0 = acc + sub * r.seg + off;
          s1 = s0 + piece_begin(r.seg, n, q + 1) - off;
        }
      } else if (start < acc + m * segv) {
        const int rel = start - acc;
        sub = rel / segv;
        off = rel % segv;
        s0 = start;
        s1 = end;
      }
      if (sub >= 0) {
        loc[0] = i;
        loc[1] = sub;
        loc[2] = off;
        loc[3] = r.q0;
        loc[4] = r.q0 + r.k;
        loc[5] = r.ctx;
        loc[6] = s0;
        loc[7] = s1;
        break;
      }
      acc += m * segv;
      acc_pc += m * n;
    }
  }
  __syncthreads();
  auto uni = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const bool has = uni(seg_mode ? b < total_pc : start < total_v) != 0;
  TreeShare sh;
  sh.lead = uni(lead);
  sh.start = has ? uni(loc[6]) : 0;
  sh.end = has ? uni(loc[7]) : 0;
  sh.i = uni(loc[0]);
  sh.sub = uni(loc[1]);
  sh.off = uni(loc[2]);
  const int q0 = uni(loc[3]), q1 = uni(loc[4]), ctx = uni(loc[5]);
  sh.first = tree_meta(p, q0, q1, ctx);
  return sh;
}

// ------------------------------------------------------------------------ pieces
// A piece: the workgroup's keys [key_begin, key_end) of request i, KV head g, row
// group rg.
struct TreePiece {
  int i, g, rg, key_begin, key_end, slot, prio_end;
  bool complete;
  TreeMeta rq;
  int rows;  // of the row group
};

// The wave's query operands and its rows' masks.
template <int D, int TW>
struct TreeQ {
  bf16x8 r[TW][D / 32];
  unsigned long long mask[TW];
};

// A row past the live ones loads row 0 of the request and is zeroed.
template <int D, int TW>
__device__ __forceinline__ void load_tree_q(const TreeParams &p, const TreePiece &x, int tile0,
                                            int lane, TreeQ<D, TW> &qv) {
  const int kq = lane >> 4, n = lane & 15;
  const int lg = __builtin_ctz(p.group);
  u32x4 w[TW][D / 32];
  bool valid[TW];
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    const int rr = (tile0 + t) * 16 + n;
    valid[t] = rr < x.rows;
    const int at = valid[t] ? x.rg * p.group_rows + rr : 0;
    const int j = at >> lg, hh = at & (p.group - 1);
    qv.mask[t] = p.masks ? p.masks[x.rq.q0 + j] : (2ull << j) - 1;
    const uint16_t *row = p.q + ((size_t)(x.rq.q0 + j) * p.hq + (size_t)x.g * p.group + hh) * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      w[t][c] = *reinterpret_cast<const u32x4 *>(row + 32 * c + 8 * kq);
  }
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    const uint32_t keep = valid[t] ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      qv.r[t][c] = as_bf16x8(__builtin_bit_cast(uint4, w[t][c] & u32x4{keep, keep, keep, keep}));
  }
}

// Masks of a step that holds keys past the context.  Element (h, q) of a lane is key
// t0 + 16h + 4*(lane>>4) + q.
template <int TW>
__device__ __forceinline__ void tree_mask(int t0, int se, int ctx,
                                          const unsigned long long (&mask)[TW], int lane,
                                          Scores<TW> &s) {
  const int kq = lane >> 4;
  const int node = t0 - ctx;  // of key t0: negative in the context
  const uint32_t inside = se - t0 >= 32 ? 0xFFFFFFFFu : (1u << (se - t0)) - 1;
#pragma unroll
  for (int t = 0; t < TW; ++t) {
    uint32_t seen;  // bit b: the row sees key t0 + b
    if (node >= 0)
      seen = (uint32_t)(mask[t] >> node);
    else if (node > -32)
      seen = (uint32_t)mask[t] << -node | ((1u << -node) - 1);
    else
      seen = 0xFFFFFFFFu;
    seen = (seen & inside) >> (4 * kq);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // in integers, as in only_finite
        const uint32_t keep = (uint32_t)((int)(seen << (31 - 16 * h - q)) >> 31);
        s.x[t][h][q] = __uint_as_float((__float_as_uint(s.x[t][h][q]) & keep) | (0xFF800000u & ~keep));
      }
  }
}

// -------------------------------------------------------------------------- ring
// What a wave needs to run the ring over one sub-piece.  Of every stage a wave loads one
// tile: page wave >> 1, K or V by wave & 1.
constexpr int kIdRegs = 4;  // windows of 64 stages whose page ids a wave holds
struct TreeRing {
  const char *base;       // the wave's tile in page 0, plus the lane's offset
  const uint8_t *scales;  // its scales in page 0, plus the lane's slot (8-bit cache)
  uint32_t page_bytes, scale_bytes;
  u32x4 id;               // lane j of id[w]: the page of stage 64w + j
  int ns;                 // stages
  int sb, se, ctx;        // first key, end of the keys, committed context
  int prio_end;           // key at which the wave priority returns to the default
  int *not_finite;        // LDS: a V cell of a node was left out
};

// A wave's tile of one stage on its way to LDS: bf16 cells, or codes with the scale of
// slot lane & 15.
template <int D, bool kFp8>
struct TreeStage {
  u32x4 x[kFp8 ? D / 64 : D / 32];
  uint32_t e;
};

// A step's V scales by key, of the lane's eight keys.
template <bool kFp8>
struct VScales {
  static constexpr bool kOn = kFp8;
  f32x4 x[2];
};

// Page ids of the sub-piece's stages, each wave for its own tiles and straight into
// registers: through LDS they took a barrier at the start and a wait in every step.  An
// id outside [0, num_pages) breaks the contract and reads page 0 instead; pages past the
// sub-piece read page 0 and are masked.
template <int NW>
__device__ __forceinline__ void load_ids(const TreeParams &p, int i, int wave, int lane,
                                         TreeRing &c) {
  constexpr int kPages = NW / 2;
  const int32_t *pt = p.page_table + (size_t)i * p.max_pages + c.sb / kPage;
  const int npg = (c.se - c.sb + kPage - 1) / kPage;
  auto load = [&](int w) {
    const int at = kPages * (64 * w + lane) + (wave >> 1);
    const int id = at < npg ? pt[at] : 0;
    return (unsigned)id < (unsigned)p.num_pages ? (uint32_t)id : 0u;
  };
  c.id = u32x4{load(0), load(1), load(2), load(3)};
}

// Loads the wave's tile of stage b.  Past the last stage it reads page 0 (in cache, never
// used): the loop then has one shape, and the compiler can wait for exactly the stage
// each step writes.
template <int D, bool kFp8>
__device__ __forceinline__ void tree_ring_load(const TreeRing &c, int b, TreeStage<D, kFp8> &r) {
  const int w = b >> 6;
  const u32x4 all = c.id;
  const uint32_t lo = w & 1 ? all[1] : all[0], hi = w & 1 ? all[3] : all[2];
  const int ids = (int)(w & 2 ? hi : lo);
  const uint32_t id = b < c.ns ? __builtin_amdgcn_readlane(ids, b & 63) : 0;
  const char *t = c.base + (size_t)id * c.page_bytes;
#pragma unroll
  for (int x = 0; x < (kFp8 ? D / 64 : D / 32); ++x)
    r.x[x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(t + 1024 * x));
  if (kFp8) r.e = c.scales[(size_t)id * c.scale_bytes];
}

// Two codes (the low or high half of a word) times a power of two, as bf16: exact.
template <bool kHigh>
__device__ __forceinline__ uint32_t bf16_of_codes(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, kHigh));
}

// Leaves out the cells of a V tile, the lane's sixteen or eight slots of a dim from key
// on, that lie past the keys or are not finite, and notes the latter.  (Cells of the context
// too, where a stage holds both: add_not_finite brings them back.)
template <bool kFp8>
__device__ __forceinline__ u32x4 only_finite(u32x4 x, int key, int se, int *not_finite) {
  // in integer arithmetic on whole words: conditions by cell would take scalar registers
  // that the key loop needs (8-bit cache, one node: 90 us a call with them, 78 without)
  constexpr int kPer = kFp8 ? 4 : 2, kBits = 32 / kPer;  // cells of a word, bits of a cell
  constexpr uint32_t kSpecial = kFp8 ? 0x7F7F7F7Fu : 0x7F807F80u;  // a cell's bits if not finite
  constexpr uint32_t kOne = kFp8 ? 0x01010101u : 0x00800080u;      // carries those to its top bit
  constexpr uint32_t kTop = kFp8 ? 0x80808080u : 0x80008000u;
  uint32_t found = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int cells = min(max(se - key - kPer * w, 0), kPer);  // before the end
    const uint32_t keep = (uint32_t)((1ull << (kBits * cells)) - 1);
    const uint32_t top = ((x[w] & kSpecial) + kOne) & kTop;
    const uint32_t odd = (top - (top >> (kBits - 1))) | top;  // whole cells
    found |= odd & keep;
    x[w] &= keep & ~odd;
  }
  if (found) *not_finite = 1;
  return x;
}

// Writes a wave's tile to the ring.  8-bit K: lane l holds sixteen dims of slot l & 15,
// two of the ring's 8-dim chunks.  8-bit V: a dim's sixteen slots; the scales of the
// stage's keys go to vscale.  A scale is its exponent's bits; 255, which no writer leaves
// and a slot past the keys may hold, would be an infinity that turns weights of 0 to NaN.
template <int D, int NW, bool kFp8>
__device__ __forceinline__ void tree_ring_store(const TreeRing &c, int b, char *stage,
                                                float *vscale, int wave, int lane,
                                                TreeStage<D, kFp8> &r) {
  using R = Ring<D, NW>;
  static_assert(R::kTiles == 1, "one tile to a wave");
  const int page = wave >> 1, kind = wave & 1;
  char *tile = stage + (kind * R::kPages + page) * R::kTile;
  const int t0 = c.sb + b * R::kKeys;
  if (kind && t0 + R::kKeys > min(c.ctx, c.se)) {
    const int key = t0 + kPage * page + (kFp8 ? 0 : 8 * (v_unit_inv(lane) & 1));
#pragma unroll
    for (int x = 0; x < (kFp8 ? D / 64 : D / 32); ++x)
      r.x[x] = only_finite<kFp8>(r.x[x], key, c.se, c.not_finite);
  }
  if constexpr (!kFp8) {
#pragma unroll
    for (int x = 0; x < D / 32; ++x) *reinterpret_cast<u32x4 *>(tile + 1024 * x + 16 * lane) = r.x[x];
  } else {
    const float scale = __uint_as_float(min(r.e, 254u) << 23);
    const float by = kind ? 1.f : scale;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
      const int dim = 64 * x + lane;  // V's; K: chunk 2 * (4x + lane / 16) of slot lane & 15
      char *k_to = tile + 16 * (2 * (4 * x + (lane >> 4)) * 16 + (lane & 15));
      char *v_to = tile + 1024 * (dim / 32);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a = r.x[x][2 * h], b2 = r.x[x][2 * h + 1];
        *reinterpret_cast<u32x4 *>(kind ? v_to + 16 * v_unit(2 * (dim % 32) + h) : k_to + 256 * h) =
            u32x4{bf16_of_codes<false>(a, by), bf16_of_codes<true>(a, by),
                  bf16_of_codes<false>(b2, by), bf16_of_codes<true>(b2, by)};
      }
    }
    if (kind && lane < kPage) vscale[kPage * page + lane] = scale;
  }
}

// One stage in ring slot S: write it, load the stage kStages ahead, and after the
// barrier compute the wave's steps of it.
template <int D, int TW, int NE, int NW, bool kFp8, int S>
__device__ __forceinline__ void tree_ring_step(const TreeRing &c, char *ring, float *vscales,
                                               int b, int wave,
                                               int lane, TreeStage<D, kFp8> &r,
                                               const TreeQ<D, TW> &qv, const Role &role,
                                               float scale_log2, RowState<TW, NE> &st) {
  using R = Ring<D, NW>;
  char *stage = ring + S * R::kStage;
  float *vscale = vscales + S * R::kKeys;
  tree_ring_store<D, NW, kFp8>(c, b, stage, vscale, wave, lane, r);
  tree_ring_load<D, kFp8>(c, b + R::kStages, r);
  __syncthreads();
  if (c.sb + b * R::kKeys >= c.prio_end) __builtin_amdgcn_s_setprio(0);
  if (!role.active) return;
  const int kq = lane >> 4, m = lane & 15;
  const char *vb = stage + (R::kPages + (kq & 1)) * R::kTile + 16 * v_unit(2 * m + (kq >> 1)) +
                   512 * role.e_lo;
#pragma unroll 1
  for (int sub = 0; sub < R::kSteps; ++sub) {
    const int t0 = c.sb + b * R::kKeys + sub * kBlockKeys;
    if (t0 >= c.se) break;
    KRegs<D> k;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
        k.x[h][x] = *reinterpret_cast<const u32x4 *>(
            stage + (sub * 2 + h) * R::kTile + 1024 * x + 16 * lane);
    Scores<TW> s;
    step_scores<D, TW>(k, qv, s);
    VRegs<NE> v;
#pragma unroll
    for (int u = 0; u < NE; ++u)
      v.x[u] = *reinterpret_cast<const u32x4 *>(vb + sub * 2 * R::kTile + 512 * u);
    VScales<kFp8> vs;
    if (kFp8)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        vs.x[h] = *reinterpret_cast<const f32x4 *>(vscale + sub * kBlockKeys + kPage * h + 4 * kq);
    if (t0 + kBlockKeys > min(c.ctx, c.se))
      tree_mask<TW>(t0, c.se, c.ctx, qv.mask, lane, s);
    step_update<TW, NE>(s, v, scale_log2, st, vs);
  }
}

template <int D, int TW, int NE, int NW, bool kFp8>
__device__ __forceinline__ void tree_ring_run(const TreeRing &c, char *ring, float *vscales,
                                              int wave, int lane,
                                              const TreeQ<D, TW> &qv, const Role &role,
                                              float scale_log2, RowState<TW, NE> &st) {
  constexpr int kStages = Ring<D, NW>::kStages;
  TreeStage<D, kFp8> r[kStages];
  // in stage order (the empty asm keeps the compiler from reordering them), so that
  // each step waits only for its own stage
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    tree_ring_load<D, kFp8>(c, s, r[s]);
    asm volatile("" ::: "memory");
  }
  for (int b = 0; b < c.ns; b += kStages) {
    tree_ring_step<D, TW, NE, NW, kFp8, 0>(c, ring, vscales, b, wave, lane, r[0], qv, role, scale_log2, st);
    tree_ring_step<D, TW, NE, NW, kFp8, 1>(c, ring, vscales, b + 1, wave, lane, r[1], qv, role, scale_log2, st);
    tree_ring_step<D, TW, NE, NW, kFp8, 2>(c, ring, vscales, b + 2, wave, lane, r[2], qv, role, scale_log2, st);
  }
}

// Writes NE d blocks from e_lo of a finished row tile: bf16 output when the piece is
// the whole segment, else the fp32 partial in this workgroup's slot (0: the segment
// where its share starts, 1: where it ends).
template <int D, int NE>
__device__ __forceinline__ void write_tree_rows(const TreeParams &p, const TreePiece &x, int rt,
                                                int e_lo, int lane, float m, float l,
                                                const f32x4 (&o)[NE]) {
  const int kq = lane >> 4;
  const int rr = rt * 16 + (lane & 15);
  if (rr >= x.rows) return;
  const int dim = 16 * e_lo + 4 * kq;
  if (x.complete) {
    const int at = x.rg * p.group_rows + rr;
    const int j = at >> __builtin_ctz(p.group), hh = at & (p.group - 1);
    const size_t row = (size_t)(x.rq.q0 + j) * p.hq + (size_t)x.g * p.group + hh;
    // a row whose keys have no weight is 0, whatever their values are
    const float inv = 1.f / l;
    const uint32_t keep = l == 0.f ? 0u : 0xFFFFFFFFu;
#pragma unroll
    for (int u = 0; u < NE; ++u) {
      uint2 w;
      w.x = pack_bf16x2(o[u][0] * inv, o[u][1] * inv) & keep;
      w.y = pack_bf16x2(o[u][2] * inv, o[u][3] * inv) & keep;
      *reinterpret_cast<uint2 *>(p.out + row * D + dim + 16 * u) = w;
    }
  } else {
    const size_t prow = ((size_t)blockIdx.x * 2 + x.slot) * p.group_rows + rr;
#pragma unroll
    for (int u = 0; u < NE; ++u)
      *reinterpret_cast<f32x4 *>(p.part_o + prow * D + dim + 16 * u) = o[u];
    if (e_lo == 0 && kq == 0) p.part_ml[prow] = make_float2(m, l);
  }
}

// Adds the V cells that are not finite of the stages in which the ring left them out, to
// the rows that see them.  Those are the stages from the one on that reaches past the
// context or past the piece's end (tree_ring_store's condition); every row sees the keys
// before ctx, also those of a piece that ends inside the context.
template <int D, int TW, int NE, int NW, bool kFp8>
__device__ __forceinline__ void add_not_finite(const TreeParams &p, const TreePiece &x,
                                               const Role &role, int lane,
                                               const unsigned long long (&mask)[TW],
                                               RowState<TW, NE> &st) {
  constexpr int kKeys = Ring<D, NW>::kKeys;  // stages lie at multiples of it from key_begin
  const int kq = lane >> 4, ctx = x.rq.ctx;
  const int whole = max(min(ctx, x.key_end) - x.key_begin, 0) / kKeys;  // stages as they are
#pragma unroll 1
  for (int key = x.key_begin + whole * kKeys; key < x.key_end; ++key) {
    const int id = p.page_table[(size_t)x.i * p.max_pages + key / kPage];
    const size_t page = (unsigned)id < (unsigned)p.num_pages ? id : 0;
    const size_t tile = ((page * 2 + 1) * p.hkv + x.g) * kPage * D + key % kPage;
#pragma unroll
    for (int u = 0; u < NE; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const size_t at = tile + (size_t)(16 * (role.e_lo + u) + 4 * kq + q) * kPage;
        float v = 0.f;
        if constexpr (kFp8)
          v = (((const uint8_t *)p.kv)[at] & 0x7F) == 0x7F ? NAN : 0.f;
        else
          v = __uint_as_float((uint32_t)((const uint16_t *)p.kv)[at] << 16);
        if (fabsf(v) < INFINITY) continue;
#pragma unroll
        for (int t = 0; t < TW; ++t)
          if (key < ctx || (mask[t] >> (key - ctx) & 1)) st.o[t][u][q] += v;
      }
  }
}

// Wave roles as run_piece in attn.hip: with NE < D/16 d blocks the waves split one
// tile's dims (or two tiles', half of the waves each), else each has TW tiles to itself.
template <int D, int TW, int NE, int NW, bool kFp8>
__device__ __forceinline__ void run_tree_piece(const TreeParams &p, char *buf, float *vscales,
                                               int *not_finite, const TreePiece &x,
                                               int wave, int lane) {
  using R = Ring<D, NW>;
  constexpr int kParts = D / 16 / NE;  // waves to a tile
  constexpr int kCell = kFp8 ? 1 : 2;
  Role role;
  role.tile0 = wave / kParts * TW;
  role.e_lo = wave % kParts * NE;
  role.active = role.tile0 * 16 < x.rows;
  RowState<TW, NE> st;
  TreeQ<D, TW> qv;
  load_tree_q<D, TW>(p, x, role.tile0, lane, qv);
  clear_state<TW, NE>(st);
  TreeRing c;
  const int kind = wave & 1;
  c.page_bytes = (uint32_t)(2 * p.hkv * kPage * D * kCell);
  c.base = reinterpret_cast<const char *>(p.kv) + (size_t)(kind * p.hkv + x.g) * kPage * D * kCell +
           16 * (!kFp8 && kind ? v_unit_inv(lane) : lane);
  c.scales = p.scales + (size_t)x.g * 2 * kPage + kind * kPage + (lane & 15);
  c.scale_bytes = (uint32_t)(p.hkv * 2 * kPage);
  c.ctx = x.rq.ctx;
  c.prio_end = x.prio_end;
  c.not_finite = not_finite;
  if (threadIdx.x == 0) *not_finite = 0;
  __syncthreads();
  constexpr int kSub = 64 * kIdRegs * R::kKeys;
  for (int sb = x.key_begin; sb < x.key_end; sb += kSub) {
    c.sb = sb;
    c.se = min(x.key_end, sb + kSub);
    c.ns = (c.se - sb + R::kKeys - 1) / R::kKeys;
    load_ids<NW>(p, x.i, wave, lane, c);
    if (sb > x.key_begin) __syncthreads();  // the last stages have been read
    tree_ring_run<D, TW, NE, NW, kFp8>(c, buf, vscales, wave, lane, qv, role, p.scale_log2, st);
  }
  if (!role.active) return;
  // set, if at all, before the last stage's barrier
  if (__builtin_amdgcn_readfirstlane(*not_finite) != 0)
    add_not_finite<D, TW, NE, NW, kFp8>(p, x, role, lane, qv.mask, st);
#pragma unroll
  for (int t = 0; t < TW; ++t)
    write_tree_rows<D, NE>(p, x, role.tile0 + t, role.e_lo, lane, st.m[t], row_sum4(st.l[t]),
                           st.o[t]);
}

// NW waves, each with up to kTW row tiles: group_rows = 16 * NW * kTW.
constexpr int tree_waves_per_simd(int D, int NW, int kTW) {
  return D == 64 && NW == 4 ? (kTW == 1 ? 4 : (kTW == 2 ? 3 : 2)) : 2;
}
template <int D, int NW, int kTW, bool kFp8>
__global__ __launch_bounds__(NW *kWave, tree_waves_per_simd(D, NW, kTW)) void tree_attn_kernel(
    TreeParams p) {
  __shared__ __attribute__((aligned(1024))) char buf[Ring<D, NW>::kBytes];
  __shared__ __attribute__((aligned(16))) float vscales[kFp8 ? Ring<D, NW>::kStages * Ring<D, NW>::kKeys : 4];
  __shared__ int not_finite;
  __shared__ int lds_plan[2 * NW + 8 + (kNumPieceCaps / 2 + 2) * NW];

  const TreeShare sh = tree_plan<D, NW>(p, lds_plan);
  if (sh.start >= sh.end) return;
  int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int lane = threadIdx.x % kWave;

  // the workgroups placed after the first on a CU, over half of their share
  const bool boost = (int)blockIdx.x >= p.num_cu;
  if (boost) __builtin_amdgcn_s_setprio(1);
  const int boost_end = boost ? sh.start + (int)((long long)(sh.end - sh.start) * kBoostPct / 100) : -1;

  TreePiece x;
  x.i = sh.i;
  x.rq = sh.first;
  int sub = sh.sub, off = sh.off, pos = sh.start, piece = 0, i_meta = sh.i;
  while (pos < sh.end && x.i < p.num_reqs) {
    if (x.i != i_meta) {
      const int q0 = __builtin_amdgcn_readfirstlane(p.cu[x.i]);
      const int q1 = __builtin_amdgcn_readfirstlane(p.cu[x.i + 1]);
      const int ctx = __builtin_amdgcn_readfirstlane(p.ctx[x.i]);
      x.rq = tree_meta(p, q0, q1, ctx);
      i_meta = x.i;
    }
    if (x.rq.seg == 0) {  // no rows, or metadata out of range: no keys in the plan
      ++x.i;
      continue;
    }
    const int segv = x.rq.seg + sh.lead;
    const int take = min(segv - off, sh.end - pos);
    x.key_begin = max(off - sh.lead, 0);
    x.key_end = min(x.rq.len, off + take - sh.lead);
    if (x.key_end <= x.key_begin) break;  // the share ends inside the lead-in
    x.complete = off <= sh.lead && off + take == segv;
    x.slot = piece == 0 ? 0 : 1;
    x.prio_end = boost ? x.key_begin + boost_end - pos : 0x7FFFFFFF;
    x.g = sub / x.rq.groups;
    x.rg = sub % x.rq.groups;
    x.rows = min(p.group_rows, p.group * x.rq.k - x.rg * p.group_rows);
    if (piece > 0) __syncthreads();  // the last piece's LDS has been read

    asm volatile("" : "+v"(lane), "+s"(wave));  // no offsets of all the forms ahead of the loop
    const int nt = (x.rows + 15) / 16;  // row tiles
    constexpr int kBlocks = D / 16;
    if (NW == 4 && nt == 1)
      run_tree_piece<D, 1, kBlocks / 4, NW, kFp8>(p, buf, vscales, &not_finite, x, wave, lane);
    else if (NW == 4 && nt == 2)
      run_tree_piece<D, 1, kBlocks / 2, NW, kFp8>(p, buf, vscales, &not_finite, x, wave, lane);
    else if (kTW == 1 || nt <= NW)
      run_tree_piece<D, 1, kBlocks, NW, kFp8>(p, buf, vscales, &not_finite, x, wave, lane);
    else if (kTW == 2 || nt <= 2 * NW)
      run_tree_piece<D, 2, kBlocks, NW, kFp8>(p, buf, vscales, &not_finite, x, wave, lane);
    else
      run_tree_piece<D, kTW, kBlocks, NW, kFp8>(p, buf, vscales, &not_finite, x, wave, lane);

    pos += take;
    off += take;
    ++piece;
    if (off == segv) {
      off = 0;
      if (++sub == x.rq.groups * p.hkv) {
        sub = 0;
        ++x.i;
      }
    }
  }
}

// Merges the partials of segments cut at share boundaries, in workgroup order, and
// zeroes the tail rows.  Workgroup (x, y, i) owns kCombThreads / (D/4) rows of segment y
// of request i; a thread four dims of a row.
template <int D>
__global__ __launch_bounds__(kCombThreads) void tree_combine_kernel(TreeParams p) {
  constexpr int kLanesPerRow = D / 4;
  constexpr int kRows = kCombThreads / kLanesPerRow;
  const int sub = blockIdx.y, i = blockIdx.z;
  if (i == p.num_reqs) {
    const int live = min(max(p.cu[p.num_reqs], 0), p.cap);
    const long long total = (long long)(p.cap - live) * p.hq * (D / 8);
    uint4 *tail = reinterpret_cast<uint4 *>(p.out + (size_t)live * p.hq * D);
    const long long step = (long long)gridDim.x * gridDim.y * kCombThreads;
    for (long long n = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * kCombThreads + threadIdx.x;
         n < total; n += step)
      tail[n] = make_uint4(0, 0, 0, 0);
    return;
  }
  // one round trip: the empty asm uses every word before the first branch
  int prefix = p.plan[i], share = p.plan[p.num_reqs + 1];
  int pc_prefix = p.plan[p.num_reqs + 2 + i];
  int cq0 = p.cu[i], cq1 = p.cu[i + 1], cctx = p.ctx[i];
  asm volatile("" : "+s"(prefix), "+s"(share), "+s"(pc_prefix), "+s"(cq0), "+s"(cq1), "+s"(cctx));
  const TreeMeta rq = tree_meta(p, cq0, cq1, cctx);
  if (sub >= rq.groups * p.hkv) return;
  const int seg = rq.seg + (share > 0 ? kLeadKeys : 0);
  const int start = prefix + sub * seg;
  const int skew = share > 0 ? share_skew(share) : 0;
  int b0, b1;
  if (share <= 0) {
    const int n = seg_pieces(seg, -share);
    b0 = pc_prefix + sub * n;
    b1 = b0 + n - 1;
  } else {
    b0 = share_owner(start + kLeadKeys, share, skew);
    b1 = share_owner(start + seg - 1, share, skew);
  }
  if (b0 == b1) return;  // one workgroup held the whole segment
  const int g = sub / rq.groups, rg = sub % rq.groups;
  const int rr = blockIdx.x * kRows + threadIdx.x / kLanesPerRow;
  if (rr >= min(p.group_rows, p.group * rq.k - rg * p.group_rows)) return;
  const int d4 = threadIdx.x % kLanesPerRow;
  const int at = rg * p.group_rows + rr;
  const int j = at >> __builtin_ctz(p.group), hh = at & (p.group - 1);
  const size_t row = (size_t)(rq.q0 + j) * p.hq + (size_t)g * p.group + hh;
  const int n_parts = b1 - b0 + 1;
  auto prow = [&](int u) -> size_t {
    const int b = b0 + u;
    const int slot = share <= 0 || share_begin(b, share, skew) >= start ? 0 : 1;
    return ((size_t)b * 2 + slot) * p.group_rows + rr;
  };
  float mx = -INFINITY;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
  if (n_parts > 8)
    for (int u0 = 0; u0 < n_parts; u0 += 8) {
      float m8[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        m8[u] = u0 + u < n_parts ? p.part_ml[prow(u0 + u)].x : -INFINITY;
#pragma unroll
      for (int u = 0; u < 8; ++u) mx = fmaxf(mx, m8[u]);
    }
  for (int u0 = 0; u0 < n_parts; u0 += 8) {
    float2 l8[8];
    f32x4 o8[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool in = u0 + u < n_parts;
      const size_t pr = prow(u0 + u);
      l8[u] = in ? p.part_ml[pr] : make_float2(-INFINITY, 0.f);
      o8[u] = in ? *reinterpret_cast<const f32x4 *>(p.part_o + pr * D + 4 * d4)
                 : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (n_parts <= 8)
#pragma unroll
      for (int u = 0; u < 8; ++u) mx = fmaxf(mx, l8[u].x);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = exp2f(l8[u].x - mx);
      den += w * l8[u].y;
      acc += w * o8[u];
    }
  }
  const float inv = 1.f / den;
  const uint32_t keep = den == 0.f ? 0u : 0xFFFFFFFFu;
  uint2 w2;
  w2.x = pack_bf16x2(acc[0] * inv, acc[1] * inv) & keep;
  w2.y = pack_bf16x2(acc[2] * inv, acc[3] * inv) & keep;
  *reinterpret_cast<uint2 *>(p.out + row * D + 4 * d4) = w2;
}

// ------------------------------------------------------------------------- masks
// One wave per request, lane j node j: what a node sees is itself and what its parent
// sees, closed by doubling (six rounds for 64 nodes).  A parent that does not come before
// its node makes the node a root.
__global__ __launch_bounds__(kWave) void tree_masks_kernel(const int32_t *parents,
                                                          const int32_t *cu, const int32_t *ctx,
                                                          unsigned long long *masks,
                                                          int32_t *positions, int32_t cap) {
  const int i = blockIdx.x, j = threadIdx.x;
  const int o = cu[i], k = cu[i + 1] - o;
  if (k <= 0 || k > kMaxNodes || o < 0 || o + k > cap) return;
  int up = j < k ? parents[o + j] : -1;
  if (up < 0 || up >= j) up = -1;
  unsigned long long mask = 1ull << j;
  int depth = up >= 0 ? 1 : 0;
#pragma unroll
  for (int round = 0; round < 6; ++round) {
    const int from = max(up, 0);
    const unsigned long long m = __shfl(mask, from);
    const int d = __shfl(depth, from), u = __shfl(up, from);
    if (up >= 0) {
      mask |= m;
      depth += d;
      up = u;
    }
  }
  if (j < k) {
    masks[o + j] = mask;
    if (positions) positions[o + j] = ctx[i] + depth;
  }
}

// The split kernel for a batch's dims: as many row tiles as the largest tree has, up to
// what a workgroup's registers hold.  D = 128: four waves of one or two tiles, two
// workgroups to a CU; above eight tiles eight waves of two, one to a CU.  D = 64: four waves
// of one, two or four tiles, four, three and two workgroups to a CU.  The host knows only the
// bound max_nodes, and trees far below it pay for the larger form.  B=32, 32/8 heads,
// contexts to 8K, us a call with a bound of the trees' own size and of 64: D = 128, 8-bit
// cache, 1 node 73 and 115, 8 nodes 83 and 121, 16 nodes 95 and 125, 32 nodes 145 and 161;
// bf16 100 and 113, 109 and 122, 118 and 129, 151 and 169; D = 64, 8-bit, 1 node 45 and 57, 16
// nodes 61 and 67; bf16 57 and 59, 68 and 71.
struct TreeKernel {
  int index;  // of the form, below kTreeKernels
  void (*fn)(TreeParams);
  int threads, group_rows, max_grid;
};
constexpr int kTreeKernels = 12;
template <bool kFp8>
TreeKernel tree_kernel(const dsv_tree_dims &d) {
  const int tiles = (d.num_q_heads / d.num_kv_heads * d.max_nodes + 15) / 16;
  constexpr int k4 = 4 * kWave, k8 = 8 * kWave, at = kFp8 ? kTreeKernels / 2 : 0;
  if (d.head_dim == 128) {
    if (tiles <= 4) return {at, tree_attn_kernel<128, 4, 1, kFp8>, k4, 64, 512};
    if (tiles <= 8) return {at + 1, tree_attn_kernel<128, 4, 2, kFp8>, k4, 128, 512};
    return {at + 2, tree_attn_kernel<128, 8, 2, kFp8>, k8, 256, 256};
  }
  if (tiles <= 4) return {at + 3, tree_attn_kernel<64, 4, 1, kFp8>, k4, 64, 1024};
  if (tiles <= 8) return {at + 4, tree_attn_kernel<64, 4, 2, kFp8>, k4, 128, 768};
  return {at + 5, tree_attn_kernel<64, 4, 4, kFp8>, k4, 256, 512};
}
TreeKernel tree_kernel_of(const dsv_tree_dims &d) {
  return d.kv_dtype == DSV_FP8 ? tree_kernel<true>(d) : tree_kernel<false>(d);
}

int32_t tree_grid_cap(const dsv_tree_dims &d, const TreeKernel &k) {
  const int rows = d.num_q_heads / d.num_kv_heads * d.max_nodes;
  const long long groups = (rows + k.group_rows - 1) / k.group_rows;
  const long long blocks = (long long)d.num_reqs * d.num_kv_heads * groups *
                           ((d.max_kv_len + kBlockKeys - 1) / kBlockKeys);
  return (int32_t)(blocks < k.max_grid ? blocks : k.max_grid);
}

}  // namespace

// Workgroups the current device holds at once (cached per device and form), capped; 0
// if a device query failed.
int32_t tree_grid(const dsv_tree_dims &d) {
  static std::atomic<int> cache[64][kTreeKernels];
  const TreeKernel k = tree_kernel_of(d);
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
  int resident = cache[dev][k.index].load(std::memory_order_relaxed);
  if (resident <= 0) {
    int per_cu = 0;
    const hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(
        &per_cu, reinterpret_cast<const void *>(k.fn), k.threads, 0);
    resident = attn_num_cu() * per_cu;
    if (e != hipSuccess || resident <= 0) {
      (void)hipGetLastError();
      return 0;
    }
    cache[dev][k.index].store(resident, std::memory_order_relaxed);
  }
  const int32_t cap = tree_grid_cap(d, k);
  return resident < cap ? resident : cap;
}

TreeWorkspace tree_workspace_layout(const dsv_tree_dims &d) {
  const TreeKernel k = tree_kernel_of(d);
  TreeWorkspace w;
  w.group_rows = k.group_rows;
  const int rows = d.num_q_heads / d.num_kv_heads * d.max_nodes;
  w.row_groups = (rows + k.group_rows - 1) / k.group_rows;
  const size_t parts = (size_t)tree_grid_cap(d, k) * 2 * (size_t)k.group_rows;
  w.plan_off = 0;
  w.part_ml_off = align_up((size_t)(2 * d.num_reqs + 3) * sizeof(int32_t), 256);
  w.part_o_off = align_up(w.part_ml_off + parts * sizeof(float2), 256);
  w.total = align_up(w.part_o_off + parts * d.head_dim * sizeof(float), 256);
  return w;
}

hipError_t launch_tree_attn(const TreeParams &p, const dsv_tree_dims &d, int32_t grid,
                            hipStream_t s) {
  const TreeKernel k = tree_kernel_of(d);
  const int comb_rows = kCombThreads / (d.head_dim / 4);
  const TreeWorkspace w = tree_workspace_layout(d);
  const int rows = p.group * p.max_nodes < w.group_rows ? p.group * p.max_nodes : w.group_rows;
  launch_kernel(k.fn, dim3(grid), dim3(k.threads), s, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  launch_kernel(d.head_dim == 128 ? tree_combine_kernel<128> : tree_combine_kernel<64>,
                dim3((rows + comb_rows - 1) / comb_rows, p.hkv * w.row_groups, p.num_reqs + 1),
                dim3(kCombThreads), s, p);
  return hipGetLastError();
}

hipError_t launch_tree_masks(const int32_t *parents, const int32_t *cu, const int32_t *ctx,
                             unsigned long long *masks, int32_t *positions, int32_t num_reqs,
                             int32_t cap, hipStream_t s) {
  launch_kernel(tree_masks_kernel, dim3(num_reqs), dim3(kWave), s, parents, cu, ctx, masks,
                positions, cap);
  return hipGetLastError();
}

}  // namespace dsv
