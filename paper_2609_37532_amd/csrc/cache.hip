// cache.hip -- writing, reading back and moving rows of the paged KV cache (gfx950).
//
// What it computes:
//  * rope_append: rotary positions on q and k, and k and v written to their slots of
//    the cache.  Pair i of a head turns by theta = position * inv_freq[i]:
//    (a, b) -> scale * (a cos - b sin, b cos + a sin).
//  * kv_read: slots gathered into dense rows.
//  * tree_commit: the rows of an accepted path moved to the positions that follow the
//    context.
// In an 8-bit cache each row (token, KV head, K or V) has a scale 2^e, the least power of
// two with |x| <= 448 * 2^e: the codes use the top binade of e4m3, and value = code * 2^e
// is exact in bf16, which the attention and kv_read rely on.
//
// How:
//  * A cell of a page is reached by its slot, and V lies d-major there, so 16 rows
//    that fill a page are one contiguous tile and a row alone is D cells 16 or 32 bytes
//    apart.  The kernels therefore work in runs: consecutive rows on consecutive slots of
//    one page.  A workgroup owns the runs that begin in its 16 rows, whole, up to 15 rows
//    beyond them; it finds them with a few ballots over the slots.
//  * V passes through LDS, where it is transposed; K needs no transposing.
//  * Angles are products of whole positions and fp32 frequencies, exact in two doubles,
//    brought to [-pi/4, pi/4] in two parts of pi/2 and summed as Taylor series, for each
//    row and frequency, by each workgroup for its heads.  k is rotated in double precision
//    too, within 5.5 * 2^-53 * (|a| + |b|) * |scale| of the exact value (2.5 from sin and cos,
//    one each from their factor, a product and the sum), and brought to fp32 with its last
//    bit set if anything was cut, so that there is one rounding to bf16 or to 8 bits, and a
//    cache hardly depends on how its writer rounds.  q is rotated in fp32.
//
// What bounds it, and what it measured (MI355X):
//  * rope_append, 8,191 rows, 32/8 heads, D = 128, bf16 cache (201 MB): 50 us, 4.1 TB/s,
//    where a copy of that size reaches 5.4.  q alone takes 31 and the cache alone 31: the
//    cache writers' chain of slots, angles, then turns, a stage of V and two barriers for
//    each head in turn.  8-bit cache (185 MB) 48, fp32 inputs 68, D = 64 27 us: bf16 inputs
//    hold four workgroups to a CU with a bf16 cache at D = 64 and with an 8-bit one at D =
//    128, the others three (LDS or registers), and those with four are no nearer to their
//    floor.  rotary_dim not a multiple of 16 with the half layout moves by single elements:
//    144 us.
//  * rope_append of one row 5.6 us, of a step's 739 rows 6.6: two round trips (slots, rows),
//    the angles, a barrier.
//  * kv_read, 60,001 rows of the 8-bit cache in whole pages (370 MB): 73 us, 5.1 TB/s; 7,500
//    scattered rows 35 us (each V row costs its whole tile's lines).  fp32 outputs, 20,001
//    rows (205 MB): 62 us, 3.3 TB/s, one head to a workgroup.
//  * tree_commit: 3.7 us for one request's layer, 4.6 for 32.
// Tried, and slower: two heads to a pass with K on all four waves (their stages leave a CU
// two workgroups: 62 us); q in a launch of its own (70); one or eight heads to a
// workgroup at 8,191 rows (81 before loads ran ahead, 56 after).
#include "dsv_internal.h"

#include <math.h>

namespace dsv {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;             // rows in which a workgroup's runs begin
constexpr int kMaxRows = kChunk + 15;  // rows they can span
constexpr int kMinExp = -60;           // of a quantised row's scale: tiny rows become 0
constexpr float kFp8Max = 448.f;
// From so many (chunk, KV head) pairs on a workgroup takes several heads: two, and from
// twice as many on four.  It saves the angles of the others and loads ahead; below, there
// are too few workgroups.  us a call, 8 KV heads and 32 query heads, one / two / four heads, a
// bf16 | an 8-bit cache: 739 rows 9.1 / 12.0 / 19.4 | 9.5 / 13.2 / 21.8; 2,100 rows 16.9 / 16.0 /
// 22.5 | 15.5 / 17.6 / 25.5; 3,000 21.8 / 20.8 / 23.4 | 20.3 / 19.0 / 26.6; 4,200 29.0 / 26.1 /
// 24.7 | 26.9 / 24.6 / 27.1; 6,000 42.7 / 37.6 / 36.3 | 38.8 / 34.2 / 33.3; 8,191 58.6 / 51.7 /
// 49.9 | 55.8 / 49.9 / 48.7.  (An 8-bit cache would change over a little later.)
constexpr int kManyBlocks = 1024, kAppendHeads = 4;

// Chunk of a K tile: dims of one slot that lie together.
template <bool kFp8>
constexpr int kKChunk = kFp8 ? 16 : 8;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// ------------------------------------------------------------------------- runs
// The runs that begin in rows [r0, r0 + 16), found by every wave for itself.  Lane l
// stands for row r0 + l; bit l of a mask likewise.
struct Runs {
  int ref;                    // this lane's slot
  unsigned long long valid;   // rows with a slot inside the cache
  unsigned long long start;   // rows that begin a run
  int first, end;             // the owned rows lie in [first, end); none if first == end
  __device__ __forceinline__ bool owns(int l) const {
    return l >= first && l < end && (valid >> l & 1) != 0;
  }
};

__device__ __forceinline__ Runs find_runs(const int32_t *refs, int r0, int live, int num_slots,
                                          int lane) {
  Runs x;
  const int row = r0 + lane;
  const bool in = lane < kMaxRows && row < live;
  x.ref = in ? refs[row] : -1;
  const int before = in && row > 0 ? refs[row - 1] : -2;
  const bool valid = in && x.ref >= 0 && x.ref < num_slots;
  const bool start = valid && ((x.ref & (kPage - 1)) == 0 || before < 0 || x.ref != before + 1);
  x.valid = __ballot(valid);
  x.start = __ballot(start);
  const unsigned mine = (unsigned)x.start & ((1u << kChunk) - 1);
  x.first = x.end = 0;
  if (mine) {
    x.first = __builtin_ctz(mine);
    // and rows past the chunk that go on with its last run; bit 31 is never set
    const unsigned on = (unsigned)(x.valid & ~x.start);
    x.end = kChunk + __builtin_ctz(~(on >> kChunk));
    x.end = min(x.end, 64 - __builtin_clzll(x.valid));  // nor past the last row with a slot
  }
  return x;
}

// How many V cells of one dim a row's lane writes at once: 16 or 4 where this row begins
// that many aligned slots of a run, 0 where an earlier row's lane writes this one's.
__device__ __forceinline__ int lead_of(const Runs &x, int lane) {
  const unsigned on = (unsigned)(x.valid & ~x.start);
  const int slot = x.ref & (kPage - 1);
  const bool owned = x.owns(lane);
  const unsigned next = lane < 31 ? on >> (lane + 1) : 0;  // rows that follow in the run
  const unsigned l16 = (unsigned)__ballot(owned && slot == 0 && (next & 0x7FFF) == 0x7FFF);
  const unsigned l4 = (unsigned)__ballot(owned && slot % 4 == 0 && (next & 7) == 7);
  if (!owned) return 0;
  if (lane >= slot && (l16 >> (lane - slot) & 1)) return slot == 0 ? 16 : 0;
  const int b = slot % 4;
  if (lane >= b && (l4 >> (lane - b) & 1)) return b == 0 ? 4 : 0;
  return 1;
}

// ----------------------------------------------------------------------- angles
// sin and cos of the angle position * freq in double precision, each within 2.5 * 2^-53, for
// angles up to 2^40.  The product has up to 55 bits: a and what its rounding left.  n = a /
// (pi/2) rounded (the quotient is off by at most 2^-12 there, so r hardly leaves [-pi/4,
// pi/4]), pi/2 in two parts (106 bits), and the Taylor series of sin and cos to r^17 and r^16,
// whose remainders at pi/4 are 8e-20 and 2e-18.
__device__ __forceinline__ void sincos64(int position, float freq, double &s, double &c) {
  const double p = position, f = freq;
  const double a = p * f, left = __builtin_fma(p, f, -a);
  const double n = __builtin_rint(a * 0.63661977236758138);
  double r = __builtin_fma(-n, 1.5707963267948966, a);
  r = __builtin_fma(-n, 6.123233995736766e-17, r) + left;
  const double z = r * r;
  double ps = 1.0 / 355687428096000.0;  // 1/17!
  ps = __builtin_fma(ps, z, -1.0 / 1307674368000.0);
  ps = __builtin_fma(ps, z, 1.0 / 6227020800.0);
  ps = __builtin_fma(ps, z, -1.0 / 39916800.0);
  ps = __builtin_fma(ps, z, 1.0 / 362880.0);
  ps = __builtin_fma(ps, z, -1.0 / 5040.0);
  ps = __builtin_fma(ps, z, 1.0 / 120.0);
  ps = __builtin_fma(ps, z, -1.0 / 6.0);
  const double sr = __builtin_fma(ps * z, r, r);
  double pc = 1.0 / 20922789888000.0;  // 1/16!
  pc = __builtin_fma(pc, z, -1.0 / 87178291200.0);
  pc = __builtin_fma(pc, z, 1.0 / 479001600.0);
  pc = __builtin_fma(pc, z, -1.0 / 3628800.0);
  pc = __builtin_fma(pc, z, 1.0 / 40320.0);
  pc = __builtin_fma(pc, z, -1.0 / 720.0);
  pc = __builtin_fma(pc, z, 1.0 / 24.0);
  pc = __builtin_fma(pc, z, -0.5);
  const double cr = __builtin_fma(pc, z, 1.0);
  const double m = n * 0.25;
  const int quarter = (int)((m - __builtin_floor(m)) * 4.0);  // n mod 4
  const bool odd = quarter & 1;
  const double s0 = odd ? cr : sr, c0 = odd ? sr : cr;
  s = quarter & 2 ? -s0 : s0;
  c = (quarter + 1) & 2 ? -c0 : c0;
}

// d in fp32, cut towards zero with the last bit set if anything was cut: rounding the
// result to fewer bits, or comparing it with a value of fewer bits, gives what d gives.
__device__ __forceinline__ float to_odd(double d) {
  const float f = (float)d;
  const double back = (double)f;
  uint32_t bits = __float_as_uint(f);
  if (back != d) bits = (bits - (__builtin_fabs(back) > __builtin_fabs(d) ? 1u : 0u)) | 1u;
  return __uint_as_float(bits);
}

// ---------------------------------------------------------------- a thread's dims
// D / 16 threads share a head; thread t holds the eight pairs p = 8t .. 8t+7 as a[e],
// b[e].  Which dims a pair is depends on the layout; pairs from rot / 2 on do not turn.
//   0 half, rot / 2 a multiple of 8: (p, p + rot / 2), else two vectors past rot
//   1 interleaved (and every use without rotation): (2p, 2p + 1)
//   2 half, other rot: as 0 by single elements, past rot (2p, 2p + 1)
enum PairMode { kHalfVec = 0, kAdjacent = 1, kHalfAny = 2 };

struct PairDims {
  int a, b, step;  // dims of pair e: a + step * e, b + step * e
};
// kHalfAny has no single form for a thread's eight pairs: by element.
__device__ __forceinline__ PairDims pair_dims(int mode, int rot, int t) {
  if (mode == kHalfVec) {
    if (16 * t < rot) return {8 * t, 8 * t + rot / 2, 1};
    return {16 * t, 16 * t + 8, 1};
  }
  return {16 * t, 16 * t + 1, 2};
}
__device__ __forceinline__ void any_dims(int rot, int p, int &da, int &db) {
  da = 2 * p < rot ? p : 2 * p;
  db = 2 * p < rot ? p + rot / 2 : 2 * p + 1;
}

// Sixteen values as they lie in memory: two vectors of eight dims.
template <bool kF32>
struct Raw {
  u32x4 x[kF32 ? 4 : 2];
};
template <bool kF32>
__device__ __forceinline__ void load_raw(const void *row, int mode, int rot, int t, Raw<kF32> &r) {
  constexpr int kBytes = kF32 ? 4 : 2;
  if (mode == kHalfAny) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      int da, db;
      any_dims(rot, 8 * t + e, da, db);
      if constexpr (kF32) {
        r.x[e / 4][e % 4] = ((const uint32_t *)row)[da];
        r.x[2 + e / 4][e % 4] = ((const uint32_t *)row)[db];
      } else {
        r.x[e / 4][e % 4] = (uint32_t)((const uint16_t *)row)[da] |
                            (uint32_t)((const uint16_t *)row)[db] << 16;
      }
    }
    return;
  }
  const PairDims d = pair_dims(mode, rot, t);
  const char *a = (const char *)row + d.a * kBytes;
  const char *b = (const char *)row + (mode == kHalfVec ? d.b : d.a + 8) * kBytes;
#pragma unroll
  for (int q = 0; q < (kF32 ? 2 : 1); ++q) {
    r.x[q] = *reinterpret_cast<const u32x4 *>(a + 16 * q);
    r.x[(kF32 ? 2 : 1) + q] = *reinterpret_cast<const u32x4 *>(b + 16 * q);
  }
}
// As pairs.
template <bool kF32>
__device__ __forceinline__ void pairs_of(const Raw<kF32> &r, int mode, float (&a)[8], float (&b)[8]) {
  if constexpr (kF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // two vectors of a, then b; or sixteen dims in order
      const float pa = __uint_as_float(r.x[e / 4][e % 4]), pb = __uint_as_float(r.x[2 + e / 4][e % 4]);
      const float qa = __uint_as_float(r.x[e / 2][2 * (e % 2)]);
      const float qb = __uint_as_float(r.x[e / 2][2 * (e % 2) + 1]);
      a[e] = mode == kAdjacent ? qa : pa;
      b[e] = mode == kAdjacent ? qb : pb;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // a word of each vector holds two dims of it; or a pair (kHalfAny likewise)
      const uint32_t wa = r.x[0][e / 2], wb = r.x[1][e / 2], w = r.x[e / 4][e % 4];
      const float pa = e % 2 ? bf16_hi(wa) : bf16_lo(wa), pb = e % 2 ? bf16_hi(wb) : bf16_lo(wb);
      a[e] = mode == kHalfVec ? pa : bf16_lo(w);
      b[e] = mode == kHalfVec ? pb : bf16_hi(w);
    }
  }
}

// A thread's sixteen values as bf16: w[0..3] and w[4..7] are the vectors at dims
// pair_dims().a and .b (kHalfVec) or .a and .a + 8.
__device__ __forceinline__ void bf16_words(int mode, const float (&a)[8], const float (&b)[8],
                                           uint32_t (&w)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = mode == kHalfVec ? pack_bf16x2(a[2 * e], a[2 * e + 1]) : pack_bf16x2(a[e], b[e]);
    w[4 + e] = mode == kHalfVec ? pack_bf16x2(b[2 * e], b[2 * e + 1])
                                : pack_bf16x2(a[4 + e], b[4 + e]);
  }
}

__device__ __forceinline__ uint32_t fp8_word(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// The same as 8-bit codes: w[0..1] and w[2..3].
__device__ __forceinline__ void fp8_words(int mode, const float (&a)[8], const float (&b)[8],
                                          uint32_t (&w)[4]) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int q = 4 * e, h = 2 * e;
    w[e] = mode == kHalfVec ? fp8_word(a[q], a[q + 1], a[q + 2], a[q + 3])
                            : fp8_word(a[h], b[h], a[h + 1], b[h + 1]);
    w[2 + e] = mode == kHalfVec ? fp8_word(b[q], b[q + 1], b[q + 2], b[q + 3])
                                : fp8_word(a[4 + h], b[4 + h], a[5 + h], b[5 + h]);
  }
}

// Scales a row held by `threads` adjacent lanes to 8-bit range: the exponent of the
// row's scale, by its largest finite value.  Values that are not finite become NaN.
template <int kTph>
__device__ __forceinline__ int scale_row(float (&a)[8], float (&b)[8]) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = fabsf(a[e]), y = fabsf(b[e]);
    top = fmaxf(top, x < INFINITY ? x : 0.f);
    top = fmaxf(top, y < INFINITY ? y : 0.f);
  }
#pragma unroll
  for (int o = 1; o < kTph; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  const uint32_t bits = __float_as_uint(top);
  // 448 = 1.75 * 2^8
  const int e = max(kMinExp, (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0));
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    a[q] *= inv;
    b[q] *= inv;
    if (!(fabsf(a[q]) <= kFp8Max)) a[q] = NAN;
    if (!(fabsf(b[q]) <= kFp8Max)) b[q] = NAN;
  }
  return e;
}

// ------------------------------------------------------------------------ append
// Cells of one V stage in LDS: [dim][row], the rows at r - first + the first one's slot,
// so that aligned slots of its run are aligned words.  The pitch is an odd number of
// words, which spreads the dims of a wave over the banks.
template <bool kFp8>
struct VStage {
  using Cell = typename std::conditional<kFp8, uint8_t, uint16_t>::type;
  static constexpr int kPitch = kFp8 ? 52 : 50;
};

template <bool kF32, bool kFp8, int D>
__device__ void append_kv(const AppendParams &p, char *lds, int block, int live) {
  constexpr int kTph = D / 16;
  using Stage = VStage<kFp8>;
  using Cell = typename Stage::Cell;
  double2 *cs = reinterpret_cast<double2 *>(lds);  // [row][pair] cos, sin
  Cell *stage = reinterpret_cast<Cell *>(lds + kMaxRows * (D / 2) * sizeof(double2));
  __shared__ int refs[kMaxRows];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int chunks = (p.rows + kChunk - 1) / kChunk;
  const int r0 = block % chunks * kChunk;
  const int g0 = block / chunks * p.heads_per_block;
  const int g1 = min(p.hkv, g0 + p.heads_per_block);
  const Runs x = find_runs(p.refs, r0, live, p.num_pages * kPage, lane);
  if (x.first == x.end) return;
  const int lead = lead_of(x, lane);
  const int nr = x.end - x.first;
  if ((int)threadIdx.x < kMaxRows) refs[lane] = x.ref;
  // stage row - row
  const int shift = (__builtin_amdgcn_readlane(x.ref, x.first) & (kPage - 1)) - x.first;
  const int half = p.rot / 2;
  // item n: thread n % kTph of a row's K, then of the rows' V; the first one of a head is
  // loaded ahead, under the angles and under the head before
  auto load_item = [&](int n, int g, Raw<kF32> &r) {
    const bool is_v = n >= nr * kTph;
    const int at = is_v ? n - nr * kTph : n;
    const int l = x.first + at / kTph;
    if (n >= 2 * nr * kTph || !x.owns(l)) return;
    const char *src = (const char *)(is_v ? p.v : p.k) +
                      ((size_t)(r0 + l) * (size_t)(is_v ? p.v_stride : p.k_stride) + (size_t)g * D) *
                          (kF32 ? 4 : 2);
    load_raw<kF32>(src, is_v ? (int)kAdjacent : p.mode, p.rot, at % kTph, r);
  };
  // every head's first item is loaded ahead, under the angles
  Raw<kF32> ahead[kAppendHeads];
#pragma unroll
  for (int h = 0; h < kAppendHeads; ++h)
    if (g0 + h < g1) load_item(threadIdx.x, g0 + h, ahead[h]);
#pragma unroll 1
  for (int n = threadIdx.x; n < nr * half; n += kThreads) {
    const int r = n / half, i = n - r * half;
    double s, c;
    sincos64(p.pos[r0 + x.first + r], p.inv_freq[i], s, c);
    cs[r * (D / 2) + i] = make_double2(c * (double)p.rope_scale, s * (double)p.rope_scale);
  }
  __syncthreads();
  const size_t tile = (size_t)kPage * D;
#pragma unroll 1
  for (int g = g0; g < g1; ++g) {
    if (g > g0) __syncthreads();  // the last head's stage has been read
    Raw<kF32> item = ahead[0];
#pragma unroll
    for (int h = 1; h < kAppendHeads; ++h)
      if (g == g0 + h) item = ahead[h];
#pragma unroll 1
    for (int n = threadIdx.x; n < 2 * nr * kTph; n += kThreads) {
      const bool is_v = n >= nr * kTph;
      const int at = is_v ? n - nr * kTph : n;
      const int l = x.first + at / kTph, t = at % kTph;
      if (n >= kThreads) load_item(n, g, item);
      if (!x.owns(l)) continue;
      const int mode = is_v ? (int)kAdjacent : p.mode;
      float a[8], b[8];
      pairs_of<kF32>(item, mode, a, b);
      if (!is_v) {
        const double2 *turn = cs + (l - x.first) * (D / 2) + 8 * t;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * t + e < half) {
            asm volatile("" ::: "memory");  // one pair's factors at a time: 120 registers less
            const double2 w = turn[e];
            const double u = a[e], v = b[e];
            a[e] = to_odd(__builtin_fma(u, w.x, -(v * w.y)));
            b[e] = to_odd(__builtin_fma(v, w.x, u * w.y));
          }
      }
      const int ref = refs[l];
      const int page = ref / kPage, slot = ref % kPage;
      uint32_t w[kFp8 ? 4 : 8];
      if constexpr (kFp8) {
        const int e = scale_row<kTph>(a, b);
        if (t == 0) p.scales[(((size_t)page * p.hkv + g) * 2 + (is_v ? 1 : 0)) * kPage + slot] = (uint8_t)(e + 127);
        fp8_words(mode, a, b, w);
      } else {
        bf16_words(mode, a, b, w);
      }
      if (is_v) {
        Cell *to = stage + (size_t)16 * t * Stage::kPitch + l + shift;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          constexpr int kPer = kFp8 ? 4 : 2;
          to[e * Stage::kPitch] = (Cell)(w[e / kPer] >> (e % kPer * 8 * (int)sizeof(Cell)));
        }
        continue;
      }
      Cell *kt = (Cell *)p.pages + ((size_t)page * 2 * p.hkv + g) * tile;
      constexpr int kC = kKChunk<kFp8>;
      auto cell = [&](int d) { return kt + (d / kC * kPage + slot) * kC + d % kC; };
      if (mode == kHalfAny) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          int da, db;
          any_dims(p.rot, 8 * t + e, da, db);
          // the words hold the adjacent order: pair e is elements 2e and 2e + 1
          constexpr int kPer = kFp8 ? 4 : 2;
          *cell(da) = (Cell)(w[2 * e / kPer] >> (2 * e % kPer * 8 * (int)sizeof(Cell)));
          *cell(db) = (Cell)(w[(2 * e + 1) / kPer] >> ((2 * e + 1) % kPer * 8 * (int)sizeof(Cell)));
        }
      } else {
        const PairDims d = pair_dims(mode, p.rot, t);
        const int d1 = mode == kHalfVec ? d.b : d.a + 8;
        if constexpr (kFp8) {
          *reinterpret_cast<uint2 *>(cell(d.a)) = make_uint2(w[0], w[1]);
          *reinterpret_cast<uint2 *>(cell(d1)) = make_uint2(w[2], w[3]);
        } else {
          *reinterpret_cast<u32x4 *>(cell(d.a)) = u32x4{w[0], w[1], w[2], w[3]};
          *reinterpret_cast<u32x4 *>(cell(d1)) = u32x4{w[4], w[5], w[6], w[7]};
        }
      }
    }
    __syncthreads();
    for (int l = x.first + wave; l < x.end; l += kThreads / kWave) {
      const int count = __builtin_amdgcn_readlane(lead, l);
      if (count == 0) continue;
      const int ref = __builtin_amdgcn_readlane(x.ref, l);
      const int page = ref / kPage, slot = ref % kPage;
      Cell *vt = (Cell *)p.pages + ((size_t)page * 2 * p.hkv + p.hkv + g) * tile + slot;
      const int at = l + shift;
      // word reads where the stage's rows are as aligned as the slots
      const bool words = (at - slot) % 4 == 0;
#pragma unroll
      for (int d0 = 0; d0 < D; d0 += kWave) {
        const int d = d0 + lane;
        const Cell *from = stage + (size_t)d * Stage::kPitch + at;
        Cell *to = vt + (size_t)d * kPage;
        if (count == 1) {
          *to = *from;
        } else if (!words) {
          for (int q = 0; q < count; ++q) to[q] = from[q];
        } else {
          const uint32_t *fw = reinterpret_cast<const uint32_t *>(from);
          if (count == 16) {
            reinterpret_cast<u32x4 *>(to)[0] = u32x4{fw[0], fw[1], fw[2], fw[3]};
            if (!kFp8) reinterpret_cast<u32x4 *>(to)[1] = u32x4{fw[4], fw[5], fw[6], fw[7]};
          } else if (kFp8) {
            *reinterpret_cast<uint32_t *>(to) = fw[0];
          } else {
            *reinterpret_cast<uint2 *>(to) = make_uint2(fw[0], fw[1]);
          }
        }
      }
    }
  }
}

// Dense outputs go past the L2 caches, which the kernels' other traffic uses and a reader
// on another XCD does not (through them and past them: kv_read of 60,001 8-bit rows 76.9 and
// 72.4 us, append of 8,191 rows 52.2 and 49.8, into an 8-bit cache 49.3 and 47.8).
__device__ __forceinline__ void store16(void *to, u32x4 x) {
  __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(to));
}


template <bool kF32, int D>
__device__ void append_q(const AppendParams &p, char *lds, int block, int live) {
  constexpr int kTph = D / 16;
  float2 *cs = reinterpret_cast<float2 *>(lds);
  const int r0 = block * p.q_rows;
  const int nr = min(p.q_rows, live - r0);
  if (nr <= 0) return;
  const int half = p.rot / 2;
#pragma unroll 1
  for (int n = threadIdx.x; n < nr * half; n += kThreads) {
    const int r = n / half, i = n - r * half;
    double s, c;
    sincos64(p.pos[r0 + r], p.inv_freq[i], s, c);
    cs[r * (D / 2) + i] = make_float2((float)(c * (double)p.rope_scale),
                                      (float)(s * (double)p.rope_scale));
  }
  __syncthreads();
  // four items of a thread in flight at a time
  const int per_row = p.hq * kTph, total = nr * per_row;
  constexpr int kItems = kF32 ? 2 : 4;
  for (int n0 = threadIdx.x; n0 < total; n0 += kItems * kThreads) {
    Raw<kF32> raw[kItems];
#pragma unroll
    for (int y = 0; y < kItems; ++y) {
      const int n = n0 + y * kThreads, r = n / per_row, i = n - r * per_row;
      if (n >= total) continue;
      const char *src = (const char *)p.q + ((size_t)(r0 + r) * (size_t)p.q_stride +
                                             (size_t)(i / kTph) * D) * (kF32 ? 4 : 2);
      load_raw<kF32>(src, p.mode, p.rot, i % kTph, raw[y]);
    }
#pragma unroll
    for (int y = 0; y < kItems; ++y) {
      const int n = n0 + y * kThreads, r = n / per_row, i = n - r * per_row;
      if (n >= total) continue;
      const int h = i / kTph, t = i % kTph;
      float a[8], b[8];
      pairs_of<kF32>(raw[y], p.mode, a, b);
      const float2 *turn = cs + r * (D / 2) + 8 * t;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * t + e < half) {
          const float2 w = turn[e];
          const float u = a[e], v = b[e];
          a[e] = __builtin_fmaf(u, w.x, -(v * w.y));
          b[e] = __builtin_fmaf(v, w.x, u * w.y);
        }
      uint32_t w[8];
      bf16_words(p.mode, a, b, w);
      uint16_t *out = p.q_out + ((size_t)(r0 + r) * p.hq + h) * D;
      if (p.mode == kHalfAny) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          int da, db;
          any_dims(p.rot, 8 * t + e, da, db);
          out[da] = (uint16_t)w[e];
          out[db] = (uint16_t)(w[e] >> 16);
        }
      } else {
        const PairDims d = pair_dims(p.mode, p.rot, t);
        store16(out + d.a, u32x4{w[0], w[1], w[2], w[3]});
        store16(out + (p.mode == kHalfVec ? d.b : d.a + 8), u32x4{w[4], w[5], w[6], w[7]});
      }
    }
  }
}

// Workgroups [0, kv_blocks) write the cache, the others rotate q.
template <bool kF32, bool kFp8, int D>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(AppendParams p) {
  constexpr int kLds = kMaxRows * (D / 2) * (int)sizeof(double2) +
                       D * VStage<kFp8>::kPitch * (int)sizeof(typename VStage<kFp8>::Cell);
  __shared__ __attribute__((aligned(16))) char lds[kLds];
  const int live = p.num_live ? min(max(__builtin_amdgcn_readfirstlane(*p.num_live), 0), p.rows)
                              : p.rows;
  if ((int)blockIdx.x < p.kv_blocks)
    append_kv<kF32, kFp8, D>(p, lds, blockIdx.x, live);
  else
    append_q<kF32, D>(p, lds, blockIdx.x - p.kv_blocks, live);
}

// -------------------------------------------------------------------------- read
// Sixteen values as fp32 out of codes and a scale, or out of bf16.
__device__ __forceinline__ void fp8_values(u32x4 w, float scale, float (&x)[16]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    x[4 * q] = __builtin_amdgcn_cvt_f32_fp8((int)w[q], 0) * scale;
    x[4 * q + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[q], 1) * scale;
    x[4 * q + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[q], 2) * scale;
    x[4 * q + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[q], 3) * scale;
  }
}
__device__ __forceinline__ float scale_of(uint8_t e) { return __uint_as_float((uint32_t)e << 23); }

// Eight values to eight dims of an output row.  As fp32 a thread's sixteen dims are four
// stores and a wave's lanes lie 64 bytes apart, quarters of lines that only a cache brings
// together: ordinary stores (20,001 8-bit rows, D = 128, 205 MB: 62 us, past the L2 141).
template <bool kF32>
__device__ __forceinline__ void store8(void *row, int d, const float (&x)[8]) {
  if (kF32) {
    const f32x4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
    *reinterpret_cast<f32x4 *>((float *)row + d) = lo;
    *reinterpret_cast<f32x4 *>((float *)row + d + 4) = hi;
  } else {
    store16((uint16_t *)row + d,
            u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                  pack_bf16x2(x[6], x[7])});
  }
}

// Most KV heads to a workgroup, from kManyBlocks pairs on: two at D = 128, four at D = 64.  us,
// one / two / four heads, 8 KV heads in whole pages.  D = 128, 8-bit: 2,000 rows (below
// kManyBlocks) 4.5 / 5.2 / 7.0, 8,000 10.3 / 11.0 / 13.3, 30,001 31 / 37 / -, 60,001 88 / 72 / -;
// bf16: 2,000 4.6 / 5.5 / 7.5, 40,001 64 / 65 / 65.  D = 64, 8-bit: 2,000 3.9 / 4.0 / 4.8, 30,001
// 22.3 / 16.6 / 18.6, 60,001 42 / 30 / 34; bf16: 40,001 28.6 / 27.2 / 28.5.  (So the rule is the
// largest reads' at D = 128; two heads would do a little better at D = 64.)
constexpr int read_heads(int dim) { return 256 / dim; }
template <bool kFp8, bool kF32, int D>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(ReadParams p) {
  constexpr int kTph = D / 16;
  using Out = typename std::conditional<kF32, float, uint16_t>::type;
  constexpr int kPitch = D + 16 / sizeof(Out);  // rows 16 bytes apart in the banks
  __shared__ __attribute__((aligned(16))) Out rows[(kF32 ? 1 : read_heads(D)) * kMaxRows * kPitch];  // V
  __shared__ int run_row[kChunk], refs[kMaxRows];
  const int lane = threadIdx.x % kWave;
  const int chunks = (p.rows + kChunk - 1) / kChunk;
  const int r0 = blockIdx.x % chunks * kChunk, g0 = blockIdx.x / chunks * p.heads_per_block;
  const int heads = min(p.heads_per_block, p.hkv - g0);
  const Runs x = find_runs(p.refs, r0, p.rows, p.num_pages * kPage, lane);
  const size_t tile = (size_t)kPage * D;
  auto out_row = [&](void *base, int l, int h) {
    return (Out *)base + ((size_t)(r0 + l) * p.hkv + g0 + h) * D;
  };
  // rows of this chunk without a slot in the cache
  if (((unsigned)~x.valid & ((1u << kChunk) - 1)) != 0)
    for (int n = threadIdx.x; n < heads * kChunk * (D / 8); n += kThreads) {
      const int l = n / (D / 8) % kChunk, h = n / (D / 8 * kChunk), d = n % (D / 8) * 8;
      if (r0 + l >= p.rows || (x.valid >> l & 1)) continue;
      const float zero[8] = {};
      store8<kF32>(out_row(p.k_out, l, h), d, zero);
      store8<kF32>(out_row(p.v_out, l, h), d, zero);
    }
  if (x.first == x.end) return;
  const int nr = x.end - x.first;
  const unsigned starts = (unsigned)x.start & ((1u << kChunk) - 1);
  const int num_runs = __builtin_popcount(starts);
  if ((int)threadIdx.x < kChunk && (starts >> lane & 1))
    run_row[__builtin_popcount(starts & ((1u << lane) - 1))] = lane;
  if ((int)threadIdx.x < kMaxRows) refs[lane] = x.ref;
  __syncthreads();
  // V: a thread takes one dim of a run, 16 slots at once, into rows
  for (int n = threadIdx.x; n < heads * num_runs * D; n += kThreads) {
    const int d = n % D, h = n / D % heads, l = run_row[n / D / heads];
    const unsigned on = (unsigned)(x.valid & ~x.start);
    const int len = 1 + __builtin_ctz(~(on >> (l + 1)));
    const int ref = refs[l];
    const int page = ref / kPage, slot = ref % kPage;
    const size_t at = ((size_t)page * 2 * p.hkv + p.hkv + g0 + h) * tile + (size_t)d * kPage;
    Out *to = rows + (h * kMaxRows + l - x.first) * kPitch + d;
    auto put = [&](int row, float v) {
      if constexpr (kF32)
        to[row * kPitch] = v;
      else
        to[row * kPitch] = (uint16_t)(__float_as_uint(v) >> 16);  // exact: bf16 holds it
    };
    const uint8_t *sc = kFp8 ? p.scales + (((size_t)page * p.hkv + g0 + h) * 2 + 1) * kPage : nullptr;
    if (len == 1) {
      put(0, kFp8 ? __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)p.pages)[at + slot], 0) *
                        scale_of(sc[slot])
                  : __uint_as_float((uint32_t)((const uint16_t *)p.pages)[at + slot] << 16));
      continue;
    }
    float v[16];
    if constexpr (kFp8) {
      const u32x4 w = *reinterpret_cast<const u32x4 *>((const uint8_t *)p.pages + at);
      const u32x4 e = *reinterpret_cast<const u32x4 *>(sc);
      fp8_values(w, 1.f, v);
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] *= scale_of((uint8_t)(e[q / 4] >> (q % 4 * 8)));
    } else {
      const u32x4 *w = reinterpret_cast<const u32x4 *>((const uint16_t *)p.pages + at);
      const u32x4 lo = w[0], hi = w[1];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[2 * q] = bf16_lo(lo[q]);
        v[2 * q + 1] = bf16_hi(lo[q]);
        v[8 + 2 * q] = bf16_lo(hi[q]);
        v[8 + 2 * q + 1] = bf16_hi(hi[q]);
      }
    }
    if (len == kPage) {
#pragma unroll
      for (int q = 0; q < 16; ++q) put(q, v[q]);
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q)
        if (q >= slot && q < slot + len) put(q - slot, v[q]);
    }
  }
  // K: a thread takes sixteen dims of a row; a wave eight rows of a head, whose chunks and
  // output rows lie together
  for (int n = threadIdx.x; n < heads * nr * kTph; n += kThreads) {
    const int t = n % kTph, l = x.first + n / kTph % nr, h = n / kTph / nr;
    if (!x.owns(l)) continue;
    const int ref = refs[l];
    const int page = ref / kPage, slot = ref % kPage;
    const size_t at = ((size_t)page * 2 * p.hkv + g0 + h) * tile;
    u32x4 w[2];
    float lo[8], hi[8];
    if constexpr (kFp8) {
      w[0] = *reinterpret_cast<const u32x4 *>((const uint8_t *)p.pages + at +
                                              (size_t)(t * kPage + slot) * 16);
      float v[16];
      fp8_values(w[0], scale_of(p.scales[((size_t)page * p.hkv + g0 + h) * 2 * kPage + slot]), v);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        lo[q] = v[q];
        hi[q] = v[8 + q];
      }
    } else {
      const uint16_t *k = (const uint16_t *)p.pages + at;
      w[0] = *reinterpret_cast<const u32x4 *>(k + (size_t)(2 * t * kPage + slot) * 8);
      w[1] = *reinterpret_cast<const u32x4 *>(k + (size_t)((2 * t + 1) * kPage + slot) * 8);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        lo[2 * q] = bf16_lo(w[0][q]);
        lo[2 * q + 1] = bf16_hi(w[0][q]);
        hi[2 * q] = bf16_lo(w[1][q]);
        hi[2 * q + 1] = bf16_hi(w[1][q]);
      }
    }
    store8<kF32>(out_row(p.k_out, l, h), 16 * t, lo);
    store8<kF32>(out_row(p.k_out, l, h), 16 * t + 8, hi);
  }
  __syncthreads();
  constexpr int kVec = 16 / sizeof(Out);
  for (int n = threadIdx.x; n < heads * nr * (D / kVec); n += kThreads) {
    const int d = n % (D / kVec) * kVec, l = x.first + n / (D / kVec) % nr, h = n / (D / kVec) / nr;
    if (!x.owns(l)) continue;
    store16(out_row(p.v_out, l, h) + d,
            *reinterpret_cast<const u32x4 *>(rows + (h * kMaxRows + l - x.first) * kPitch + d));
  }
}

// ------------------------------------------------------------------------ commit
// One workgroup per KV head and request: all rows that move are read into LDS before the
// first is written, since a row's new slot may be another row's old one.
template <bool kFp8, int D>
__global__ __launch_bounds__(kThreads) void tree_commit_kernel(CommitParams p) {
  using Cell = typename std::conditional<kFp8, uint8_t, uint16_t>::type;
  __shared__ __attribute__((aligned(16))) Cell ks[kMaxNodes * D], vs[kMaxNodes * D];
  __shared__ uint8_t es[2 * kMaxNodes];
  __shared__ int from[kMaxNodes], to[kMaxNodes];  // slots of the rows that move
  __shared__ int moves;
  const int g = blockIdx.x, i = blockIdx.y;
  const int o = p.cu[i], k = p.cu[i + 1] - o, ctx = p.ctx[i];
  if (k <= 0 || k > kMaxNodes || o < 0 || o + k > p.cap || ctx < 0 ||
      (long long)ctx + k > (long long)p.max_pages * kPage)
    return;
  if (threadIdx.x < kWave) {
    const int j = threadIdx.x;
    const int node = j < k ? p.path[o + j] : -1;
    // the path ends at its first entry that is no node
    const unsigned long long bad = __ballot(node < 0 || node >= k);
    const int len = bad ? __builtin_ctzll(bad) : kWave;
    bool move = j < len && node != j;
    int a = -1, b = -1;
    if (move) {
      const int32_t *table = p.page_table + (size_t)i * p.max_pages;
      const int pa = table[(ctx + node) / kPage], pb = table[(ctx + j) / kPage];
      move = (unsigned)pa < (unsigned)p.num_pages && (unsigned)pb < (unsigned)p.num_pages;
      a = pa * kPage + (ctx + node) % kPage;
      b = pb * kPage + (ctx + j) % kPage;
    }
    const unsigned long long mm = __ballot(move);
    if (move) {
      const int at = __builtin_popcountll(mm & ((1ull << j) - 1));
      from[at] = a;
      to[at] = b;
    }
    if (j == 0) moves = __builtin_popcountll(mm);
  }
  __syncthreads();
  const int n = moves;
  if (n == 0) return;
  constexpr int kC = kKChunk<kFp8>, kChunks = D / kC;
  const size_t tile = (size_t)kPage * D;
  Cell *pages = (Cell *)p.pages;
  auto k_at = [&](int ref, int c) {
    return pages + ((size_t)(ref / kPage) * 2 * p.hkv + g) * tile + (c * kPage + ref % kPage) * kC;
  };
  auto v_at = [&](int ref, int d) {
    return pages + ((size_t)(ref / kPage) * 2 * p.hkv + p.hkv + g) * tile + d * kPage + ref % kPage;
  };
  auto e_at = [&](int ref, int kind) {
    return p.scales + (((size_t)(ref / kPage) * p.hkv + g) * 2 + kind) * kPage + ref % kPage;
  };
#pragma unroll 4
  for (int x = threadIdx.x; x < n * D; x += kThreads) vs[x] = *v_at(from[x / D], x % D);
  for (int x = threadIdx.x; x < n * kChunks; x += kThreads)
    reinterpret_cast<u32x4 *>(ks)[x] = *reinterpret_cast<const u32x4 *>(k_at(from[x / kChunks], x % kChunks));
  if (kFp8)
    for (int x = threadIdx.x; x < 2 * n; x += kThreads) es[x] = *e_at(from[x / 2], x & 1);
  __syncthreads();
#pragma unroll 4
  for (int x = threadIdx.x; x < n * D; x += kThreads) *v_at(to[x / D], x % D) = vs[x];
  for (int x = threadIdx.x; x < n * kChunks; x += kThreads)
    *reinterpret_cast<u32x4 *>(k_at(to[x / kChunks], x % kChunks)) = reinterpret_cast<const u32x4 *>(ks)[x];
  if (kFp8)
    for (int x = threadIdx.x; x < 2 * n; x += kThreads) *e_at(to[x / 2], x & 1) = es[x];
}

template <bool kF32, bool kFp8>
void (*append_kernel(int dim))(AppendParams) {
  return dim == 128 ? rope_append_kernel<kF32, kFp8, 128> : rope_append_kernel<kF32, kFp8, 64>;
}
template <bool kFp8, bool kF32>
void (*read_kernel(int dim))(ReadParams) {
  return dim == 128 ? kv_read_kernel<kFp8, kF32, 128> : kv_read_kernel<kFp8, kF32, 64>;
}

}  // namespace

hipError_t launch_rope_append(AppendParams p, int dim, bool f32, bool fp8, hipStream_t s) {
  p.mode = p.interleaved || p.rot == 0 ? kAdjacent : (p.rot % 16 == 0 ? kHalfVec : kHalfAny);
  const int chunks = (p.rows + kChunk - 1) / kChunk;
  const long long pairs = (long long)chunks * p.hkv;
  p.heads_per_block = pairs < kManyBlocks ? 1 : (pairs < 2 * kManyBlocks ? 2 : kAppendHeads);
  p.kv_blocks = chunks * ((p.hkv + p.heads_per_block - 1) / p.heads_per_block);
  // one row of q to a workgroup and four: 2,047 rows 15.3 and 15.9 us, 3,000 20.6 and 20.5, 8,191
  // 58.9 and 49.8 (8-bit cache 50.5 and 47.9)
  p.q_rows = p.rows >= 2048 ? 4 : 1;
  const int q_blocks = p.hq > 0 ? (p.rows + p.q_rows - 1) / p.q_rows : 0;
  auto fn = f32 ? (fp8 ? append_kernel<true, true>(dim) : append_kernel<true, false>(dim))
                : (fp8 ? append_kernel<false, true>(dim) : append_kernel<false, false>(dim));
  launch_kernel(fn, dim3(p.kv_blocks + q_blocks), dim3(kThreads), s, p);
  return hipGetLastError();
}

hipError_t launch_kv_read(ReadParams p, int dim, bool fp8, bool f32, hipStream_t s) {
  const int chunks = (p.rows + kChunk - 1) / kChunk;
  // as fp32 the stage holds one head's V
  p.heads_per_block = f32 || (long long)chunks * p.hkv < kManyBlocks ? 1 : read_heads(dim);
  const int groups = (p.hkv + p.heads_per_block - 1) / p.heads_per_block;
  auto fn = fp8 ? (f32 ? read_kernel<true, true>(dim) : read_kernel<true, false>(dim))
                : (f32 ? read_kernel<false, true>(dim) : read_kernel<false, false>(dim));
  launch_kernel(fn, dim3(chunks * groups), dim3(kThreads), s, p);
  return hipGetLastError();
}

hipError_t launch_tree_commit(const CommitParams &p, int num_reqs, int dim, bool fp8,
                              hipStream_t s) {
  auto fn = fp8 ? (dim == 128 ? tree_commit_kernel<true, 128> : tree_commit_kernel<true, 64>)
                : (dim == 128 ? tree_commit_kernel<false, 128> : tree_commit_kernel<false, 64>);
  launch_kernel(fn, dim3(p.hkv, num_reqs), dim3(kThreads), s, p);
  return hipGetLastError();
}

}  // namespace dsv
