// Tree-masked grouped-query attention over the 4-bit KV cache (quant.h), with an optional
// sliding window whose first tokens stay visible.
//
// Row r of a session of P slots sits at position P + depth(r).  It sees the P slots and, of the
// tree, its ancestors and itself; with a window w > 0 only what is at a position less than w
// behind its own, or below `sinks`.  Of the P slots the complete blocks of 32 are records, the
// rest and the tree's rows the tail in the model's type, taken as blocks of 32 slots too.
//
// Query rows are the G query heads of the kv head times the tree rows (row = tree_row * G +
// head) in tiles of 16.  The work is divided by slots, not by queries: a wave holds all TPW
// tiles of its workgroup (as accumulators; one or two) and takes blocks of its own, so a block's
// codes are read by one wave, straight into the registers that the matrix instructions read, and
// serve all the tiles.  No barrier and no LDS traffic but the queries' fragments.
//  * S^T = K Q^T by 16x16 products: a lane holds 8 scores of ONE query, for 8 consecutive
//    slots.  Its running reference, exp2 and the probabilities stay in the lane, and these are
//    its B operand of O^T = V^T P^T.
//  * bf16 model: the keys' codes and scale bytes ARE the operand of the scaled product
//    (v_mfma_scale_f32_16x16x128_f8f6f4, a scale per 32 elements), so keys are never decoded.
//    The queries are the other operand in pieces, hi the nearest e4m3 and each next one the
//    nearest to what is left, each with its own scale per 32 head dims.  A bf16 query (8
//    significant bits) is held exactly by hi and an e4m3 lo, but for what lies 2^22 below its
//    group's largest, and fp16's own range.  An fp16 one (the verify step's, 11 bits) is held
//    exactly by hi and two e3m2 pieces from 1/64 of its group's largest on, below that to
//    2^-17 of it, which is what fp32 sums of 128 products may lose; e3m2 multiplies at twice
//    e4m3's rate (a layer of the 8B step: 69.8 us, with three e4m3 pieces 71.5; with two, which
//    are off by up to 2^-9 of an element, 66.5).
//    Values are decoded to fp16 (exactly) and multiplied by fp16 weights
//    (v_mfma_f32_16x16x32_f16), the tail's keys and values widened to fp16.  A weight is rounded
//    once (2^-11 of it; below 2^-25 of the row's largest it may count as 0), their sum stays
//    fp32: an output moves by 2e-4 in the norm, before it is rounded to bf16 by 1.7e-3.
//  * fp32 model: keys and values decoded to fp32 (exactly), v_mfma_f32_16x16x4_f32.
//  * The reference of a query's exponents moves only when a score exceeds it by about 2^8
//    (LAZY_LOG2), and only then are the four lanes of a query reduced and the accumulators
//    rescaled: one rare branch for all tiles, so that one tile's exponents fill the matrix
//    pipe's time on the others.
// At the end the waves of a workgroup, and then the splits of a session, are joined by their
// (maximum, sum) pairs.
//
// What bounds it: a single row, the way from memory to L2 (64 sessions x 2048 slots x 8 kv heads of
// 128: 156 MB counted there in 25.3 us, repeated, the MALL keeping some; 27.5 us with the records in
// HBM, 5.7 TB/s); 17 rows there, vector issue (69 % busy in 60.2 us, 65 from HBM; of a block's 760
// cycles for two tiles 300 decode the values, 176 are exponentials) and two rounds' fixed part of
// about 9 us each (tail, queries, join); 65 rows over 16384 slots, vector issue (74 %, matrix
// cores 50 %; 158.6 us, 140 GFLOP).  Few rows: the chain of loads, products and join, 6 to 10 us.
// Slower as measured: keys decoded to fp16 (92 us where this took 70), records through a ring in
// LDS (72 and 181 against 69 and 167), weights through LDS with waves taking head dims (79, 240).
//
// Not finite: a group of 32 marked so reads as NaN.  NaN and inf reach the rows that see them
// and no others: where a mask applies, values that are not finite count as 0 in the products and
// are added at the end, to the rows that see their slots.
#include "quant.h"

#include <type_traits>
#include <utility>

namespace {

constexpr float LAZY_LOG2 = 8.f;
constexpr float LAZY_SUM = 8 * 256.f;   // of 8 weights none of which exceeds 2^LAZY_LOG2
constexpr float LOG2E = 1.4426950408889634f;
constexpr int SLOW = 3;   // what a masked block costs a wave, in blocks that every row sees whole

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
// The operand arithmetic of a model's type: eight elements of a lane.
template <typename T> struct Ops;
template <> struct Ops<bf16> {
  typedef f16x8 F8;
  typedef f16 E;
  static AS_DEVICE F8 decode(uint32_t c, float s) { return q4_decode_f16(c, s); }
  typedef bf16x8 Raw;
  static AS_DEVICE Raw raw(const bf16 *p) { return *(const bf16x8 *)p; }
  static AS_DEVICE F8 wide(bf16x8 v) { return bf16x8_to_f16x8(v); }
  static AS_DEVICE f32x4 mma(F8 a, F8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Ops<float> {
  typedef f32x8 F8;
  typedef float E;
  static AS_DEVICE F8 decode(uint32_t c, float s) { return q4_decode_f32(c, s); }
  typedef F8 Raw;
  static AS_DEVICE F8 raw(const float *p) {
    const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
    return F8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static AS_DEVICE F8 wide(F8 v) { return v; }
  static AS_DEVICE f32x4 mma(F8 a, F8 b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// n / d by one multiplication, for 0 <= n and (n + 1) d <= 2^32: a workgroup's own indices cost
// a chain of eight divisions otherwise (some 250 scalar instructions before its first load).
struct Div {
  uint32_t m;
  explicit Div(int d) : m(0xffffffffu / (uint32_t)d) {}
  AS_DEVICE int operator()(int n) const { return (int)__umulhi((uint32_t)n + 1u, m); }
};

struct QuantAttnArgs {
  const void *q;            // [rows][H hd]: T (rows_io) or the activation type
  const uint8_t *blocks;    // records of the layer
  const void *tk, *tv;      // tail of the layer
  // The trees: prepared as pos and anc, or else as the caller's parents [rows] and lengths [B],
  // and status [B] to write.
  const int32_t *pos;       // [rows] P + depth
  const uint64_t *anc;      // [rows] visible drafted rows (bit j - 1)
  const int32_t *parents, *prefix;
  int32_t *status;
  void *out;
  float *part_o, *part_ml;
  int rows, n1, H, Hkv, G, nblk, tcap, nsplit, nqg, each, more, window, sinks;   // G = H / Hkv; a
                            // group has each tiles, the first `more` of them one more
  Div by_nqg, by_nsplit, by_Hkv, by_G;
  int rows_io;              // 1: q and out are row-major in T; 0: q row-major and out in the
                            // activation layout, fp16 (bf16 model; fp32: the same as 1)
};

// What a query row sees.
struct RowView {
  int lo;         // slots of the prefix from here on, and below `sinks`
  int root;       // whether it sees the root
  uint64_t anc;   // drafted rows
};
// Bit j: whether it sees tree row tr0 + j or, where that is negative, position pos0 + j of the
// prefix (j < 8).
AS_DEVICE uint32_t visible(const RowView &w, int sinks, int tr0, int pos0) {
  auto ones = [](int n) { return (1u << min(max(n, 0), 8)) - 1u; };   // the first n of 8
  const uint32_t prefix = ones(-tr0) & (~ones(w.lo - pos0) | ones(sinks - pos0));
  uint32_t tree;
  if (tr0 >= 1) tree = tr0 <= 64 ? (uint32_t)(w.anc >> (tr0 - 1)) : 0u;
  else tree = tr0 > -8 ? (((uint32_t)w.anc << 1) | (uint32_t)w.root) << -tr0 : 0u;
  return (prefix | tree) & 255u;
}

// The drafted rows of a session's tree from the caller's parents, in one wave: lane j holds row
// j + 1, `parent` its parent and rows n1 - 1.  Each row's ancestors are folded in by pointer
// jumping over shuffles; a malformed tree (`ok` false) becomes a chain.
struct TreeRow {
  uint64_t anc;   // visible drafted rows
  int depth;
};
AS_DEVICE TreeRow tree_row(const QuantAttnArgs &a, int lane, int P, int parent, bool ok) {
  const bool in = lane + 1 < a.n1;
  int jump = !in ? 0 : ok ? parent : lane;   // the next ancestor's row, 0 (the root): none
  uint64_t anc = in ? 1ull << lane : 0ull;
  for (int span = 1; span < a.n1; span *= 2) {
    const uint64_t up = __shfl((unsigned long long)anc, max(jump - 1, 0));
    const int next = __shfl(jump, max(jump - 1, 0));
    if (jump) anc |= up, jump = next;
  }
  const int depth = __popcll(anc);
  if (a.window && __any(depth >= a.window))   // ancestors too far back
    for (int j = 0; j + 1 < a.n1; ++j) {
      const int dj = __shfl(depth, j);
      if (depth - dj >= a.window && P + dj >= a.sinks) anc &= ~(1ull << j);
    }
  return {anc, depth};
}

// Eight consecutive elements of a query row as they are, and as operands; four of an output row.
AS_DEVICE u32x4 load_q(const QuantAttnArgs &a, bf16, size_t off) {
  return *(const u32x4 *)((const uint16_t *)a.q + off);
}
template <bool FP16> AS_DEVICE f16x8 wide_q(u32x4 v) {   // FP16: so they are already
  return FP16 ? __builtin_bit_cast(f16x8, v) : bf16x8_to_f16x8(__builtin_bit_cast(bf16x8, v));
}
AS_DEVICE f32x8 load_q(const QuantAttnArgs &a, float, size_t off) {
  return Ops<float>::raw((const float *)a.q + off);
}
// What a thread of NT loads of a workgroup's queries: element e = i NT + its number is a piece of
// 8 head dims, e % (HD / 8), of query e / (HD / 8).  Asked for first of all, as nothing else
// need be known for it.
template <typename T, int HD, int TPW, int NT> struct Asked {
  static constexpr int ALL = TPW * 16 * (HD / 8), N = (ALL + NT - 1) / NT;
  decltype(load_q(std::declval<const QuantAttnArgs &>(), T(), 0)) v[N];
  AS_DEVICE void load(const QuantAttnArgs &a, int qbase, int QR, int g, int row0, int tid) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * NT + tid, qi = qbase + e / (HD / 8), r = a.by_G(qi), h = g * a.G + (qi - r * a.G);
      v[i] = {};
      if ((ALL % NT == 0 || e < ALL) && qi < QR)
        v[i] = load_q(a, T(), (size_t)(row0 + r) * (a.H * HD) + h * HD + e % (HD / 8) * 8);
    }
  }
};
AS_DEVICE void store_out(const QuantAttnArgs &a, bf16, int row, int col, int width, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  if (a.rows_io)
    *(bf16x4 *)((bf16 *)a.out + (size_t)row * width + col) =
        bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  else
    *(f16x4 *)((f16 *)a.out + act_off(row, col, a.rows, width)) =
        f16x4{(f16)v[0], (f16)v[1], (f16)v[2], (f16)v[3]};
}
AS_DEVICE void add_out(const QuantAttnArgs &a, bf16, int row, int col, int width, float v) {
  if (a.rows_io) {
    bf16 *p = (bf16 *)a.out + (size_t)row * width + col;
    *p = (bf16)((float)*p + v);
  } else {
    f16 *p = (f16 *)a.out + act_off(row, col, a.rows, width);
    *p = (f16)((float)*p + v);
  }
}
AS_DEVICE void add_out(const QuantAttnArgs &a, float, int row, int col, int width, float v) {
  ((float *)a.out)[(size_t)row * width + col] += v;
}
AS_DEVICE void store_out(const QuantAttnArgs &a, float, int row, int col, int width, f32x4 v) {
  *(f32x4 *)((float *)a.out + (size_t)row * width + col) = v;
}

AS_DEVICE bool not_finite(f16 v) { return (__builtin_bit_cast(uint16_t, v) & 0x7c00) == 0x7c00; }
AS_DEVICE bool not_finite(float v) { return abs_bits(v) >= 0x7f800000u; }
template <typename F8> AS_DEVICE F8 finite(F8 v) {   // 0 for what is not
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = not_finite(v[j]) ? 0.f : v[j];
  return v;
}
// Whether one is not, for many at once: an exponent of ones carries into the sign's place.
AS_DEVICE uint32_t carries(f16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t |= (w[i] & 0x7c007c00u) + 0x04000400u;
  return t & 0x80008000u;
}
AS_DEVICE uint32_t carries(f32x8 v) {
  uint32_t t = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) t |= (__float_as_uint(v[j]) & 0x7f800000u) + 0x00800000u;
  return t & 0x80000000u;
}
// The first n of eight (none, or all, where n is below or above that), 0 for the others.
AS_DEVICE f16x8 first_of(f16x8 v, int n) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= n >= 2 * i + 2 ? ~0u : n > 2 * i ? 0xffffu : 0u;
  return __builtin_bit_cast(f16x8, w);
}
AS_DEVICE f32x8 first_of(f32x8 v, int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] : 0.f;
  return v;
}

// The queries of a workgroup's tiles as operands of the scores, in LDS.
//
// fp32 model: [tile][hd / 32 fragments][lane][8], head dims lg * hd/4 + 8 s .. of query lr.
template <typename T, int HD, int TPW, bool FP16> struct Queries {
  float x[TPW][HD / 32][64][8];
  AS_DEVICE f32x8 plain(int i, int s, int lane) const { return *(const f32x8 *)x[i][s][lane]; }
  template <int NT> AS_DEVICE void fill(const Asked<T, HD, TPW, NT> &q, int tid) {
#pragma unroll
    for (int i = 0; i < q.N; ++i) {
      const int e = i * NT + tid, qi = e / (HD / 8), c = e % (HD / 8);
      if (q.ALL % NT == 0 || e < q.ALL)
        *(f32x8 *)x[qi >> 4][c % (HD / 32)][c / (HD / 32) * 16 + (qi & 15)] = q.v[i];
    }
  }
};
// bf16 model, bf16 queries: e4m3 pieces [tile][piece][half][lane][16 bytes] and their scale bytes
// [tile][lane].  Element k of the 128 that a product contracts is byte k % 16 of lane group
// k % 64 / 16 in half k / 64 (measured; an e2m1 operand's is nibble k % 32 of lane group k / 32),
// its scale that of lane group k / 32.  hd 128: pieces hi and lo, their scales bytes 0 and 1.
// hd 64: one product, the first half hi and the second lo (the keys' lane groups 2 and 3 repeat 0
// and 1, so one product adds both).
// FP16: hi alone (hd 64: the second half is 0), scale byte 0, and e3m2 pieces lo and rest, which
// lie as e2m1 does, in 6 bits an element: 16 bytes of a lane and 8 more.  hd 128: products 0 and
// 1, scale bytes 1 and 2.  hd 64: one product, lane groups 0 and 1 lo, 2 and 3 rest, scale byte 1.
template <int HD, int TPW, bool FP16> struct Queries<bf16, HD, TPW, FP16> {
  static constexpr int NP = HD / 64, N8 = FP16 ? 1 : NP;   // products of a half or whole; e4m3 ones
  u32x4 x[TPW][N8][2][64];
  u32x4 six[TPW][FP16 ? NP : 1][64];
  uint2 six2[TPW][FP16 ? NP : 1][64];
  f16x8 wide[TPW][HD / 32][64];   // fp16, for the tail: as in the fp32 model
  typename std::conditional<FP16, uint32_t, uint16_t>::type scale[TPW][64];
  AS_DEVICE f16x8 plain(int i, int s, int lane) const { return wide[i][s][lane]; }
  AS_DEVICE i32x8 piece(int i, int p, int lane) const {
    const u32x4 a = x[i][p][0][lane], b = FP16 && HD == 64 ? u32x4{} : x[i][p][1][lane];
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
  }
  AS_DEVICE i32x8 piece6(int i, int p, int lane) const {
    const u32x4 a = six[i][p][lane];
    const uint2 b = six2[i][p][lane];
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b.x, (int)b.y, 0, 0};
  }
  // The nearest e3m2 (sign, 3 bits of exponent with bias 3, 2 of mantissa) of eight values of at
  // most 28, piece `at` of a lane's four; what they leave.  At 2^-12 of a value fp16's exponent is
  // e3m2's, subnormals among them, so its upper bits, rounded, are the code.
  AS_DEVICE void put6(f16x2 (&v)[4], int i, int p, int lane, int at) {
    uint32_t c[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t h = __builtin_bit_cast(uint32_t, v[w] * (f16)0x1p-12);
      const uint32_t r = h + 0x007f007fu + ((h >> 8) & 0x00010001u);
      v[w] -= __builtin_bit_cast(f16x2, r & 0xff00ff00u) * (f16)0x1p12;
      const uint32_t t = ((r >> 8) & 0x001f001fu) | ((r >> 10) & 0x00200020u);
      c[w] = (t | (t >> 10)) & 0xfffu;
    }
    const uint32_t word[2] = {c[0] | (c[1] << 12) | (c[2] << 24), (c[2] >> 8) | (c[3] << 4)};
#pragma unroll
    for (int j = 0; j < 3; ++j) {   // 48 bits
      const int u = at * 3 + j;
      uint16_t *to = u < 8 ? (uint16_t *)&six[i][p][lane] + u : (uint16_t *)&six2[i][p][lane] + (u - 8);
      *to = (uint16_t)(word[j >> 1] >> (16 * (j & 1)));
    }
  }
  template <int NT> AS_DEVICE void fill(const Asked<bf16, HD, TPW, NT> &q, int tid) {
#pragma unroll
    for (int i = 0; i < q.N; ++i) {
      const int e = i * NT + tid;
      if (q.ALL % NT && e >= q.ALL) break;
      const int qi = e / (HD / 8), tile = qi >> 4, piece = e % (HD / 8), lr = qi & 15, c = piece >> 2;   // c: group
      const f16x8 v = wide_q<FP16>(q.v[i]);
      wide[tile][piece % (HD / 32)][piece / (HD / 32) * 16 + lr] = v;
      float f[8];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[j] = (float)v[j];
        top = max(top, abs_bits(f[j]));
      }
      top = max(top, (uint32_t)__shfl_xor((int)top, 1));   // four lanes a group
      top = max(top, (uint32_t)__shfl_xor((int)top, 2));
      // hi: the largest in [128, 256); what it leaves is at most 8.  An e4m3 lo holds 16 times
      // that; an e3m2 one twice that, leaving at most 1 of 16, of which rest holds 16 times
      const int ex = max((int)(top >> 23), 30) - 7;      // biased; fp16 queries are 2^-24 or 0
      const bool bad = top >= 0x7f800000u;               // NaN or inf: every score is NaN
      const float down = bad ? 0.f : __uint_as_float((uint32_t)(254 - ex) << 23);
      uint32_t hi[2], lo[2];
      f16x2 left[4];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        float y[4], d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = bad ? 0.f : f[4 * w + j] * down;
        hi[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        hi[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], hi[w], true);
        d[0] = (y[0] - __builtin_amdgcn_cvt_f32_fp8(hi[w], 0)) * (FP16 ? 2.f : 16.f);
        d[1] = (y[1] - __builtin_amdgcn_cvt_f32_fp8(hi[w], 1)) * (FP16 ? 2.f : 16.f);
        d[2] = (y[2] - __builtin_amdgcn_cvt_f32_fp8(hi[w], 2)) * (FP16 ? 2.f : 16.f);
        d[3] = (y[3] - __builtin_amdgcn_cvt_f32_fp8(hi[w], 3)) * (FP16 ? 2.f : 16.f);
        if (FP16) {   // (at most 7 bits)
          left[2 * w] = f16x2{(f16)d[0], (f16)d[1]};
          left[2 * w + 1] = f16x2{(f16)d[2], (f16)d[3]};
        } else {
          lo[w] = __builtin_amdgcn_cvt_pk_fp8_f32(d[0], d[1], 0, false);
          lo[w] = __builtin_amdgcn_cvt_pk_fp8_f32(d[2], d[3], lo[w], true);
        }
      }
      auto scaled = [&](int down) { return bad ? 255u : (uint32_t)(ex - down); };
      const int half = piece >> 1 & 1, at = piece & 1;   // of the group's 32 bytes: which 8
      const bool one = (piece & 3) == 0;
      const int l = (HD == 128 ? (c & 1) * 2 + half : c * 2 + half) * 16 + lr, lane = c * 16 + lr;
      ((uint2 *)&x[tile][0][HD == 128 ? c >> 1 : 0][l])[at] = make_uint2(hi[0], hi[1]);
      if constexpr (FP16) {
        put6(left, tile, 0, lane, piece & 3);
#pragma unroll
        for (int w = 0; w < 4; ++w) left[w] *= (f16)16.f;
        put6(left, tile, NP - 1, HD == 128 ? lane : lane + 32, piece & 3);
        if (one) {
          if (HD == 128) {
            scale[tile][lane] = scaled(0) | (scaled(1) << 8) | (scaled(5) << 16);
          } else {
            scale[tile][lane] = scaled(0) | (scaled(1) << 8);
            scale[tile][lane + 32] = scaled(5) << 8;
          }
        }
      } else if constexpr (HD == 128) {
        ((uint2 *)&x[tile][N8 - 1][c >> 1][l])[at] = make_uint2(lo[0], lo[1]);
        if (one) scale[tile][lane] = (uint16_t)(scaled(0) | (scaled(4) << 8));
      } else {
        ((uint2 *)&x[tile][0][1][l])[at] = make_uint2(lo[0], lo[1]);
        if (one) {
          scale[tile][lane] = (uint16_t)scaled(0);
          scale[tile][lane + 32] = (uint16_t)scaled(4);
        }
      }
    }
  }
};

// 16 bytes of a record's codes; ONCE: past the caches, as no other workgroup reads them.
template <bool ONCE> AS_DEVICE u32x4 codes(const uint8_t *p) {
  return ONCE ? __builtin_nontemporal_load((const u32x4 *)p) : *(const u32x4 *)p;
}
// What a lane holds of a block's keys, and the scores of a tile against them.
template <typename T, int HD> struct Keys {   // fp32 model
  u32x4 k[HD / 64];
  uint32_t ks;
  struct Op { f32x8 f[2][HD / 32]; };          // decoded
  template <bool ONCE> AS_DEVICE void load(const uint8_t *rec, int lane) {
    const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) k[h] = codes<ONCE>(rec + h * 1024 + lane * 16);
    ks = *(const uint16_t *)(rec + 32 * HD + (lr * (HD / 32) + (HD == 128 ? lg : lg >> 1)) * 2);
  }
  AS_DEVICE Op operand() const {
    Op o;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int s = 0; s < HD / 32; ++s)
        o.f[kk][s] = q4_decode_f32(HD == 128 ? k[kk * (HD / 128)][s] : k[0][kk * 2 + s],
                                   q4_scale((ks >> (8 * kk)) & 255u));
    return o;
  }
  template <typename Q> static AS_DEVICE void score(const Op &o, const Q &q, int i, int lane, f32x4 (&sc)[2]) {
    sc[0] = sc[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < HD / 32; ++s) {
      const f32x8 qf = q.plain(i, s, lane);
      sc[0] = Ops<T>::mma(o.f[0][s], qf, sc[0]);
      sc[1] = Ops<T>::mma(o.f[1][s], qf, sc[1]);
    }
  }
};
template <int HD> struct Keys<bf16, HD> {     // bf16 model: as they are
  u32x4 k[2];
  uint32_t ks;
  struct Op { i32x8 f[2]; int ks; };
  template <bool ONCE> AS_DEVICE void load(const uint8_t *rec, int lane) {
    const int lr = lane & 15, lg = lane >> 4;
    if constexpr (HD == 128) {
      k[0] = codes<ONCE>(rec + lane * 16);
      k[1] = codes<ONCE>(rec + 1024 + lane * 16);
      ks = *(const uint16_t *)(rec + 32 * HD + (lr * 4 + lg) * 2);
    } else {   // both 16-dim halves of group lg % 2, each with both operands' keys
      k[0] = codes<ONCE>(rec + ((lg & 1) * 32 + lr) * 16);
      k[1] = codes<ONCE>(rec + ((lg & 1) * 32 + 16 + lr) * 16);
      ks = *(const uint16_t *)(rec + 32 * HD + (lr * 2 + (lg & 1)) * 2);
    }
  }
  AS_DEVICE Op operand() const {
    Op o = {};
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int j = 0; j < 4; ++j) o.f[kk][j] = (int)(HD == 128 ? k[kk][j] : k[j >> 1][kk * 2 + (j & 1)]);
    o.ks = (int)ks;
    return o;
  }
  template <int TPW, bool FP16>
  static AS_DEVICE void score(const Op &o, const Queries<bf16, HD, TPW, FP16> &q, int i, int lane,
                              f32x4 (&sc)[2]) {
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const int qs = q.scale[i][lane];
    // operand formats: 4 e2m1 (keys), 0 e4m3, 3 e3m2; scale byte kk of ks, and the piece's of qs
    const i32x8 a = q.piece(i, 0, lane);
    sc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[0], a, zero, 4, 0, 0, o.ks, 0, qs);
    sc[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[1], a, zero, 4, 0, 1, o.ks, 0, qs);
    if constexpr (FP16) {
      const i32x8 b = q.piece6(i, 0, lane);
      sc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[0], b, sc[0], 4, 3, 0, o.ks, 1, qs);
      sc[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[1], b, sc[1], 4, 3, 1, o.ks, 1, qs);
      if constexpr (HD == 128) {
        const i32x8 d = q.piece6(i, 1, lane);
        sc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[0], d, sc[0], 4, 3, 0, o.ks, 2, qs);
        sc[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[1], d, sc[1], 4, 3, 1, o.ks, 2, qs);
      }
    } else if constexpr (HD == 128) {
      const i32x8 b = q.piece(i, 1, lane);
      sc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[0], b, sc[0], 4, 0, 0, o.ks, 1, qs);
      sc[1] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(o.f[1], b, sc[1], 4, 0, 1, o.ks, 1, qs);
    }
  }
};
// ... and of its values.
template <int HD> struct Values {
  u32x4 v[HD / 64];
  uint32_t vs[HD / 64];   // byte nb % 4 of word nb / 4
  template <bool ONCE> AS_DEVICE void load(const uint8_t *rec, int lane) {
#pragma unroll
    for (int h = 0; h < HD / 64; ++h) {
      v[h] = codes<ONCE>(rec + 16 * HD + h * 1024 + lane * 16);
      vs[h] = *(const uint32_t *)(rec + 33 * HD + (lane & 15) * (HD / 16) + h * 4);
    }
  }
  AS_DEVICE float scale(int nb) const { return q4_scale((vs[nb >> 2] >> (8 * (nb & 3))) & 255u); }
};

template <typename T, int HD, int TPW, int NW, bool FP16> struct Shared {
  // value operands a wave joins (8 waves and head dim 64: only the first four do)
  static constexpr int OWN = HD / 16 > NW ? HD / 16 / NW : 1;
  union {
    Queries<T, HD, TPW, FP16> q;
    f32x4 part[TPW][HD / 16 / OWN][OWN * (NW - 1)][64];   // accumulators other waves join
  };
  RowView view[TPW * 16];
  float2 ml[NW][TPW * 16];
};

template <typename T, int HD, int TPW, int LDST, int NW, bool ONCE, bool FP16>
AS_DEVICE void attend(const QuantAttnArgs &a, Shared<T, HD, LDST, NW, FP16> &smem_, int item, int split, int qbase) {
  typedef Ops<T> O;
  typedef typename O::F8 F8;
  typedef typename O::E E;
  typedef typename O::Raw Raw;
  typedef Keys<T, HD> K;
  constexpr int NB = HD / 16, LD = HD / 4, OWN = Shared<T, HD, TPW, NW, FP16>::OWN;
  Shared<T, HD, TPW, NW, FP16> &sm = reinterpret_cast<Shared<T, HD, TPW, NW, FP16> &>(smem_);
  const int b = a.by_Hkv(item), g = item - b * a.Hkv;
  const int G = a.G, QR = G * a.n1;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int row0 = b * a.n1, width = a.H * HD;
  const bool own = a.parents != nullptr;
  const int given = own ? a.prefix[b] : a.pos[row0], most = a.nblk * Q4_SLOTS + Q4_SLOTS - 1;
  const int parent = own && wave == 0 && lane + 1 < a.n1 ? a.parents[row0 + lane + 1] : 0;
  const int root = own ? a.parents[row0] : -1;
  Asked<T, HD, TPW, NW * 64> asked;
  asked.load(a, qbase, QR, g, row0, tid);
  const int P = min(max(given, 0), most), t = P & (Q4_SLOTS - 1), full = P / Q4_SLOTS;

  // Complete blocks that some row sees: [0, nsink) and [wlo, full).  Those that every row sees
  // whole are [0, send) and [wend, full); a window cuts [send, nsink) and [wlo, wend).
  int nsink = 0, wlo = 0, send = 0, wend = 0;
  if (a.window) {
    wlo = min(max(P - a.window + 1, 0) / Q4_SLOTS, full);        // the root's window starts first
    nsink = min((int)(((unsigned)a.sinks + Q4_SLOTS - 1) / Q4_SLOTS), wlo);
    send = min(a.sinks / Q4_SLOTS, nsink);
    const long long last = (long long)P + a.n1 - a.window;       // the deepest row's at most here
    wend = min(max((int)((last > 0 ? last : 0) + Q4_SLOTS - 1) / Q4_SLOTS, wlo), full);
  }
  // Masked blocks, the tail's first, then the cut ones; then the whole ones.  A masked block
  // counts as SLOW whole ones in the shares of the splits and of the waves.
  const int ntail = (t + a.n1 + Q4_SLOTS - 1) / Q4_SLOTS;
  const int nmask = ntail + nsink - send + wend - wlo, nwhole = send + full - wend;
  const int per = a.by_nsplit(nmask * SLOW + nwhole + a.nsplit - 1);
  const int u0 = split * per, u1 = u0 + per;
  const int m0 = min((u0 + SLOW - 1) / SLOW, nmask), m1 = min((u1 + SLOW - 1) / SLOW, nmask);
  const int w0 = min(max(u0 - nmask * SLOW, 0), nwhole), w1 = min(max(u1 - nmask * SLOW, 0), nwhole);
  auto masked_block = [&](int m) {   // m >= ntail: a record
    m -= ntail;
    return m < nsink - send ? send + m : wlo + m - (nsink - send);
  };
  auto whole_block = [&](int c) { return c < send ? c : wend + c - send; };
  // Of the split's masked blocks wave w takes every NW-th; the first `odd` waves one more than
  // the others, which have SLOW rounds of whole blocks to themselves.
  const int odd = (m1 - m0) % NW;
  auto whole_of_round = [&](int r) {
    const int alone = SLOW * (NW - odd);
    return r < SLOW ? w0 + r * (NW - odd) + wave - odd : w0 + alone + (r - SLOW) * NW + wave;
  };

  const uint8_t *rec0 = a.blocks + (size_t)item * a.nblk * q4_bytes(HD);
  const T *tk = (const T *)a.tk + (size_t)item * a.tcap * HD;
  const T *tv = (const T *)a.tv + (size_t)item * HD * a.tcap;
  int round = wave < odd ? SLOW : 0, c = whole_of_round(round);
  auto record = [&](int c) { return rec0 + (size_t)whole_block(min(c, nwhole - 1)) * q4_bytes(HD); };
  // A wave's first block of the tail is loaded ahead of everything.
  Raw kt[2][HD / 32], vt[NB];
  const bool early = m0 + wave < min(m1, ntail);
  if (early) {
    const int s0 = (m0 + wave) * Q4_SLOTS;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int s = 0; s < HD / 32; ++s)
        kt[kk][s] = O::raw(tk + (size_t)(s0 + q4_key(kk, lr)) * HD + lg * LD + s * 8);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      vt[nb] = O::raw(tv + (size_t)(nb * 16 + lr) * a.tcap + s0 + lg * 8);
  }

  K key;
  if (c < w1) key.template load<ONCE>(record(c), lane);
  RowView mine = {};
  if (wave == 0) {
    const int r = a.by_G(min(qbase + min(lane, TPW * 16 - 1), QR - 1));
    int depth;
    if (own) {
      const bool ok = __all(parent >= 0 && parent <= lane) && root == -1 && given == P;
      const TreeRow row = tree_row(a, lane, P, parent, ok);
      mine.anc = __shfl((unsigned long long)row.anc, max(r - 1, 0));
      depth = __shfl(row.depth, max(r - 1, 0));
      if (r == 0) mine.anc = depth = 0;
      if (lane == 0 && qbase == 0 && split == 0 && g == 0) a.status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
    } else {
      mine.anc = a.anc[row0 + r];
      depth = a.pos[row0 + r] - P;
    }
    mine.lo = a.window ? max(P + depth - a.window + 1, 0) : 0;
    mine.root = !a.window || depth < a.window || P < a.sinks;
  }
  sm.q.template fill<NW * 64>(asked, tid);
  if (tid < TPW * 16) sm.view[tid] = mine;
  __syncthreads();

  const float sscale = LOG2E / sqrtf((float)HD);   // scores -> exponents of 2
  float mb[TPW], l_run[TPW];   // reference as an exponent (-inf: none yet), sum of weights
  f32x4 o[TPW][NB];
  // Moves the reference of tile i where one of the scores exceeds it by too much; returns it, or
  // 0 where there is none.
  auto refer = [&](int i, const f32x4 (&sc)[2]) -> float {
    float mx = sc[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j >> 2][j & 3]);
    mx *= sscale;
    if (__ballot(mx > mb[i] + LAZY_LOG2)) {
      mx = rows4_max(mx);
      const float mn = mx > mb[i] + LAZY_LOG2 ? mx : mb[i];
      const float alpha = __builtin_amdgcn_exp2f(mb[i] - (mn == -INFINITY ? 0.f : mn));
      mb[i] = mn;
      l_run[i] *= alpha;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][nb][e] *= alpha;
    }
    return mb[i] == -INFINITY ? 0.f : mb[i];
  };
  // The weights of a tile's scores against reference m, as operands of the values; adds their
  // sum in the lane.
  auto weights = [&](f32x4 (&sc)[2], float m, float &sum) -> F8 {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      sc[j >> 2][j & 3] = __builtin_amdgcn_exp2f(fmaf(sc[j >> 2][j & 3], sscale, -m));
    sum = ((sc[0][0] + sc[1][0]) + (sc[0][1] + sc[1][1])) + ((sc[0][2] + sc[1][2]) + (sc[0][3] + sc[1][3]));
    F8 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = (E)sc[j >> 2][j & 3];
    return p;
  };

  // Masked blocks: those of the tail (slots of the last, incomplete block, then the tree's
  // rows) and records that a window cuts.
  bool bad = false;   // one held values that are not finite: left out here, put in at the end
  auto mask = [&](int i, int tr0, int pos0, f32x4 (&sc)[2]) {
    const uint32_t vis = visible(sm.view[i * 16 + lr], a.sinks, tr0, pos0);
#pragma unroll
    for (int j = 0; j < 8; ++j) sc[j >> 2][j & 3] = (vis >> j) & 1u ? sc[j >> 2][j & 3] : -INFINITY;
  };
  if (early) {   // nothing is summed yet
    const int s0 = (m0 + wave) * Q4_SLOTS, tr0 = s0 - t + lg * 8;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    F8 p[TPW];
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      f32x4 sc[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int s = 0; s < HD / 32; ++s)
          sc[kk] = O::mma(O::wide(kt[kk][s]), sm.q.plain(i, s, lane), s ? sc[kk] : zero);
      mask(i, tr0, full * Q4_SLOTS + s0 + lg * 8, sc);
      float mx = sc[0][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j >> 2][j & 3]);
      mb[i] = rows4_max(mx) * sscale;
      p[i] = weights(sc, mb[i] == -INFINITY ? 0.f : mb[i], l_run[i]);
    }
    F8 vf[NB];
    uint32_t nf = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      vf[nb] = first_of(O::wide(vt[nb]), a.n1 - tr0);   // slots behind the last row were never written
      nf |= carries(vf[nb]);
    }
    if (__ballot(nf)) {
      bad = true;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) vf[nb] = finite(vf[nb]);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < TPW; ++i) o[i][nb] = O::mma(vf[nb], p[i], zero);
  } else {
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      mb[i] = -INFINITY;
      l_run[i] = 0.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) o[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
#pragma unroll 1
  for (int m = m0 + wave + (early ? NW : 0); m < m1; m += NW) {
    const bool tail = m < ntail;
    const int blk = masked_block(m), s0 = m * Q4_SLOTS;   // s0: first slot within the tail
    const int tr0 = tail ? s0 - t + lg * 8 : -Q4_SLOTS;
    const int pos0 = (tail ? full * Q4_SLOTS + s0 : blk * Q4_SLOTS) + lg * 8;
    const uint8_t *rec = rec0 + (size_t)(tail ? 0 : blk) * q4_bytes(HD);
    F8 p[TPW];
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
      if (tail) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int s = 0; s < HD / 32; ++s)
            sc[kk] = O::mma(O::wide(O::raw(tk + (size_t)(s0 + q4_key(kk, lr)) * HD + lg * LD + s * 8)),
                            sm.q.plain(i, s, lane), sc[kk]);
      } else {
        K kc;
        kc.template load<ONCE>(rec, lane);
        K::score(kc.operand(), sm.q, i, lane, sc);
      }
      mask(i, tr0, pos0, sc);
      float sum;
      p[i] = weights(sc, refer(i, sc), sum);
      l_run[i] += sum;
      SCHED_FENCE();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      F8 vf;
      if (tail)
        vf = O::wide(O::raw(tv + (size_t)(nb * 16 + lr) * a.tcap + s0 + lg * 8));
      else
        vf = O::decode(*(const uint32_t *)(rec + 16 * HD + (nb >> 2) * 1024 + lane * 16 + (nb & 3) * 4),
                       q4_scale(rec[33 * HD + lr * NB + nb]));
      vf = first_of(vf, a.n1 - tr0);
      if (__ballot(carries(vf))) {
        bad = true;
        vf = finite(vf);
      }
#pragma unroll
      for (int i = 0; i < TPW; ++i) o[i][nb] = O::mma(vf, p[i], o[i][nb]);
      if (nb % 2) SCHED_FENCE();
    }
  }
  // Whole blocks.  The next block's keys are asked for once the scores have read this one's,
  // its values once they are multiplied: a wave's loads cross the other half of its work.
  // A lane does not look for its largest score: a reference that is too low (or, before the
  // first, -inf) shows in the sum of the weights (inf, or NaN where a score is -inf itself), and
  // the scores are then computed again.
  Values<HD> val;
  if (c < w1) val.template load<ONCE>(record(c), lane);
  while (c < w1) {
    c = whole_of_round(++round);
    F8 p[TPW];
    float add[TPW];
    bool over = false;
    const typename K::Op kop = key.operand();
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
      f32x4 sc[2];
      K::score(kop, sm.q, i, lane, sc);
      p[i] = weights(sc, mb[i], add[i]);
      over |= !(add[i] <= LAZY_SUM);
    }
    if (__ballot(over)) {
#pragma unroll
      for (int i = 0; i < TPW; ++i) {
        f32x4 sc[2];
        K::score(kop, sm.q, i, lane, sc);
        p[i] = weights(sc, refer(i, sc), add[i]);
        SCHED_FENCE();
      }
    }
    key.template load<ONCE>(record(c), lane);
#pragma unroll
    for (int i = 0; i < TPW; ++i) l_run[i] += add[i];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const F8 vf = O::decode(val.v[nb >> 2][nb & 3], val.scale(nb));
#pragma unroll
      for (int i = 0; i < TPW; ++i) o[i][nb] = O::mma(vf, p[i], o[i][nb]);
    }
    val.template load<ONCE>(record(c), lane);
  }

  // Join the waves: o[i][nb][e] is head dim 16 nb + 4 lg + e of query 16 i + lr.  Wave w joins
  // the operands nb = w OWN .. and hands the others' to their waves.
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    const float l = rows4_sum(l_run[i]);
    if (lg == 0)
      sm.ml[wave][i * 16 + lr] = make_float2(mb[i], l);
  }
  const bool any_bad = __syncthreads_or(bad);   // (and the queries are read)
  float top[TPW], sum[TPW];
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    float M = -INFINITY, L = 0.f, f = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sm.ml[w][i * 16 + lr].x);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 e = sm.ml[w][i * 16 + lr];
      const float fw = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - M);
      L += fw * e.y;
      f = w == wave ? fw : f;
    }
    top[i] = M;
    sum[i] = L;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][nb][e] *= f;
  }
  // (qi: the query, acc: what the other waves handed over, for operand nb)
  auto finish = [&](int i, int nb, f32x4 acc) {
    const int qi = qbase + i * 16 + lr;
#pragma unroll
    for (int w = 0; w < NW - 1; ++w) {
      const f32x4 v = sm.part[i][wave][w * OWN + nb % OWN][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += v[e];
    }
    if (qi < QR) {
      const int r = a.by_G(qi), h = g * G + (qi - r * G);
      if (a.nsplit == 1) {
        const float inv = 1.f / sum[i];                  // every row sees itself
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= inv;
        store_out(a, T(), row0 + r, h * HD + nb * 16 + lg * 4, width, acc);
      } else {
        const size_t q = ((size_t)item * a.nsplit + split) * QR + qi;
        *(f32x4 *)(a.part_o + q * HD + nb * 16 + lg * 4) = acc;
        if (nb == 0 && lg == 0) *(float2 *)(a.part_ml + q * 2) = make_float2(top[i], sum[i]);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < TPW; ++i)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      if (nb / OWN != wave)
        sm.part[i][nb / OWN][(wave - (wave > nb / OWN)) * OWN + nb % OWN][lane] = o[i][nb];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TPW; ++i)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      if (nb / OWN == wave) finish(i, nb, o[i][nb]);
  if (!any_bad) return;
  // Values that are not finite, in the masked blocks of this split (rare): added to the rows
  // that see their slots, and to no others.
  __threadfence();
  __syncthreads();
#pragma unroll 1
  for (int x = tid; x < TPW * 16 * HD; x += NW * 64) {
    const int e = x / HD, d = x % HD, qi = qbase + e;
    if (qi >= QR) break;
    const RowView w = sm.view[e];
    float v = 0.f;
#pragma unroll 1
    for (int m = m0; m < m1; ++m) {
      const bool tail = m < ntail;
      const int blk = masked_block(m), s0 = m * Q4_SLOTS;
      const int n = tail ? min(Q4_SLOTS, t + a.n1 - s0) : Q4_SLOTS;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        if (!(visible(w, a.sinks, tail ? s0 + j - t : -Q4_SLOTS,
                      tail ? full * Q4_SLOTS + s0 + j : blk * Q4_SLOTS + j) & 1u))
          continue;
        const float y = tail ? (float)(E)(float)tv[(size_t)d * a.tcap + s0 + j]
                             : q4_scale(rec0[(size_t)blk * q4_bytes(HD) + 33 * HD + d % 16 * NB + d / 16]);
        if (not_finite(y)) v += tail ? y : __builtin_nanf("");
      }
    }
    if (v == 0.f) continue;
    const int r = a.by_G(qi), h = g * G + (qi - r * G);
    if (a.nsplit == 1) add_out(a, T(), row0 + r, h * HD + d, width, v);
    else a.part_o[(((size_t)item * a.nsplit + split) * QR + qi) * HD + d] += v;
  }
}

// Waves a SIMD holds, by the registers of the accumulators (hd 128: 32 a tile) and of the fp32
// model's decoded keys.
template <typename T> constexpr int waves_per_simd(int tpw) {
  return sizeof(T) == 4 ? 2 : tpw == 1 ? 4 : 3;
}

// A workgroup: TPW tiles of a session's kv head (or one less: the tiles are dealt evenly to nqg
// groups) over one of nsplit shares of its blocks.  FP16: the queries are fp16 (not those of the
// standalone call, which two pieces hold).
template <typename T, int HD, int TPW, int NW, bool ONCE, bool FP16>
__global__ __launch_bounds__(NW * 64, waves_per_simd<T>(TPW)) void quant_attn_kernel(QuantAttnArgs a) {
  __shared__ __attribute__((aligned(16))) Shared<T, HD, TPW, NW, FP16> sm;
  // The query groups and the splits of a session's kv head follow each other on one XCD: the
  // groups read the same records.
  const int id = xcd_tile(blockIdx.x, gridDim.x);
  const int pair = a.by_nqg(id), grp = id - pair * a.nqg;
  const int item = a.by_nsplit(pair), split = pair - item * a.nsplit;
  const int qbase = (grp * a.each + min(grp, a.more)) * 16;
  if (TPW == 1 || a.each + (grp < a.more) == TPW) attend<T, HD, TPW, TPW, NW, ONCE, FP16>(a, sm, item, split, qbase);
  else attend<T, HD, (TPW > 1 ? TPW - 1 : 1), TPW, NW, ONCE, FP16>(a, sm, item, split, qbase);
}

// Joins the splits: one thread per 4 head dims of a query row.
template <typename T>
__global__ __launch_bounds__(256) void quant_combine_kernel(QuantAttnArgs a, int HD) {
  const int item = blockIdx.y, b = a.by_Hkv(item), g = item - b * a.Hkv;
  const int G = a.G, QR = G * a.n1, hd4 = HD >> 2;
  const int idx = blockIdx.x * 256 + threadIdx.x;
  if (idx >= QR * hd4) return;
  const int qi = idx / hd4, d = (idx - qi * hd4) * 4;
  const size_t q0 = (size_t)item * a.nsplit * QR + qi;
  const float2 *ml = (const float2 *)a.part_ml + q0;
  const float *po = a.part_o + q0 * HD + d;
  float M = -INFINITY;
#pragma unroll 8
  for (int s = 0; s < a.nsplit; ++s) M = fmaxf(M, ml[(size_t)s * QR].x);
  f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
#pragma unroll 8
  for (int s = 0; s < a.nsplit; ++s) {
    const float2 e = ml[(size_t)s * QR];
    const f32x4 v = *(const f32x4 *)(po + (size_t)s * QR * HD);
    const float w = e.x == -INFINITY ? 0.f : exp2f(e.x - M);   // (a split without slots)
    den += w * e.y;
#pragma unroll
    for (int j = 0; j < 4; ++j) num[j] += w * v[j];
  }
  const float inv = 1.f / den;
#pragma unroll
  for (int j = 0; j < 4; ++j) num[j] *= inv;
  const int r = a.by_G(qi), h = g * G + (qi - r * G);
  store_out(a, T(), b * a.n1 + r, h * HD + d, a.H * HD, num);
}

template <typename T, int HD, bool FP16>
void launch_tiles(int tpw, int waves, bool once, unsigned grid, hipStream_t s, const QuantAttnArgs &a) {
  auto kernel = once       ? quant_attn_kernel<T, HD, 1, 4, true, FP16>
                : tpw == 1 ? quant_attn_kernel<T, HD, 1, 4, false, FP16>
                           : quant_attn_kernel<T, HD, 2, 4, false, FP16>;
  if constexpr (sizeof(T) == 2)
    if (waves == 8) kernel = quant_attn_kernel<T, HD, 1, 8, false, FP16>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(waves * 64), 0, s, a);
}

}  // namespace

namespace acespec {

template <typename T>
hipError_t launch_attention_quant(const void *q, const uint8_t *blocks, const T *tk, const T *tv,
                                  const TreeMeta &meta, const int32_t *parents,
                                  const int32_t *prefix, int32_t *status, void *out, float *part_o,
                                  float *part_ml, long long part_capacity, int B, int n1, int H, int Hkv, int hd,
                                  int capacity, int tcap, int window, int sinks, int rows_io,
                                  int cus, hipStream_t s) {
  // The lengths are on the device, so that all that follows goes by the capacity: right for any
  // prefix, chosen for long ones.  Much shorter prefixes pay for it (17 rows over 32 heads: 8
  // sessions of 300 slots 8.1 us in a cache of 320 and 17.8 in one of 32768, of 2000 slots 19.3
  // and 22.0; 64 of 2048 58.7 and 58.5).
  const int QR = H / Hkv * n1, tiles = (QR + 15) / 16, items = B * Hkv;
  const long long seen = window ? (long long)window + n1 + sinks + 2 * Q4_SLOTS : capacity;
  const int blocks_seen = (int)((seen < capacity ? seen : capacity) / Q4_SLOTS) + 3;
  const long long work = (long long)items * tiles;
  // No more tiles than CUs: a workgroup of eight waves on each CU, one tile each (bf16; one
  // session of 17 rows, 1500 slots: 10.2 us against 11.1 with four waves, 24 x one row, 4000
  // slots: 21 against 27).  Below 16 blocks eight waves have nothing to share.
  const bool wide = sizeof(T) == 4, few = work <= cus;
  const int waves = few && !wide && blocks_seen >= 16 ? 8 : 4;
  // One tile a session (a token, as in plain decoding) otherwise, and more than 96 MB of records:
  // they pass the caches (64 sessions x 2048 slots, 143 MB: 29.6 us against 31.8; 26
  // MB, which a repeated call finds there: 13.9 against 12.4).
  const bool once = tiles == 1 && !few && items * (long long)blocks_seen * q4_bytes(hd) > (96 << 20);
  // Tiles a workgroup otherwise: two share a block's decoding and its read (70b fan-out: 85 us
  // against 106), so they are taken for many tiles, for long prefixes and where they leave a CU
  // one workgroup (8 sessions of 17 rows x 2000: 17.0 us against 19.0; x 2: 6.5 against 5.9, so
  // not below 32 blocks); one keeps two or three on each CU and the CUs even (12 x 2000: 19.7 against 23.9; fp32 model: 3 sessions of 60 rows,
  // 8.8 against 11.6, one workgroup a CU or not).  Three were slower than two at head
  // dim 128 (90 against 85) and mixed at 64 (36 against 33 with 5 tiles, 57 against 64 with 17).
  const bool even = wide ? work <= 2LL * cus
                         : blocks_seen < 128 && work <= 3LL * cus &&
                               (blocks_seen < 32 || items * ((tiles + 1LL) / 2) > cus);
  const int most = few || even ? 1 : 2;
  const int nqg = (tiles + most - 1) / most, tpw = (tiles + nqg - 1) / nqg;
  // Splits, where a CU would have less than two workgroups: as many as it holds at once, of eight
  // waves one; from 128 blocks on (few tiles: from 64), of 32 at least, which pays for their
  // joining (40 single rows x 2000: 21.5 us in two, 19.4 in one).  fp32 model: of 12, as a block
  // takes longer there (4 sessions x 1000: 22 us in two, 28 in one).  A prefix of 384 blocks or
  // more is read in four parts also by up to three workgroups a CU: small ones end closer
  // together (16384 slots, 576 workgroups: 169 us against 179).
  const int each = wide ? 12 : 32, from = wide || few ? 2 * each : 128;
  const long long splits = blocks_seen >= from ? blocks_seen / each : 1;
  const long long groups = (long long)items * nqg;
  long long nsplit = 1;
  if (groups < 2LL * cus) nsplit = (waves == 8 ? 1LL : tpw == 1 ? 4LL : 3LL) * cus / groups;
  if (waves == 4 && groups < 3LL * cus && nsplit < 4 && blocks_seen >= 384) nsplit = 4;
  nsplit = nsplit < splits ? nsplit : splits;
  if (nsplit < 1) nsplit = 1;
  while (nsplit > 1 && (long long)items * nsplit * QR * hd > part_capacity) --nsplit;
  const int G = H / Hkv, nblk = capacity / Q4_SLOTS;
  // (what Div divides; only a long cache can bring a number of splits to the limit)
  while (nsplit > 1 && (nblk + 128 + nsplit) * nsplit > 0x80000000LL) --nsplit;
  if ((groups * nsplit + 1) * nqg > 0xffffffffLL || (items + 1LL) * Hkv > 0xffffffffLL ||
      (QR + 33LL) * G > 0xffffffffLL)
    return hipErrorInvalidValue;
  const QuantAttnArgs a{q, blocks, tk, tv, meta.pos, meta.anc, parents, prefix, status, out, part_o, part_ml,
                        B * n1, n1, H, Hkv, G, nblk, tcap, (int)nsplit, nqg, tiles / nqg, tiles % nqg, window,
                        sinks, Div(nqg), Div((int)nsplit), Div(Hkv), Div(G), rows_io};
  const unsigned grid = (unsigned)(groups * nsplit);
  auto launch = hd == 128 ? launch_tiles<T, 128, false> : launch_tiles<T, 64, false>;
  if constexpr (sizeof(T) == 2)
    if (!rows_io) launch = hd == 128 ? launch_tiles<T, 128, true> : launch_tiles<T, 64, true>;
  launch(tpw, waves, once, grid, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nsplit == 1) return e;
  hipLaunchKernelGGL(quant_combine_kernel<T>, dim3((QR * (hd / 4) + 255) / 256, items), dim3(256), 0,
                     s, a, hd);
  return hipGetLastError();
}

template hipError_t launch_attention_quant<float>(const void *, const uint8_t *, const float *,
                                                  const float *, const TreeMeta &, const int32_t *,
                                                  const int32_t *, int32_t *, void *, float *, float *,
                                                  long long, int, int, int, int, int, int,
                                                  int, int, int, int, int, hipStream_t);
template hipError_t launch_attention_quant<bf16>(const void *, const uint8_t *, const bf16 *,
                                                 const bf16 *, const TreeMeta &, const int32_t *,
                                                 const int32_t *, int32_t *, void *, float *, float *,
                                                 long long, int, int, int, int, int, int,
                                                 int, int, int, int, int, hipStream_t);

}  // namespace acespec
