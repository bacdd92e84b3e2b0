// How the work over shared prefixes is dealt out, and how its partial results are joined with those
// of a session's own slots.
#pragma once
#include "tree.h"

// Units of work (a 64-slot record for a tile of kSharedTile rows) lie on a line: group after group,
// tile after tile, record after record, and the workgroups of a kv head take it in pieces, of which
// each leaves a partial result a tile.  The line is cut in one of two ways:
//  * evenly, so that all workgroups finish together whatever the lengths; a piece may then reach
//    over tiles, and each of them costs its queries' way in and its results' way out;
//  * every tile into the same number of pieces, which is taken where the longest of these is
//    shorter than an even piece and the price of a second tile in it (six records: eight sessions of
//    17 rows behind 2000 slots, three tiles, 44 us evenly cut and 37 tile by tile).
// An even piece has LEAST records at least, unless there are more tiles than such pieces; tile by tile
// the longest tile's pieces follow from LEAST, and a shorter tile beside it is cut into as many (ten of
// one record where the longest has ten of four).  Short pieces finish sooner, but each leaves its rows'
// results to be written and read (64 single tokens behind 8192 slots: 61.0 us at two records, 58.1 at
// four, 59.6 at eight; 32 behind 2048 34.9, 35.3 and 38.0).
struct SharedLine {
  static constexpr int LEAST = 4;
  int n, each, more;   // workgroups; evenly: records of each, and one more for the first `more`
  int pieces;          // of a tile, or 0: evenly
  // total: units, -, tiles, most records of a tile
  AS_DEVICE SharedLine(int4 total, int wgs) {
    const int units = total.x, tiles = total.z;
    n = min(max((units + LEAST - 1) / LEAST, tiles), wgs);
    each = n > 0 ? units / n : 0;
    more = units - n * each;
    pieces = tiles > 0 && tiles <= wgs ? min(wgs / tiles, (total.w + LEAST - 1) / LEAST) : 0;
    if (pieces && (total.w + pieces - 1) / pieces <= each + 6)
      n = tiles * pieces;
    else
      pieces = 0;
  }
  AS_DEVICE int begin(int w) const { return w * each + (w < more ? w : more); }
  // records of a piece of a tile of nblk
  AS_DEVICE int piece(int nblk) const { return (nblk + pieces - 1) / pieces; }
  // The workgroups of a tile (the tiles-th, from unit u0 on): the first, and how many.
  AS_DEVICE void workers(int tiles, int u0, int nblk, int *first, int *count) const {
    if (pieces) {
      *first = tiles * pieces;
      *count = (nblk + piece(nblk) - 1) / piece(nblk);
    } else {
      *first = worker(u0);
      *count = worker(u0 + nblk - 1) - *first + 1;
    }
  }

 private:
  AS_DEVICE int worker(int u) const {
    const int front = more * (each + 1);
    return u < front ? u / (each + 1) : more + (u - front) / each;
  }
};
// Where the partial rows of (a group's first member, tile, workgroup) begin, of one kv head: rows
// and workgroups both only grow along the line, so no two meet.
AS_DEVICE long long shared_rows_at(int first, int QR, int tile, int w) {
  return (long long)first * QR + (long long)(tile + w) * acespec::kSharedTile;
}

// The shared partial results of a row: `parts` of them, the first at ml (largest exponent, sum) and
// o, the next ones a tile's rows on.
struct SharedParts {
  const float2 *ml;
  const float *o;
  int parts;
};
template <int HD>
AS_DEVICE SharedParts shared_parts(const SharedJoin &j, const SharedSession &me, int4 total, int g,
                                   int qi, int QR) {
  SharedParts p{nullptr, nullptr, 0};
  if (me.place < 0) return p;
  const int nblk = (me.slots + 63) >> 6;
  const int local = (me.place - me.first) * QR + qi, tile = local / acespec::kSharedTile;
  const SharedLine line(total, j.wgs);
  int w0;
  line.workers(me.tiles + tile, me.units + tile * nblk, nblk, &w0, &p.parts);
  const long long at = g * j.rows_total + shared_rows_at(me.first, QR, tile, w0) +
                       (local - tile * acespec::kSharedTile);
  p.ml = (const float2 *)j.ml + at;
  p.o = j.o + at * HD;
  return p;
}

// A row's own partial result (largest exponent M in base 2, sum l, outputs o of four head dims from
// dim(i) on) joined with the shared ones, and written.  me, total: j.sm's, asked for in time.  bad:
// tree rows with values that are not finite, which were left out: whatever weight such a value has,
// an infinity or a NaN comes of it in the rows that see its slot.  sets: the session's ancestor sets;
// vb: the tree's values, [head dim][capacity].
template <int HD, int N, typename F>
AS_DEVICE void shared_finish(const SharedJoin &j, const SharedSession &me, int4 total,
                             const uint64_t *sets, const bf16 *vb, int capacity,
                             const uint32_t *bad, int b, int g, int qi, int n1, int H, int Hkv,
                             int rows, float M, float l, f32x4 (&o)[N], F dim) {
  typedef bf16 b4 __attribute__((ext_vector_type(4)));
  typedef f16 h4 __attribute__((ext_vector_type(4)));
  const int G = H / Hkv, r = qi / G, h = g * G + qi - r * G;
  const SharedParts p = shared_parts<HD>(j, me, total, g, qi, G * n1);
  float top = M;
#pragma unroll 4
  for (int s = 0; s < p.parts; ++s) top = fmaxf(top, p.ml[(size_t)s * acespec::kSharedTile].x);
  if (top == -INFINITY) top = 0.f;
  const float w = __builtin_amdgcn_exp2f(M - top);
  l *= w;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] *= w;
  constexpr int UNROLL = N == 1 ? 8 : 1;
#pragma unroll UNROLL
  for (int s = 0; s < p.parts; ++s) {
    const float2 e = p.ml[(size_t)s * acespec::kSharedTile];
    const float x = __builtin_amdgcn_exp2f(e.x - top);
    l += x * e.y;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      o[i] += x * *(const f32x4 *)(p.o + (size_t)s * acespec::kSharedTile * HD + dim(i));
      if (i % 8 == 7) SCHED_FENCE();   // (no more loads at a time than there are registers)
    }
  }
  if (bad[0] | bad[1] | bad[2]) {
    __asm__ volatile("");   // (seldom: a branch)
    const uint64_t anc = sets[r];
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll 1
      for (int t = 0; t < n1; ++t) {
        if (!((bad[t >> 5] >> (t & 31)) & 1u) || (t > 0 && !((anc >> (t - 1)) & 1ull))) continue;
        const bf16 *v = vb + (size_t)dim(i) * capacity + t;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = (float)(f16)(float)v[(size_t)e * capacity];
          if (!(fabsf(x) <= 65504.f)) o[i][e] += x;
        }
      }
      SCHED_FENCE();   // (few registers: the loops' addresses are not kept side by side)
    }
  }
  const float inv = 1.f / l;   // (a row sees itself)
  const int row = b * n1 + r;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const f32x4 y = o[i] * inv;
    if (j.rows_out)
      *(b4 *)((bf16 *)j.out + (size_t)row * H * HD + h * HD + dim(i)) =
          b4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    else
      *(h4 *)((f16 *)j.out + act_off(row, h * HD + dim(i), rows, H * HD)) =
          h4{(f16)y[0], (f16)y[1], (f16)y[2], (f16)y[3]};
  }
}
