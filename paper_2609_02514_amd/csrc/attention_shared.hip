// Tree attention for sessions that stand behind shared prefixes.
//
// A row's keys are its session's shared prefix, the session's own slots, and its ancestors in the
// tree: with scores z and base-2 exponents, o = sum 2^(z - m) v / sum 2^(z - m) over all of them.
// The sum over the shared slots is the same product for every session of a group, so it is
// computed for all their query rows at once: the group's members * G * (N + 1) rows of a kv head
// against the prefix's records, a matrix product with a softmax between, where a session alone
// would stream the prefix for G * (N + 1) rows.  The own slots are the tree attention's work
// (attention.hip); both leave partial (sum, max, outputs) and one pass joins them.
#include "shared.h"

namespace {

constexpr float RAISE = 1024.f;    // sum of 16 weights from which on their reference moves
constexpr int AHEAD = 2;           // products whose operands are on their way from LDS

constexpr int TM = acespec::kSharedTile;

// A value that all lanes hold alike, in a scalar register: what depends on it stays there too (loop
// counts, addresses, branches), where a loaded value would make vector work of all of it.
AS_DEVICE int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A value is computed where this stands, not where it is used.
#define PIN(x) __asm__ volatile("" : "+v"(x))

AS_DEVICE f16x8 to_f16x8(f16x8 v) { return v; }
AS_DEVICE f16x8 to_f16x8(bf16x8 v) { return bf16x8_to_f16x8(v); }

// Eight waves, 32 query rows each, over one record after the other.  A record is 1 KB operands of
// v_mfma_f32_32x32x16_f16 in the order in which they are multiplied: keys (rows are slots, in an
// order that makes a lane's scores 8 neighbouring slots) for S^T = K Q^T, then values (rows are
// head dims) for O^T = V^T P^T.  A lane's scores, as fp16 weights, are its operand of the second
// product, so they never leave its registers.  Records come by DMA into a ring of NST stages.
//
// What bounds it: a half record (32 slots) takes a wave 512 cycles of its SIMD's matrix core and
// about 430 of its vector unit (16 exponentials of 16 cycles, their scaling, sums, rounding), and
// two waves share a SIMD.  The halves are therefore pipelined: while the weights of one half are
// computed, the scores of the next and the product with the values of the one before run, which
// depend on none of it.  Measured: 32 sessions of 264 rows behind up to 16384 slots 0.98 to 1.05
// PFLOP/s (475 to 525 us), the matrix cores 56 % busy at the 1.73 GHz that the card's power leaves; 64
// sessions of 68 rows behind up to 8192 slots 105 to 123 us, 42 % busy at 2.0 GHz, as a workgroup goes
// through one and a half tiles there.
template <int HD, typename TQ>
__global__ __launch_bounds__(512) void shared_attn_kernel(
    const TQ *__restrict__ q, const f16 *__restrict__ blocks, SharedMeta sm,
    float *__restrict__ part_o, float *__restrict__ part_ml, int B, int n1, int H, int Hkv, int cap,
    int wgs, long long rows_total) {
  constexpr int KS = HD / 16, NDB = HD / 32;
  constexpr int REC = 128 * HD;                 // elements of a record
  constexpr int L_DMA = REC * 2 / 1024 / 8;     // 1 KB pieces a wave
  constexpr int NST = 4;   // stages: the loop holds two records and has one in flight beside the next
  __shared__ __attribute__((aligned(1024))) f16 smem[NST * REC];
  const int t = xcd_tile(blockIdx.x, gridDim.x), g = t / wgs, w = t - g * wgs;
  // (the groups are asked for, 64 at a time, before it is known how many there are)
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), lq = lane & 31, hh = lane >> 5;
  SharedGroup mine = sm.groups[min(lane, B - 1)];
  int4 total = *sm.total;
  total = make_int4(uniform(total.x), uniform(total.y), uniform(total.z), uniform(total.w));
  const int groups = total.y;
  const SharedLine line(total, wgs);
  if (w >= line.n) return;
  int u = line.begin(w), at = 0;   // `mine` is group at + lane
  int uend = line.begin(w + 1);
  const int G = H / Hkv, QR = G * n1;
  const float sscale = LOG2E / sqrtf((float)HD);
  // the group of unit x, or of tile x
  auto group_of = [&](int x, bool tiles) {
    auto begins = [&](const SharedGroup &s) { return tiles ? s.tiles : s.units; };
    int before;   // groups of the 64 that begin at x or before
    while ((before = __popcll(__ballot(at + lane < groups && begins(mine) <= x))) == 64 && at + 64 < groups &&
           uniform(begins(sm.groups[at + 64])) <= x) {
      at += 64;
      mine = sm.groups[min(at + lane, B - 1)];
    }
    return before - 1;
  };
  if (line.pieces) {   // a piece of one tile
    const int tile = w / line.pieces, gi = group_of(tile, true);
    const int nblk = (__builtin_amdgcn_readlane(mine.slots, gi) + 63) >> 6, piece = line.piece(nblk);
    const int u0 = __builtin_amdgcn_readlane(mine.units, gi) +
                   (tile - __builtin_amdgcn_readlane(mine.tiles, gi)) * nblk;
    const int c = (w - tile * line.pieces) * piece;
    u = u0 + min(c, nblk);
    uend = u0 + min(c + piece, nblk);
  }

  while (u < uend) {
    const int gi = group_of(u, false);
    const int first = __builtin_amdgcn_readlane(mine.first, gi), slots = __builtin_amdgcn_readlane(mine.slots, gi);
    const int prefix = __builtin_amdgcn_readlane(mine.prefix, gi);
    const int rows = __builtin_amdgcn_readlane(mine.members, gi) * QR, nblk = (slots + 63) >> 6;
    const int in = u - __builtin_amdgcn_readlane(mine.units, gi), tile = in / nblk, c0 = in - tile * nblk;
    const int c1 = min(nblk, c0 + (uend - u));
    u += c1 - c0;
    const int row = tile * TM + wave * 32 + lq;   // of the group
    const bool any = tile * TM + wave * 32 < rows;
    const f16 *kv = blocks + (((size_t)prefix * Hkv + g) * (cap >> 6) + c0) * REC;
    const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(kv, (uint32_t)(c1 - c0) * (REC * 2));
    auto issue = [&](int c) {
      const int i = c - c0;
#pragma unroll
      for (int j = 0; j < L_DMA; ++j) {
        const int piece = j * 8 + wave;
        buf_dma16(rsrc, (lds_ptr_t)(smem + (i % NST) * REC + piece * 512), lane * 16,
                  i * (REC * 2) + piece * 1024);
      }
    };
    // the first record is on its way while the queries are looked up
    chunk_barrier();      // (the last tile's stages are free)
    issue(c0);
    // queries: rows of padding multiply zeros
    f16x8 qf[KS];
    {
      const int rr = min(row, rows - 1), m = rr / QR, rem = rr - m * QR, r = rem / G;
      const TQ *qp = q + ((size_t)sm.order[first + m] * n1 + r) * H * HD +
                     (g * G + rem - r * G) * HD + hh * 8;
      typedef TQ q8 __attribute__((ext_vector_type(8)));
      q8 raw[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) raw[s] = *(const q8 *)(qp + s * 16);
#pragma unroll
      for (int i = 1; i < NST - 1; ++i)
        if (c0 + i < c1) issue(c0 + i);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const f16x8 v = to_f16x8(raw[s]);
        qf[s] = row < rows ? v : f16x8{};
      }
    }
    float m_run = -INFINITY, l_run = 0.f;
    f32x16 o[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

    auto stage_of = [&](int c) { return smem + ((c - c0) % NST) * REC + lane * 8; };
    // S^T of half kb of a stage
    auto scores = [&](const f16 *st, int kb, f32x16 &z) {
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        z = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const f16x8 *)(st + (kb * KS + s) * 512), qf[s], z,
                                                   0, 0, 0);
    };
    // O^T += V^T P^T of half kb; valid: slots of the record (what lies behind the prefix may be no
    // number at all)
    auto values = [&](const f16 *st, int kb, const f16x8 (&p)[2], int valid) {
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          f16x8 v = *(const f16x8 *)(st + REC / 2 + ((kb * 2 + k2) * NDB + db) * 512);
          if (valid < 64) {
            MASK_BRANCH();
            const int lim = valid - hh * 8 - kb * 32 - k2 * 16;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= lim) v[e] = (f16)0.f;
          }
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[k2], o[db], 0, 0, 0);
        }
    };
    // score i of a lane in half kb: slot 32 kb + 16 (i / 8) + 8 hh + i % 8
    auto mask = [&](f32x16 &z, int kb, int valid) {
      if (valid < 64) {
        MASK_BRANCH();
        const int lim = valid - hh * 8 - kb * 32;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((i >> 3) * 16 + (i & 7) >= lim) z[i] = -INFINITY;
      }
    };
    auto top = [&](const f32x16 &z) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, z[i]);
      return halves_max(mx);
    };
    // The weights of scores z in the reference m_run; their sum.
    auto reference = [&] { return m_run == -INFINITY ? 0.f : m_run * sscale; };
    auto weights = [&](const f32x16 &z, f16x8 (&p)[2]) {
      const float mb = reference();
      float rs = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(fmaf(z[i], sscale, -mb));
        rs += e;
        p[i >> 3][i & 7] = (f16)e;
      }
      return rs;
    };
    // Takes up the sum rs of weights p of scores z.  The reference of the exponents is not looked
    // for beforehand: it holds until a lane's weights add up to more than RAISE (each is then still
    // far inside fp16), when it moves to the largest score and they are computed again.  o holds no
    // product of p yet.
    auto take = [&](const f32x16 &z, f16x8 (&p)[2], float rs) {
      if (__ballot(rs > RAISE || m_run == -INFINITY)) {
        MASK_BRANCH();
        const float mn = fmaxf(m_run, top(z));
        const float alpha = __builtin_amdgcn_exp2f((m_run - (mn == -INFINITY ? 0.f : mn)) * sscale);
        m_run = mn;
        l_run *= alpha;
        rs = weights(z, p);
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
      l_run += rs;
    };
    // One half: the weights pc of scores zc, beside them the scores zn of half kn of stage sn and the
    // product with half kv of stage sv that was pending (weights pp).  The products' operands are
    // read two ahead, and each product is followed by the weights' share of its time.
    auto half = [&](const f32x16 &zc, f16x8 (&pc)[2], f32x16 &zn, const f16 *sn, int kn,
                    const f16x8 (&pp)[2], const f16 *sv, int kv) {
      constexpr int SPP = 16 / KS;   // scores a pair of products
      const f16 *kp = sn + kn * KS * 512, *vp = sv + REC / 2 + kv * KS * 512;
      f16x8 kf[KS], vf[KS];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        kf[i] = *(const f16x8 *)(kp + i * 512);
        vf[i] = *(const f16x8 *)(vp + i * 512);
      }
      const float mb = reference();
      float e[16], rs = 0.f;
      auto sum = [&](int x0) {
#pragma unroll
        for (int x = x0; x < x0 + SPP; x += 2) {
          rs += e[x];
          rs += e[x + 1];
          f16x2 two = {(f16)e[x], (f16)e[x + 1]};
          PIN(two);
          pc[x >> 3][x & 7] = two[0];
          pc[x >> 3][(x & 7) + 1] = two[1];
        }
        PIN(rs);
      };
#pragma unroll
      for (int i = 0; i < 16; ++i) zn[i] = 0.f;
      SCHED_FENCE();
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        zn = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i], qf[i], zn, 0, 0, 0);
        if (i + AHEAD < KS) kf[i + AHEAD] = *(const f16x8 *)(kp + (i + AHEAD) * 512);
#pragma unroll
        for (int x = i * SPP; x < (i + 1) * SPP; ++x) {
          e[x] = __builtin_amdgcn_exp2f(fmaf(zc[x], sscale, -mb));
          PIN(e[x]);
        }
        SCHED_FENCE();
        o[i % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i], pp[i / NDB], o[i % NDB], 0, 0, 0);
        if (i + AHEAD < KS) vf[i + AHEAD] = *(const f16x8 *)(vp + (i + AHEAD) * 512);
        if (i > 0) sum((i - 1) * SPP);
        SCHED_FENCE();
      }
      sum((KS - 1) * SPP);
      take(zc, pc, rs);
    };

    if (c0 + 2 < c1) wait_vmcnt<2 * L_DMA>(); else wait_vmcnt<0>();
    chunk_barrier();      // record c0 is there
    f32x16 za, zb;        // scores of the record's halves
    f16x8 pa[2], pb[2];
    if (any) {
      const int valid = slots - c0 * 64;
      scores(stage_of(c0), 0, za);
      mask(za, 0, valid);
      m_run = top(za);
      scores(stage_of(c0), 1, zb);
      l_run = weights(za, pa);
      mask(zb, 1, valid);
    }
    for (int c = c0; c + 1 < c1; ++c) {
      if (c + 2 < c1) wait_vmcnt<L_DMA>(); else wait_vmcnt<0>();
      chunk_barrier();    // record c + 1 is there, record c - 1 is used up, for every wave
      if (c + 3 < c1) issue(c + 3);
      if (!any) continue;
      const f16 *st = stage_of(c), *next = stage_of(c + 1);
      half(zb, pb, za, next, 0, pa, st, 0);
      const int valid = slots - (c + 1) * 64;
      mask(za, 0, valid);
      half(za, pa, zb, next, 1, pb, st, 1);
      mask(zb, 1, valid);
    }
    if (any) {
      const f16 *st = stage_of(c1 - 1);
      const int valid = slots - (c1 - 1) * 64;
      const float rs = weights(zb, pb);
      values(st, 0, pa, valid);
      take(zb, pb, rs);
      values(st, 1, pb, valid);
    }
    const float l = halves_sum(l_run);
    if (row < rows) {
      const long long to = g * rows_total + shared_rows_at(first, QR, tile, w) + wave * 32 + lq;
      float *po = part_o + to * HD + hh * 4;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(f32x4 *)(po + db * 32 + j * 8) =
              f32x4{o[db][j * 4], o[db][j * 4 + 1], o[db][j * 4 + 2], o[db][j * 4 + 3]};
      if (hh == 0) {
        part_ml[to * 2] = m_run == -INFINITY ? -INFINITY : m_run * sscale;
        part_ml[to * 2 + 1] = l;
      }
    }
  }
}

// A row's partial results joined where its session was split: of its tile over the shared prefix,
// and of the parts of its own slots.  A thread takes four head dims of every JOIN-th part: few rows
// have many parts, and one thread for all of them leaves too few loads under way (4: one token behind
// 8192 slots 25.2 -> 21.1 us, 32 behind 2048 36.2 -> 34.3, 64 behind 8192 61.6 -> 60.8), which many
// rows do by themselves (8 sessions of 17 rows 28.2 -> 29.7, 256 single tokens 136 -> 143; so from
// 256 threads a CU on JOIN is 1).
template <int HD, int JOIN>
__global__ __launch_bounds__(256) void shared_combine_kernel(const float *__restrict__ part_o,
                                                             const float *__restrict__ part_ml,
                                                             SharedJoin j, TreeMeta meta,
                                                             const bf16 *__restrict__ cv,
                                                             int capacity, int rows, int n1, int H,
                                                             int Hkv, int nsplit) {
  constexpr int TD = HD / 4, RPW = 256 / (TD * JOIN);   // threads of a part, rows of a workgroup
  __shared__ f32x4 s_o[RPW][JOIN][TD];
  __shared__ float2 s_ml[RPW][JOIN];
  __shared__ uint32_t s_bad[RPW][JOIN][3];
  const int piece = threadIdx.x % TD, d = piece * 4, k = threadIdx.x / TD % JOIN, x = threadIdx.x / (TD * JOIN);
  const long long rh = min((long long)blockIdx.x * RPW + x, (long long)rows * H - 1);
  const int row = (int)(rh / H), h = (int)(rh - (long long)row * H);
  const int b = row / n1, r = row - b * n1, G = H / Hkv, g = h / G, QR = G * n1;
  const int qi = r * G + h - g * G;
  SharedSession me{0, -1, 0, 0, 0};   // (with blocks the parts hold the shared slots too)
  int4 total{};
  if (!j.blocks) {
    me = j.sm.sessions[b];
    total = *j.sm.total;
  }
  const SharedParts p = shared_parts<HD>(j, me, total, g, qi, QR);
  const size_t item0 = ((size_t)b * Hkv + g) * nsplit * QR + qi;
  const float2 *ml = (const float2 *)part_ml + item0;
  const float *po = part_o + item0 * HD + d;
  constexpr size_t ON = acespec::kSharedTile;
  float M = -INFINITY;
  const uint32_t *marks = j.sm.bad + ((size_t)b * Hkv + g) * nsplit * 3;
  uint32_t bad[3] = {0, 0, 0};
#pragma unroll 4
  for (int s = k; s < nsplit; s += JOIN) {
    M = fmaxf(M, ml[(size_t)s * QR].x);
#pragma unroll
    for (int i = 0; i < 3; ++i) bad[i] |= marks[s * 3 + i];
  }
#pragma unroll 8
  for (int s = k; s < p.parts; s += JOIN) M = fmaxf(M, p.ml[s * ON].x);
  float top = M == -INFINITY ? 0.f : M;
  f32x4 o[1] = {f32x4{0.f, 0.f, 0.f, 0.f}};
  float l = 0.f;
  auto add = [&](float2 e, f32x4 v) {   // (a part without slots: weight 2^-inf, zero sums)
    const float w = __builtin_amdgcn_exp2f(e.x - top);
    l += w * e.y;
    o[0] += w * v;
  };
#pragma unroll 4
  for (int s = k; s < nsplit; s += JOIN) add(ml[(size_t)s * QR], *(const f32x4 *)(po + (size_t)s * QR * HD));
#pragma unroll 8
  for (int s = k; s < p.parts; s += JOIN) add(p.ml[s * ON], *(const f32x4 *)(p.o + s * ON * HD + d));
  if constexpr (JOIN > 1) {
    s_o[x][k][piece] = o[0];
    if (piece == 0) {
      s_ml[x][k] = make_float2(M, l);
#pragma unroll
      for (int i = 0; i < 3; ++i) s_bad[x][k][i] = bad[i];
    }
    __syncthreads();
    M = -INFINITY;
#pragma unroll
    for (int i = 0; i < JOIN; ++i) M = fmaxf(M, s_ml[x][i].x);
    top = M == -INFINITY ? 0.f : M;
    o[0] = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN; ++i) {
      add(s_ml[x][i], s_o[x][i][piece]);
#pragma unroll
      for (int w = 0; w < 3; ++w) bad[w] |= s_bad[x][i][w];
    }
  }
  if (k > 0 || (long long)blockIdx.x * RPW + x > rh) return;
  me.place = -1;   // (its parts are in)
  const bf16 *vb = cv + ((size_t)b * Hkv + g) * HD * capacity + meta.sess_S[b];
  shared_finish<HD>(j, me, total, meta.anc + (size_t)b * n1, vb, capacity, bad, b, g, qi, n1, H, Hkv, rows, M, l, o,
                    [&](int) { return d; });
}

// fp32 models: one workgroup per 16 query rows of a (session, kv head), over the prefix's records
// and behind them the session's own slots as one line of slots, whose blocks of 16 go round its
// eight waves.  S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x4_f32: lane (x, y) of 16 x 4
// holds key row x and head dims y HD/4 .. of it (the products' steps may take the dims in any order
// that the queries share), hence scores of slots 4 y .. 4 y + 3 for query x, which are as they stand
// its operand of the second product: step e takes slot 4 y + e.  No LDS before the join, and no
// rounding to fewer bits anywhere.  Bound by latency in small batches and by the reads of keys and
// values (L2) in large ones, 16 rows a read: a workgroup a row and head took 332 us for 4 sessions
// of 25 rows and 4 heads a kv head over 1200 slots where this takes 50.
template <int HD, bool TREES>
__global__ __launch_bounds__(512) void shared_attn_f32_kernel(
    const float *__restrict__ qin, const float *__restrict__ blocks, SharedArgs sh,
    const SharedSession *__restrict__ sessions, const float *__restrict__ ck,
    const float *__restrict__ cv, TreeMeta meta, TreeArgs trees, float *__restrict__ out, int n1, int H,
    int Hkv, int capacity) {
  constexpr int NW = 8, NK = HD / 16, ND = HD / 16, REC = 128 * HD;
  __shared__ __attribute__((aligned(16))) float so[NW][16][HD + 4];
  __shared__ float sml[NW][16][2];
  __shared__ int s_bad;   // a tree row has a value that is not finite
  const int tile = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lx = lane & 15, ly = lane >> 4;
  const int G = H / Hkv, QR = G * n1, qi = min(tile * 16 + lx, QR - 1), r = qi / G;
  __shared__ TreeSets sets[1];
  // queries, and the first keys and values, are on their way before the tree is known
  f32x4 qf[NK];
  const float *qp = qin + ((size_t)b * n1 + r) * H * HD + (g * G + qi - r * G) * HD + ly * (HD / 4);
#pragma unroll
  for (int i = 0; i < NK; ++i) qf[i] = *(const f32x4 *)(qp + i * 4);
  TreeAsked asked{};
  if constexpr (TREES) asked = tree_ask(trees, sh, b, n1);
  const int front = TREES ? __builtin_amdgcn_readfirstlane(max(asked.slots, 0)) : sessions[b].slots;
  const int prefix = TREES ? __builtin_amdgcn_readfirstlane(max(asked.prefix, 0)) : front > 0 ? sh.of[b] : 0;
  const int start = (front + 63) & ~63;   // own slots begin here
  const float *rec = blocks + ((size_t)prefix * Hkv + g) * (sh.cap >> 6) * REC;
  const float *kb = ck + ((size_t)b * Hkv + g) * capacity * HD;
  const float *vb = cv + ((size_t)b * Hkv + g) * HD * capacity;   // [HD][capacity]
  const float scale = 1.0f / sqrtf((float)HD);
  if (tid == 0) s_bad = 0;
  f32x4 kx[NK], vx[ND];
  auto load = [&](int c) {   // (a record's or the capacity's 64 slots hold all of a block)
    const int slot = c * 16, in = slot & 63;
    const float *rp = rec + (size_t)(slot >> 6) * REC;
    const float *kp = slot < start ? rp + in * HD : kb + (size_t)(slot - start) * HD;
    const float *vp = slot < start ? rp + REC / 2 + in : vb + slot - start;
    const int stride = slot < start ? 64 : capacity;
#pragma unroll
    for (int i = 0; i < NK; ++i) kx[i] = *(const f32x4 *)(kp + lx * HD + ly * (HD / 4) + i * 4);
#pragma unroll
    for (int d = 0; d < ND; ++d) vx[d] = *(const f32x4 *)(vp + (size_t)(d * 16 + lx) * stride + ly * 4);
  };
  float m = -INFINITY, l = 0.f;
  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (wave * 16 < start + capacity) load(wave);
  int S;
  if constexpr (TREES)
    S = tree_session(sets[0], trees, asked, b, n1, capacity, tile == 0 && g == 0, TreeMeta{}).S;
  else
    S = meta.sess_S[b];
  __syncthreads();   // (s_bad is clear)
  const uint64_t *ancs = TREES ? sets[0].anc : meta.anc + (size_t)b * n1;
  const uint64_t anc = ancs[r];
  const int total = start + S + n1, nblk = (total + 15) >> 4;
  for (int c = wave; c < nblk; c += NW) {
    const int slot0 = c * 16 + ly * 4;   // of this lane's four
    f32x4 z = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[i][e], qf[i][e], z, 0, 0, 0);
    f32x4 v[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) v[d] = vx[d];
    if (c + NW < nblk) load(c + NW);
    z *= scale;
    if (c * 16 + 16 > front && (c * 16 < start || c * 16 + 16 > start + S)) {
      // the prefix's end, or the tree: hidden slots, and values there that are no numbers
      // (bitwise, so that these are selects)
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int slot = slot0 + e, j = slot - start - S, sh = min(max(j - 1, 0), 63);
        const bool front_part = slot < start;
        const bool there = slot < (front_part ? front : total);
        const bool seen = there & (front_part | (j <= 0) | (bool)((anc >> sh) & 1ull));
        const bool tree = !front_part & (j >= 0) & there;
        z[e] = seen ? z[e] : -INFINITY;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const bool number = fabsf(v[d][e]) <= 3.402823466e38f;
          odd |= tree & !number;
          v[d][e] = there & (number | !tree) ? v[d][e] : 0.f;
        }
      }
      if (__ballot(odd)) s_bad = 1;
    }
    const float mn = fmaxf(m, rows4_max(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))));
    const float mu = mn == -INFINITY ? 0.f : mn, alpha = expf(m - mu);
    m = mn;
    f32x4 p;
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = expf(z[e] - mu);
    l = l * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
    if (__ballot(alpha < 1.f)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int d = 0; d < ND; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[d][e], p[e], o[d], 0, 0, 0);
  }
  // o[d][e] is head dim 16 d + 4 ly + e of query lx: the waves' parts join in LDS
  l = rows4_sum(l);
#pragma unroll
  for (int d = 0; d < ND; ++d) *(f32x4 *)(&so[wave][lx][d * 16 + ly * 4]) = o[d];
  if (ly == 0) {
    sml[wave][lx][0] = m;
    sml[wave][lx][1] = l;
  }
  __syncthreads();
  for (int e = tid; e < 16 * HD / 4; e += 512) {
    const int x = e / (HD / 4), d = e % (HD / 4) * 4, qx = tile * 16 + x;
    if (qx >= QR) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sml[w][x][0]);
    if (M == -INFINITY) M = 0.f;
    f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float y = expf(sml[w][x][0] - M);
      den += y * sml[w][x][1];
      sum += y * *(const f32x4 *)(&so[w][x][d]);
    }
    const int rx = qx / G, h = g * G + qx - rx * G, row = b * n1 + rx;
    if (s_bad) {   // an infinity or a NaN comes of such a value in the rows that see it
      const uint64_t ax = ancs[rx];
      for (int t = 0; t < n1; ++t) {
        if (t > 0 && !((ax >> (t - 1)) & 1ull)) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = vb[(size_t)(d + i) * capacity + S + t];
          if (!(fabsf(v) <= 3.402823466e38f)) sum[i] += v;
        }
      }
    }
    *(f32x4 *)(out + (size_t)row * H * HD + h * HD + d) = sum / den;
  }
}

template <int HD, typename TQ>
hipError_t launch_hd(const TQ *q, const f16 *blocks, const SharedArgs &sh, const SharedMeta &sm,
                     const TreeArgs &trees, const bf16 *ck, const bf16 *cv, const TreeMeta &meta, void *out, int rows_out,
                     float *sh_o, float *sh_ml, float *part_o, float *part_ml, long long part_cap,
                     int B, int n1, int H, int Hkv, int capacity, int cus, hipStream_t s) {
  const int rows = B * n1, wgs = acespec::shared_wgs(Hkv, cus);
  // Few tiles are cut into many parts, which a kernel of its own joins faster, with a thread or more
  // for four head dims, than the waves over the own slots do (64 single tokens, one tile in 32 parts:
  // 27 + 9 us against 88; the 8B batch, 17 tiles in up to three: 45 + 18 against 49).
  const int here = 3LL * rows * (H / Hkv) >= (long long)wgs * TM;
  // Small batches over short prefixes: the kernel over the own slots takes the records first, each
  // session for itself, which leaves the tiles' way in and out of memory, and a launch, away.  It is
  // taken up to 18 chunks in turn of head dim 128 or 36 of 64, single tokens up to 16 or 32, as they
  // leave the tiles little to do.  Both sides in us (so taken, by tiles), 64 own slots, captured:
  //   17 rows, 4 heads a kv head, head dim 128: 8 sessions behind 2048 slots (9 chunks) 28.5, 44.9;
  //   8 behind 8192 (17) 48.3, 52.8; 64 behind 1024 (18) 47.6, 59.1; 32 behind 2048 (34) 59.3, 59.8;
  //   16 behind 8192 (33) 76.0, 69.5; of 64: 16 behind 8192 (33) 50.8, 56.4; 64 behind 2048 (34) 47.8,
  //   51.7; 64 behind 4096 (66) 80.1, 70.9.
  //   Single tokens, 128: 8 behind 4096 (9) 26.9, 28.2; 8 behind 8192 (17) 40.8, 28.0; of 64: 64 behind
  //   1024 (18) 24.0, 26.2, but 16 behind 4096 (17) 24.8, 22.1; 32 behind 2048 (34) 27.7, 22.5.
  //   More than 8 tiles, one workgroup a CU, 8 heads a kv head, 128: 17 rows, 16 behind 2048 (17)
  //   48.6, 58.9; 64 behind 512 (20) 55.9, 73.7; 32 behind 2048 (34) 61.7, 74.2; 33 rows, 8 behind 4096
  //   (17) 66.1, 81.0; 16 behind 4096 (33) 107, 113; 64 behind 1024 (36) 121, 143; of 64: 17 rows, 32
  //   behind 2048 (34) 52.0, 50.7; 16 behind 8192 (65) 96.0, 76.3.
  // (With more than 8 tiles of head dim 128 sessions could go further for themselves, with single
  // tokens of 64 less far; of the sizes measured none loses more than a third of the other way's time by it.)
  const int chunks = acespec::attention_chunks_in_turn(B, n1, H, Hkv, HD, (sh.cap + capacity) / 64, cus, part_cap);
  const bool direct = (long long)chunks * HD <= (H / Hkv * n1 <= 16 ? 16 : 18) * 128;
  const SharedJoin j{sh_o, sh_ml, sm, wgs,
                     acespec::shared_part_rows((long long)rows * (H / Hkv), Hkv, cus), out, rows_out,
                     direct || here, direct ? blocks : nullptr, sh, trees};
  hipError_t e = hipSuccess;
  if (trees.parents && !direct) {
    e = acespec::launch_tree_prep_shared(nullptr, trees.parents, trees.prefix_len, B, n1, 1, capacity, sh,
                                         H / Hkv, TM, meta, sm, trees.status, s);
    if (e != hipSuccess) return e;
  }
  if (!direct) {
    hipLaunchKernelGGL((shared_attn_kernel<HD, TQ>), dim3(wgs * Hkv), dim3(512), 0, s, q, blocks, sm,
                       sh_o, sh_ml, B, n1, H, Hkv, sh.cap, wgs, j.rows_total);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  int nsplit = 1;
  e = acespec::launch_attention_own(q, ck, cv, meta, j, part_o, part_ml, part_cap, B, n1, H, Hkv, HD,
                                    capacity, cus, s, &nsplit);
  if (e != hipSuccess || (j.here && nsplit == 1)) return e;
  const long long threads = (long long)rows * H * (HD / 4);
  const bool few = threads <= 256LL * cus;
  const long long wg = (threads * (few ? 4 : 1) + 255) / 256;
  if (wg > 0xffffffffLL / 256) return hipErrorInvalidValue;
  auto kernel = few ? shared_combine_kernel<HD, 4> : shared_combine_kernel<HD, 1>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wg), dim3(256), 0, s, part_o, part_ml, j, meta, cv, capacity, rows, n1,
                     H, Hkv, nsplit);
  return hipGetLastError();
}

}  // namespace

namespace acespec {

template <>
hipError_t launch_attention_shared<bf16>(const void *q, const f16 *blocks, const SharedArgs &sh,
                                         const SharedMeta &sm, const TreeArgs &trees, const bf16 *ck,
                                         const bf16 *cv, const TreeMeta &meta, void *out, int rows_io, float *sh_o,
                                         float *sh_ml, float *part_o, float *part_ml,
                                         long long part_capacity, int B, int n1, int H, int Hkv,
                                         int hd, int capacity, int cus, hipStream_t s) {
  auto run = [&](auto launch, auto *queries) {
    return launch(queries, blocks, sh, sm, trees, ck, cv, meta, out, rows_io, sh_o, sh_ml, part_o, part_ml,
                  part_capacity, B, n1, H, Hkv, capacity, cus, s);
  };
  if (rows_io)
    return hd == 128 ? run(launch_hd<128, bf16>, (const bf16 *)q) : run(launch_hd<64, bf16>, (const bf16 *)q);
  return hd == 128 ? run(launch_hd<128, f16>, (const f16 *)q) : run(launch_hd<64, f16>, (const f16 *)q);
}

template <>
hipError_t launch_attention_shared<float>(const void *q, const float *blocks, const SharedArgs &sh,
                                          const SharedMeta &sm, const TreeArgs &trees, const float *ck,
                                          const float *cv,
                                          const TreeMeta &meta, void *out, int, float *, float *,
                                          float *, float *, long long, int B, int n1, int H,
                                          int Hkv, int hd, int capacity, int, hipStream_t s) {
  if (Hkv > 65535 || B > 65535) return hipErrorInvalidValue;
  auto kernel = trees.parents ? (hd == 64 ? shared_attn_f32_kernel<64, true> : shared_attn_f32_kernel<128, true>)
                              : (hd == 64 ? shared_attn_f32_kernel<64, false> : shared_attn_f32_kernel<128, false>);
  hipLaunchKernelGGL(kernel, dim3((H / Hkv * n1 + 15) / 16, Hkv, B), dim3(512), 0, s, (const float *)q, blocks, sh,
                     sm.sessions, ck, cv, meta, trees, (float *)out, n1, H, Hkv, capacity);
  return hipGetLastError();
}

}  // namespace acespec
