// Tree-masked grouped-query attention over the 4-bit KV cache (quant.h), with an optional
// sliding window whose first tokens stay visible.
//
// Row r of a session of P slots sits at position P + depth(r).  It sees the P slots and, of the
// tree, its ancestors and itself; with a window w > 0 only what is at a position less than w
// behind its own, or below `sinks`.  Of the P slots the complete blocks of 32 are records, the
// rest and the tree's rows the tail in the model's type; both go through the same code as blocks
// of 32 slots.
//
// Query rows are the G query heads of the kv head times the tree rows (row = tree_row * G +
// head) in tiles of 16.  The work is divided by slots, not by queries: a wave holds all TPW
// tiles of its workgroup (as accumulators) and takes blocks of its own, so a block's codes are
// read once, by one wave, straight into the registers that the matrix instructions read, and
// are decoded once for all the tiles.  No barrier and no LDS traffic but the queries' fragments.
//  * S^T = K Q^T by 16x16 products: a lane holds 8 scores of ONE query, for 8 consecutive
//    slots.  Its running reference, exp2 and the probabilities stay in the lane, and these are
//    its B operand of O^T = V^T P^T.  Head dims are dealt to the products so that a lane's codes
//    of a key are consecutive (head dims lg * hd/4 ..), the queries' fragments alike.
//  * A decoded element is e2m1 times a power of two: exact in fp16.  The bf16 model multiplies
//    in fp16 (v_mfma_f32_16x16x32_f16), the fp32 model in fp32 (v_mfma_f32_16x16x4_f32).
//  * The reference of a query's exponents moves only when a score exceeds it by more than
//    2^8 (LAZY_LOG2): a lane compares its own scores, and only then are the four lanes of a query
//    reduced and the accumulators rescaled.
// At the end the waves of a workgroup, and then the splits of a session, are joined by their
// (maximum, sum) pairs.
//
// Not finite: a group of 32 marked so reads as NaN.  NaN and inf reach the rows that see them
// and no others: where a mask applies, slots with such values are taken one at a time.
#include "quant.h"

namespace {

constexpr float LAZY_LOG2 = 8.f;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int NW = 4;   // waves of a workgroup

// The operand arithmetic of a model's type: eight elements of a lane.
template <typename T> struct Ops;
template <> struct Ops<bf16> {
  typedef f16x8 F8;
  typedef f16 E;
  static AS_DEVICE F8 decode(uint32_t c, float s) { return q4_decode_f16(c, s); }
  static AS_DEVICE F8 load(const bf16 *p) { return bf16x8_to_f16x8(*(const bf16x8 *)p); }
  static AS_DEVICE f32x4 mma(F8 a, F8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Ops<float> {
  typedef f32x8 F8;
  typedef float E;
  static AS_DEVICE F8 decode(uint32_t c, float s) { return q4_decode_f32(c, s); }
  static AS_DEVICE F8 load(const float *p) {
    const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
    return F8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static AS_DEVICE f32x4 mma(F8 a, F8 b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

struct QuantAttnArgs {
  const void *q;            // [rows][H hd]: T (rows_io) or the activation type
  const uint8_t *blocks;    // records of the layer
  const void *tk, *tv;      // tail of the layer
  const int32_t *pos;       // [rows] P + depth
  const uint64_t *anc;      // [rows] visible drafted rows (bit j - 1)
  void *out;
  float *part_o, *part_ml;
  int B, n1, H, Hkv, nblk, tcap, nsplit, nqg, window, sinks;
  int rows_io;              // 1: q and out are row-major in T; 0: q row-major and out in the
                            // activation layout, fp16 (bf16 model; fp32: the same as 1)
};

// What a query row sees.
struct RowView {
  int lo;         // slots of the prefix from here on, and below `sinks`
  int root;       // whether it sees the root
  uint64_t anc;   // drafted rows
};

// Eight consecutive elements of a query row, and four of an output row.
AS_DEVICE f16x8 load_q(const QuantAttnArgs &a, bf16, size_t off) {
  if (a.rows_io) return bf16x8_to_f16x8(*(const bf16x8 *)((const bf16 *)a.q + off));
  return *(const f16x8 *)((const f16 *)a.q + off);
}
AS_DEVICE f32x8 load_q(const QuantAttnArgs &a, float, size_t off) {
  return Ops<float>::load((const float *)a.q + off);
}
AS_DEVICE void store_out(const QuantAttnArgs &a, bf16, int row, int col, int width, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  if (a.rows_io)
    *(bf16x4 *)((bf16 *)a.out + (size_t)row * width + col) =
        bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  else
    *(f16x4 *)((f16 *)a.out + act_off(row, col, a.B * a.n1, width)) =
        f16x4{(f16)v[0], (f16)v[1], (f16)v[2], (f16)v[3]};
}
AS_DEVICE void store_out(const QuantAttnArgs &a, float, int row, int col, int width, f32x4 v) {
  *(f32x4 *)((float *)a.out + (size_t)row * width + col) = v;
}

AS_DEVICE bool not_finite(f16 v) { return (__builtin_bit_cast(uint16_t, v) & 0x7c00) == 0x7c00; }
AS_DEVICE bool not_finite(float v) { return abs_bits(v) >= 0x7f800000u; }

template <typename T, int HD, int TPW, int WPS>
__global__ __launch_bounds__(NW * 64, WPS) void quant_attn_kernel(QuantAttnArgs a) {
  typedef Ops<T> O;
  typedef typename O::F8 F8;
  constexpr int KS = HD / 32, NB = HD / 16, LD = HD / 4;
  __shared__ __attribute__((aligned(16))) typename O::E qs[TPW * 16 * HD];  // [tile][s][lane][8]
  __shared__ RowView view[TPW * 16];
  __shared__ f32x4 mo[NW * NB * 64];
  __shared__ float2 ml[NW][TPW * 16];

  // The query groups and the splits of a session's kv head follow each other on one XCD: the
  // groups read the same records.
  const int id = xcd_tile(blockIdx.x, gridDim.x);
  const int grp = id % a.nqg, split = id / a.nqg % a.nsplit, item = id / (a.nqg * a.nsplit);
  const int b = item / a.Hkv, g = item - b * a.Hkv;
  const int G = a.H / a.Hkv, QR = G * a.n1, qbase = grp * TPW * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const int row0 = b * a.n1, width = a.H * HD;
  const int P = a.pos[row0], t = P & (Q4_SLOTS - 1), full = P / Q4_SLOTS;
  // Blocks that some row sees: [0, nsink) and [wlo, full), then the tail's.
  int nsink = 0, wlo = 0;
  if (a.window) {
    const int lo = max(P - a.window + 1, 0);           // the root's window, the furthest back
    wlo = min(lo / Q4_SLOTS, full);
    nsink = min((int)(((unsigned)a.sinks + Q4_SLOTS - 1) / Q4_SLOTS), wlo);
  }
  const int nq = nsink + full - wlo, total = nq + (t + a.n1 + Q4_SLOTS - 1) / Q4_SLOTS;
  const int per = (total + a.nsplit - 1) / a.nsplit;
  const int c0 = min(split * per, total), c1 = min(c0 + per, total);

  for (int e = tid; e < TPW * 16 * (HD / 8); e += NW * 64) {
    const int qi = e / (HD / 8), c = e % (HD / 8);     // query of the group, piece of 8 head dims
    const int s = c % KS, l = c / KS * 16 + (qi & 15);
    F8 v{};
    if (qbase + qi < QR) {
      const int r = (qbase + qi) / G, h = g * G + (qbase + qi - r * G);
      v = load_q(a, T(), (size_t)(row0 + r) * width + h * HD + c * 8);
    }
    *(F8 *)(qs + (((qi >> 4) * KS + s) * 64 + l) * 8) = v;
  }
  for (int e = tid; e < TPW * 16; e += NW * 64) {
    const int r = min(qbase + e, QR - 1) / G, p = a.pos[row0 + r];
    view[e].lo = a.window ? p - a.window + 1 : -1;
    view[e].root = !a.window || p - P < a.window || P < a.sinks;
    view[e].anc = a.anc[row0 + r];
  }
  __syncthreads();

  const float sscale = LOG2E / sqrtf((float)HD), lazy = LAZY_LOG2 / sscale;
  float m_run[TPW], l_run[TPW];
  f32x4 o[TPW][NB];
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[i][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // The scores of tile i against a block's keys and their step of the online softmax; `vis`
  // has a bit for each of the lane's 8 slots.
  auto soft = [&](int i, const F8 (&kf)[2][KS], uint32_t vis, bool masked) -> F8 {
    f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const F8 qf = *(const F8 *)(qs + ((i * KS + s) * 64 + lane) * 8);
      sc[0] = O::mma(kf[0][s], qf, sc[0]);
      sc[1] = O::mma(kf[1][s], qf, sc[1]);
    }
    if (masked) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!((vis >> j) & 1u)) sc[j >> 2][j & 3] = -INFINITY;
    }
    float mx = sc[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j >> 2][j & 3]);
    if (__ballot(mx > m_run[i] + lazy)) {
      mx = rows4_max(mx);
      const float mn = mx > m_run[i] + lazy ? mx : m_run[i];
      const float alpha = __builtin_amdgcn_exp2f((m_run[i] - (mn == -INFINITY ? 0.f : mn)) * sscale);
      m_run[i] = mn;
      l_run[i] *= alpha;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][nb][e] *= alpha;
    }
    const float mb = m_run[i] == -INFINITY ? 0.f : m_run[i] * sscale;
    F8 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = __builtin_amdgcn_exp2f(fmaf(sc[j >> 2][j & 3], sscale, -mb));
      l_run[i] += v;
      p[j] = (typename O::E)v;
    }
    return p;
  };
  // O^T += V^T P^T for head dims 16 nb .. where rows do not all see the same slots: slots whose
  // value is not finite go one at a time, to the rows that see them (0 * NaN is NaN).
  auto weigh = [&](int nb, F8 vf, const F8 (&p)[TPW], const uint32_t (&vis)[TPW]) {
    uint32_t bad = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) bad |= (uint32_t)not_finite(vf[j]) << j;
    if (__ballot(bad != 0)) {
      for (int js = 0; js < Q4_SLOTS; ++js) {
        const bool mine = lg == js >> 3;
        const int je = js & 7;
        if (!__ballot(mine && ((bad >> je) & 1u))) continue;
        F8 v1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v1[j] = mine && j == je ? vf[j] : (typename O::E)0.f;
          vf[j] = mine && j == je ? (typename O::E)0.f : vf[j];
        }
#pragma unroll
        for (int i = 0; i < TPW; ++i) {
          F8 p1;
#pragma unroll
          for (int j = 0; j < 8; ++j) p1[j] = mine && j == je ? p[i][j] : (typename O::E)0.f;
          const bool sees = ((uint32_t)__shfl((int)vis[i], (js >> 3) * 16 + lr) >> je) & 1u;
          const f32x4 n = O::mma(v1, p1, o[i][nb]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][nb][e] = sees ? n[e] : o[i][nb][e];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TPW; ++i) o[i][nb] = O::mma(vf, p[i], o[i][nb]);
  };

  const uint8_t *rec0 = a.blocks + (size_t)item * a.nblk * q4_bytes(HD);
  const T *tk = (const T *)a.tk + (size_t)item * a.tcap * HD;
  const T *tv = (const T *)a.tv + (size_t)item * HD * a.tcap;
  auto block_of = [&](int c) { return c < nsink ? c : wlo + c - nsink; };
  Q4Regs<HD> cur, nxt;
  if (c0 + wave < min(c1, nq)) q4_load<HD>(cur, rec0 + (size_t)block_of(c0 + wave) * q4_bytes(HD), lane);
  for (int c = c0 + wave; c < c1; c += NW) {
    if (c + NW < min(c1, nq)) q4_load<HD>(nxt, rec0 + (size_t)block_of(c + NW) * q4_bytes(HD), lane);
    const int slot0 = block_of(c) * Q4_SLOTS;
    F8 kf[2][KS], p[TPW];
    // Every row sees the whole block unless a window ends in it.
    if (c < nq && (a.window == 0 || slot0 + Q4_SLOTS <= a.sinks || slot0 >= P + a.n1 - a.window)) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int s = 0; s < KS; ++s)
          kf[kk][s] = O::decode(q4_kword<HD>(cur, kk, s), q4_kscale<HD>(cur, kk));
#pragma unroll
      for (int i = 0; i < TPW; ++i) p[i] = soft(i, kf, 0, false);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const F8 vf = O::decode(q4_vword<HD>(cur, nb), q4_vscale<HD>(cur, nb));
#pragma unroll
        for (int i = 0; i < TPW; ++i) o[i][nb] = O::mma(vf, p[i], o[i][nb]);
      }
    } else {
      // A block that a window cuts, or one of the tail: slots of the last, incomplete block,
      // then the tree's rows.
      const bool tail = c >= nq;
      const int s0 = tail ? (c - nq) * Q4_SLOTS : 0;       // first slot within the tail
      const int tr0 = tail ? s0 - t + lg * 8 : -Q4_SLOTS;  // tree row of the lane's first slot
      const int pos0 = (tail ? full * Q4_SLOTS + s0 : slot0) + lg * 8;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int s = 0; s < KS; ++s)
          kf[kk][s] = tail ? O::load(tk + (size_t)(s0 + q4_key(kk, lr)) * HD + lg * LD + s * 8)
                           : O::decode(q4_kword<HD>(cur, kk, s), q4_kscale<HD>(cur, kk));
      uint32_t vis[TPW];
#pragma unroll
      for (int i = 0; i < TPW; ++i) {
        const RowView w = view[i * 16 + lr];
        vis[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int tr = tr0 + j, slot = pos0 + j;
          const bool see = tr < 0 ? slot < a.sinks || slot >= w.lo
                                  : tr == 0 ? w.root != 0 : tr < a.n1 && ((w.anc >> (tr - 1)) & 1ull);
          vis[i] |= (uint32_t)see << j;
        }
        p[i] = soft(i, kf, vis[i], true);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        F8 vf;
        if (tail) {
          vf = O::load(tv + (size_t)(nb * 16 + lr) * a.tcap + s0 + lg * 8);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (tr0 + j >= a.n1) vf[j] = (typename O::E)0.f;   // never written
        } else {
          vf = O::decode(q4_vword<HD>(cur, nb), q4_vscale<HD>(cur, nb));
        }
        weigh(nb, vf, p, vis);
      }
    }
    cur = nxt;
  }

  // Join the waves: o[i][nb][e] is head dim 16 nb + 4 lg + e of query 16 i + lr.
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    const float l = rows4_sum(l_run[i]);
    if (lg == 0)
      ml[wave][i * 16 + lr] = make_float2(m_run[i] == -INFINITY ? -INFINITY : m_run[i] * sscale, l);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TPW; ++i) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[w][i * 16 + lr].x);
    float f = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 e = ml[w][i * 16 + lr];
      const float fw = e.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(e.x - M);
      L += fw * e.y;
      f = w == wave ? fw : f;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      f32x4 v = o[i][nb];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= f;
      mo[(wave * NB + nb) * 64 + lane] = v;
    }
    __syncthreads();
    const int qi = qbase + i * 16 + lr;
    if (qi < QR) {
      const int r = qi / G, h = g * G + (qi - r * G);
#pragma unroll
      for (int x = 0; x < NB / NW; ++x) {
        const int nb = wave * (NB / NW) + x;
        f32x4 acc = mo[nb * 64 + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
          const f32x4 v = mo[(w * NB + nb) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += v[e];
        }
        if (a.nsplit == 1) {
          const float inv = 1.f / L;                   // every row sees itself
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] *= inv;
          store_out(a, T(), row0 + r, h * HD + nb * 16 + lg * 4, width, acc);
        } else {
          const size_t q = ((size_t)item * a.nsplit + split) * QR + qi;
          *(f32x4 *)(a.part_o + q * HD + nb * 16 + lg * 4) = acc;
          if (nb == 0 && lg == 0) *(float2 *)(a.part_ml + q * 2) = make_float2(M, L);
        }
      }
    }
    if (i + 1 < TPW) __syncthreads();
  }
}

// Joins the splits: one thread per 4 head dims of a query row.
template <typename T>
__global__ __launch_bounds__(256) void quant_combine_kernel(QuantAttnArgs a, int HD) {
  const int item = blockIdx.y, b = item / a.Hkv, g = item - b * a.Hkv;
  const int G = a.H / a.Hkv, QR = G * a.n1, hd4 = HD >> 2;
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
  const int r = qi / G, h = g * G + (qi - r * G);
  store_out(a, T(), b * a.n1 + r, h * HD + d, a.H * HD, num);
}

template <typename T, int HD>
void launch_tiles(int tpw, unsigned grid, hipStream_t s, const QuantAttnArgs &a) {
  auto kernel = tpw == 1 ? quant_attn_kernel<T, HD, 1, 2> : quant_attn_kernel<T, HD, 2, 2>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(NW * 64), 0, s, a);
}

}  // namespace

namespace acespec {

template <typename T>
hipError_t launch_attention_quant(const void *q, const uint8_t *blocks, const T *tk, const T *tv,
                                  const TreeMeta &meta, void *out, float *part_o, float *part_ml,
                                  long long part_capacity, int B, int n1, int H, int Hkv, int hd,
                                  int capacity, int tcap, int window, int sinks, int rows_io,
                                  int cus, hipStream_t s) {
  constexpr int MAXT = 2;
  const int QR = H / Hkv * n1, tiles = (QR + 15) / 16;
  const int tpw = (tiles + (tiles + MAXT - 1) / MAXT - 1) / ((tiles + MAXT - 1) / MAXT);
  const int nqg = (tiles + tpw - 1) / tpw, items = B * Hkv;
  // Splits: two workgroups a CU, and at least two blocks a wave.
  const long long seen = window ? (long long)window + n1 + sinks + 2 * Q4_SLOTS : capacity;
  const int blocks_seen = (int)((seen < capacity ? seen : capacity) / Q4_SLOTS) + 3;
  int nsplit = 2 * cus / (items * nqg);
  nsplit = nsplit < blocks_seen / (2 * NW) ? nsplit : blocks_seen / (2 * NW);
  if (nsplit < 1) nsplit = 1;
  while (nsplit > 1 && (long long)items * nsplit * QR * hd > part_capacity) --nsplit;
  const QuantAttnArgs a{q, blocks, tk, tv, meta.pos, meta.anc, out, part_o, part_ml, B, n1, H, Hkv,
                        capacity / Q4_SLOTS, tcap, nsplit, nqg, window, sinks, rows_io};
  const unsigned grid = (unsigned)(items * nqg * nsplit);
  if (hd == 128) launch_tiles<T, 128>(tpw, grid, s, a);
  else launch_tiles<T, 64>(tpw, grid, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nsplit == 1) return e;
  hipLaunchKernelGGL(quant_combine_kernel<T>, dim3((QR * (hd / 4) + 255) / 256, items), dim3(256), 0,
                     s, a, hd);
  return hipGetLastError();
}

template hipError_t launch_attention_quant<float>(const void *, const uint8_t *, const float *,
                                                  const float *, const TreeMeta &, void *, float *,
                                                  float *, long long, int, int, int, int, int, int,
                                                  int, int, int, int, int, hipStream_t);
template hipError_t launch_attention_quant<bf16>(const void *, const uint8_t *, const bf16 *,
                                                 const bf16 *, const TreeMeta &, void *, float *,
                                                 float *, long long, int, int, int, int, int, int,
                                                 int, int, int, int, int, hipStream_t);

}  // namespace acespec
