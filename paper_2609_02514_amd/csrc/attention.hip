// Tree-masked grouped-query attention of the verify pass.
//
// Every drafted node of a session is verified in one forward pass (Section III-C): a
// node attends to the whole verified context (the KV prefix) and, among the tree's own
// slots, only to its ancestors and itself; the root is every node's ancestor.  Keys and
// values of tree row j sit in cache slot prefix_len + j, so one contiguous key range
// [0, prefix_len + N + 1) covers everything and the mask applies to its tail only.
//
// bf16 model.  One workgroup of 16 waves (8 with more than 16 tiles) per (key split, kv
// head, session).  Query rows are the G query heads of the kv head times the N+1 tree rows
// (row = tree_row * G + head), in tiles of 16 rows, one a wave (more than 16 tiles: the
// 32-row kernel below).  The key range of the split streams through LDS in chunks of 64 slots:
//  * HBM -> LDS by direct DMA (buffer loads to LDS, 16 bytes a lane, nontemporal: the
//    cache is read once per step, and streaming it past L2 and the MALL measured 15 %
//    faster at the 8B shape) into a ring of NST stages.  The buffer form rather than the
//    global one: the compiler counts it on vmcnt alone, so its waits for the fragment
//    reads stay exact (1-3 % faster).  A stage holds the chunk's keys as [64 slots][head_dim] and its values,
//    read from the head-dim-major value cache, as [head_dim][64 slots].  The 16-byte
//    pieces of every row are XOR-swizzled so that the fragment reads below hit distinct
//    banks; the DMA fixes where each lane's bytes land, so the swizzle is applied to the
//    global source addresses.
//  * One chunk ahead of its use, the stage is widened from bf16 to fp16 in place (exact
//    in the fp16 normal range), so the MFMAs run on fp16 operands like the rest of the
//    pass, and the value columns past the last tree slot are zeroed (their probability
//    is 0, but 0 * NaN would not be).  Waves without a query tile do the widening when
//    there are any, which keeps it off the SIMD that holds two tile waves.
//  * Scores are computed transposed, S^T = K Q^T with v_mfma_f32_16x16x32_f16 (16 keys
//    as rows, 16 queries as columns), so each lane holds 16 scores of ONE query.  The
//    tree mask, the running max (reduced over the query's 4 lanes by two row swaps) and
//    exp2 stay in the lane, and the lane's probabilities, rounded to fp16, are exactly
//    its B operand of O^T = V^T P^T (the keys are assigned to MFMA rows so that a lane's
//    8 probabilities are 8 consecutive keys, whose V^T fragment is one 16-byte read).  The O^T
//    accumulator lane holds 4 head dims of its query, so the online-softmax rescale is
//    lane-local (and skipped when no running max moved).
//  * Barrier protocol at chunk c: a wave waits for its own DMA of chunk c+1; one LDS
//    barrier then certifies that chunk c+1 landed for every wave, that every wave
//    widened its share of chunk c, and that chunk c-1 is consumed, so its stage takes the
//    DMA of chunk c+NST-1.  NST-2 chunks are in flight while chunk c is computed.
//  With several splits, unnormalised partial outputs and (max, sum) pairs are merged by
//  a small combine kernel.
//
// Behind shared prefixes (attention_shared.hip) the same kernels go over the sessions' own slots and
// join the prefix's partial results (MODE 1), or over the prefix's records and then the own slots
// (MODE 2: records come in the order of 32 x 32 operands and in fp16, so the DMA's source addresses
// undo that order, and nothing of them is widened).  Up to 8 tiles they take 8 waves and two stages, two
// workgroups a CU: 64 sessions of 17 rows over up to 512 own slots 47 us, 20 of it their stream at
// 5 TB/s, 7 the prefix's parts; 64 single tokens 27.
//
// fp32 kernel (small models): one workgroup per (tree row, query head).
#include <algorithm>

#include "shared.h"

namespace {

constexpr int KC = 64;            // slots per chunk
// Online softmax with a lazy reference: the exponent's reference m moves to a new block
// maximum only when that maximum exceeds m by more than LAZY_LOG2 in base 2 (or m is
// unset), so the accumulators are rescaled a few times per query instead of at most
// blocks; the probabilities stay below 2^LAZY_LOG2, far inside fp16, and o / l is
// unchanged because numerator and denominator share the reference.
constexpr float LAZY_LOG2 = 8.f;
AS_DEVICE float lazy_ref(float m, float mx, float lazy) { return mx > m + lazy ? mx : m; }


AS_DEVICE bool tree_visible(int slot, int S, int n1, uint64_t anc) {
  if (slot < S) return true;
  const int j = slot - S;
  if (j >= n1) return false;
  return j == 0 || ((anc >> (j - 1)) & 1ull);
}

// Order of the keys inside each 32-key group of a chunk: A row m of key block kk (16
// rows) holds key (kk/2)*32 + (m/4)*8 + (kk%2)*4 + m%4.  The score block's output row
// lg*4 + e is then key (kk/2)*32 + lg*8 + (kk%2)*4 + e, so the lane with row group lg
// holds the 8 consecutive keys (kk/2)*32 + lg*8 .. + 7 of its query -- one contiguous
// 16-byte read of a V^T row gives its A operand of O^T = V^T P^T.
AS_DEVICE int key_of_row(int kk, int m) { return (kk >> 1) * 32 + (m >> 2) * 8 + (kk & 1) * 4 + (m & 3); }
AS_DEVICE int key_of_score(int kk, int lg, int e) { return (kk >> 1) * 32 + lg * 8 + (kk & 1) * 4 + e; }

// XOR swizzles of the 16-byte pieces of a row, chosen so that each fragment read -- 16
// lanes at one logical piece of 16 rows (keys m = 0..15 of a block above, or 16
// consecutive V^T rows) -- runs at the LDS's full rate; measured on gfx950 with the
// kernel's own lane patterns (256-byte K rows: about 200 B/clk/CU with this key swizzle;
// 128-byte V^T rows: 210 B/clk/CU with row / 2, where row ^ (row / 8) halved it).
// K rows are 2*HD bytes.
template <int HD> AS_DEVICE int ksw(int key) {
  if (HD == 128) return (((key >> 3) & 3) << 2) | (key & 3);
  return ((key & 1) ^ ((key >> 4) & 1)) | (((key >> 1) & 1) << 1) | (((key >> 3) & 1) << 2);
}
AS_DEVICE int vsw(int row) { return (row >> 1) & 7; }
// K swizzle of the 32-row-tile kernel: its 16-lane fragment groups read 16 consecutive
// keys (bits 0-3 vary) in the main tiles and keys with bits 0, 1, 3, 4 varying in the
// remainder tile's quarter units; the XOR value below takes 16 (head_dim 128: 256-byte
// rows, one bank round each) or 2 x 8 (head_dim 64: rows alternate between the two
// halves of a bank round) distinct values on both sets.
template <int HD> AS_DEVICE int ksw32(int key) {
  const int b24 = ((key >> 2) ^ (key >> 4)) & 1;
  if (HD == 128) return (key & 0xB) | (b24 << 2);
  return ((key >> 1) & 1) | (b24 << 1) | (((key >> 3) & 1) << 2);
}
template <int HD, bool T32> AS_DEVICE int kswz(int key) {
  return T32 ? ksw32<HD>(key) : ksw<HD>(key);
}

// Element offset of piece `piece` of key row `key` in a stage's K part.
template <int HD> AS_DEVICE int k_off(int key, int piece) {
  return key * HD + ((piece ^ ksw<HD>(key)) << 3);
}
// Element offset of piece `piece` (8 slots) of head-dim row `row` in a stage's V^T part
// (rows of 64 slots = 128 bytes).
AS_DEVICE int v_off(int row, int piece) { return row * KC + ((piece ^ vsw(row)) << 3); }

// DMA of one chunk (keys key0 .. key0 + 63) into a stage: HD/8 blocks of 1 KB for K and
// as many for V^T, dealt to the NW waves in turn.
template <int HD, int NW, bool T32 = false>
AS_DEVICE void issue_chunk(uint16_t *stage, __amdgpu_buffer_rsrc_t kr,
                           __amdgpu_buffer_rsrc_t vr, int key0,
                           int capacity, int wave, int lane) {
  constexpr int BLOCKS = HD / 8;
  static_assert((2 * BLOCKS) % NW == 0, "DMA blocks per wave");
#pragma unroll
  for (int j = 0; j < 2 * BLOCKS / NW; ++j) {
    const int blk = wave + NW * j;
    if (blk < BLOCKS) {
      const int e = blk * 512 + lane * 8;          // element offset this lane's bytes land at
      const int key = e / HD, piece = (e % HD) >> 3;
      buf_dma16_stream(kr, (lds_ptr_t)(stage + blk * 512),
                       (uint32_t)((key0 + key) * HD + ((piece ^ kswz<HD, T32>(key)) << 3)) * 2u);
    } else {
      const int i = blk - BLOCKS;
      const int row = i * 8 + (lane >> 3), piece = lane & 7;
      buf_dma16_stream(vr, (lds_ptr_t)(stage + KC * HD + i * 512),
                       (uint32_t)(row * capacity + key0 + ((piece ^ vsw(row)) << 3)) * 2u);
    }
  }
}

// The same of a record of a shared prefix (fp16, pieces in the order of 32 x 32 operands) at byte
// `at` of its plane.
template <int HD, int NW, bool T32 = false>
AS_DEVICE void issue_record(uint16_t *stage, __amdgpu_buffer_rsrc_t rr, int at, int wave, int lane) {
  constexpr int BLOCKS = HD / 8;
#pragma unroll
  for (int j = 0; j < 2 * BLOCKS / NW; ++j) {
    const int blk = wave + NW * j;
    int from;   // the piece
    if (blk < BLOCKS) {
      const int e = blk * 512 + lane * 8, key = e / HD, d8 = ((e % HD) >> 3) ^ kswz<HD, T32>(key);
      const int row = (key & 16) + ((key >> 3) & 1) * 4 + ((key >> 2) & 1) * 8 + (key & 3);
      from = ((key >> 5) * (HD / 16) + (d8 >> 1)) * 64 + (d8 & 1) * 32 + row;
    } else {
      const int row = (blk - BLOCKS) * 8 + (lane >> 3), s8 = (lane & 7) ^ vsw(row);
      from = KC * HD / 8 + ((s8 >> 1) * (HD / 32) + (row >> 5)) * 64 + (s8 & 1) * 32 + (row & 31);
    }
    buf_dma16(rr, (lds_ptr_t)(stage + blk * 512), (uint32_t)from * 16, at);
  }
}

// Zeroes the values of a record's slots >= valid in a stage.
template <int HD>
AS_DEVICE void cut_record(uint16_t *stage, int t, int stride, int valid) {
  for (int vp = t; vp < KC * HD / 8; vp += stride) {
    uint16_t *p = stage + KC * HD + vp * 8;
    const int s0 = ((vp & 7) ^ vsw(vp >> 3)) << 3;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (s0 + e >= valid) p[e] = 0;
  }
}

// Tree rows whose values are not all finite: three words.
AS_DEVICE void mark_row(uint32_t *bad, int row) { atomicOr(bad + (row >> 5), 1u << (row & 31)); }

// bf16 -> fp16 in place for pieces t, t + stride, ... of a stage (t: the thread's index
// among the widening threads); value slots >= total are zeroed.
// PART: values that are not finite are zeroed in the tree's slots (>= S) too, and their rows
// marked in bad (in LDS); the join of the parts brings them to the rows that see them.
template <int HD, bool PART = false>
AS_DEVICE void widen_chunk(uint16_t *stage, int t, int stride, int key0, int total, int S = 0,
                           uint32_t *bad = nullptr) {
  constexpr int KPIECES = KC * HD / 8;
  const bool tail = key0 + KC > total;
  for (int pc = t; pc < 2 * KPIECES; pc += stride) {
    uint16_t *p = stage + pc * 8;
    f16x8 h = bf16x8_to_f16x8(*(const bf16x8 *)p);
    if (tail && pc >= KPIECES) {
      const int vp = pc - KPIECES, row = vp >> 3;
      const int s0 = key0 + (((vp & 7) ^ vsw(row)) << 3);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (s0 + e >= total) h[e] = (f16)0.f;
    }
    if (PART && key0 + KC > S && pc >= KPIECES) {
      const int vp = pc - KPIECES, row = vp >> 3;
      const int j0 = key0 + (((vp & 7) ^ vsw(row)) << 3) - S;   // the piece's first tree row
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (j0 + e >= 0 && !(fabsf((float)h[e]) <= 65504.f)) {
          h[e] = (f16)0.f;
          mark_row(bad, j0 + e);
        }
    }
    *(f16x8 *)p = h;
  }
}

template <int HD, int NW, int NST, int MODE = 0, typename TQ = f16>
__global__ __launch_bounds__(NW * 64, 4) void tree_attn_mfma_kernel(
    const TQ *__restrict__ qin, const bf16 *__restrict__ ck, const bf16 *__restrict__ cv,
    TreeMeta meta, f16 *__restrict__ out, float *__restrict__ part_o,
    float *__restrict__ part_ml, int n1, int H, int Hkv, int capacity, int nsplit, SharedJoin join) {
  // MODE 0: the verify pass; 1: own slots behind a shared prefix, joined with its partial results or
  // left as some; 2: its records first, then the own slots
  constexpr bool PART = MODE > 0, RECORDS = MODE == 2;
  constexpr bool TREES = RECORDS && std::is_same<TQ, bf16>::value;   // (a call of the attention alone)
  constexpr int KSTEPS = HD / 32, NB = HD / 16;
  constexpr int STAGE = 2 * KC * HD;     // elements: K [KC][HD], then V^T [HD][KC]
  constexpr int L_DMA = HD / 4 / NW;     // DMA instructions per wave per chunk
  // Two stages: a chunk is widened once it is there, between two barriers, with the next one in
  // flight; the shorter ring leaves room for a second workgroup on the CU, whose loads and products
  // fill these gaps.  Otherwise the widening runs one stage ahead of the MFMAs.
  constexpr bool SYNC = NST == 2;
  __shared__ __attribute__((aligned(1024))) uint16_t smem[NST * STAGE];

  const int g = blockIdx.y, b = blockIdx.z;
  const int G = H / Hkv, QR = G * n1, ntiles = (QR + 15) / 16, split = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lr = lane & 15, lg = lane >> 4;
  __shared__ uint32_t bad[PART ? 3 : 1];   // tree rows with values that are not finite
  if (PART && threadIdx.x < 3) bad[threadIdx.x] = 0;   // (before the prologue's barrier)
  SharedSession me{};          // (asked for here, well before the join needs it)
  int4 total_units{};
  if (PART && !TREES && (RECORDS || join.here)) {
    me = join.sm.sessions[b];
    total_units = *join.sm.total;
  }
  __shared__ TreeSets sets[1];
  TreeSession session{};
  if constexpr (TREES)
    session = tree_session(sets[0], join.trees, tree_ask(join.trees, join.sh, b, n1), b, n1, capacity, blockIdx.x == 0 && g == 0, meta);
  // chunks of the session's shared prefix, in front of its own, if they are taken here
  const int front = TREES ? session.front : RECORDS ? __builtin_amdgcn_readfirstlane(me.slots) : 0;
  const int fc = RECORDS ? (front + KC - 1) / KC : 0;
  const size_t plane = RECORDS && fc > 0 ? (size_t)join.sh.cap * 2 * HD : 0;
  const int prefix = TREES ? session.prefix : RECORDS && fc > 0 ? __builtin_amdgcn_readfirstlane(join.sh.of[b]) : 0;
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(join.blocks + ((size_t)prefix * Hkv + g) * plane,
                                              (uint32_t)(plane * 2));
  if (RECORDS) me.place = -1;   // nothing to join
  const int S = TREES ? session.S : meta.sess_S[b];
  const uint64_t *ancs = TREES ? sets[0].anc : meta.anc + (size_t)b * n1;
  const int total = S + n1;
  const int nchunks = fc + (total + KC - 1) / KC;
  const int cps = (nchunks + nsplit - 1) / nsplit;
  const int c0 = split * cps;
  const int c1 = min(nchunks, c0 + cps);
  const bf16 *kb = ck + ((size_t)b * Hkv + g) * capacity * HD;
  const bf16 *vb = cv + ((size_t)b * Hkv + g) * HD * capacity;
  const __amdgpu_buffer_rsrc_t kr = make_rsrc(kb, (uint32_t)((size_t)capacity * HD * 2));
  const __amdgpu_buffer_rsrc_t vr = make_rsrc(vb, (uint32_t)((size_t)capacity * HD * 2));
  const size_t row0 = (size_t)b * n1;
  const int q_stride = H * HD, rows_all = gridDim.z * n1;
  const float sscale = LOG2E / sqrtf((float)HD);   // scores -> base-2 exponent
  const float lazy = LAZY_LOG2 / sscale;           // reference threshold in score units

  // Query tile `wave`: query fragments (B operand of S^T = K Q^T), ancestor mask, running
  // softmax state.
  f16x8 qf[KSTEPS];
  uint64_t anc;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 o[NB];
  {
    const int qi = min(wave * 16 + lr, QR - 1);
    const int r = qi / G, h = g * G + (qi - r * G);
    const TQ *qp = qin + (row0 + r) * q_stride + h * HD;
    // padding rows of the last tile multiply zeros (their outputs are dropped; zero
    // operands keep the MFMA's switching, and so its power draw, down)
    const bool pad = wave * 16 + lr >= QR;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
      const f16x8 v = load_f16x8(qp + s * 32 + lg * 8);
      qf[s] = pad ? f16x8{} : v;
    }
    anc = ancs[r];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) o[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  wait_vmcnt<0>();   // the loop's vmcnt accounting covers the DMA only

  auto stage_of = [&](int c) { return smem + ((c - c0) % NST) * STAGE; };
  auto issue = [&](int c) {
    if (RECORDS && c < fc)
      issue_record<HD, NW>(stage_of(c), rr, c * (STAGE * 2), wave, lane);
    else
      issue_chunk<HD, NW>(stage_of(c), kr, vr, (c - fc) * KC, capacity, wave, lane);
  };
  auto widen = [&](int c, int t, int stride) {
    if (!RECORDS || c >= fc)
      widen_chunk<HD, PART>(stage_of(c), t, stride, (c - fc) * KC, total, S, bad);
    else if (front - c * KC < KC)
      cut_record<HD>(stage_of(c), t, stride, front - c * KC);
  };
  // The widening goes to the waves without a tile when there are any (one SIMD then
  // holds no more than its share of tile work plus widening), else to every wave.
  const int wbeg = ntiles < NW ? ntiles : 0;
  const int wt = (wave - wbeg) * 64 + lane, wstride = (NW - wbeg) * 64;
  const bool widener = wave >= wbeg;

  // Prologue: chunks c0 .. c0+NST-2 in flight, chunk c0 widened.
#pragma unroll
  for (int i = 0; i < NST - 1; ++i)
    if (c0 + i < c1) issue(c0 + i);
  if (!SYNC && c0 < c1) {
    if (c0 + NST - 2 < c1) wait_vmcnt<(NST - 2) * L_DMA>(); else wait_vmcnt<0>();
    lds_barrier();
    if (widener) widen(c0, wt, wstride);
  }

  // Fragment offsets: the swizzles depend on the lane only, so the read of K block kk at
  // k-step s is koff[s] + key_of_row(kk, 0) * HD and that of V^T block nb at key step ks is
  // voff[ks] + nb * 16 * KC -- a few lane registers plus compile-time constants.
  const int ksw_l = ksw<HD>(key_of_row(0, lr));
  int koff[KSTEPS], voff[2];
#pragma unroll
  for (int s = 0; s < KSTEPS; ++s)
    koff[s] = key_of_row(0, lr) * HD + (((s * 4 + lg) ^ ksw_l) << 3);
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) voff[ks] = v_off(lr, ks * 4 + lg);

  for (int c = c0; c < c1; ++c) {
    if constexpr (SYNC) {
      wait_vmcnt<0>();
      chunk_barrier();
      if (c + 1 < c1)
        issue(c + 1);
      widen(c, tid, NW * 64);
      chunk_barrier();
    } else {
      if (c + 1 < c1) {
        if (c + NST - 2 < c1) wait_vmcnt<(NST > 3 ? NST - 3 : 0) * L_DMA>(); else wait_vmcnt<0>();
      }
      chunk_barrier();
      if (c + NST - 1 < c1)
        issue(c + NST - 1);
      if (c + 1 < c1 && widener)
        widen(c + 1, wt, wstride);
    }

    const uint16_t *st = stage_of(c);
    const f16 *sk = (const f16 *)st;
    const f16 *sv = (const f16 *)(st + KC * HD);
    // (a record's slots in front of the prefix's end are seen by all, those behind it by none)
    const bool record = RECORDS && c < fc;
    const int key0 = record ? 0 : (c - fc) * KC, Sc = record ? front - c * KC : S, n1c = record ? 0 : n1;
    const bool tree_chunk = key0 + KC > Sc;
    if (wave < ntiles) {
      // S^T for 4 blocks of 16 keys: sc[kk][e] is the score of slot
      // key0 + key_of_score(kk, lg, e) against this lane's query.
      f32x4 sc[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) sc[kk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const f16x8 kf = *(const f16x8 *)(sk + koff[s] + key_of_row(kk, 0) * HD);
          sc[kk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[s], sc[kk], 0, 0, 0);
        }
      if (tree_chunk) {
        MASK_BRANCH();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // the slot is tree row j (a prefix slot if j < 0)
            const int j = key0 + key_of_score(kk, lg, e) - Sc;
            const int sh = min(max(j - 1, 0), 63);
            const bool vis = (j < 0) | ((j < n1c) & ((j == 0) | (bool)((anc >> sh) & 1ull)));
            sc[kk][e] = vis ? sc[kk][e] : -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, sc[kk][e]);
      mx = rows4_max(mx);
      const float m_new = lazy_ref(m_run, mx, lazy);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      // raw v_exp_f32: results below 2^-126 flush to zero, which a softmax weight can spare
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_use) * sscale);
      m_run = m_new;
      const float mb = m_use * sscale;
      f16x8 pb[2];
      float rs = 0.f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sc[kk][e], sscale, -mb));
          rs += p;
          pb[kk >> 1][(kk & 1) * 4 + e] = (f16)p;
        }
      l_run = l_run * alpha + rs;
      if (__ballot(alpha < 1.f)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[nb][e] *= alpha;
      }
      // O^T += V^T P^T over two k-steps of 32 keys.
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f16x8 va = *(const f16x8 *)(sv + voff[ks] + nb * 16 * KC);
          o[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, pb[ks], o[nb], 0, 0, 0);
        }
    }
  }
  wait_vmcnt<0>();
  if (PART) {
    __syncthreads();   // the marks are complete
    if (!join.here && tid < 3) join.sm.bad[(((size_t)b * Hkv + g) * nsplit + split) * 3 + tid] = bad[tid];
  }
  const bf16 *vtree = vb + S;   // the tree's values

  // o[nb][e] is head dim nb*16 + lg*4 + e of query wave*16 + lr.
  if (wave < ntiles) {
    const float l = rows4_sum(l_run);
    const int qi = wave * 16 + lr;
    if (qi >= QR) return;
    const int r = qi / G, h = g * G + (qi - r * G);
    if (PART && join.here) {
      shared_finish<HD>(join, me, total_units, ancs, vtree, capacity, bad, b, g, qi, n1, H, Hkv, rows_all,
                        m_run == -INFINITY ? -INFINITY : m_run * sscale, l, o,
                        [&](int nb) { return nb * 16 + lg * 4; });
    } else if (!PART && nsplit == 1) {
      const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        f16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (f16)(o[nb][e] * inv);
        *(f16x4 *)(out + act_off((int)row0 + r, h * HD + nb * 16 + lg * 4, rows_all, q_stride)) = v;
      }
    } else {
      const size_t item = ((size_t)b * Hkv + g) * nsplit + split;
      float *po = part_o + (item * QR + qi) * HD + lg * 4;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *(f32x4 *)(po + nb * 16) = o[nb];
      if (lg == 0) {
        part_ml[(item * QR + qi) * 2 + 0] = m_run == -INFINITY ? -INFINITY : m_run * sscale;
        part_ml[(item * QR + qi) * 2 + 1] = l;
      }
    }
  }
}

// ------------------------------------------------------------------------------------
// 32-row query tiles, for kv heads whose query rows exceed 16 tiles of 16 (a 64-node tree
// under 4 or more query heads per kv head).  Eight waves, one 32-row tile each, on
// v_mfma_f32_32x32x16_f16: every 16-byte K or V^T fragment read now feeds 32 queries
// instead of 16, which halves the LDS fragment traffic per query, and each wave's chains
// are twice as long.  A remainder of at most 16 rows is one 16-row tile split into four
// quarter units (one 16-key block of every chunk each) on waves 4-7, which share SIMDs
// with waves 0-3, merged through LDS at the end.  At most 8 x 32 + 16 rows per workgroup;
// more rows are dealt to query groups of equal size.
//  * S^T = K Q^T per 32-key block: A row r holds key p32(r) of the block, B holds the 32
//    queries, so a lane holds 16 scores of one query (lane % 32) for keys
//    key32_of_score(i, lane / 32).  The two lanes of a query reduce their running max with
//    one 32-lane swap.
//  * O^T = V^T P^T per 16-key step: lane half h needs keys 8h .. 8h+7 of the step as its
//    B operand, which is exactly what p32 put in its scores; the matching V^T fragment is
//    one contiguous 16-byte read of a head-dim row.
// ------------------------------------------------------------------------------------
// key (within a 32-key block) held by A row r of a 32 x 32 score block
AS_DEVICE int p32(int r) {
  return ((r >> 4) & 1) * 16 + ((r >> 2) & 1) * 8 + ((r >> 3) & 1) * 4 + (r & 3);
}
// key (within the block) of score i = 4 j + e of a lane in half h: output row 8 j + 4 h + e
AS_DEVICE int key32_of_score(int i, int h) {
  const int j = i >> 2, e = i & 3;
  return (j >> 1) * 16 + h * 8 + (j & 1) * 4 + e;
}

template <int HD, int NST, int MODE = 0, typename TQ = f16>
__global__ __launch_bounds__(512) void tree_attn_t32_kernel(
    const TQ *__restrict__ qin, const bf16 *__restrict__ ck, const bf16 *__restrict__ cv,
    TreeMeta meta, f16 *__restrict__ out, float *__restrict__ part_o,
    float *__restrict__ part_ml, int n1, int H, int Hkv, int capacity, int nsplit, int rpg,
    SharedJoin join) {
  constexpr bool PART = MODE > 0, RECORDS = MODE == 2;
  constexpr bool TREES = RECORDS && std::is_same<TQ, bf16>::value;   // (a call of the attention alone)
  constexpr int NW = 8;
  constexpr int KS16 = HD / 16;   // 16-dim k-steps of a 32-row tile's S^T
  constexpr int NDB = HD / 32;    // 32-dim blocks of its O^T
  constexpr int KS32 = HD / 32;   // 32-dim k-steps of the remainder tile's S^T
  constexpr int NB16 = HD / 16;   // 16-dim blocks of the remainder tile's O^T
  constexpr int STAGE = 2 * KC * HD;
  constexpr int L_DMA = HD / 4 / NW;
  static_assert(NST >= 3, "the widening runs one stage ahead of the MFMAs");
  __shared__ __attribute__((aligned(1024))) uint16_t smem[NST * STAGE];

  const int g = blockIdx.y, b = blockIdx.z;
  const int G = H / Hkv, QR = G * n1;
  const int nqg = (QR + rpg - 1) / rpg;
  const int split = blockIdx.x / nqg, grp = blockIdx.x - split * nqg;
  const int rlo = grp * rpg, rows = min(rpg, QR - rlo);
  int n32 = rows >> 5, rem = rows & 31;
  if (rem > 16) {  // a remainder beyond 16 rows is a (padded) 32-row tile of its own
    ++n32;
    rem = 0;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lq = lane & 31, hh = lane >> 5;   // 32 x 32 layout: query column, lane half
  const int lr = lane & 15, lg = lane >> 4;   // 16 x 16 layout (remainder tile)
  const bool t32 = wave < n32;
  const bool quarter = rem > 0 && wave >= NW - 4;
  const int qk = wave & 3;                    // a quarter unit's key block in each chunk
  __shared__ uint32_t bad[PART ? 3 : 1];   // tree rows with values that are not finite
  if (PART && threadIdx.x < 3) bad[threadIdx.x] = 0;   // (before the prologue's barrier)
  SharedSession me{};          // (asked for here, well before the join needs it)
  int4 total_units{};
  if (PART && !TREES && (RECORDS || join.here)) {
    me = join.sm.sessions[b];
    total_units = *join.sm.total;
  }
  __shared__ TreeSets sets[1];
  TreeSession session{};
  if constexpr (TREES)
    session = tree_session(sets[0], join.trees, tree_ask(join.trees, join.sh, b, n1), b, n1, capacity, blockIdx.x == 0 && g == 0, meta);
  // chunks of the session's shared prefix, in front of its own, if they are taken here
  const int front = TREES ? session.front : RECORDS ? __builtin_amdgcn_readfirstlane(me.slots) : 0;
  const int fc = RECORDS ? (front + KC - 1) / KC : 0;
  const size_t plane = RECORDS && fc > 0 ? (size_t)join.sh.cap * 2 * HD : 0;
  const int prefix = TREES ? session.prefix : RECORDS && fc > 0 ? __builtin_amdgcn_readfirstlane(join.sh.of[b]) : 0;
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(join.blocks + ((size_t)prefix * Hkv + g) * plane,
                                              (uint32_t)(plane * 2));
  if (RECORDS) me.place = -1;   // nothing to join
  const int S = TREES ? session.S : meta.sess_S[b];
  const uint64_t *ancs = TREES ? sets[0].anc : meta.anc + (size_t)b * n1;
  const int total = S + n1;
  const int nchunks = fc + (total + KC - 1) / KC;
  const int cps = (nchunks + nsplit - 1) / nsplit;
  const int c0 = split * cps;
  const int c1 = min(nchunks, c0 + cps);
  const bf16 *kb = ck + ((size_t)b * Hkv + g) * capacity * HD;
  const bf16 *vb = cv + ((size_t)b * Hkv + g) * HD * capacity;
  const __amdgpu_buffer_rsrc_t kr = make_rsrc(kb, (uint32_t)((size_t)capacity * HD * 2));
  const __amdgpu_buffer_rsrc_t vr = make_rsrc(vb, (uint32_t)((size_t)capacity * HD * 2));
  const size_t row0 = (size_t)b * n1;
  const int q_stride = H * HD, rows_all = gridDim.z * n1;
  const float sscale = LOG2E / sqrtf((float)HD);
  const float lazy = LAZY_LOG2 / sscale;

  // This wave's 32-row tile: query rlo + 32 wave + lq.  Padding rows (and the tile of a
  // wave without one) multiply zeros; their outputs are dropped.
  f16x8 qf[KS16];
  uint64_t anc;
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 o[NDB];
  {
    const int qv = rlo + wave * 32 + lq;
    const bool pad = !t32 || qv >= rlo + rows;
    const int qi = min(qv, QR - 1);
    const int r = qi / G, h = g * G + (qi - r * G);
    const TQ *qp = qin + (row0 + r) * q_stride + h * HD;
#pragma unroll
    for (int s = 0; s < KS16; ++s) {
      const f16x8 v = load_f16x8(qp + s * 16 + hh * 8);
      qf[s] = pad ? f16x8{} : v;
    }
    anc = ancs[r];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  }
  // The remainder tile (quarter waves): query rlo + 32 n32 + lr.
  f16x8 qq[KS32];
  uint64_t ancq;
  float mq = -INFINITY, lsq = 0.f;
  f32x4 oq[NB16];
  {
    const int qv = rlo + n32 * 32 + lr;
    const bool pad = !quarter || lr >= rem;
    const int qi = min(qv, QR - 1);
    const int r = qi / G, h = g * G + (qi - r * G);
    const TQ *qp = qin + (row0 + r) * q_stride + h * HD;
#pragma unroll
    for (int s = 0; s < KS32; ++s) {
      const f16x8 v = load_f16x8(qp + s * 32 + lg * 8);
      qq[s] = pad ? f16x8{} : v;
    }
    ancq = ancs[r];
#pragma unroll
    for (int nb = 0; nb < NB16; ++nb) oq[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  wait_vmcnt<0>();   // the loop's vmcnt accounting covers the DMA only

  auto stage_of = [&](int c) { return smem + ((c - c0) % NST) * STAGE; };
  auto issue = [&](int c) {
    if (RECORDS && c < fc)
      issue_record<HD, NW, true>(stage_of(c), rr, c * (STAGE * 2), wave, lane);
    else
      issue_chunk<HD, NW, true>(stage_of(c), kr, vr, (c - fc) * KC, capacity, wave, lane);
  };
  auto widen = [&](int c, int t, int stride) {
    if (!RECORDS || c >= fc)
      widen_chunk<HD, PART>(stage_of(c), t, stride, (c - fc) * KC, total, S, bad);
    else if (front - c * KC < KC)
      cut_record<HD>(stage_of(c), t, stride, front - c * KC);
  };
  const int wt = tid, wstride = NW * 64;   // every wave widens its share

  // Prologue: chunks c0 .. c0+NST-2 in flight, chunk c0 widened.
#pragma unroll
  for (int i = 0; i < NST - 1; ++i)
    if (c0 + i < c1)
      issue(c0 + i);
  if (c0 < c1) {
    if (c0 + NST - 2 < c1) wait_vmcnt<(NST - 2) * L_DMA>(); else wait_vmcnt<0>();
    lds_barrier();
    widen(c0, wt, wstride);
  }

  // Fragment offsets (lane registers; blocks add compile-time constants): K row p32(lq)
  // (+32 for the second key block) at piece 2 s + hh; V^T row lq (+32 db) at piece
  // 2 ks + hh; the quarter unit's K row key_of_row(qk, lr) at piece 4 s + lg and its V^T
  // half-piece.
  const int krow = p32(lq), ksl = ksw32<HD>(krow);
  int koff[KS16];
#pragma unroll
  for (int s = 0; s < KS16; ++s) koff[s] = krow * HD + (((s * 2 + hh) ^ ksl) << 3);
  int voff[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) voff[ks] = lq * KC + (((ks * 2 + hh) ^ vsw(lq)) << 3);
  const int qkey = key_of_row(qk, lr), qksl = ksw32<HD>(qkey);
  int qkoff[KS32];
#pragma unroll
  for (int s = 0; s < KS32; ++s) qkoff[s] = qkey * HD + (((s * 4 + lg) ^ qksl) << 3);
  const int qvoff = lr * KC + (((((qk >> 1) * 4) + lg) ^ vsw(lr)) << 3) + (qk & 1) * 4;

  for (int c = c0; c < c1; ++c) {
    if (c + 1 < c1) {
      if (c + NST - 2 < c1) wait_vmcnt<(NST - 3) * L_DMA>(); else wait_vmcnt<0>();
    }
    chunk_barrier();
    if (c + NST - 1 < c1)
      issue(c + NST - 1);
    if (c + 1 < c1)
      widen(c + 1, wt, wstride);

    const uint16_t *st = stage_of(c);
    const f16 *sk = (const f16 *)st;
    const f16 *sv = (const f16 *)(st + KC * HD);
    // (a record's slots in front of the prefix's end are seen by all, those behind it by none)
    const bool record = RECORDS && c < fc;
    const int key0 = record ? 0 : (c - fc) * KC, Sc = record ? front - c * KC : S, n1c = record ? 0 : n1;
    const bool tree_chunk = key0 + KC > Sc;
    if (t32) {
      // S^T for the chunk's two 32-key blocks: sc[kb][i] is the score of slot
      // key0 + 32 kb + key32_of_score(i, hh) against this lane's query.  Both blocks are
      // issued first; then each block gets its own online-softmax step and its P.V
      // products, so block 0's softmax runs on the VALU while block 1's scores are still
      // in the matrix pipe, and block 1's softmax while block 0's P.V runs.
      f32x16 sc[2];
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb2][i] = 0.f;
#pragma unroll
        for (int s = 0; s < KS16; ++s) {
          const f16x8 kf = *(const f16x8 *)(sk + koff[s] + kb2 * 32 * HD);
          sc[kb2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[s], sc[kb2], 0, 0, 0);
        }
      }
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2) {
        SCHED_FENCE();
        f32x16 &z = sc[kb2];
        if (tree_chunk) {
          MASK_BRANCH();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = key0 + kb2 * 32 + key32_of_score(i, hh) - Sc;  // tree row, or < 0
            const int sh = min(max(j - 1, 0), 63);
            const bool vis = (j < 0) | ((j < n1c) & ((j == 0) | (bool)((anc >> sh) & 1ull)));
            z[i] = vis ? z[i] : -INFINITY;
          }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, z[i]);
        mx = halves_max(mx);
        const float m_new = lazy_ref(m_run, mx, lazy);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f((m_run - m_use) * sscale);
        m_run = m_new;
        const float mb = m_use * sscale;
        // the block's probabilities as the B operands of its two 16-key steps: step
        // (j / 2) takes scores 4 j + e at positions (j % 2) * 4 + e
        f16x8 pk[2];
        float rs = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float pz = __builtin_amdgcn_exp2f(fmaf(z[i], sscale, -mb));
          rs += pz;
          const int j = i >> 2, e = i & 3;
          pk[j >> 1][(j & 1) * 4 + e] = (f16)pz;
        }
        l_run = l_run * alpha + rs;
        if (__ballot(alpha < 1.f)) {
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        }
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const f16x8 va = *(const f16x8 *)(sv + voff[kb2 * 2 + k2] + db * 32 * KC);
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va, pk[k2], o[db], 0, 0, 0);
          }
      }
      SCHED_FENCE();
    }
    if (quarter) {
      // key block qk of the chunk for the remainder tile: 4 scores a lane
      f32x4 sq = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS32; ++s) {
        const f16x8 kf = *(const f16x8 *)(sk + qkoff[s]);
        sq = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qq[s], sq, 0, 0, 0);
      }
      if (tree_chunk) {
        MASK_BRANCH();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = key0 + key_of_score(qk, lg, e) - Sc;
          const int sh = min(max(j - 1, 0), 63);
          const bool vis = (j < 0) | ((j < n1c) & ((j == 0) | (bool)((ancq >> sh) & 1ull)));
          sq[e] = vis ? sq[e] : -INFINITY;
        }
      }
      float mx = fmaxf(fmaxf(sq[0], sq[1]), fmaxf(sq[2], sq[3]));
      mx = rows4_max(mx);
      const float m_new = lazy_ref(mq, mx, lazy);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f((mq - m_use) * sscale);
      mq = m_new;
      const float mb = m_use * sscale;
      f16x4 pq;
      float rs = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sq[e], sscale, -mb));
        rs += p;
        pq[e] = (f16)p;
      }
      lsq = lsq * alpha + rs;
      if (__ballot(alpha < 1.f)) {
#pragma unroll
        for (int nb = 0; nb < NB16; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) oq[nb][e] *= alpha;
      }
#pragma unroll
      for (int nb = 0; nb < NB16; ++nb) {
        const f16x4 va = *(const f16x4 *)(sv + qvoff + nb * 16 * KC);
        oq[nb] = __builtin_amdgcn_mfma_f32_16x16x16f16(va, pq, oq[nb], 0, 0, 0);
      }
    }
  }
  wait_vmcnt<0>();
  if (PART) {
    __syncthreads();   // the marks are complete
    if (!join.here && tid < 3) join.sm.bad[(((size_t)b * Hkv + g) * nsplit + split) * 3 + tid] = bad[tid];
  }
  const bf16 *vtree = vb + S;   // the tree's values

  if (rem > 0) {
    // Merge the remainder tile's four quarter units (the ring is free once every wave is
    // past its last chunk); quarter wave qk finalises head-dim blocks qk * NB16/4 ...
    __syncthreads();
    f32x4 *mo = (f32x4 *)smem;                                 // [quarter][NB16][64 lanes]
    float *mml = (float *)smem + (size_t)4 * NB16 * 64 * 4;    // [quarter][16 queries][2]
    if (quarter) {
      const float l = rows4_sum(lsq);
#pragma unroll
      for (int nb = 0; nb < NB16; ++nb) mo[(qk * NB16 + nb) * 64 + lane] = oq[nb];
      if (lg == 0) {
        mml[(qk * 16 + lr) * 2 + 0] = mq == -INFINITY ? -INFINITY : mq * sscale;
        mml[(qk * 16 + lr) * 2 + 1] = l;
      }
    }
    __syncthreads();
    if (quarter) {
      float mj[4], wj[4];
      float M = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mj[j] = mml[(j * 16 + lr) * 2];
        M = fmaxf(M, mj[j]);
      }
      float L = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        wj[j] = mj[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mj[j] - M);
        L += wj[j] * mml[(j * 16 + lr) * 2 + 1];
      }
      const int qi = rlo + n32 * 32 + lr;
      if (lr < rem) {
        const int r = qi / G, h = g * G + (qi - r * G);
        const size_t item = ((size_t)b * Hkv + g) * nsplit + split;
        f32x4 all[NB16 / 4];
#pragma unroll
        for (int i = 0; i < NB16 / 4; ++i) {
          const int nb = qk * (NB16 / 4) + i;
          f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4 v = mo[(j * NB16 + nb) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += wj[j] * v[e];
          }
          all[i] = acc;
          if (PART && join.here) continue;
          if (!PART && nsplit == 1) {
            const float inv = L > 0.f ? 1.0f / L : 0.f;
            f16x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (f16)(acc[e] * inv);
            *(f16x4 *)(out + act_off((int)row0 + r, h * HD + nb * 16 + lg * 4, rows_all, q_stride)) = v;
          } else {
            *(f32x4 *)(part_o + (item * QR + qi) * HD + nb * 16 + lg * 4) = acc;
          }
        }
        if (PART && join.here)
          shared_finish<HD>(join, me, total_units, ancs, vtree, capacity, bad, b, g, qi, n1, H, Hkv, rows_all, M, L, all,
                            [&](int i) { return (qk * (NB16 / 4) + i) * 16 + lg * 4; });
        if ((PART ? !join.here : nsplit > 1) && qk == 0 && lg == 0) {
          part_ml[(item * QR + qi) * 2 + 0] = M;
          part_ml[(item * QR + qi) * 2 + 1] = L;
        }
      }
    }
  }

  // o[db][4 j + e] is head dim 32 db + 8 j + 4 hh + e of query rlo + 32 wave + lq.
  if (t32) {
    const float l = halves_sum(l_run);
    const int qi = rlo + wave * 32 + lq;
    if (qi < rlo + rows) {
      const int r = qi / G, h = g * G + (qi - r * G);
      if (PART && join.here) {
        f32x4 all[4 * NDB];
#pragma unroll
        for (int i = 0; i < 4 * NDB; ++i)
          all[i] = f32x4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2],
                         o[i >> 2][4 * (i & 3) + 3]};
        shared_finish<HD>(join, me, total_units, ancs, vtree, capacity, bad, b, g, qi, n1, H, Hkv, rows_all,
                          m_run == -INFINITY ? -INFINITY : m_run * sscale, l, all,
                          [&](int i) { return 8 * i + 4 * hh; });
      } else if (!PART && nsplit == 1) {
        const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f16x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (f16)(o[db][j * 4 + e] * inv);
            *(f16x4 *)(out + act_off((int)row0 + r, h * HD + db * 32 + j * 8 + hh * 4, rows_all,
                                     q_stride)) = v;
          }
      } else {
        const size_t item = ((size_t)b * Hkv + g) * nsplit + split;
        float *po = part_o + (item * QR + qi) * HD + hh * 4;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *(f32x4 *)(po + db * 32 + j * 8) =
                f32x4{o[db][j * 4], o[db][j * 4 + 1], o[db][j * 4 + 2], o[db][j * 4 + 3]};
        if (hh == 0) {
          part_ml[(item * QR + qi) * 2 + 0] = m_run == -INFINITY ? -INFINITY : m_run * sscale;
          part_ml[(item * QR + qi) * 2 + 1] = l;
        }
      }
    }
  }
}

// Merge of the split partials.  grid: (ceil(QR * HD / 4 / 256), kv heads, sessions); one
// thread per 4 head dims of one query row.  part_ml holds (max in base-2 exponent units,
// sum) per (item, query row).
__global__ __launch_bounds__(256) void attn_combine_kernel(const float *__restrict__ part_o,
                                                           const float *__restrict__ part_ml,
                                                           f16 *__restrict__ out, int n1, int H,
                                                           int Hkv, int HD, int nsplit) {
  const int g = blockIdx.y, b = blockIdx.z;
  const int G = H / Hkv, QR = G * n1, hd4 = HD >> 2;
  const int idx = blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= QR * hd4) return;
  const int qi = idx / hd4, d = (idx - qi * hd4) * 4;
  const size_t item0 = ((size_t)b * Hkv + g) * nsplit;
  // (the splits' loads are independent and in flight together: one after the other they
  // took 10.6 us at 12 splits of a single session)
  const float2 *ml = (const float2 *)part_ml + item0 * QR + qi;
  const float *po = part_o + (item0 * QR + qi) * HD + d;
  const size_t so = (size_t)QR * HD;
  float M = -INFINITY;
#pragma unroll 8
  for (int s = 0; s < nsplit; ++s) M = fmaxf(M, ml[(size_t)s * QR].x);
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
  float den = 0.f;
#pragma unroll 8
  for (int s = 0; s < nsplit; ++s) {
    const float2 e = ml[(size_t)s * QR];
    const float4 v = *(const float4 *)(po + s * so);
    const float w = e.x == -INFINITY ? 0.f : exp2f(e.x - M);   // (a split without slots)
    den += w * e.y;
    num.x += w * v.x;
    num.y += w * v.y;
    num.z += w * v.z;
    num.w += w * v.w;
  }
  const float inv = den > 0.f ? 1.f / den : 0.f;
  const int r = qi / G, h = g * G + (qi - r * G);
  *(f16x4 *)(out + act_off(b * n1 + r, h * HD + d, gridDim.z * n1, H * HD)) =
      f16x4{(f16)(num.x * inv), (f16)(num.y * inv), (f16)(num.z * inv), (f16)(num.w * inv)};
}

// fp32 path: one workgroup per (tree row, query head).  256 slots at a time: scores with
// HD / 4 lanes a slot (16-byte pieces of a key row, summed by lane swaps), a softmax step
// over the block with the usual running maximum, then the values: 16 lanes x 4 slots of a
// head dim, whose sums stay in registers until the end.  (One wave walking the slots one by
// one, each behind a reduction over the wave, took 62 us at 137 slots, this 10.)
template <int HD>
__global__ __launch_bounds__(256) void tree_attn_f32_kernel(
    const float *__restrict__ qin, const float *__restrict__ ck, const float *__restrict__ cv,
    TreeMeta meta, float *__restrict__ out, int n1, int H, int Hkv, int capacity) {
  constexpr int LPS = HD / 4, SPW = 64 / LPS;   // lanes a slot, slots a wave and load
  constexpr int NCH = 256, STEPS = NCH / 4 / SPW;
  constexpr int DJ = HD / 16;                   // head dims a lane sums
  __shared__ __attribute__((aligned(16))) float p[NCH];
  __shared__ float red[8];
  const int h = blockIdx.x, row = blockIdx.y;
  const int b = row / n1;
  const int G = H / Hkv, g = h / G, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int S = meta.sess_S[b], total = S + n1;
  const uint64_t anc = meta.anc[row];
  const float *kb = ck + ((size_t)b * Hkv + g) * capacity * HD;
  const float *vb = cv + ((size_t)b * Hkv + g) * HD * capacity;   // [HD][capacity]
  const float4 q4 = *(const float4 *)(qin + (size_t)row * H * HD + h * HD + lane % LPS * 4);
  const float scale = 1.0f / sqrtf((float)HD);
  float m = -INFINITY, l = 0.f, o[DJ];
#pragma unroll
  for (int j = 0; j < DJ; ++j) o[j] = 0.f;
  for (int c0 = 0; c0 < total; c0 += NCH) {
    // scores of slots c0 + wave * 64 + i * SPW + lane / LPS
    float4 kv[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int slot = c0 + wave * 64 + i * SPW + lane / LPS;
      kv[i] = *(const float4 *)(kb + (size_t)min(slot, total - 1) * HD + lane % LPS * 4);
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int ls = wave * 64 + i * SPW + lane / LPS, slot = c0 + ls;
      float d = q4.x * kv[i].x + q4.y * kv[i].y + q4.z * kv[i].z + q4.w * kv[i].w;
#pragma unroll
      for (int x = 1; x < LPS; x <<= 1) d += __shfl_xor(d, x);
      if (lane % LPS == 0) p[ls] = tree_visible(slot, S, n1, anc) ? d * scale : -INFINITY;
    }
    __syncthreads();
    const float s = p[tid];
    float mx = wave_max(s);
    if (lane == 0) red[wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float mn = fmaxf(m, mx);      // finite from the first block on: the root is visible,
    const float mu = mn == -INFINITY ? 0.f : mn;   // and prefix slots are
    const bool vis = tree_visible(c0 + tid, S, n1, anc);
    const float e = vis ? expf(s - mu) : 0.f, a = expf(m - mu);
    m = mn;
    p[tid] = vis ? e : -1.f;            // (a hidden slot's value is left out, not times 0)
    const float ls = wave_sum(e);
    if (lane == 0) red[4 + wave] = ls;
    __syncthreads();
    l = l * a + ((red[4] + red[5]) + (red[6] + red[7]));
#pragma unroll
    for (int j = 0; j < DJ; ++j) o[j] *= a;
    // values: lane % 16 takes slots 4 (lane % 16) + 64 i, for head dims wave * 4 + lane / 16
    // + 16 j (the capacity is a multiple of 64: reads past the last slot stay in the row)
    for (int i = 0; i < NCH / 64 && c0 + i * 64 < total; ++i) {
      const int ls4 = i * 64 + lane % 16 * 4, slot = c0 + ls4;
      const float4 w = *(const float4 *)(p + ls4);
#pragma unroll
      for (int j = 0; j < DJ; ++j) {
        const float4 v = *(const float4 *)(vb + (size_t)(wave * 4 + lane / 16 + 16 * j) * capacity + slot);
        if (w.x >= 0.f) o[j] += w.x * v.x;
        if (w.y >= 0.f) o[j] += w.y * v.y;
        if (w.z >= 0.f) o[j] += w.z * v.z;
        if (w.w >= 0.f) o[j] += w.w * v.w;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < DJ; ++j) {
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) o[j] += __shfl_xor(o[j], x);
    if (lane % 16 == 0)
      out[(size_t)row * (H * HD) + h * HD + wave * 4 + lane / 16 + 16 * j] = o[j] / l;
  }
}

// Ring depth: 4 stages of 32 KB (head_dim 128) or 16 KB (head_dim 64).
template <int HD> struct AttnCfg { static constexpr int NST = 4; };

template <int HD, int NW, int NST, int MODE, typename TQ>
void launch_mfma(dim3 grid, hipStream_t s, const TQ *q, const bf16 *ck, const bf16 *cv,
                 const TreeMeta &meta, f16 *out, float *po, float *pml, int n1, int H, int Hkv,
                 int capacity, int nsplit, const SharedJoin &join) {
  hipLaunchKernelGGL((tree_attn_mfma_kernel<HD, NW, NST, MODE, TQ>), grid,
                     dim3(NW * 64), 0, s, q, ck, cv, meta, out, po, pml, n1, H, Hkv,
                     capacity, nsplit, join);
}

// Key splits: as many as the CUs hold at once, rounded down, for a second round of a few
// workgroups costs what the first does (6 sessions of 8 kv heads: six splits, 288
// workgroups, took 29.2 us, five 24.6; where the items do not divide the CUs some idle).
// A split is at least 4 chunks, as the merge's launch and its fp32 partials cost about as
// much as three (16 sessions of 8 kv heads, 300 slots, two splits 27.3 us, whole 21.0),
// but 2 for up to 32 items, whose few partials cost little, if the chunks' query tiles add
// up to some work (one session of 1500 slots: 16.2 us against 17.3 at 4 chunks; 65 rows of
// 8 query heads over 300 slots: 26 against 33 whole).
int workgroups_a_cu(int all_tiles) { return all_tiles <= 8 ? 2 : 1; }   // behind shared prefixes
int attn_items(int B, int n1, int H, int Hkv) {
  const int QR = H / Hkv * n1;
  return B * Hkv * (QR > 256 ? (QR + 271) / 272 : 1);   // (the query groups of launch_tree_attn)
}
int attn_splits(int B, int n1, int H, int Hkv, int hd, int nchunks, int cus, long long part_capacity,
                bool part) {
  const int QR = H / Hkv * n1, all_tiles = (QR + 15) / 16, items = attn_items(B, n1, H, Hkv);
  int nsplit = cus / items;
  const int least = items <= 32 && nchunks * all_tiles >= 48 ? 2 : 4;
  nsplit = nsplit < nchunks / least ? nsplit : nchunks / least;
  // Behind shared prefixes two workgroups share a CU up to 8 tiles: items that are split already are
  // split for both where five chunks are left of each (17 rows, 8 kv heads: 8 sessions of 4096 slots
  // 39.0 -> 35.2 us, 12 of 2048 40.9 -> 34.4; 8 of 2048, four chunks, 27.5 -> 28.6, two chunks 22.3 ->
  // 26.7, and items that were whole 37.4 -> 41.0).
  if (part && nsplit > 1 && workgroups_a_cu(all_tiles) == 2 && nchunks / 5 >= 2 * cus / items)
    nsplit = std::max(nsplit, 2 * cus / items);
  if (nsplit < 1) nsplit = 1;
  while (nsplit > 1 && (long long)B * Hkv * nsplit * QR * hd > part_capacity) --nsplit;
  return nsplit;
}

// The kernels of one layer, without the merge of their splits.
template <int MODE, typename TQ>
hipError_t launch_tree_attn(const TQ *q, const bf16 *ck, const bf16 *cv, const TreeMeta &meta,
                            f16 *out, float *part_o, float *part_ml, long long part_capacity, int B,
                            int n1, int H, int Hkv, int hd, int capacity, int cus, hipStream_t s,
                            int *nsplit_used, SharedJoin join) {
  constexpr bool PART = MODE > 0;
  const int G = H / Hkv, QR = G * n1;
  const int all_tiles = (QR + 15) / 16;
  if (capacity % KC != 0) return hipErrorInvalidValue;
  // Up to 16 tiles of 16 rows: 16 waves, one tile per wave, the others widen (measured
  // fastest on the 8B shape: 5 tiles).  More rows: 8 waves of 32-row tiles plus a
  // remainder of at most 16 rows, i.e. up to 272 rows a workgroup; beyond that the rows
  // are dealt to query groups of equal size (8 query heads per kv head under a 64-node
  // tree: 520 rows, two groups of 260), each streaming the key range once.
  const bool t32 = all_tiles > 16;
  const int nqg = t32 ? (QR + 271) / 272 : 1;
  const int rpg = (QR + nqg - 1) / nqg;
  const int nsplit = attn_splits(B, n1, H, Hkv, hd,
                                 capacity / KC + (MODE == 2 ? join.sh.cap / KC : 0), cus,
                                 part_capacity, PART);
  *nsplit_used = nsplit;
  if (PART && nsplit > 1) join.here = 0;
  const dim3 grid(nsplit * nqg, Hkv, B);
  if (t32) {
    if (hd == 128)
      hipLaunchKernelGGL((tree_attn_t32_kernel<128, AttnCfg<128>::NST, MODE, TQ>), grid, dim3(512), 0, s,
                         q, ck, cv, meta, out, part_o, part_ml, n1, H, Hkv, capacity, nsplit,
                         rpg, join);
    else
      hipLaunchKernelGGL((tree_attn_t32_kernel<64, AttnCfg<64>::NST, MODE, TQ>), grid, dim3(512), 0, s,
                         q, ck, cv, meta, out, part_o, part_ml, n1, H, Hkv, capacity, nsplit,
                         rpg, join);
  } else {
    auto launch = hd == 128 ? launch_mfma<128, 16, 4, MODE, TQ> : launch_mfma<64, 16, 4, MODE, TQ>;
    if constexpr (PART)
      if (workgroups_a_cu(all_tiles) == 2)
        launch = hd == 128 ? launch_mfma<128, 8, 2, MODE, TQ> : launch_mfma<64, 8, 4, MODE, TQ>;
    launch(grid, s, q, ck, cv, meta, out, part_o, part_ml, n1, H, Hkv, capacity, nsplit, join);
  }
  return hipGetLastError();
}

}  // namespace

namespace acespec {

template <>
hipError_t launch_attention<bf16>(const f16 *q, const bf16 *ck, const bf16 *cv,
                                  const TreeMeta &meta, f16 *out, float *part_o,
                                  float *part_ml, long long part_capacity, int B, int n1, int H,
                                  int Hkv, int hd, int capacity, int cus, hipStream_t s,
                                  int *nsplit_used) {
  const hipError_t e = launch_tree_attn<0, f16>(q, ck, cv, meta, out, part_o, part_ml, part_capacity, B,
                                               n1, H, Hkv, hd, capacity, cus, s, nsplit_used, SharedJoin{});
  const int nsplit = *nsplit_used;
  if (e != hipSuccess || nsplit == 1) return e;
  const int QR = H / Hkv * n1, cblocks = (QR * (hd / 4) + 255) / 256;
  hipLaunchKernelGGL(attn_combine_kernel, dim3(cblocks, Hkv, B), dim3(256), 0, s, part_o,
                     part_ml, out, n1, H, Hkv, hd, nsplit);
  return hipGetLastError();
}

int attention_chunks_in_turn(int B, int n1, int H, int Hkv, int hd, int nchunks, int cus,
                             long long part_capacity) {
  const int nsplit = attn_splits(B, n1, H, Hkv, hd, nchunks, cus, part_capacity, true);
  const int at_once = cus * workgroups_a_cu((H / Hkv * n1 + 15) / 16);
  const int rounds = (attn_items(B, n1, H, Hkv) * nsplit + at_once - 1) / at_once;
  return rounds * ((nchunks + nsplit - 1) / nsplit);
}

template <typename TQ>
hipError_t launch_attention_own(const TQ *q, const bf16 *ck, const bf16 *cv, const TreeMeta &meta,
                                const SharedJoin &j, float *part_o, float *part_ml,
                                long long part_capacity, int B, int n1, int H, int Hkv, int hd,
                                int capacity, int cus, hipStream_t s, int *nsplit) {
  auto launch = j.blocks ? launch_tree_attn<2, TQ> : launch_tree_attn<1, TQ>;
  return launch(q, ck, cv, meta, nullptr, part_o, part_ml, part_capacity, B, n1, H, Hkv, hd, capacity, cus,
                s, nsplit, j);
}
template hipError_t launch_attention_own<f16>(const f16 *, const bf16 *, const bf16 *,
                                              const TreeMeta &, const SharedJoin &, float *, float *,
                                              long long, int, int, int, int, int, int, int,
                                              hipStream_t, int *);
template hipError_t launch_attention_own<bf16>(const bf16 *, const bf16 *, const bf16 *,
                                               const TreeMeta &, const SharedJoin &, float *,
                                               float *, long long, int, int, int, int, int, int, int,
                                               hipStream_t, int *);

template <>
hipError_t launch_attention<float>(const float *q, const float *ck, const float *cv,
                                   const TreeMeta &meta, float *out, float *, float *,
                                   long long, int B, int n1, int H, int Hkv, int hd,
                                   int capacity, int, hipStream_t s, int *nsplit_used) {
  *nsplit_used = 1;
  auto kernel = hd == 64 ? tree_attn_f32_kernel<64> : tree_attn_f32_kernel<128>;
  hipLaunchKernelGGL(kernel, dim3(H, B * n1), dim3(256), 0, s, q, ck, cv, meta, out, n1, H, Hkv,
                     capacity);
  return hipGetLastError();
}

}  // namespace acespec
