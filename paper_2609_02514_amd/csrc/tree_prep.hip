// Tree preparation: validates each session's drafted tree and derives the per-row data
// the forward pass needs.  All drafted nodes of a session go through the target in one
// pass (Section III-C); a node may attend to the verified context and to its own
// ancestral sequence only, so each row gets the set of its ancestors as a bit mask over
// the drafted rows (the root, row 0, is every row's ancestor and is always visible).
// Positions: siblings share a position, prefix_len + depth; keys/values of row r live
// in cache slot prefix_len + r.
// Behind a shared prefix positions start at its end; the sessions of a prefix become a group.
// Over a cache in 4 bits the tree's rows go behind the prefix_len % 32 slots of the tail, and a
// sliding window takes ancestors that are too far back out of a row's set.
#include "tree.h"

namespace {

constexpr int TP_THREADS = TREE_ROWS;  // one thread per tree row (at most 65 rows)

// One workgroup per session.  A row's depth is its set's population count.
// tokens may be NULL.  front: positions before the prefix (-1: a shared prefix that is not one).
template <bool QUANT>
AS_DEVICE void prepare_tree(int b, const int32_t *__restrict__ tokens,
                            const int32_t *__restrict__ parents,
                            const int32_t *__restrict__ prefix_len, int n1, int V, int capacity,
                            int window, int sinks, int front, const TreeMeta &meta,
                            int32_t *__restrict__ status) {
  __shared__ TreeSets sets;
  const int r = threadIdx.x;
  const size_t base = (size_t)b * n1;
  const bool in = r < n1;
  const int pr = in ? parents[base + r] : 0;
  const int tk = in && tokens ? tokens[base + r] : 0;
  int S = prefix_len[b], p;
  // largest prefix: with QUANT full blocks and a full tail behind them
  const long long most = QUANT ? (long long)capacity + 31 : (long long)capacity - n1;
  const bool ok = tree_sets(sets, n1, pr, tk >= 0 && tk < V && S >= 0 && S <= most && front >= 0, &p);
  if (front < 0) front = 0;
  if (S < 0) S = 0;
  if (S > most) S = (int)most;
  if (r == 0) {
    meta.sess_S[b] = QUANT ? S & 31 : S;
    status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
  }
  uint64_t anc = sets.anc[r];
  const int depth = __popcll(anc);
  if (QUANT) __syncthreads();   // (other rows' sets are read)
  if (!in) return;
  if (QUANT && window > 0)
    for (uint64_t rest = anc; rest; rest &= rest - 1) {
      const int j = __builtin_ctzll(rest) + 1, dj = __popcll(sets.anc[j]);
      if (depth - dj >= window && S + dj >= sinks) anc &= ~(1ull << (j - 1));
    }
  if (tokens) meta.tok[base + r] = tk < 0 ? 0 : (tk >= V ? V - 1 : tk);
  meta.par[base + r] = p;
  meta.depth[base + r] = depth;
  meta.anc[base + r] = anc;
  meta.pos[base + r] = front + S + depth;
}

template <bool QUANT>
__global__ __launch_bounds__(TP_THREADS) void tree_prep_kernel(
    const int32_t *__restrict__ tokens, const int32_t *__restrict__ parents,
    const int32_t *__restrict__ prefix_len, int B, int n1, int V, int capacity, int window,
    int sinks, TreeMeta meta, int32_t *__restrict__ status) {
  prepare_tree<QUANT>(blockIdx.x, tokens, parents, prefix_len, n1, V, capacity, window, sinks, 0,
                      meta, status);
}

AS_DEVICE int group_tiles(int members, int QR, int tile_rows) {
  return (members * QR + tile_rows - 1) / tile_rows;
}

// The groups of at most 64 sessions, a lane each of one wave: in the order of their first members.
AS_DEVICE void group_few(int B, int QR, const SharedArgs &sh, int tile_rows, const SharedMeta &sm) {
  const int b = threadIdx.x;
  if (b >= 64) return;
  int slots = 0, groups = 0, units = 0, tiles = 0, most = 0, grouped = 0;
  const int p = b < B ? shared_prefix(sh, b, &slots) : -1;
  SharedSession mine{max(slots, 0), -1, 0, 0, 0};
  for (uint64_t rest = __ballot(p >= 0); rest;) {
    const int lead = __builtin_ctzll(rest);
    const uint64_t with = __ballot(p == __builtin_amdgcn_readlane(p, lead));
    const int members = __popcll(with), n = __builtin_amdgcn_readlane(slots, lead);
    if ((with >> b) & 1) {
      mine = SharedSession{slots, grouped + (int)__popcll(with & ((1ull << b) - 1)), grouped, units, tiles};
      if (b == lead) sm.groups[groups] = SharedGroup{p, grouped, members, n, units, tiles};
    }
    ++groups;
    grouped += members;
    units += group_tiles(members, QR, tile_rows) * ((n + 63) / 64);
    tiles += group_tiles(members, QR, tile_rows);
    most = max(most, (n + 63) / 64);
    rest &= ~with;
  }
  if (b < B) {
    sm.sessions[b] = mine;
    if (mine.place >= 0) sm.order[mine.place] = b;
  }
  if (b == 0) *sm.total = make_int4(units, groups, tiles, most);
}

// More sessions: in the order of their prefixes.  Each session's workgroup counts the sessions before
// its own (one pass over prefix_of), and a launch behind it puts the groups together.  (One workgroup
// for all of it took 324 us for 1024 sessions, this 5 and 6.)
AS_DEVICE void group_one(int b, int B, const SharedArgs &sh, const SharedMeta &sm) {
  __shared__ int s_count[4][TP_THREADS / 64];
  const int tid = threadIdx.x, mine = sh.of[b];
  int slots, count[4] = {0, 0, 0, 0};   // of lower prefixes, of this before b, of this, of any
  shared_prefix(sh, b, &slots);
#pragma unroll 4
  for (int i = tid; i < B; i += TP_THREADS) {
    const int o = sh.of[i];
    const bool in = o >= 0 && o < sh.P;
    count[0] += in && o < mine;
    count[1] += o == mine && i < b;
    count[2] += o == mine;
    count[3] += in;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = wave_sum_i32(count[k]);
    if (tid % 64 == 0) s_count[k][tid / 64] = c;
  }
  __syncthreads();
  if (tid > 0) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    count[k] = 0;
    for (int w = 0; w < TP_THREADS / 64; ++w) count[k] += s_count[k][w];
  }
  // (a prefix that is empty or malformed keeps its places, and has no group)
  const bool in = mine >= 0 && mine < sh.P;
  sm.sessions[b] = SharedSession{max(slots, 0), -1, count[0], count[2], 0};
  if (in) sm.order[count[0] + count[1]] = b;
  if (b == 0) *sm.total = make_int4(count[3], 0, 0, 0);
}

// A place a thread: sums over the groups before follow from a scan in which a group counts at its
// first place.
constexpr int GT = 1024;
__global__ __launch_bounds__(GT) void group_kernel(int QR, int tile_rows, SharedArgs sh, SharedMeta sm) {
  __shared__ int s_sum[4][GT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int places = sm.total->x;
  int units = 0, tiles = 0, groups = 0, most = 0;   // of the groups so far
  for (int x0 = 0; x0 < places; x0 += GT) {
    const int x = x0 + tid, b = x < places ? sm.order[x] : 0;
    SharedSession me = x < places ? sm.sessions[b] : SharedSession{0, -1, 0, 0, 0};
    const bool live = me.slots > 0, lead = live && me.first == x;
    const int members = me.units, nblk = (me.slots + 63) / 64, t = live ? group_tiles(members, QR, tile_rows) : 0;
    int sum[3] = {lead ? t * nblk : 0, lead ? t : 0, lead ? 1 : 0};   // with the lanes' before
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int v = __shfl_up(sum[k], o);
        if (lane >= o) sum[k] += v;
      }
    int top = nblk;
    for (int o = 1; o < 64; o <<= 1) top = max(top, __shfl_xor(top, o));
    __syncthreads();
    if (lane == 63) {
#pragma unroll
      for (int k = 0; k < 3; ++k) s_sum[k][wave] = sum[k];
      s_sum[3][wave] = top;
    }
    __syncthreads();
    int all[3] = {0, 0, 0};
    for (int w = 0; w < GT / 64; ++w) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int v = s_sum[k][w];
        all[k] += v;
        if (w < wave) sum[k] += v;
      }
      most = max(most, s_sum[3][w]);
    }
    if (live) {
      me.place = x;
      me.units = units + sum[0] - t * nblk;
      me.tiles = tiles + sum[1] - t;
      sm.sessions[b] = me;
      if (lead)
        sm.groups[groups + sum[2] - 1] = SharedGroup{sh.of[b], x, members, me.slots, me.units, me.tiles};
    }
    units += all[0];
    tiles += all[1];
    groups += all[2];
  }
  __syncthreads();   // (all have read how many places there are)
  if (tid == 0) *sm.total = make_int4(units, groups, tiles, most);
}

// Workgroups: the groups, then a session each.
__global__ __launch_bounds__(TP_THREADS) void tree_prep_shared_kernel(
    const int32_t *__restrict__ tokens, const int32_t *__restrict__ parents,
    const int32_t *__restrict__ prefix_len, int B, int n1, int V, int capacity, SharedArgs sh,
    int QR, int tile_rows, TreeMeta meta, SharedMeta sm,
    int32_t *__restrict__ status) {
  const int w = blockIdx.x;
  if (w == 0) {
    if (B <= 64) group_few(B, QR, sh, tile_rows, sm);
  } else {
    int slots;
    shared_prefix(sh, w - 1, &slots);
    prepare_tree<false>(w - 1, tokens, parents, prefix_len, n1, V, capacity, 0, 0, slots, meta,
                        status);
    if (B > 64) group_one(w - 1, B, sh, sm);
  }
}

}  // namespace

namespace acespec {

hipError_t launch_tree_prep(const int32_t *tokens, const int32_t *parents,
                            const int32_t *prefix_len, int B, int n1, int V, int capacity,
                            TreeMeta meta, int32_t *status, hipStream_t s) {
  if (n1 > TP_THREADS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(tree_prep_kernel<false>, dim3(B), dim3(TP_THREADS), 0, s, tokens, parents,
                     prefix_len, B, n1, V, capacity, 0, 0, meta, status);
  return hipGetLastError();
}

hipError_t launch_tree_prep_quant(const int32_t *tokens, const int32_t *parents,
                                  const int32_t *prefix_len, int B, int n1, int V, int capacity,
                                  int window, int sinks, TreeMeta meta, int32_t *status,
                                  hipStream_t s) {
  if (n1 > TP_THREADS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(tree_prep_kernel<true>, dim3(B), dim3(TP_THREADS), 0, s, tokens, parents,
                     prefix_len, B, n1, V, capacity, window, sinks, meta, status);
  return hipGetLastError();
}

hipError_t launch_tree_prep_shared(const int32_t *tokens, const int32_t *parents,
                                   const int32_t *prefix_len, int B, int n1, int V, int capacity,
                                   const SharedArgs &sh, int G, int tile_rows, TreeMeta meta,
                                   const SharedMeta &sm, int32_t *status, hipStream_t s) {
  if (n1 > TP_THREADS) return hipErrorInvalidValue;
  hipLaunchKernelGGL(tree_prep_shared_kernel, dim3(1 + B), dim3(TP_THREADS), 0, s, tokens, parents,
                     prefix_len, B, n1, V, capacity, sh, G * n1, tile_rows, meta, sm, status);
  if (B > 64) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(group_kernel, dim3(1), dim3(GT), 0, s, G * n1, tile_rows, sh, sm);
  }
  return hipGetLastError();
}

}  // namespace acespec
