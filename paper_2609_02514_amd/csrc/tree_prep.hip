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

// The groups of any number of sessions, by one workgroup, in the order of their prefixes: a
// session's place follows from counts over all the sessions (B^2 / 128 reads from LDS a thread).
constexpr int GROUP_TILE = 1024;   // sessions in LDS at a time
AS_DEVICE void group_many(int B, int QR, const SharedArgs &sh, int tile_rows, const SharedMeta &sm) {
  __shared__ int s_p[GROUP_TILE];
  const int tid = threadIdx.x;
  int grouped = 0;
  for (int b0 = 0; b0 < B; b0 += TP_THREADS) {
    const int b = b0 + tid;
    int slots = 0, before = 0, rank = 0, members = 0;
    const int p = b < B ? shared_prefix(sh, b, &slots) : -1;
    grouped = 0;
    for (int t0 = 0; t0 < B; t0 += GROUP_TILE) {
      const int n = min(GROUP_TILE, B - t0);
      int unused;
      __syncthreads();
      for (int i = tid; i < n; i += TP_THREADS) s_p[i] = shared_prefix(sh, t0 + i, &unused);
      __syncthreads();
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const int o = s_p[i];
        grouped += o >= 0;
        before += o >= 0 && o < p;
        members += o == p;
        rank += o == p && t0 + i < b;
      }
    }
    if (b >= B) continue;
    sm.sessions[b] = SharedSession{max(slots, 0), p < 0 ? -1 : before + rank, before, 0, 0};
    if (p < 0) continue;
    sm.order[before + rank] = b;
    // a group's entry waits at its first place until the ones before it are known
    sm.groups[before + rank] = SharedGroup{p, before, rank == 0 ? members : 0, slots, 0, 0};
  }
  __syncthreads();
  // one wave closes the gaps, and sums the units
  if (tid < 64) {
    int count = 0, units = 0, tiles = 0, most = 0;
    for (int x0 = 0; x0 < grouped; x0 += 64) {
      const int x = x0 + tid;
      SharedGroup g = x < grouped ? sm.groups[x] : SharedGroup{0, 0, 0, 0, 0, 0};
      const bool lead = g.members > 0;
      const int t = lead ? group_tiles(g.members, QR, tile_rows) : 0, mine = t * ((g.slots + 63) / 64);
      int sum = mine, sum_t = t;   // of this lane's and the ones' before
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(sum, o), vt = __shfl_up(sum_t, o);
        if (tid >= o) {
          sum += v;
          sum_t += vt;
        }
      }
      const uint64_t leads = __ballot(lead);
      g.units = units + sum - mine;
      g.tiles = tiles + sum_t - t;
      if (lead) {
        most = max(most, (g.slots + 63) / 64);
        sm.groups[count + __popcll(leads & ((1ull << tid) - 1))] = g;   // (at most x: read already)
      }
      count += __popcll(leads);
      units += __shfl(sum, 63);
      tiles += __shfl(sum_t, 63);
    }
    for (int o = 1; o < 64; o <<= 1) most = max(most, __shfl_xor(most, o));
    if (tid == 0) *sm.total = make_int4(units, count, tiles, most);
    __threadfence_block();   // (the entries were moved by other lanes)
    // and its members learn what lies before their group
    for (int x = tid; x < grouped; x += 64) {
      int lo = 0, hi = count - 1;   // the last group that begins at place x or before
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (sm.groups[mid].first <= x) lo = mid; else hi = mid - 1;
      }
      SharedSession &m = sm.sessions[sm.order[x]];
      m.units = sm.groups[lo].units;
      m.tiles = sm.groups[lo].tiles;
    }
  }
}

// Workgroups: the groups, then a session each.
__global__ __launch_bounds__(TP_THREADS) void tree_prep_shared_kernel(
    const int32_t *__restrict__ tokens, const int32_t *__restrict__ parents,
    const int32_t *__restrict__ prefix_len, int B, int n1, int V, int capacity, SharedArgs sh,
    int QR, int tile_rows, TreeMeta meta, SharedMeta sm,
    int32_t *__restrict__ status) {
  const int w = blockIdx.x;
  if (w == 0) {
    if (B <= 64)
      group_few(B, QR, sh, tile_rows, sm);
    else
      group_many(B, QR, sh, tile_rows, sm);
  } else {
    int slots;
    shared_prefix(sh, w - 1, &slots);
    prepare_tree<false>(w - 1, tokens, parents, prefix_len, n1, V, capacity, 0, 0, slots, meta,
                        status);
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
  return hipGetLastError();
}

}  // namespace acespec
