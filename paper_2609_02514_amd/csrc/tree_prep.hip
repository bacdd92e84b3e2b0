// Tree preparation: validates each session's drafted tree and derives the per-row data
// the forward pass needs.  All drafted nodes of a session go through the target in one
// pass (Section III-C); a node may attend to the verified context and to its own
// ancestral sequence only, so each row gets the set of its ancestors as a bit mask over
// the drafted rows (the root, row 0, is every row's ancestor and is always visible).
// Positions: siblings share a position, prefix_len + depth; keys/values of row r live
// in cache slot prefix_len + r.
// Over a cache in 4 bits the tree's rows go behind the prefix_len % 32 slots of the tail, and a
// sliding window takes ancestors that are too far back out of a row's set.
#include "common.h"

namespace {

constexpr int TP_THREADS = 128;  // one thread per tree row (at most 65 rows)

// One workgroup per session.  A row's ancestor mask is its own bit and its ancestors'
// (the root carries none); it is built by pointer jumping, every row doubling the span of
// ancestors it has folded in per round (7 rounds cover 65 rows), and the row's depth is
// the mask's population count.
template <bool QUANT>
__global__ __launch_bounds__(TP_THREADS) void tree_prep_kernel(
    const int32_t *__restrict__ tokens, const int32_t *__restrict__ parents,
    const int32_t *__restrict__ prefix_len, int B, int n1, int V, int capacity, int window,
    int sinks, TreeMeta meta, int32_t *__restrict__ status) {
  __shared__ int s_jump[TP_THREADS];
  __shared__ uint64_t s_anc[TP_THREADS];
  const int b = blockIdx.x, r = threadIdx.x;
  const size_t base = (size_t)b * n1;
  const bool in = r < n1;
  const int pr = in ? parents[base + r] : 0;
  const int tk = in ? tokens[base + r] : 0;
  int S = prefix_len[b];
  const bool row_ok = !in || (((r == 0) ? (pr == -1) : (pr >= 0 && pr < r)) && tk >= 0 && tk < V);
  // largest prefix: with QUANT full blocks and a full tail behind them
  const long long most = QUANT ? (long long)capacity + 31 : (long long)capacity - n1;
  const bool ok = __syncthreads_and(row_ok) && S >= 0 && S <= most;
  if (S < 0) S = 0;
  if (S > most) S = (int)most;
  const int p = !in || r == 0 ? -1 : (ok ? pr : r - 1);  // malformed trees become a chain
  s_jump[r] = p < 0 ? 0 : p;
  s_anc[r] = (in && r > 0) ? (1ull << (r - 1)) : 0ull;
  for (int round = 0; round < 7; ++round) {
    __syncthreads();
    const int jr = s_jump[r];
    const uint64_t a = s_anc[r] | s_anc[jr];
    const int jj = s_jump[jr];
    __syncthreads();
    s_anc[r] = a;
    s_jump[r] = jj;
  }
  if (r == 0) {
    meta.sess_S[b] = QUANT ? S & 31 : S;
    status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
  }
  if (!in) return;
  uint64_t anc = s_anc[r];
  const int depth = __popcll(anc);
  if (QUANT && window > 0)
    for (uint64_t rest = anc; rest; rest &= rest - 1) {
      const int j = __builtin_ctzll(rest) + 1, dj = __popcll(s_anc[j]);
      if (depth - dj >= window && S + dj >= sinks) anc &= ~(1ull << (j - 1));
    }
  meta.tok[base + r] = tk < 0 ? 0 : (tk >= V ? V - 1 : tk);
  meta.par[base + r] = p;
  meta.depth[base + r] = depth;
  meta.anc[base + r] = anc;
  meta.pos[base + r] = S + depth;
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

}  // namespace acespec
