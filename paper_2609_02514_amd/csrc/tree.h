// A session's tree inside a workgroup: which rows a row descends from, and the shared prefix that
// the session stands behind.
#pragma once
#include "common.h"

constexpr int TREE_ROWS = 128;   // (at most 65 are in use)
struct TreeSets {
  int jump[TREE_ROWS];
  uint64_t anc[TREE_ROWS];       // bit (j-1) set iff drafted row j is r or an ancestor of r
};

// All threads of the workgroup come here, thread r with row r's parent.  A row's set is its own bit
// and its ancestors' (the root carries none); it is built by pointer jumping, every row doubling
// the span of ancestors it has folded in per round until the span covers n1 rows.  good: the row, and
// what else the caller asks of its session, is well-formed; otherwise the tree becomes a chain and
// the result is false.  *up: the row's parent in the tree as it is taken.  A row's own set is there
// at the end, another's behind a barrier.
AS_DEVICE bool tree_sets(TreeSets &t, int n1, int parent, bool good, int *up) {
  const int r = threadIdx.x;
  const bool in = r < n1, held = r < TREE_ROWS;
  const bool ok = __syncthreads_and(good && (!in || (r == 0 ? parent == -1 : parent >= 0 && parent < r)));
  const int p = !in || r == 0 ? -1 : (ok ? parent : r - 1);
  if (held) {
    t.jump[r] = p < 0 ? 0 : p;
    t.anc[r] = (in && r > 0) ? (1ull << (r - 1)) : 0ull;
  }
  for (int span = 1; span < n1; span *= 2) {
    __syncthreads();
    const int jr = held ? t.jump[r] : 0, jj = t.jump[jr];
    const uint64_t a = held ? t.anc[r] | t.anc[jr] : 0ull;
    __syncthreads();
    if (held) {
      t.anc[r] = a;
      t.jump[r] = jj;
    }
  }
  *up = p;
  return ok;
}

// Session b's shared prefix, -1 where it has none (or an empty or malformed one); *slots its
// length, -1 where malformed.
AS_DEVICE int shared_prefix(const SharedArgs &sh, int b, int *slots) {
  const int p = sh.of[b];
  *slots = p == -1 ? 0 : -1;
  if (p < 0 || p >= sh.P) return -1;
  const int n = sh.len[p];
  if (n < 0 || n > sh.cap) return -1;
  *slots = n;
  return n > 0 ? p : -1;
}

// A call that prepares its trees in the attention itself asks for what session b is, in time,
struct TreeAsked {
  int parent, S, prefix, slots;   // (of this thread's row), own slots, shared prefix and its slots, as they are given
};
AS_DEVICE TreeAsked tree_ask(const TreeArgs &a, const SharedArgs &sh, int b, int n1) {
  TreeAsked x;
  x.parent = (int)threadIdx.x < n1 ? a.parents[(size_t)b * n1 + threadIdx.x] : 0;
  x.S = a.prefix_len[b];
  x.prefix = shared_prefix(sh, b, &x.slots);
  return x;
}
// and makes of it the sets and the session's own slots S, its shared prefix and the slots of it.
// writes: this workgroup leaves the status (and, with meta.anc given, what joins parts of the session
// later) for all of the session's.
struct TreeSession {
  int S, prefix, front;
};
AS_DEVICE TreeSession tree_session(TreeSets &t, const TreeArgs &a, const TreeAsked &x, int b, int n1,
                                   int capacity, bool writes, const TreeMeta &meta) {
  const int r = threadIdx.x, most = capacity - n1;
  int up;
  const bool ok = tree_sets(t, n1, x.parent, x.S >= 0 && x.S <= most && x.slots >= 0, &up);
  const int S = min(max(x.S, 0), most);
  if (writes) {
    if (r == 0) {
      a.status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
      if (meta.anc) meta.sess_S[b] = S;
    }
    if (r < n1 && meta.anc) meta.anc[(size_t)b * n1 + r] = t.anc[r];
  }
  __syncthreads();
  return TreeSession{__builtin_amdgcn_readfirstlane(S), __builtin_amdgcn_readfirstlane(max(x.prefix, 0)),
                     __builtin_amdgcn_readfirstlane(max(x.slots, 0))};
}
