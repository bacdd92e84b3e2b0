"""Sessions behind shared prefixes, as their users call them.

Each case is one pass through an operator:

  attend  acespec_attention_shared: tree attention of one layer for a batch whose sessions
          stand behind prefixes that several of them share, computed once for all of them
  share   acespec_share_prefix: a session's first slots taken over into the store of shared
          prefixes, in the order in which the attention reads them
  rotate  acespec_qk_norm_rope: a projection's queries and keys normalised head by head and
          rotated to their positions, the tree's keys and values written into the cache
  fork    acespec_fork_kv: sessions that take over another session's slots, in another cache
          or in the same one

The attention.  Session b has prefix_of[b] = p, the shared prefix that it stands behind (-1:
none), and P own slots behind that prefix's n slots.  Tree row r sits at position n + P +
depth(r) and sees the n shared slots, the P own ones, its ancestors and itself.

The store.  Records of 64 slots, in fp16 for a bf16 model.  With bits of a slot's number in its
record k, s4, s3, s2, ss (1, 1, 1, 1 and 2 of them) and a head dim's number 16 s + 8 h + e, keys
are ordered [k][s][h][s4][s2][s3][ss][e]; behind them the values, a slot's number being 32 k +
16 j + 8 h + e and a head dim's 32 d + r, [k][j][d][h][r][e].  An fp32 model's record is
[64][head_dim] keys and [head_dim][64] values.  Slots of the last record behind a prefix's end
are 0.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False  # True: the framework's kernels; False: the plain forms below

DEV = "cuda"
BLOCK = 64

# Query heads, kv heads, head dim of the decoder shapes the repository's workloads use.
HEADS = {"tiny": (4, 4, 64), "1b": (32, 8, 64), "8b": (32, 8, 128), "70b": (64, 8, 128)}


def listed():
    return [
        # Two sessions of the small fp32 model behind one prompt: latency is everything.
        attend("attend_tiny_f32", "tiny", B=2, P=1, S=128, T=40, shape="chain_sib", a=4, b=1, dtype="f32"),
        # Plain decoding behind one system prompt: one token a session.
        attend("attend_one_token", "8b", B=64, P=1, S=8192, T=512, ragged=True, shape="chain", a=0),
        # The headline batch, 17 rows a session, behind one system prompt.
        attend("attend_8b", "8b", B=64, P=1, S=8192, T=512, ragged=True, shape="widths"),
        # Eight samples of one prompt, as they start: nothing of their own yet.
        attend("attend_samples", "8b", B=8, P=1, S=2000, T=0, shape="widths"),
        # A serving batch of the 1B-class model: six tenants' prompts, some sessions with none.
        attend("attend_tenants", "1b", B=48, P=6, S=4000, T=300, ragged=True, loose=True, shape="chain_sib", a=8, b=1),
        # Many questions about one long document, eight query heads a kv head, wide trees.
        attend("attend_document", "70b", B=32, P=1, S=16384, T=512, ragged=True, shape="fanout"),
        # Two system prompts of some layers, as they are taken over after their prefill.
        dict(name="share_8b", call="share", L=8, B=4, P=2, Hkv=8, hd=128, S=8192, ragged=True, dtype="bf16"),
        # The small fp32 model's.
        dict(name="share_tiny_f32", call="share", L=2, B=2, P=1, Hkv=4, hd=64, S=137, ragged=False, dtype="f32"),
        # One layer's projection of the headline batch.
        rotate("rotate_8b", "8b", B=64, P=1, S=8192, T=512, shape="widths"),
        # One token of one session: latency again.
        rotate("rotate_one_token", "70b", B=1, P=1, S=2000, T=100, shape="chain", a=0),
        # Beam search: sixteen rows continue four of the sessions, some layers.
        fork("fork_beams", L=8, Hkv=8, hd=128, source=4, B=16, S=2048, ragged=True),
        # A batch of the small fp32 model closes its gaps, in place.
        fork("fork_gaps_f32", L=2, Hkv=4, hd=64, source=0, B=4, S=137, dtype="f32"),
    ]


def attend(name, model, B, P, S, T, shape, a=0, b=0, ragged=False, loose=False, dtype="bf16", heads=None):
    H, Hkv, hd = heads or HEADS[model]
    c = dict(call="attend", H=H, Hkv=Hkv, hd=hd, B=B, P=P, S=S, T=T, ragged=ragged, loose=loose,
             shape=shape, a=a, b=b, dtype=dtype)
    return dict(c, name=name) if name else c


def rotate(name, model, B, P, S, T, shape, a=0, b=0, ragged=True, loose=False, dtype="bf16", heads=None):
    return dict(attend(name, model, B, P, S, T, shape, a, b, ragged, loose, dtype, heads), call="rotate")


def fork(name, L, Hkv, hd, source, B, S, ragged=False, cut=0, dtype="bf16"):
    """source: sessions of the cache that is copied from, 0 for the same cache; cut: up to so
    many of a session's first slots are left out."""
    c = dict(call="fork", L=L, Hkv=Hkv, hd=hd, source=source, B=B, S=S, ragged=ragged, cut=cut, dtype=dtype)
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.random()
    Hkv, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    f32 = rng.random() < 0.2
    if kind < 0.68:
        shape, a, b = rng.choice([("widths", 0, 0), ("chain", rng.randint(0, 24), 0),
                                  ("chain_sib", rng.randint(1, 8), rng.randint(0, 7)),
                                  ("random", rng.randint(1, 64), 0), ("fanout", 0, 0)])
        G = rng.choice([1, 2, 4] if f32 else [1, 2, 4, 7, 8])
        B = _log(rng, 1, 4 if f32 else 64)
        P = min(B, _log(rng, 1, 8))
        rows = len(_parents(dict(B=1, shape=shape, a=a, b=b), 0)[0])
        make = attend if kind < 0.5 else rotate
        most = 1024 if f32 else max(64, min(16384, 8 * 10 ** 9 // (B * rows * Hkv * G * hd)))
        return make("", "", B=B, P=P, S=_log(rng, 1, most), T=_log(rng, 1, max(2, min(1024, most))) - 1,
                    shape=shape, a=a, b=b, ragged=rng.random() < 0.6, loose=rng.random() < 0.3,
                    dtype="f32" if f32 else "bf16", heads=(Hkv * G, Hkv, hd))
    L, B, dtype = _log(rng, 1, 16), _log(rng, 1, 16), "f32" if f32 else "bf16"
    S = _log(rng, 1, max(64, min(8192, (1 << 18) // (L * B * Hkv))))
    if kind < 0.84:
        return dict(call="share", L=L, B=B, P=_log(rng, 1, B), Hkv=Hkv, hd=hd, S=S,
                    ragged=rng.random() < 0.6, dtype=dtype)
    return fork("", L=L, Hkv=Hkv, hd=hd, source=rng.choice([0, 1, _log(rng, 1, 16)]), B=B, S=S,
                ragged=rng.random() < 0.6, cut=rng.choice([0, 0, S]), dtype=dtype)


# --------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _held(case):
    """The type of the store."""
    return torch.float32 if case["dtype"] == "f32" else torch.float16


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1_000_003 + stream * 10_007) & 0x7FFF_FFFF_FFFF_FFFF)
    return g


def _parents(case, seed):
    """[B][N + 1] parent rows, -1 for the root."""
    B, a, b = case["B"], case["a"], case["b"]
    if case["shape"] == "random":  # a tree of its own for each session, a nodes
        r = random.Random(seed)
        return [[-1] + [r.randint(max(0, i - 9), i - 1) for i in range(1, a + 1)]
                for _ in range(B)]
    if case["shape"] == "widths":  # widths 2, 4, 5, 5: 16 nodes
        p = [-1, 0, 0, 1, 1, 2, 2, 3, 3, 4, 5, 6, 7, 7, 8, 9, 10]
    elif case["shape"] == "chain":
        p = list(range(-1, a))
    else:  # a main chain, siblings of its nodes as leaves
        sib = [b] * a if case["shape"] == "chain_sib" else [4, 4, 3, 3, 3, 3, 2, 2]
        p, main = [-1], 0
        for n in sib:
            row = len(p)
            p += [main] * (1 + n)
            main = row
    return [p] * B


def _keys_values(case, rows, slots, g):
    """Keys [rows, slots, hd], whose channels differ in spread and mean, and values
    [rows, hd, slots]."""
    hd, dt = case["hd"], _dt(case)
    k = torch.randn((rows, slots, hd), generator=g, device=DEV, dtype=dt)
    spread = torch.empty(hd, device=DEV).uniform_(0.5, 1.5, generator=g).to(dt)
    mean = torch.empty(hd, device=DEV).uniform_(-0.5, 0.5, generator=g).to(dt)
    k.mul_(spread).add_(mean)
    v = torch.randn((rows, hd, slots), generator=g, device=DEV, dtype=dt)
    return k, v


def _lengths(r, most, ragged, n):
    return [r.randint((most + 1) // 2, most) if ragged else most for _ in range(n)]


def _layout(case):
    """Slots of each prefix, own slots of each session and the prefix it stands behind: the same
    for every seed."""
    c = case
    r = random.Random(1000 * c["S"] + c["B"])
    held = _lengths(r, c["S"], c["ragged"], c["P"])
    mine = _lengths(r, c["T"], c["ragged"], c["B"])
    of = [b % c["P"] for b in range(c["B"])]
    r.shuffle(of)
    if c["loose"]:
        of = [-1 if r.random() < 0.2 else p for p in of]
    return held, mine, of


def _moves(case):
    """Of a fork or a take-over: each source's slots, each receiver's source (-1: none) and the
    first slot that it takes (a fork) or how many (a take-over)."""
    c = case
    r = random.Random(1000 * c["S"] + 10 * c["L"] + c["B"])
    if c["call"] == "share":
        S = _lengths(r, c["S"], c["ragged"], c["B"])
        frm = r.sample(range(c["B"]), c["P"])
        return S, frm, [r.randint((S[s] + 1) // 2, S[s]) if c["ragged"] else S[s] for s in frm]
    n = c["source"] or c["B"]
    S = _lengths(r, c["S"], c["ragged"], n)
    if c["source"]:
        frm = [r.randrange(n) if r.random() < 0.9 else -1 for _ in range(c["B"])]
    else:  # the last sessions close gaps in front
        frm = [-1] * n
        gaps = sorted(r.sample(range(n), n // 3 if n < 4 else max(1, n // 4)))
        left = [b for b in range(n) if b not in gaps]
        for g in gaps:
            if left and left[-1] > g:
                frm[g] = left.pop()
    return S, frm, [r.randint(0, min(c["cut"], S[f])) if f >= 0 else 0 for f in frm]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _up(n, to):
    return max(1, -(-n // to)) * to


def prepare(case, seed):
    c, g = case, _gen(seed, 0)
    B, Hkv, hd, dt = c["B"], c["Hkv"], c["hd"], _dt(c)
    s = SimpleNamespace(case=dict(c), status=_ints([0] * B))
    L, H, N, most = c.get("L", 1), c.get("H", Hkv), 0, B
    if c["call"] in ("attend", "rotate"):
        par = _parents(c, seed)
        N, P = len(par[0]) - 1, c["P"]
        s.parents, s.n1 = _ints(par), N + 1
        s.held, s.mine, s.of = _layout(c)
        s.len, s.prefix, s.prefix_of = _ints(s.held), _ints(s.mine), _ints(s.of)
        s.cap, s.scap = _up(max(s.mine) + s.n1, 64), _up(max(s.held), BLOCK)
        k, v = _keys_values(c, B * Hkv, s.cap, g)
        s.k, s.v = k.view(1, B, Hkv, s.cap, hd), v.view(1, B, Hkv, hd, s.cap)
        s.blocks = torch.zeros((1, P, Hkv, s.scap // BLOCK, 2 * BLOCK * hd), dtype=_held(c), device=DEV)
        s.q = torch.randn((B, s.n1, H, hd), generator=g, device=DEV, dtype=dt)
        s.out = torch.empty_like(s.q)
        if c["call"] == "attend":
            for p in range(P):
                k, v = _keys_values(c, Hkv, s.scap, g)
                k[:, s.held[p]:], v[..., s.held[p]:] = 0, 0
                s.blocks[0, p] = _records(k, v, _held(c))
        else:
            s.qkv = torch.randn((B, s.n1, (H + 2 * Hkv) * hd), generator=g, device=DEV, dtype=dt).mul_(3)
            s.q_gain, s.k_gain = (torch.empty(hd, device=DEV).uniform_(0.5, 2, generator=g).to(dt)
                                  for _ in range(2))
    else:
        s.S, s.frm, s.cut = _moves(c)
        n = len(s.S)
        s.cap = _up(max(s.S), 64)
        s.prefix, s.take, s.mark = _ints(s.S), _ints(s.frm), _ints(s.cut)
        k, v = _keys_values(c, L * n * Hkv, s.cap, g)
        s.k, s.v = k.view(L, n, Hkv, s.cap, hd), v.view(L, n, Hkv, hd, s.cap)
        most = max(n, B)
        if c["call"] == "share":
            s.blocks = torch.zeros((L, c["P"], Hkv, s.cap // BLOCK, 2 * BLOCK * hd), dtype=_held(c), device=DEV)
            s.len, s.new = _ints([0] * c["P"]), _ints([0] * c["P"])
            s.scap = s.cap
        else:
            s.dk, s.dv, s.dcap, s.dlen = s.k, s.v, s.cap, s.prefix
            if c["source"]:
                s.dcap = s.cap + 64
                s.dk = torch.ones((L, B, Hkv, s.dcap, hd), dtype=dt, device=DEV)
                s.dv = torch.ones((L, B, Hkv, hd, s.dcap), dtype=dt, device=DEV)
                s.dlen = _ints([1] * B)
            s.new = _ints([0] * B)
    if own:
        from paper_2609_02514_amd import acespec as ac
        s.ver = ac.Verifier(L, 64, H, Hkv, hd, 64, 64, c["dtype"], most, N)
        if c["call"] != "fork":
            s.shared = ac.SharedPrefix(s.blocks, s.scap, s.len)
    return s


# --------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------


def run(s):
    c = s.case
    if c["call"] == "attend":
        if own:
            s.ver.attention_shared(s.shared, s.prefix_of, s.k, s.v, s.cap, s.prefix, 0, s.q, s.parents, s.out, s.status)
            return s.out
        return _attend(s)
    if c["call"] == "rotate":
        if own:
            s.ver.qk_norm_rope(s.qkv, s.q_gain, s.k_gain, s.k, s.v, s.cap, s.prefix, 0, s.parents, s.out, s.status,
                               s.shared, s.prefix_of)
            return dict(q=s.out, k=s.k, v=s.v)
        return _rotate(s)
    if c["call"] == "share":
        if own:
            s.ver.share_prefix(s.k, s.v, s.cap, s.prefix, s.take, s.shared, s.new, s.mark)
            return dict(blocks=s.blocks, len=s.new)
        return _share(s)
    if own:
        s.ver.fork_kv(s.k, s.v, s.cap, s.prefix, s.dk, s.dv, s.dcap, s.dlen, s.take, s.new, s.mark)
        return dict(k=s.dk, v=s.dv, len=s.new)
    return _fork(s)


# --------------------------------------------------------------------------------------
# The plain forms
# --------------------------------------------------------------------------------------


def _records(k, v, held):
    """Records [rows, slots / 64, 128 hd] of keys [rows, slots, hd] and values [rows, hd, slots]."""
    rows, slots, hd = k.shape
    nb = slots // BLOCK
    k, v = k.to(held), v.to(held)
    if held == torch.float32:
        k, v = k.reshape(rows, nb, -1), v.view(rows, hd, nb, BLOCK).transpose(1, 2).reshape(rows, nb, -1)
    else:
        k = k.view(rows, nb, 2, 2, 2, 2, 4, hd // 16, 2, 8).permute(0, 1, 2, 7, 8, 3, 5, 4, 6, 9).reshape(rows, nb, -1)
        v = v.view(rows, hd // 32, 32, nb, 2, 2, 2, 8).permute(0, 3, 4, 5, 1, 6, 2, 7).reshape(rows, nb, -1)
    return torch.cat([k, v], -1)


def _unpacked(blocks, hd):
    """Keys [rows, slots, hd] and values [rows, hd, slots] in 32 bits."""
    rows, nb, n = blocks.shape
    k, v = blocks.float().view(rows, nb, 2, n // 2).unbind(2)
    if blocks.dtype == torch.float32:
        return k.reshape(rows, -1, hd), v.reshape(rows, nb, hd, BLOCK).transpose(1, 2).reshape(rows, hd, -1)
    k = k.reshape(rows, nb, 2, hd // 16, 2, 2, 2, 2, 4, 8).permute(0, 1, 2, 5, 7, 6, 8, 3, 4, 9)
    v = v.reshape(rows, nb, 2, 2, hd // 32, 2, 32, 8).permute(0, 4, 6, 1, 2, 3, 5, 7)
    return k.reshape(rows, nb * BLOCK, hd), v.reshape(rows, hd, nb * BLOCK)


def _reach(parents):
    """[B, n1, n1]: whether row j is row r's ancestor or r itself."""
    n1 = parents.shape[1]
    reach = torch.eye(n1, device=DEV) + (parents.long().unsqueeze(-1) == torch.arange(n1, device=DEV))
    for _ in range(6):  # 64 generations
        reach = (reach @ reach).clamp_max(1)
    return reach > 0


def _softmax_values(z, v):
    """softmax(z) v^T for scores z [m, rows, slots] and values [m, hd, slots]."""
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    z.div_(z.sum(-1, keepdim=True))
    return torch.matmul(z, v.transpose(1, 2).contiguous())


def _attend(s):
    c, n1, cap = s.case, s.n1, s.cap
    B, H, Hkv, hd = c["B"], c["H"], c["Hkv"], c["hd"]
    G = H // Hkv
    out = torch.empty((B, Hkv, n1 * G, hd), device=DEV)
    q = s.q.float().view(B, n1, Hkv, G, hd).transpose(1, 2).reshape(B, Hkv, n1 * G, hd) / math.sqrt(hd)
    # of the own slots: the prefix, and the tree's rows as far as they are ancestors
    t = torch.arange(cap, device=DEV).view(1, 1, cap)
    P = s.prefix.long().view(B, 1, 1)
    row = (t - P).clamp(0, n1 - 1).expand(B, n1, cap)
    seen = (t < P) | ((t < P + n1) & _reach(s.parents).gather(2, row))
    seen = seen.view(B, 1, n1, 1, cap).expand(B, 1, n1, G, cap).reshape(B, 1, n1 * G, cap)
    for p in range(-1, c["P"]):
        b = [i for i in range(B) if s.of[i] == p]
        if not b:
            continue
        k, v = s.k[0, b].float(), s.v[0, b].float()
        qb = q[b]
        z = torch.matmul(qb, k.transpose(2, 3).contiguous()).masked_fill_(~seen[b], -math.inf)
        if p >= 0:  # all the sessions' rows against the prefix in one product
            n, m = s.held[p], len(b)
            ks, vs = _unpacked(s.blocks[0, p], hd)
            ks, vs = ks[:, :n], vs[..., :n]
            zs = torch.matmul(qb.transpose(0, 1).reshape(Hkv, -1, hd), ks.transpose(1, 2).contiguous())
            z = torch.cat([zs.view(Hkv, m, n1 * G, n).transpose(0, 1), z], -1)
            z = z.sub_(z.amax(-1, keepdim=True)).exp_()
            z.div_(z.sum(-1, keepdim=True))
            o = torch.matmul(z[..., :n].transpose(0, 1).reshape(Hkv, -1, n), vs.transpose(1, 2).contiguous())
            o = o.view(Hkv, m, n1 * G, hd).transpose(0, 1) + torch.matmul(z[..., n:], v.transpose(2, 3).contiguous())
        else:
            o = _softmax_values(z.flatten(0, 1), v.flatten(0, 1)).view(len(b), Hkv, n1 * G, hd)
        out[b] = o
    return out.view(B, Hkv, n1, G, hd).transpose(1, 2).reshape(B, n1, H, hd).to(s.q.dtype)


def _rotate(s):
    c, n1 = s.case, s.n1
    B, H, Hkv, hd = c["B"], c["H"], c["Hkv"], c["hd"]
    x = s.qkv.float().view(B, n1, H + 2 * Hkv, hd)
    heads = x[:, :, :H + Hkv]
    gain = torch.cat([s.q_gain.float().expand(H, hd), s.k_gain.float().expand(Hkv, hd)])
    y = heads * torch.rsqrt(heads.square().mean(-1, keepdim=True) + 1e-5) * gain
    shared = torch.where(s.prefix_of >= 0, s.len[s.prefix_of.clamp_min(0).long()], 0)
    pos = (shared + s.prefix).view(B, 1) + _reach(s.parents).sum(-1) - 1
    freq = 10000.0 ** (-2 * torch.arange(hd // 2, device=DEV, dtype=torch.float64) / hd)
    angle = pos.double().unsqueeze(-1) * freq
    cos, sin = angle.cos().float().unsqueeze(2), angle.sin().float().unsqueeze(2)
    y1, y2 = y[..., :hd // 2], y[..., hd // 2:]
    y = torch.cat([y1 * cos - y2 * sin, y2 * cos + y1 * sin], -1).to(s.qkv.dtype)
    t = torch.arange(s.cap, device=DEV).view(1, s.cap) - s.prefix.view(B, 1)
    tree, row = (t >= 0) & (t < n1), t.clamp(0, n1 - 1).long()
    at = row.view(B, s.cap, 1, 1).expand(B, s.cap, Hkv, hd)
    k = y[:, :, H:].gather(1, at).transpose(1, 2)
    v = x[:, :, H + Hkv:].to(s.qkv.dtype).gather(1, at).permute(0, 2, 3, 1)
    s.k[0] = torch.where(tree.view(B, 1, s.cap, 1), k, s.k[0])
    s.v[0] = torch.where(tree.view(B, 1, 1, s.cap), v, s.v[0])
    return dict(q=y[:, :, :H].contiguous(), k=s.k, v=s.v)


def _share(s):
    L, Hkv, hd = s.case["L"], s.case["Hkv"], s.case["hd"]
    there = torch.arange(s.cap, device=DEV) < s.mark.view(-1, 1)  # [P, cap]
    frm = s.take.long()
    k = s.k[:, frm] * there.view(1, -1, 1, s.cap, 1)
    v = s.v[:, frm] * there.view(1, -1, 1, 1, s.cap)
    s.blocks.copy_(_records(k.view(-1, s.cap, hd), v.view(-1, hd, s.cap), s.blocks.dtype).view(s.blocks.shape))
    return dict(blocks=s.blocks, len=s.mark.clone())


def _fork(s):
    new = s.dlen.clone()
    for b, f in enumerate(s.frm):
        if f < 0:
            continue
        n = s.S[f] - s.cut[b]
        s.dk[:, b, :, :n] = s.k[:, f, :, s.cut[b]:s.S[f]]
        s.dv[:, b, :, :, :n] = s.v[:, f, :, :, s.cut[b]:s.S[f]]
        new[b] = n
    return dict(k=s.dk, v=s.dv, len=new)


def work(case):
    """Inputs read once, outputs written once."""
    c = case
    es, hd, Hkv = 4.0 if c["dtype"] == "f32" else 2.0, c["hd"], c["Hkv"]
    if c["call"] in ("share", "fork"):
        S, frm, mark = _moves(c)
        if c["call"] == "share":
            read = wrote = sum(mark)
        else:
            first = {}
            for f, m in zip(frm, mark):
                first[f] = min(m, first.get(f, m)) if f >= 0 else 0
            read = sum(S[f] - m for f, m in first.items() if f >= 0)
            wrote = sum(S[f] - m for f, m in zip(frm, mark) if f >= 0)
        return dict(bytes=max(2 * es, 2 * es * c["L"] * Hkv * hd * (read + wrote)), flops=0.0)
    held, mine, of = _layout(c)
    B, H, n1 = c["B"], c["H"], len(_parents(c, 0)[0])
    if c["call"] == "rotate":
        return dict(bytes=2 * es * B * n1 * (H + 2 * Hkv) * hd, flops=12.0 * B * n1 * (H + Hkv) * hd)
    used = sum(held[p] for p in set(of) if p >= 0)
    seen = sum(held[p] for p in of if p >= 0) + sum(mine) + B * (n1 + 1) / 2
    return dict(bytes=2 * es * Hkv * hd * (used + sum(mine) + B * n1) + 2 * es * B * n1 * H * hd,
                flops=4.0 * H * hd * n1 * seen)


# --------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# --------------------------------------------------------------------------------------


def _places(hd, packed):
    """Where in a record slot i's head dim d is: of the keys [64, hd], of the values [hd, 64]."""
    i, d = torch.arange(BLOCK, device=DEV).view(-1, 1), torch.arange(hd, device=DEV)
    if not packed:
        return i * hd + d, BLOCK * hd + d.view(-1, 1) * BLOCK + i.view(1, -1)
    j = i % 32
    lane = d % 16 // 8 * 32 + j // 16 * 16 + j // 4 % 2 * 8 + j // 8 % 2 * 4 + j % 4
    k = ((i // 32 * (hd // 16) + d // 16) * 64 + lane) * 8 + d % 8
    i, d = i.view(1, -1), d.view(-1, 1)
    lane = i % 16 // 8 * 32 + d % 32
    return k, BLOCK * hd + ((i // 16 * (hd // 32) + d // 32) * 64 + lane) * 8 + i % 8


def exact(case, seed):
    c = case
    if c["call"] == "attend":
        if c["B"] * c["H"] * len(_parents(c, 0)[0]) * (c["S"] + c["T"]) * c["hd"] > 4e11:
            return None
        return _attend64(c, seed)
    s = prepare(c, seed)
    if c["call"] == "rotate":
        return _rotate64(s)
    if c["L"] * max(c["B"], len(s.S)) * c["Hkv"] * c["hd"] * s.cap > 6e8:
        return None
    if c["call"] == "share":
        at_k, at_v = _places(c["hd"], s.blocks.dtype == torch.float16)
        blocks = torch.zeros(s.blocks.shape, dtype=torch.float64, device=DEV)
        for p, f in enumerate(s.frm):
            for x in range(0, s.cut[p], BLOCK):
                n, rec = min(BLOCK, s.cut[p] - x), blocks[:, p, :, x // BLOCK]
                rec[:, :, at_k[:n].flatten()] = s.k[:, f, :, x:x + n].double().flatten(2)
                rec[:, :, at_v[:, :n].flatten()] = s.v[:, f, :, :, x:x + n].double().flatten(2)
        return dict(blocks=blocks, len=None)
    k, v = s.dk.double(), s.dv.double()
    for b, f in enumerate(s.frm):
        if f >= 0:
            src = torch.arange(s.cut[b], s.S[f], device=DEV)
            k[:, b].index_copy_(2, src - s.cut[b], s.k[:, f].double().index_select(2, src))
            v[:, b].index_copy_(3, src - s.cut[b], s.v[:, f].double().index_select(3, src))
    return dict(k=k, v=v, len=None)


def _lines(par):
    """Each row's ancestors from the root on, and itself."""
    line = [[0]]
    for r in range(1, len(par)):
        line.append(line[par[r]] + [r])
    return line


def _rotate64(s):
    """One row after the other, as complex numbers."""
    c, n1 = s.case, s.n1
    B, H, Hkv, hd = c["B"], c["H"], c["Hkv"], c["hd"]
    x = s.qkv.double().view(B, n1, H + 2 * Hkv, hd)
    k, v = s.k.double(), s.v.double()
    parents = s.parents.tolist()
    pos = [[(s.held[p] if p >= 0 else 0) + m + len(y) - 1 for y in _lines(t)]
           for p, m, t in zip(s.of, s.mine, parents)]
    i = torch.arange(hd // 2, device=DEV, dtype=torch.float64)
    angle = torch.tensor(pos, dtype=torch.float64, device=DEV).unsqueeze(-1) / torch.pow(10000.0, i / (hd // 2))
    turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(2)

    def turned(y, gain):
        y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / hd + 1e-5) * gain.double()
        z = torch.complex(y[..., :hd // 2], y[..., hd // 2:]) * turn
        return torch.cat([z.real, z.imag], -1)

    q, kk = turned(x[:, :, :H], s.q_gain), turned(x[:, :, H:H + Hkv], s.k_gain)
    for b, m in enumerate(s.mine):
        k[0, b, :, m:m + n1] = kk[b].transpose(0, 1)
        v[0, b, :, :, m:m + n1] = x[b, :, H + Hkv:].permute(1, 2, 0)
    return dict(q=q, k=k, v=v)


def _attend64(c, seed):
    """One session and kv head after the other, each over its own line of slots."""
    s = prepare(c, seed)
    H, Hkv, hd, n1 = c["H"], c["Hkv"], c["hd"], s.n1
    G = H // Hkv
    at_k, at_v = _places(hd, s.blocks.dtype == torch.float16)
    parents = s.parents.tolist()
    out = torch.zeros((c["B"], n1, H, hd), dtype=torch.float64, device=DEV)
    for g in range(Hkv):
        rec = s.blocks[0, :, g].double()
        front = [(r[:, at_k.flatten()].view(-1, hd)[:n], r[:, at_v.t().flatten()].view(-1, hd)[:n])
                 for r, n in zip(rec, s.held)]
        for b, m in enumerate(s.mine):
            k, v = s.k[0, b, g, :m + n1].double(), s.v[0, b, g, :, :m + n1].double().t().contiguous()
            n = 0
            if s.of[b] >= 0:
                fk, fv = front[s.of[b]]
                n, k, v = len(fk), torch.cat([fk, k]), torch.cat([fv, v])
            hide = torch.zeros((n1, n + m + n1), dtype=torch.bool)
            hide[:, n + m:] = True
            for r, y in enumerate(_lines(parents[b])):
                hide[r, [n + m + j for j in y]] = False
            z = (s.q[b, :, g * G:(g + 1) * G].double().reshape(n1 * G, hd) @ k.t().contiguous()) / math.sqrt(hd)
            z = z.view(n1, G, -1).masked_fill(hide.to(DEV).unsqueeze(1), -math.inf)
            o = torch.softmax(z, -1).view(n1 * G, -1) @ v
            out[b, :, g * G:(g + 1) * G] = o.view(n1, G, hd)
    return out
