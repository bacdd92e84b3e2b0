"""Shared prefixes read by tiles whose parts the own slots' kernel joins itself (large batches), malformed
sessions on the ways by tiles, packed weights behind prefixes, and what a context takes.  Which way a
call takes is counted by the kernels of its captured graph, and sizes follow the card's CUs."""
import ctypes as C
import math
import random

import pytest
import torch

import synth
from oracle import model as om
from tests import harness as hz
from tests import shared_ref as sr
from tests.test_gpu_shared import DT, bound, gains, i32, random_cache, random_parents, start, store, up64, verifier, workload

pytestmark = pytest.mark.gpu


def cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def large():
    """Slots of a store that a session would not go over by itself: more than 36 chunks for each of
    two workgroups a CU."""
    return 37 * 64 * 2 * cus()


def joining_sessions(G, Hkv, N):
    """The fewest sessions whose parts the own slots' kernel joins: 3 G B (N + 1) rows a kv head for
    256 rows of each of its workgroups."""
    return -(-max(1, cus() // Hkv) * 256 // (3 * G * (N + 1)))


def kernels_of(call):
    """The kernels of a captured call, which is replayed, too."""
    with open("/proc/self/maps") as f:
        lib = C.CDLL(next(l.split()[-1] for l in f if "libamdhip64" in l))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph(keep_graph=True)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    n = C.c_size_t(0)
    assert lib.hipGraphGetNodes(C.c_void_p(graph.raw_cuda_graph()), None, C.byref(n)) == 0
    graph.instantiate()
    graph.replay()
    torch.cuda.synchronize()
    return n.value


BY_TILES = 2                 # preparation, tiles; the groups of more than 64 sessions take a kernel more
JOINED_THERE, JOINED_APART = 1, 2


def check(hd, H, Hkv, held, of, mine, N, seed, kernels, cap=None, scap=0, poison=None, sample=None, bad=None):
    """bf16 attention against 64 bits (a sample of the sessions), eager, repeated and captured.
    kernels: how many the call takes.  bad: {session: (prefix_of, own slots or None)} and
    {-1 - prefix: length}: what is malformed."""
    r, B, n1, bad = random.Random(seed), len(of), N + 1, bad or {}
    cap = cap or up64(max(mine) + n1)
    shared, sk, sv = store(1, held, Hkv, hd, "bf16", seed, scap)
    k, v = random_cache(1, B, Hkv, cap, hd, "bf16", seed + 1)
    ver = verifier(1, B, H, Hkv, hd, "bf16", N)
    parents = [random_parents(r, N) for _ in range(B)]
    q = torch.randn(B, n1, H, hd, generator=torch.Generator().manual_seed(seed + 2)).to(torch.bfloat16).cuda()
    for b, m in enumerate(mine):
        k[:, b, :, m + n1:], v[:, b, :, :, m + n1:] = math.nan, math.nan
    if poison:
        poison(sk, sv, k, v, parents, shared)
    lens, where, own, trees = list(held), list(of), list(mine), [list(p) for p in parents]
    for at, what in bad.items():
        if at < 0:
            lens[-1 - at] = what
        else:
            where[at] = what[0]
            if what[1] is not None:
                own[at] = what[1]
            if N > 1 and what == (of[at], None):
                trees[at][2] = 2                     # its own parent
    wrong = [b for b in range(B) if b in bad or (of[b] >= 0 and lens[of[b]] != held[of[b]])]
    shared.len = i32(lens)
    args = i32(where), k, v, cap, i32(own), 0, q, i32(trees)
    out, status = torch.full_like(q, -77.0), i32([9] * B)
    hz.log(f"attention_shared hd={hd} H={H}/{Hkv} held={lens[:8]} B={B} N={N} scap={scap} malformed={len(wrong)}")
    ver.attention_shared(shared, *args, out, status)
    torch.cuda.synchronize()
    from paper_2609_02514_amd.acespec import ACESPEC_EBADTREE
    assert status.tolist() == [ACESPEC_EBADTREE if b in wrong else 0 for b in range(B)]
    worst = 0.0
    for b in sample or range(B):
        if b in wrong:
            continue
        n, p, m = held[of[b]] if of[b] >= 0 else 0, max(of[b], 0), mine[b]
        want, mag, big = sr.attend(q[b], (sk[0, p, :, :n], sv[0, p, :, :, :n].transpose(1, 2)),
                                   k[0, b, :, :m + n1], v[0, b, :, :, :m + n1], m, parents[b])
        got, fine = out[b].double(), want.isfinite()
        assert torch.equal(fine, got.isfinite()), (b, fine.logical_xor(got.isfinite()).nonzero()[:5])
        err = (got - want).abs()[fine] / bound("bf16", want, mag, big, hd)[fine]
        worst = max(worst, float(err.max()) if err.numel() else 0.0)
    hz.log(f"  worst error: {worst:.3f} of its bound")
    assert worst <= 1.0
    good = torch.tensor([b for b in range(B) if b not in wrong], device="cuda")
    again = torch.full_like(q, 55.0)
    assert kernels_of(lambda: ver.attention_shared(shared, *args, again, status)) == kernels
    assert torch.equal(again[good].nan_to_num(), out[good].nan_to_num())
    again.fill_(33.0)
    ver.attention_shared(shared, *args, again, status)
    torch.cuda.synchronize()
    assert torch.equal(again[good].nan_to_num(), out[good].nan_to_num())
    ver.close()


def spread(B, held, seed):
    """Sessions behind all prefixes, some behind none, in no order; own slots up to 200."""
    r = random.Random(seed)
    of = [b % (len(held) + 1) - 1 for b in range(B)]
    r.shuffle(of)
    return of, [r.choice([0, 1, 63, 64, r.randint(0, 200)]) for _ in range(B)]


# ---- parts that the own slots' kernel joins ---------------------------------------------------


@pytest.mark.parametrize("hd, G, Hkv, N", [
    (128, 4, 8, 16),      # five tiles of 16 rows, two workgroups a CU, two stages
    (64, 4, 8, 16),       # the same of head dim 64, four stages
    (128, 8, 8, 16),      # nine tiles: 16 waves
    (64, 8, 4, 16),
    (128, 8, 8, 32),      # 264 rows: eight tiles of 32 and a remainder of 8 rows in quarter units
    (64, 8, 8, 64),       # 520 rows: two groups of 260, with a remainder of 4
    (128, 8, 8, 63),      # 512 rows: two groups of 256, none
    (128, 5, 8, 64),      # 325 rows: groups of 163
    (128, 16, 8, 0),      # single tokens of many sessions
    (64, 7, 8, 2)])
@pytest.mark.parametrize("poisoned", [False, True])
def test_parts_join_where_the_own_slots_are(hd, G, Hkv, N, poisoned):
    held = [5200, 64, 1, 1000, 2111]
    B = joining_sessions(G, Hkv, N) + 1
    of, mine = spread(B, held, N)
    sample = random.Random(N).sample(range(B), min(B, 12))

    def poison(sk, sv, k, v, parents, shared):
        leaf, a, b, c = N, sample[0], sample[1], sample[2]
        v[0, a, 0, 3, mine[a] + leaf] = math.nan
        v[0, a, 1, 5, mine[a] + (1 if N else 0)] = math.inf
        k[0, b, 0, mine[b] + leaf, 2] = math.nan
        v[0, c, 1, 1, mine[c] + N // 2] = -math.inf
        sv[0, 3, 0, 9, 20] = math.inf                # seen by all behind prefix 3
        pk, pv = sk.clone(), sv.clone()
        for p, n in enumerate(held):
            pk[:, p, :, n:], pv[:, p, :, :, n:] = math.nan, math.nan
        shared.blocks[:] = sr.records(pk, pv, True)

    check(hd, G * Hkv, Hkv, held, of, mine, N, 40 + N, BY_TILES + JOINED_THERE + (B > 64), cap=320,
          poison=poison if poisoned else None, sample=sample)


def test_parts_join_apart_one_session_short():
    """One session fewer, whose parts a kernel of their own joins."""
    for hd, G, Hkv, N in ((128, 4, 8, 16), (64, 8, 8, 32)):
        B = joining_sessions(G, Hkv, N) - 1
        of, mine = spread(B, [5200, 300], N)
        check(hd, G * Hkv, Hkv, [5200, 300], of, mine, N, 50, BY_TILES + JOINED_APART, cap=320, scap=12032,
              sample=random.Random(N).sample(range(B), 8))


# ---- what fp16 keeps --------------------------------------------------------------------------


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("N", [0, 16, 64])
def test_values_below_fp16s_normal_range_keep_multiples_of_its_least(hd, tiles, N):
    """Keys and values that are multiples of 2^-24 below 2^-14, as the store and the products hold them.
    Keys: queries of some 2^14 make scores that weights show.  Values: the
    same 3 * 2^-24 in every slot, whose mean is itself."""
    from paper_2609_02514_amd.acespec import SharedPrefix
    H, Hkv, held, mine, B, n1 = 8, 2, 200, [0, 70, 33], 3, N + 1
    cap = up64(max(mine) + n1)
    g = torch.Generator().manual_seed(hd + N)

    def least(*shape):
        return (torch.randint(-255, 256, shape, generator=g) * 2.0 ** -24).to(torch.bfloat16).cuda()
    k, v = least(1, B, Hkv, cap, hd), torch.randn(1, B, Hkv, hd, cap, generator=g).to(torch.bfloat16).cuda()
    sk, sv = least(1, 1, Hkv, up64(held), hd), torch.randn(1, 1, Hkv, hd, up64(held), generator=g).to(torch.bfloat16).cuda()
    q = (torch.randn(B, n1, H, hd, generator=g) * 2.0 ** 14).to(torch.bfloat16).clamp(-60000, 60000).cuda()
    ver, r = verifier(1, B, H, Hkv, hd, "bf16", N), random.Random(N)
    parents = [random_parents(r, N) for _ in range(B)]
    shared = SharedPrefix.alloc(1, 1, Hkv, hd, large() if tiles else held, "bf16")
    for same in (False, True):
        new = i32([0])
        if same:
            v.fill_(3 * 2.0 ** -24)
            sv.fill_(3 * 2.0 ** -24)
        ver.share_prefix(sk, sv, up64(held), i32([held]), i32([0]), shared, new)
        shared.len = new
        out, status = torch.full_like(q, -77.0), i32([9] * B)
        ver.attention_shared(shared, i32([0] * B), k, v, cap, i32(mine), 0, q, i32(parents), out, status)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * B
        for b, m in enumerate(mine):
            want, mag, big = sr.attend(q[b], (sk[0, 0, :, :held], sv[0, 0, :, :, :held].transpose(1, 2)),
                                       k[0, b, :, :m + n1], v[0, b, :, :, :m + n1], m, parents[b])
            if same:   # weights off by 2^-11 and the output by 2^-8, of which the mean keeps both
                tol = want.abs() * (2.0 ** -11 + 2.0 ** -8 + 2.0 ** -18)
            else:
                tol = bound("bf16", want, mag, big, hd)
                flat, _, _ = sr.attend(q[b], (0 * sk[0, 0, :, :held], sv[0, 0, :, :, :held].transpose(1, 2)),
                                       0 * k[0, b, :, :m + n1], v[0, b, :, :, :m + n1], m, parents[b])
                assert float(((flat - want).abs() / tol).max()) > 4   # (keys taken for zeros would show)
            assert bool(((out[b].double() - want).abs() <= tol).all()), (same, b)
    ver.close()


# ---- malformed sessions -----------------------------------------------------------------------


@pytest.mark.parametrize("lens", [{}, {-3: 1 << 30}, {-3: -5}, {-1: -1, -2: 1 << 30}, {-1: -1, -2: -1, -3: -1}])
@pytest.mark.parametrize("B", [9, 64, 65, 130])
def test_malformed_sessions_by_tiles(B, lens):
    """Prefixes that do not exist, lengths that are none, trees that are none and own lengths without
    room: flagged, and the groups of the others as if these were not there."""
    held = [100, 300, 64]
    of, mine = spread(B, held, B)
    bad = dict(lens)
    bad.update({1: (3, None), 2: (-2, None), 4: (1 << 30, None), 5: (of[5], -1), 6: (of[6], 320 - 4), 7: (of[7], None)})
    check(64, 4, 1, held, of, mine, 4, 60, BY_TILES + JOINED_APART + (B > 64), cap=320, scap=large(), bad=bad)


def test_malformed_sessions_among_more_than_a_workgroups_places():
    """1500 sessions behind 12 prefixes, of which a third is malformed: their places lie between the others'."""
    r = random.Random(1)
    held = [2400, 1, 64, 65, 100, 300, 2300, 5, 700, 20, 30, 40]
    of = [r.randint(-1, 11) for _ in range(1500)]
    bad = {-1: -1, -4: 1 << 20, -7: -(1 << 31), -12: 2 ** 31 - 1}
    bad.update({b: (r.choice([12, -2, 1 << 30, -(1 << 31)]), None) for b in r.sample(range(1500), 40)})
    for cap, joined in ((64, JOINED_APART), ):
        check(64, 1, 1, held, of, [b % 3 for b in range(1500)], 0, 70, BY_TILES + joined + 1, cap=cap, bad=bad,
              sample=r.sample(range(1500), 200), scap=36 * 64 * 4)


def test_malformed_sessions_in_a_joined_batch():
    """The same where the own slots' kernel joins the parts."""
    held = [5200, 64, 1000]
    B = joining_sessions(4, 8, 16) + 1
    of, mine = spread(B, held, 5)
    bad = {-2: -1, 1: (3, None), 3: (-5, None), 8: (of[8], None), 9: (of[9], 320)}
    check(128, 32, 8, held, of, mine, 16, 80, BY_TILES + JOINED_THERE + (B > 64), cap=320, bad=bad,
          sample=[b for b in range(B) if b % 4 < 2])


# ---- the verify step --------------------------------------------------------------------------


@pytest.mark.parametrize("kw, shared_slots", [
    (dict(B=0, H=32, Hkv=8, hd=64, d=256, S=2800, tree="widths_2455"), 2700),   # joined where the own slots are
    (dict(B=4, H=8, Hkv=2, hd=128, d=512), 70)])                                # session by session
@pytest.mark.parametrize("packed, normed", [(True, False), (True, True), (False, True)])
def test_steps_with_packed_weights_behind_one_prefix(kw, shared_slots, packed, normed):
    """All sessions behind session 0's first slots: logits against the 64-bit decoder over these and each
    session's other slots, within 2e-2 of their largest (the verify step's own bound)."""
    from paper_2609_02514_amd.acespec import SharedPrefix, Verifier
    joined = not kw["B"]
    if joined:
        kw = dict(kw, B=joining_sessions(kw["H"] // kw["Hkv"], kw["Hkv"], 16) + 1)
    w = workload("bf16", **kw, ragged=False)
    W, batch, ver = synth.make_weights(w, "cuda"), synth.make_batch(w, "cuda"), Verifier.for_workload(w)
    n1, lens = batch.tokens.shape[1], batch.prefix_len.tolist()
    assert n1 == 17 and min(lens) > shared_slots
    shared, new = SharedPrefix.alloc(w.L, 1, w.Hkv, w.hd, shared_slots, "bf16"), i32([0])
    ver.share_prefix(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, i32([0]), shared, new, i32([shared_slots]))
    shared.len = new
    cap = up64(max(lens) - shared_slots + n1)
    k, v = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in
            ((w.L, w.B, w.Hkv, cap, w.hd), (w.L, w.B, w.Hkv, w.hd, cap)))
    own = i32([0] * w.B)
    ver.fork_kv(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, k, v, cap, i32([0] * w.B), i32(list(range(w.B))), own,
                i32([shared_slots] * w.B))
    norms = gains(w) if normed else None
    outs = [ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True) for _ in range(2)]
    PW = ver.pack_weights(W) if packed else W
    ws = ver.weights_struct(PW)

    def step(o):
        ver.verify_tree_shared(ws, shared, i32([0] * w.B), k, v, cap, own, batch.tokens, batch.parents, batch.q, batch.u,
                               w.T, w.top_p, w.top_k, o, norms)
    hz.log(f"verify_tree_shared B={w.B} packed={packed} normed={normed} own={own.tolist()[:4]}")
    step(outs[0])
    step(outs[1])
    torch.cuda.synchronize()
    assert outs[0]["status"].tolist() == [0] * w.B
    for key in outs[0]:
        assert torch.equal(outs[0][key], outs[1][key]), key
    F64, dims, parents = om.F64Weights(W), om.dims_of(w), batch.parents.tolist()
    n64 = [tuple(om.to_f64(x) for x in pair) for pair in norms] if normed else None
    for b in [0, w.B - 1] if joined else range(w.B):
        at = torch.tensor([0] * shared_slots + [b] * (lens[b] - shared_slots), device="cuda")
        slots = torch.arange(lens[b], device="cuda")
        kpre = [om.to_f64(batch.kv_k[l][at, :, slots]).transpose(1, 0, 2) for l in range(w.L)]
        vpre = [om.to_f64(batch.kv_v[l][at, :, :, slots]).transpose(1, 0, 2) for l in range(w.L)]
        z, _ = sr.forward(F64, dims, kpre, vpre, batch.tokens[b].tolist(), parents[b], lens[b], n64)
        got = outs[0]["logits_out"].view(w.B, n1, w.V)[b].double().cpu().numpy()
        err = abs(got - z).max() / abs(z).max()
        hz.log(f"  session {b}: logits off by {err:.2e} of the largest")
        assert err < 2e-2
    ver.close()


@pytest.mark.parametrize("dtype, tiles", [("bf16", False), ("bf16", True), ("f32", False)])
def test_malformed_sessions_of_a_step(dtype, tiles):
    """A step in which four of six sessions are malformed, each in its way: flagged, nothing of the others'
    caches touched, and the others decide as without them (by tiles, where the prefixes are cut
    elsewhere then, up to a few roundings to fp16 of each layer's activations, 2^-11 each)."""
    from paper_2609_02514_amd.acespec import ACESPEC_EBADTREE, SharedPrefix
    w = workload(dtype, B=6, H=8, Hkv=2, hd=128, d=512)
    W, norms = synth.make_weights(w, "cuda"), gains(w)
    batch, ver, shared, of, k, v, cap, own = start(w, [60, 40, 0, 70, 30, 20])
    if tiles:
        wide = SharedPrefix.alloc(w.L, shared.prefixes, w.Hkv, w.hd, large(), dtype)
        wide.blocks[:, :, :, :shared.blocks.shape[3]] = shared.blocks
        wide.len = shared.len
        shared = wide
    n1, ws, held = batch.tokens.shape[1], ver.weights_struct(W), shared.len.tolist()
    k0, v0 = k.clone(), v.clone()

    def step(of, lens, own, parents):
        outs = ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True)
        shared.len = i32(lens)
        k.copy_(k0)
        v.copy_(v0)
        ver.verify_tree_shared(ws, shared, of, k, v, cap, own, batch.tokens, parents, batch.q, batch.u, w.T, w.top_p,
                               w.top_k, outs, norms)
        torch.cuda.synchronize()
        return outs
    good = step(of, held, own, batch.parents)
    assert good["status"].tolist() == [0] * w.B
    gk, gv = k.clone(), v.clone()
    of2, own2, parents, lens = of.clone(), own.clone(), batch.parents.clone(), list(held)
    of2[1] = shared.prefixes
    lens[of.tolist()[3]] = shared.capacity + 1
    own2[4] = cap - n1 + 1
    parents[5, 3] = 3
    hz.log(f"verify_tree_shared {dtype} tiles={tiles} with malformed sessions")
    bad = step(of2, lens, own2, parents)
    assert bad["status"].tolist() == [0, ACESPEC_EBADTREE, 0, ACESPEC_EBADTREE, ACESPEC_EBADTREE, ACESPEC_EBADTREE]
    for b in (0, 2):
        rows = slice(b * n1, (b + 1) * n1)
        if tiles:
            x, y = good["logits_out"][rows].double(), bad["logits_out"][rows].double()
            assert float((x - y).norm() / x.norm()) < 8 * 2.0 ** -11
            continue
        assert torch.equal(gk[:, b], k[:, b]) and torch.equal(gv[:, b], v[:, b])
        for name, t in good.items():
            at = slice(b, b + 1) if t.shape[0] == w.B else rows
            assert torch.equal(t[at], bad[name][at]), (name, b)
    for b, m in enumerate(own.tolist()):   # beside the tree's slots (where the call takes them to be) nothing changes
        at = min(max(own2.tolist()[b], 0), cap - n1)
        for new, was in ((k[:, b], k0[:, b]), (v[:, b].transpose(2, 3), v0[:, b].transpose(2, 3))):
            assert torch.equal(new[:, :, :at], was[:, :, :at]) and torch.equal(new[:, :, at + n1:], was[:, :, at + n1:])
    ver.close()


# ---- refusals, with tensors of the GPU --------------------------------------------------------


def test_normed_rotation_refuses_each_wrong_tensor_by_its_name():
    B, N, H, Hkv, hd, L = 2, 3, 4, 2, 64, 2
    ver = verifier(L, B, H, Hkv, hd, "bf16", N)
    shared, _, _ = store(L, [70], Hkv, hd, "bf16", 1)
    k, v = random_cache(L, B, Hkv, 128, hd, "bf16", 2)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    good = dict(qkv=torch.zeros(B, N + 1, (H + 2 * Hkv) * hd, **bf), q_gain=torch.ones(hd, **bf),
                k_gain=torch.ones(hd, **bf), kv_k=k, kv_v=v, capacity=128, prefix_len=i32([1, 2]), layer=0, parents=i32([[-1, 0, 1, 2]] * B),
                q_out=torch.zeros(B, N + 1, H, hd, **bf), status=i32([9] * B), shared=shared, prefix_of=i32([0, 0]))
    ver.qk_norm_rope(**good)
    torch.cuda.synchronize()
    assert good["status"].tolist() == [0, 0]
    for name in ("qkv", "q_gain", "k_gain", "kv_k", "kv_v", "prefix_len", "parents", "q_out", "status", "prefix_of"):
        t = good[name]
        for bad in (t.double(), t.cpu(), torch.cat([t, t], -1), torch.cat([t, t], -1)[..., :t.shape[-1]]):
            if bad.is_cuda and bad.dtype == t.dtype and bad.shape == t.shape and bad.is_contiguous():
                continue   # (a vector's first half is itself)
            with pytest.raises(ValueError, match="parents|must be" if name == "parents" else name):
                ver.qk_norm_rope(**dict(good, **{name: bad}))
    ver.close()


# ---- a context --------------------------------------------------------------------------------


def test_a_context_takes_no_memory_of_its_own_for_partial_results():
    """A bf16 model's context is an fp32 one's with activations (the normed rows, queries, attention's
    and feed-forward's outputs) of two bytes instead of four, but for a few numbers a session."""
    from paper_2609_02514_amd.acespec import Verifier
    d, H, Hkv, hd, F, B, N = 8192, 64, 8, 128, 64, 64, 64

    def taken(dtype):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        before = torch.cuda.mem_get_info()[0]
        ver = Verifier(1, d, H, Hkv, hd, F, 64, dtype, B, N)
        n = before - torch.cuda.mem_get_info()[0]
        ver.close()
        return n
    taken("bf16")
    more = taken("bf16") - taken("f32") + B * (N + 1) * (d + 2 * H * hd + F) * 2
    hz.log(f"a bf16 context takes {more / 2**20:.1f} MB more than its types say")
    assert more <= 8 << 20
