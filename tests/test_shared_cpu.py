"""What the entry points of the shared prefixes refuse, without a GPU: every check runs before
anything is enqueued (the pointers below are never dereferenced)."""
import ctypes as C

import pytest

import paper_2609_02514_amd.acespec as A
from tests.test_quant_cpu import Ctx, cache, refused

G = 1 << 32
P = 0x7F0000000000
FAR = P + 16 * G   # behind the caches of the helpers


def shared(blocks=FAR, prefixes=3, capacity=128, length=FAR + G):
    return A.KVShared(blocks, prefixes, capacity, length)


def ref(s):
    return None if s is None else C.byref(s)


def attention(ctx, sh=None, of=FAR + 2 * G, kv=None, layer=0, q=FAR + 3 * G, parents=FAR + 4 * G, B=4, N=16,
              out=FAR + 5 * G, status=FAR + 6 * G):
    return A.load().acespec_attention_shared(ctx, ref(shared() if sh is None else sh), of, ref(cache() if kv is None else kv),
                                             layer, q, parents, B, N, out, status, None)


def rotate(ctx, sh=None, of=FAR + 2 * G, kv=None, layer=0, qkv=FAR + 3 * G, parents=FAR + 4 * G, B=4, N=16,
           q=FAR + 5 * G, status=FAR + 6 * G, gains=(FAR + 7 * G, FAR + 8 * G), norm=True):
    norm = A.QKNorm(*gains) if norm else None
    sh = shared() if sh is None else sh
    return A.load().acespec_qk_norm_rope(ctx, ref(norm), None if sh is False else ref(sh), of,
                                         ref(cache() if kv is None else kv), layer, qkv, parents, B, N, q, status, None)


def share(ctx, sh=None, kv=None, B=4, frm=FAR + 2 * G, count=FAR + 3 * G, new=FAR + 4 * G):
    return A.load().acespec_share_prefix(ctx, ref(cache() if kv is None else kv), B, ref(shared() if sh is None else sh),
                                         frm, count, new, None)


def fork(ctx, src=None, dst=None, Bs=4, Bd=4, frm=FAR + 2 * G, first=FAR + 3 * G, new=FAR + 4 * G):
    far = cache(FAR + 9 * G, FAR + 10 * G, 128, FAR + 11 * G)
    return A.load().acespec_fork_kv(ctx, ref(cache() if src is None else src), Bs, ref(far if dst is None else dst), Bd,
                                    frm, first, new, None)


def verify(ctx, sh=None, of=FAR + 2 * G, kv=None, B=4, N=16, q=P, q_hat=None, norms=None, parents=P, weights=True):
    outs, params = A.Outputs(*([P] * 12)), A.Params(0.8, 0.9, 8)
    layers = (A.LayerWeights * 2)(*[A.LayerWeights(P, P, P, P, P, P)] * 2)
    w = A.Weights(P, layers, P, P, 0) if weights else None
    return A.load().acespec_verify_tree_shared(ctx, ref(w), norms, ref(shared()) if sh is None else ref(sh) if sh else None,
                                               of, ref(cache() if kv is None else kv), P, parents, q, q_hat, P, B, N,
                                               C.byref(params), C.byref(outs), None)


def test_struct_layouts_match_the_header():
    assert C.sizeof(A.KVShared) == 24 and A.KVShared.len.offset == 16
    assert C.sizeof(A.QKNorm) == 16


@pytest.mark.parametrize("kw, text", [
    (dict(blocks=None), "NULL"), (dict(length=None), "NULL"), (dict(blocks=FAR + 8), "aligned"),
    (dict(prefixes=0), "prefixes"), (dict(prefixes=-1), "prefixes"), (dict(capacity=0), "multiple of 64"),
    (dict(capacity=96), "multiple of 64"), (dict(capacity=-64), "multiple of 64")])
def test_a_bad_store_is_refused_everywhere(kw, text):
    ctx = Ctx().ptr
    for call in (attention, rotate, share, verify):
        refused(call(ctx, shared(**kw)), text)


@pytest.mark.parametrize("kw, text", [
    (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(prefix=None), "NULL"), (dict(k=P + 4 * G + 8), "aligned"),
    (dict(v=P + 5 * G + 2), "aligned"), (dict(capacity=0), "multiple of 64"), (dict(capacity=100), "multiple of 64"),
    (dict(capacity=-64), "multiple of 64")])
def test_a_bad_cache_is_refused_everywhere(kw, text):
    ctx = Ctx().ptr
    for call in (attention, rotate, share, verify):
        refused(call(ctx, kv=cache(**kw)), text)
    refused(fork(ctx, src=cache(**kw)), text)
    refused(fork(ctx, dst=cache(**kw)), text)


def test_sizes_that_offsets_do_not_hold():
    ctx = Ctx().ptr
    for call in (attention, rotate, share, verify):
        refused(call(ctx, shared(capacity=2 ** 22)), "2 GiB", A.ACESPEC_EUNSUPPORTED)
        refused(call(ctx, kv=cache(capacity=2 ** 24)), "4 GiB", A.ACESPEC_EUNSUPPORTED)
    refused(fork(ctx, dst=cache(capacity=2 ** 24)), "4 GiB", A.ACESPEC_EUNSUPPORTED)
    tiny = Ctx(dtype=A.ACESPEC_BF16, hd=64, max_nodes=16).ptr
    refused(attention(tiny, shared(capacity=2 ** 23)), "2 GiB", A.ACESPEC_EUNSUPPORTED)


def test_contexts_layers_batches_and_pairs():
    ctx, no_layers = Ctx().ptr, Ctx(L=0).ptr
    for call in (attention, rotate, share, fork, verify):
        refused(call(None), "ctx is NULL")
        refused(call(no_layers), "no layers")
    for call in (attention, rotate):
        refused(call(ctx, layer=2), "layer")
        refused(call(ctx, layer=-1), "layer")
        refused(call(ctx, status=None), "NULL")
    for call in (attention, rotate, verify):
        refused(call(ctx, B=5), "B must be")
        refused(call(ctx, B=0), "B must be")
        refused(call(ctx, N=17), "N must be")
        refused(call(ctx, N=-1), "N must be")
        refused(call(ctx, N=65), "N must be", A.ACESPEC_EUNSUPPORTED)
        refused(call(ctx, of=None), "come together")
        refused(call(ctx, parents=None), "parent_idx")
    refused(share(ctx, B=5), "B must be")
    refused(fork(ctx, Bs=5), "B must be")
    refused(fork(ctx, Bd=0), "B must be")
    refused(rotate(ctx, sh=False), "come together")
    refused(verify(ctx, sh=False), "come together")
    refused(verify(ctx, q=None), "exactly one")
    refused(verify(ctx, q_hat=P), "exactly one")
    refused(verify(ctx, weights=False), "NULL")
    refused(share(ctx, frm=None), "NULL")
    refused(share(ctx, new=None), "NULL")
    refused(fork(ctx, frm=None), "NULL")
    refused(fork(ctx, new=None), "NULL")
    refused(attention(ctx, q=None), "NULL")
    refused(attention(ctx, out=None), "NULL")
    refused(rotate(ctx, qkv=None), "NULL")
    refused(rotate(ctx, q=None), "NULL")
    refused(rotate(ctx, norm=False), "NULL")


def test_alignment():
    ctx = Ctx().ptr
    refused(attention(ctx, q=FAR + 3 * G + 8), "aligned")
    refused(attention(ctx, out=FAR + 5 * G + 4), "aligned")
    refused(rotate(ctx, qkv=FAR + 3 * G + 8), "aligned")
    refused(rotate(ctx, q=FAR + 5 * G + 2), "aligned")
    refused(rotate(ctx, gains=(FAR + 7 * G + 8, None)), "aligned")
    refused(rotate(ctx, gains=(None, FAR + 7 * G + 2)), "aligned")
    norms = (A.QKNorm * 2)(A.QKNorm(FAR, FAR), A.QKNorm(FAR, FAR + 8))
    refused(verify(ctx, norms=norms), "aligned")


def test_what_a_call_writes_lies_apart():
    ctx = Ctx().ptr
    kv, sh = cache(), shared()
    for at in (sh.blocks, sh.len, FAR + 2 * G, kv.k, kv.v, kv.prefix_len, FAR + 4 * G, FAR + 3 * G):
        refused(attention(ctx, out=at), "overlap")
        refused(attention(ctx, status=at), "overlap")
    refused(attention(ctx, status=FAR + 5 * G + 64), "overlap")
    for at in (sh.len, FAR + 2 * G, kv.k, kv.v, kv.prefix_len, FAR + 3 * G, FAR + 4 * G, FAR + 7 * G, FAR + 8 * G):
        refused(rotate(ctx, q=at), "overlap")
        refused(rotate(ctx, status=at), "overlap")
    for at in (FAR + 3 * G, FAR + 4 * G, sh.len, FAR + 7 * G):     # the caches are written too
        refused(rotate(ctx, kv=cache(k=at)), "overlap")
        refused(rotate(ctx, kv=cache(v=at)), "overlap")
    for at in (kv.k, kv.v, kv.prefix_len, FAR + 2 * G, FAR + 3 * G, sh.len):
        refused(share(ctx, sh=shared(blocks=at // 16 * 16)), "overlap")
        refused(share(ctx, new=at), "overlap")
    refused(share(ctx, new=sh.blocks), "overlap")
    refused(verify(ctx, sh=shared(blocks=kv.k)), "overlap")
    refused(verify(ctx, sh=shared(blocks=kv.v)), "overlap")
    far = (FAR + 9 * G, FAR + 10 * G, FAR + 11 * G)
    for at in (kv.k, kv.v, kv.prefix_len, FAR + 2 * G, FAR + 3 * G):
        refused(fork(ctx, dst=cache(at, far[1], 128, far[2])), "overlap")
        refused(fork(ctx, dst=cache(far[0], at, 128, far[2])), "overlap")
    for at in (kv.k, kv.prefix_len, *far, FAR + 2 * G, FAR + 3 * G):
        refused(fork(ctx, new=at), "overlap")
    # the same cache on both sides is fine only as a whole
    refused(fork(ctx, src=cache(), dst=cache(capacity=64)), "overlap")
    refused(fork(ctx, src=cache(), dst=cache(), Bd=3), "overlap")
    refused(fork(ctx, src=cache(), dst=cache(v=far[1])), "overlap")


def step(ctx, outs=None, norms=None, sh=None, **at):
    """The whole step with every array in a place of its own but those that `at` and `outs` name."""
    places = dict(of=FAR + 2 * G, tokens=FAR + 30 * G, parents=FAR + 31 * G, q=FAR + 32 * G, uniforms=FAR + 40 * G)
    places.update(at)
    where = [FAR + (50 + i) * G for i in range(11)] + [None]
    for i, p in (outs or {}).items():
        where[i] = p
    layers = (A.LayerWeights * 2)(*[A.LayerWeights(P, P, P, P, P, P)] * 2)
    return A.load().acespec_verify_tree_shared(
        ctx, C.byref(A.Weights(P, layers, P, P, 0)), norms, ref(shared() if sh is None else sh), places["of"], ref(cache()),
        places["tokens"], places["parents"], places["q"], None, places["uniforms"], 4, 16, C.byref(A.Params(0.8, 0.9, 8)),
        C.byref(A.Outputs(*where)), None)


@pytest.mark.parametrize("field", range(12))
def test_what_a_step_writes_lies_apart(field):
    ctx, kv, sh = Ctx().ptr, cache(), shared()
    norms = (A.QKNorm * 2)(A.QKNorm(FAR + 70 * G, None), A.QKNorm(None, FAR + 71 * G))
    for at in (sh.blocks, sh.len, FAR + 2 * G, kv.k, kv.v, kv.prefix_len, FAR + 30 * G, FAR + 31 * G, FAR + 32 * G,
               FAR + 40 * G, FAR + 70 * G, FAR + 71 * G, FAR + (50 + (field + 1) % 11) * G):
        refused(step(ctx, {field: at}, norms), "overlap")


def test_the_caches_of_a_step_lie_apart():
    ctx, kv = Ctx().ptr, cache()
    for at in (kv.k, kv.v):
        for name in ("of", "tokens", "parents", "q", "uniforms"):
            refused(step(ctx, **{name: at}), "overlap")
        refused(step(ctx, sh=shared(length=at)), "overlap")
        refused(step(ctx, norms=(A.QKNorm * 2)(A.QKNorm(None, None), A.QKNorm(at, None))), "overlap")
        refused(rotate(ctx, sh=shared(blocks=at)), "overlap")


def test_more_sessions_than_a_grid_takes():
    ctx = Ctx(max_batch=70000).ptr
    for call in (attention, rotate, verify):
        refused(call(ctx, B=65536), "65535", A.ACESPEC_EUNSUPPORTED)


@pytest.mark.parametrize("cap", [2 ** 24 - 64, 2 ** 23])   # 2 x 16 x 4 planes in chunks of 64 slots: 2^25 - 128, 2^24
def test_more_slots_than_a_forks_launch_takes(cap):
    ctx, T = Ctx(H=16, Hkv=16).ptr, 1 << 42   # (the caches take up to 2^39 bytes)
    src, dst = cache(T, 2 * T, cap, P), cache(3 * T, 4 * T, cap, P + 64)
    refused(fork(ctx, src, dst, frm=P + 128, first=P + 192, new=P + 256), "one launch", A.ACESPEC_EUNSUPPORTED)
