"""What Verifier's calls over shared prefixes refuse of their tensors: each bad one by its name, before the
library is called.  No GPU: the tensors are the CPU's, whose device number is -1, and the library's
entry points are replaced by a mark that a call got through."""
import pytest
import torch

import paper_2609_02514_amd.acespec as A

L, B, N, H, HKV, HD, P, CAP, SCAP, V, K = 2, 3, 4, 4, 2, 64, 2, 128, 64, 32, 8
N1, BF, I32, F32 = N + 1, torch.bfloat16, torch.int32, torch.float32


def i32(*shape):
    return torch.zeros(shape, dtype=I32)


def bf(*shape):
    return torch.zeros(shape, dtype=BF)


def store(layers=L, dtype=torch.float16, kind=A.ACESPEC_BF16):
    s = A.SharedPrefix.__new__(A.SharedPrefix)
    s.index, s._fit = -1, (layers, HKV, HD, kind)
    s._tensors = (torch.zeros(layers, P, HKV, SCAP // 64, 128 * HD, dtype=dtype), i32(P))
    s._at = tuple(t.data_ptr() for t in s._tensors)
    s._struct = A.KVShared(s._at[0], P, SCAP, s._at[1])
    return s


@pytest.fixture
def ver(monkeypatch):
    v = A.Verifier.__new__(A.Verifier)
    v.desc = A.ModelDesc(L, 64, H, HKV, HD, 64, V, 10000.0, 1e-5, A.ACESPEC_BF16)
    v.ctx, v.index, v.reached = None, -1, []
    v._kv, v._store, v._heads = (L, HKV, HD, BF, I32), (L, HKV, HD, A.ACESPEC_BF16), (H, (H + 2 * HKV) * HD, HD)
    for f in ("share_prefix", "attention_shared", "qk_norm_rope", "verify_tree_shared", "fork_kv"):
        monkeypatch.setattr(A, "acespec_" + f, lambda *a, f=f: v.reached.append(f))
    monkeypatch.setattr(A, "_stream_of", lambda index: 0)
    monkeypatch.setattr(A.Verifier, "_stream", staticmethod(lambda: 0))
    monkeypatch.setattr(A.Verifier, "_here", lambda self: -1)
    return v


def cache(sessions=B, prefix=""):
    return {prefix + "kv_k": bf(L, sessions, HKV, CAP, HD), prefix + "kv_v": bf(L, sessions, HKV, HD, CAP),
            prefix + "capacity": CAP, prefix + "prefix_len": i32(sessions)}


def bad_ones(t, name):
    """A tensor's wrong forms: absent, of another type, shape and order."""
    yield None
    yield t.double()
    yield t[:-1].clone()
    yield t.unsqueeze(0)
    if t.dim() > 1:
        yield t.transpose(-1, -2).contiguous().transpose(-1, -2)   # strides of another order


def refuses(call, good, name, t, match=None):
    for bad in bad_ones(t, name):
        with pytest.raises(ValueError, match=match or name):
            call(**dict(good, **{name: bad}))


def test_attention(ver):
    good = dict(shared=store(), prefix_of=i32(B), **cache(), layer=0, q=bf(B, N1, H, HD), parents=i32(B, N1),
                out=bf(B, N1, H, HD), status=i32(B))
    ver.attention_shared(**good)
    assert ver.reached == ["attention_shared"]
    for name in ("kv_k", "kv_v", "prefix_len", "q", "out", "status"):
        refuses(ver.attention_shared, good, name, good[name])
    for bad in list(bad_ones(good["parents"], "parents"))[:3]:   # (its shape is the call's: others may be found wrong first)
        with pytest.raises(ValueError):
            ver.attention_shared(**dict(good, parents=bad))
    with pytest.raises(ValueError, match="parents"):
        ver.attention_shared(**dict(good, parents=None))
    with pytest.raises(ValueError, match="parents"):
        ver.attention_shared(**dict(good, parents=i32(B * N1)))
    with pytest.raises(ValueError, match="come together"):
        ver.attention_shared(**dict(good, prefix_of=None))
    for bad in list(bad_ones(good["prefix_of"], "prefix_of"))[1:]:
        with pytest.raises(ValueError, match="prefix_of"):
            ver.attention_shared(**dict(good, prefix_of=bad))
    for bad in (dict(shared=None), dict(shared=None, prefix_of=None)):
        with pytest.raises(ValueError, match="shared"):
            ver.attention_shared(**dict(good, **bad))
    for bad in (store(1), store(L, F32, A.ACESPEC_F32)):
        with pytest.raises(ValueError, match="is not this"):
            ver.attention_shared(**dict(good, shared=bad))
    assert len(ver.reached) == 1


def test_normed_rotation(ver):
    good = dict(qkv=bf(B, N1, (H + 2 * HKV) * HD), q_gain=bf(HD), k_gain=bf(HD), **cache(), layer=1,
                parents=i32(B, N1), q_out=bf(B, N1, H, HD), status=i32(B), shared=store(), prefix_of=i32(B))
    ver.qk_norm_rope(**good)
    ver.qk_norm_rope(**dict(good, shared=None, prefix_of=None, q_gain=None, k_gain=None))
    assert len(ver.reached) == 2
    for name in ("qkv", "kv_k", "kv_v", "prefix_len", "q_out", "status"):
        refuses(ver.qk_norm_rope, good, name, good[name])
    for name in ("q_gain", "k_gain", "prefix_of"):
        for bad in list(bad_ones(good[name], name))[1:]:
            with pytest.raises(ValueError, match=name):
                ver.qk_norm_rope(**dict(good, **{name: bad}))
    for bad in (dict(shared=None), dict(prefix_of=None)):
        with pytest.raises(ValueError, match="come together"):
            ver.qk_norm_rope(**dict(good, **bad))
    for bad in (None, i32(B * N1)):
        with pytest.raises(ValueError, match="parents"):
            ver.qk_norm_rope(**dict(good, parents=bad))
    with pytest.raises(ValueError, match="kv_k"):
        ver.qk_norm_rope(**dict(good, capacity=64))
    assert len(ver.reached) == 2


def test_take_over(ver):
    good = dict(**cache(), from_=i32(P), shared=store(), new_len=i32(P), count=i32(P))
    ver.share_prefix(**good)
    ver.share_prefix(**dict(good, count=None))
    assert len(ver.reached) == 2
    for name in ("kv_k", "kv_v", "from_", "new_len"):
        refuses(ver.share_prefix, good, name, good[name])
    for bad in list(bad_ones(good["count"], "count"))[1:]:
        with pytest.raises(ValueError, match="count"):
            ver.share_prefix(**dict(good, count=bad))
    for bad in (None, i32(), i32(B, 1), good["prefix_len"].long()):
        with pytest.raises(ValueError, match="prefix_len"):
            ver.share_prefix(**dict(good, prefix_len=bad))
    with pytest.raises(ValueError, match="shared"):
        ver.share_prefix(**dict(good, shared=None))
    assert len(ver.reached) == 2


def test_forks(ver):
    def names(side, c):
        return {side + "_k": c["kv_k"], side + "_v": c["kv_v"], side + "_capacity": CAP, side + "_len": c["prefix_len"]}
    good = dict(**names("src", cache(2)), **names("dst", cache()), from_=i32(B), new_prefix_len=i32(B), first=i32(B))
    ver.fork_kv(**good)
    ver.fork_kv(**dict(good, first=None))
    assert len(ver.reached) == 2
    for name in ("src_k", "src_v", "dst_k", "dst_v"):
        refuses(ver.fork_kv, good, name, good[name], f"{name[:3]} kv_{name[-1]}")
    for name in ("src_len", "dst_len"):
        for bad in (None, i32(), i32(1, B), good[name].long()):
            with pytest.raises(ValueError, match=name[:3] + " prefix_len"):
                ver.fork_kv(**dict(good, **{name: bad}))
    for name in ("from_", "new_prefix_len"):
        refuses(ver.fork_kv, good, name, good[name])
    for bad in list(bad_ones(good["first"], "first"))[1:]:
        with pytest.raises(ValueError, match="first"):
            ver.fork_kv(**dict(good, first=bad))
    assert len(ver.reached) == 2


def test_steps(ver):
    rows, outs = B * N1, A.Verifier.alloc_outputs(B * N1, B, N1, K, V, "cpu", True)
    norms = [(bf(HD), bf(HD)), (None, bf(HD))]
    good = dict(wstruct=A.Weights(), shared=store(), prefix_of=i32(B), **cache(), tokens=i32(B, N1), parents=i32(B, N1),
                q=torch.zeros(B, N1, V), u=torch.zeros(B, N1, 3), T=1.0, top_p=1.0, k=K, outs=outs, norms=norms)
    ver.verify_tree_shared(**good)
    ver.verify_tree_shared(**dict(good, shared=None, prefix_of=None, norms=None, q=torch.zeros(B, N1), scalar=True))
    assert len(ver.reached) == 2
    for name in ("kv_k", "kv_v", "prefix_len", "parents"):
        refuses(ver.verify_tree_shared, good, name, good[name])
    for bad in (None, i32(rows)):
        with pytest.raises(ValueError, match="tokens"):
            ver.verify_tree_shared(**dict(good, tokens=bad))
    with pytest.raises(ValueError, match="tokens"):
        ver.verify_tree_shared(**dict(good, tokens=good["tokens"].long()))
    for name, short in (("q", torch.zeros(rows * V - 1)), ("u", torch.zeros(rows * 3 - 1))):
        for bad in (None, short, good[name].double()):
            with pytest.raises(ValueError, match=f"^{name} "):
                ver.verify_tree_shared(**dict(good, **{name: bad}))
    for name, t in outs.items():
        for bad in ([None] if name != "logits_out" else []) + [t.flatten()[:-1], t.double()]:
            with pytest.raises(ValueError, match=name):
                ver.verify_tree_shared(**dict(good, outs=dict(outs, **{name: bad})))
    for bad in (bf(HD)[:-1], torch.zeros(HD), bf(2 * HD)[::2]):
        with pytest.raises(ValueError, match=r"norms\[1\]"):
            ver.verify_tree_shared(**dict(good, norms=[norms[0], (None, bad)]))
    with pytest.raises(ValueError, match="layers"):
        ver.verify_tree_shared(**dict(good, norms=norms[:1]))
    for bad in (dict(shared=None), dict(prefix_of=None)):
        with pytest.raises(ValueError, match="come together"):
            ver.verify_tree_shared(**dict(good, **bad))
    assert len(ver.reached) == 2
