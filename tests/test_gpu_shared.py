"""Sessions behind shared prefixes, through the ABI, against plain forms in 64 bits (shared_ref)."""
import math
import random

import numpy as np
import pytest
import torch

import synth
from oracle import model as om
from tests import harness as hz
from tests import shared_ref as sr

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F16 = {"bf16": True, "f32": False}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def up64(n):
    return max(1, (n + 63) // 64) * 64


def verifier(L, B, H, Hkv, hd, dtype, N):
    from paper_2609_02514_amd.acespec import Verifier
    return Verifier(L, 64, H, Hkv, hd, 64, 64, dtype, B, N)


def random_cache(L, B, Hkv, cap, hd, dtype, seed):
    """Keys whose channels differ in size, and values."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(L, B, Hkv, cap, hd, generator=g) * torch.rand(hd, generator=g).add_(0.5)
    v = torch.randn(L, B, Hkv, hd, cap, generator=g)
    return k.to(DT[dtype]).cuda(), v.to(DT[dtype]).cuda()


def random_parents(r, n, reach=7):
    return [-1] + [r.randint(max(0, i - reach), i - 1) for i in range(1, n + 1)]


def store(L, held, Hkv, hd, dtype, seed, cap=0):
    """A store of len(held) prefixes, their keys and values [L, P, Hkv, cap, hd] / [.., hd, cap].
    Behind a prefix's end there is a NaN, as in the records of a larger capacity behind all."""
    from paper_2609_02514_amd.acespec import SharedPrefix
    more, cap = cap // 64, up64(max(held))
    k, v = random_cache(L, len(held), Hkv, cap, hd, dtype, seed)
    pk, pv = k.clone(), v.clone()
    for p, n in enumerate(held):
        pk[:, p, :, n:], pv[:, p, :, :, n:] = math.nan, math.nan
    rec = sr.records(pk, pv, F16[dtype])
    if more > rec.shape[3]:
        rec = torch.cat([rec, rec.new_full((*rec.shape[:3], more - rec.shape[3], 128 * hd), math.nan)], 3)
    return SharedPrefix(rec, rec.shape[3] * 64, i32(held)), k, v


# ---- the store ------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("L, Hkv, lens, take, count", [
    (2, 3, [137, 64, 0, 1], [1, 0], [64, 65]), (1, 1, [0], [0], [0]),
    (1, 2, [200, 127], [0, -1, 1, 0, 0], [200, 5, 127, 63, 1]), (3, 1, [1000], [0], None)])
def test_taken_over_slots_are_where_the_attention_reads_them(dtype, hd, L, Hkv, lens, take, count):
    B, P, cap, scap = len(lens), len(take), up64(max(lens)) + 64, up64(max(lens))
    from paper_2609_02514_amd.acespec import SharedPrefix
    k, v = random_cache(L, B, Hkv, cap, hd, dtype, 11)
    ver = verifier(L, B, Hkv, Hkv, hd, dtype, 0)
    shared = SharedPrefix.alloc(L, P, Hkv, hd, scap, dtype)
    shared.blocks.fill_(7)
    shared.len = i32([9] * P)
    new = i32([-5] * P)
    ver.share_prefix(k, v, cap, i32(lens), i32(take), shared, new, None if count is None else i32(count))
    torch.cuda.synchronize()
    want = torch.full_like(shared.blocks, 7)
    lens_want = []
    for p, s in enumerate(take):
        n = 9 if s < 0 else lens[s] if count is None else count[p]
        lens_want.append(n)
        if s < 0:
            continue
        pk, pv, full = k[:, s, :, :scap].clone(), v[:, s, :, :, :scap].clone(), (n + 63) // 64
        pk[:, :, n:], pv[..., n:] = 0, 0
        want[:, p, :, :full] = sr.records(pk, pv, F16[dtype])[:, :, :full]
    assert new.tolist() == lens_want
    assert torch.equal(shared.blocks, want)


def test_values_beyond_fp16_count_as_infinite_in_the_store():
    k, v = torch.full((1, 1, 1, 64, 64), 1e5, dtype=torch.bfloat16, device="cuda"), torch.full(
        (1, 1, 1, 64, 64), -65280.0, dtype=torch.bfloat16, device="cuda")
    from paper_2609_02514_amd.acespec import SharedPrefix
    ver, shared, new = verifier(1, 1, 1, 1, 64, "bf16", 0), SharedPrefix.alloc(1, 1, 1, 64, 64, "bf16"), i32([0])
    ver.share_prefix(k, v, 64, i32([64]), i32([0]), shared, new)
    torch.cuda.synchronize()
    b = shared.blocks.flatten().double()
    assert bool((b[:4096] == math.inf).all()) and bool((b[4096:] == -65280).all())


@pytest.mark.parametrize("lens, take, count", [
    ([64, 65], [2, 1, 1], [1, 66, -1]), ([-1, 65], [0, -2, 1], [0, 1, 65]), ([129, 1], [0, 1, 1], [0, 2, 1])])
def test_take_overs_that_are_refused_on_the_device_write_nothing(lens, take, count):
    """Of three prefixes of a store of 64 slots, out of a cache of 128."""
    from paper_2609_02514_amd.acespec import SharedPrefix
    k, v = random_cache(1, 2, 2, 128, 64, "bf16", 3)
    ver, shared = verifier(1, 2, 2, 2, 64, "bf16", 0), SharedPrefix.alloc(1, 3, 2, 64, 64, "bf16")
    shared.blocks.fill_(3)
    new = i32([5] * 3)
    ver.share_prefix(k, v, 128, i32(lens), i32(take), shared, new, i32(count))
    torch.cuda.synchronize()
    for p, s in enumerate(take):
        fine = 0 <= s < 2 and 0 <= lens[s] <= 128 and 0 <= count[p] <= min(lens[s], 64)
        assert new[p] == (count[p] if fine else -1)
        if not fine or count[p] == 0:
            assert bool((shared.blocks[:, p] == 3).all())


LARGE = 37 * 64 * 512   # slots: more chunks in turn than a session goes over by itself, with two workgroups on each of 256 CUs


# ---- the attention --------------------------------------------------------------------------


def bound(dtype, out, mag, big, hd):
    """|error| of an attention output, element by element.  Scores are sums of hd products in fp32:
    each is off by at most (hd + 4) 2^-24 of the sum of magnitudes `big`, the exponent by 2^-22 of
    it (its scale and reference), and a weight relatively by as much (twice: its own and the sum's).
    exp2, the sums of weights and products and the joins of parts add 2^-20 of mag = sum p |v| for
    up to a few thousand slots.  bf16 model: weights rounded to fp16 (2^-11 of mag, and 2^-25 of a
    weight where they are subnormal, at most 2^-14 of an output with values below 8 over 16384 slots
    whose largest weight is at least 1), the output to bf16 (2^-8)."""
    b = mag * (2 * big * ((hd + 4) * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -20)
    if dtype == "bf16":
        b = b + mag * 2.0 ** -11 + 2.0 ** -14
        b = b + (out.abs() + b) * 2.0 ** -8
    return b + 1e-30


def check_attention(dtype, hd, H, Hkv, held, of, mine, N, seed, L=1, layer=0, poison=None, reach=7, cap=None,
                    scap=0):
    r, B, n1, P = random.Random(seed), len(of), N + 1, len(held)
    cap = cap or up64(max(mine) + n1)
    shared, sk, sv = store(L, held, Hkv, hd, dtype, seed, scap)
    k, v = random_cache(L, B, Hkv, cap, hd, dtype, seed + 1)
    ver = verifier(L, B, H, Hkv, hd, dtype, N)
    parents = [random_parents(r, N, reach) for _ in range(B)]
    g = torch.Generator().manual_seed(seed + 2)
    q = torch.randn(B, n1, H, hd, generator=g).to(DT[dtype]).cuda()
    for b, m in enumerate(mine):   # what lies behind the tree is no number
        k[:, b, :, m + n1:], v[:, b, :, :, m + n1:] = math.nan, math.nan
    if poison:
        poison(shared, sk, sv, k, v, parents)
    out, status = torch.full_like(q, -77.0), i32([9] * B)
    hz.log(f"attention_shared {dtype} hd={hd} H={H}/{Hkv} held={held} of={of} own={mine} N={N}")
    ver.attention_shared(shared, i32(of), k, v, cap, i32(mine), layer, q, i32(parents), out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * B
    worst = 0.0
    for b, m in enumerate(mine):
        n = held[of[b]] if of[b] >= 0 else 0
        p = max(of[b], 0)
        want, mag, big = sr.attend(q[b], (sk[layer, p, :, :n], sv[layer, p, :, :, :n].transpose(1, 2)),
                                   k[layer, b, :, :m + n1], v[layer, b, :, :, :m + n1], m, parents[b])
        got, fine = out[b].double(), want.isfinite()
        assert torch.equal(fine, got.isfinite()), (b, fine.logical_xor(got.isfinite()).nonzero()[:5])
        err = (got - want).abs()[fine] / bound(dtype, want, mag, big, hd)[fine]
        if err.numel():
            worst = max(worst, float(err.max()))
    hz.log(f"  worst error: {worst:.3f} of its bound")
    assert worst <= 1.0
    ver.close()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H, Hkv, held, of, mine, N", [
    (4, 4, [128], [0], [40], 8),                                   # one session
    (8, 2, [1], [0, 0, 0], [0, 1, 63], 0),                         # one shared slot, one token each
    (8, 1, [63, 64, 65, 0], [3, 2, 1, 0, -1, 2, 1], [0, 5, 64, 65, 30, 0, 127], 16),
    (7, 1, [300, 17], [1, 0, 1, 0, 0, -1], [3, 0, 90, 1, 2, 4], 5),
    (6, 3, [700], [0, 0, 0, 0, 0, 0, 0, 0, 0], [0] * 9, 33),       # nothing of their own
    (2, 2, [5], [-1, -1], [70, 0], 3)])                            # nobody behind the prefix
@pytest.mark.parametrize("tiles", [False, True])
def test_attention_against_64_bits(dtype, hd, H, Hkv, held, of, mine, N, tiles):
    """tiles: in a store so large that a session's own way over its prefix would take too long."""
    if tiles and dtype == "f32":
        pytest.skip("fp32 goes one way")
    check_attention(dtype, hd, H, Hkv, held, of, mine, N, seed=H + N, scap=LARGE if tiles else 0)


@pytest.mark.parametrize("dtype, hd, H, Hkv, held, B, N", [
    ("bf16", 128, 32, 8, [1500], 40, 16),        # tiles cut between workgroups, rows of several sessions
    ("bf16", 64, 8, 8, [4096, 1], 70, 0),        # more sessions than a wave
    ("bf16", 128, 8, 1, [900, 70, 333], 9, 64),  # 520 rows a session
    ("bf16", 64, 64, 8, [16384], 3, 8),          # few rows, a long prefix
    ("bf16", 128, 4, 2, [64] * 33, 33, 1),       # a prefix for each session
    ("f32", 64, 4, 2, [900, 70], 9, 10)])
def test_attention_of_batches(dtype, hd, H, Hkv, held, B, N):
    r = random.Random(B)
    of = [b % len(held) for b in range(B)]
    r.shuffle(of)
    check_attention(dtype, hd, H, Hkv, held, of, [r.randint(0, 200) for _ in range(B)], N, seed=B + N)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("G, N", [(1, 0), (2, 0), (3, 0), (4, 0), (5, 0), (7, 0), (8, 0), (9, 0), (1, 7), (4, 1), (3, 1),
                                  (2, 3), (2, 2), (1, 8)])
@pytest.mark.parametrize("scap", [0, LARGE])
def test_few_rows(hd, G, N, scap):
    """Up to 8 query rows a kv head and the first sizes beyond, with own slots that one workgroup goes
    over and with ones that several share, behind prefixes of every length within a record."""
    check_attention("bf16", hd, 2 * G, 2, [200, 33, 63], [0, 1, 2, -1, 0, 1], [0, 31, 32, 33, 600, 1], N, seed=G + N, scap=scap)
    check_attention("bf16", hd, G, 1, [97], [0], [500], N, seed=G + N, scap=scap)
    r = random.Random(G + N)
    check_attention("bf16", hd, 4 * G, 4, [1030], [0] * 70, [r.randint(0, 100) for _ in range(70)], N, seed=G + N, scap=scap)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap", [128, 4096])
@pytest.mark.parametrize("scap", [0, LARGE])
def test_what_few_rows_do_not_see_does_not_reach_them(hd, cap, scap):
    """As below, with 8 rows a kv head; cap 4096: own slots shared by several workgroups."""
    def poison(shared, sk, sv, k, v, parents):
        parents[0][:] = [-1, 0, 1, 1]
        parents[1][:] = [-1, 0, 0, 2]
        v[0, 0, 0, 3, 53] = math.nan                # row 3: nobody's ancestor
        v[0, 0, 1, 5, 51] = math.inf                # row 1: of rows 2 and 3
        k[0, 1, 0, 7 + 2, 2] = math.nan             # row 2: of row 3
        v[0, 2, 1, 1, 4] = math.inf                 # an own slot, seen by all rows of session 2
        sv[0, 1, 0, 9, 20] = -math.inf              # a shared slot of prefix 1 (sessions 2 and 3)
        pk, pv = sk.clone(), sv.clone()
        pk[:, 1, :, 70:], pv[:, 1, :, :, 70:] = math.nan, math.nan
        rec = sr.records(pk, pv, True)[:, 1]
        shared.blocks[:, 1, :, :rec.shape[2]] = rec
    check_attention("bf16", hd, 4, 2, [130, 70], [0, 0, 1, 1, -1], [50, 7, 12, 0, 3], 3, seed=9, poison=poison, cap=cap,
                    scap=scap)


def test_many_groups_of_many_sessions():
    """More sessions than a wave, dealt to tiles of 70 prefixes; some stand alone, some behind none."""
    r = random.Random(3)
    held = [r.choice([1, 64, r.randint(1, 2400), 2400]) for _ in range(70)]
    of = [r.randint(-1, 69) for _ in range(60)] + [r.randint(0, 4) for _ in range(70)]
    check_attention("bf16", 64, 2, 1, held, of, [r.randint(0, 40) for _ in of], 2, seed=3)
    check_attention("bf16", 64, 8, 1, held, of, [r.randint(0, 40) for _ in of], 9, seed=4)
    of = [r.randint(-1, 9) for _ in range(1500)]      # more places than a workgroup has threads
    check_attention("bf16", 64, 1, 1, [2400, 1, 64, 65, 100, 0, 300, 2300, 5, 700], of, [b % 3 for b in range(1500)], 0, seed=5)


def test_one_layer_of_several_and_a_larger_cache():
    check_attention("bf16", 128, 8, 2, [100, 70], [1, 0, 1], [10, 20, 30], 4, seed=5, L=3, layer=1, cap=512)
    check_attention("bf16", 64, 4, 1, [100, 70], [1, 0, 1], [10, 20, 30], 4, seed=5, L=2, layer=1, cap=512, scap=LARGE)
    check_attention("f32", 64, 8, 2, [100, 70], [1, 0, 1], [10, 20, 30], 4, seed=6, L=3, layer=2, cap=320)


@pytest.mark.parametrize("reach", [1, 64])
def test_the_deepest_and_the_widest_trees(reach):
    check_attention("bf16", 128, 8, 2, [333], [0, 0], [100, 64], 64, seed=reach, reach=reach)
    check_attention("bf16", 128, 8, 2, [333], [0, 0], [100, 64], 64, seed=reach, reach=reach, scap=LARGE)


@pytest.mark.parametrize("dtype, hd, H, N", [("bf16", 128, 8, 16), ("bf16", 64, 8, 64), ("f32", 64, 4, 16),
                                             ("bf16", 128, 16, 32), ("bf16", 128, 32, 64)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, hd, H, N):
    """NaN and infinities in the tree's slots, in one session's own slots and in one of two prefixes
    reach the rows that see them, element by element, and no others."""
    def poison(shared, sk, sv, k, v, parents):
        leaf = N                                    # nobody's ancestor
        v[0, 0, 0, 3, 50 + leaf] = math.nan
        v[0, 0, 1, 5, 50 + 1] = math.inf            # a row that others may descend from
        k[0, 1, 0, 7 + leaf, 2] = math.nan
        v[0, 2, 1, 1, 4] = math.inf                 # an own slot, seen by all rows of session 2
        sv[0, 1, 0, 9, 20] = -math.inf              # a shared slot of prefix 1 (sessions 2 and 3)
        pk, pv = sk.clone(), sv.clone()
        pk[:, 1, :, 70:], pv[:, 1, :, :, 70:] = math.nan, math.nan
        rec = sr.records(pk, pv, F16[dtype])[:, 1]
        shared.blocks[:, 1, :, :rec.shape[2]] = rec
    for scap in (0, LARGE):
        check_attention(dtype, hd, H, 2, [130, 70], [0, 0, 1, 1, -1], [50, 7, 12, 0, 3], N, seed=9, poison=poison,
                        scap=scap)


def test_malformed_sessions_are_flagged_and_the_others_unharmed():
    from paper_2609_02514_amd import acespec as A
    B, N, H, Hkv, hd = 8, 4, 4, 2, 64
    shared, _, _ = store(1, [100, 200, 64], Hkv, hd, "bf16", 1)
    k, v = random_cache(1, B, Hkv, 128, hd, "bf16", 2)
    parents = [[-1, 0, 1, 1, 0] for _ in range(B)]
    of, mine = [0, 1, 0, 1, 0, 0, 2, 0], [10, 0, 30, 40, 50, 60, 70, 123]
    q = torch.randn(B, N + 1, H, hd, device="cuda").to(torch.bfloat16)

    def call(of, mine, parents, lens):
        ver = verifier(1, B, H, Hkv, hd, "bf16", N)
        shared.len = i32(lens)
        out, status = torch.zeros_like(q), i32([9] * B)
        ver.attention_shared(shared, i32(of), k, v, 128, i32(mine), 0, q, i32(parents), out, status)
        torch.cuda.synchronize()
        ver.close()
        return out, status.tolist()

    good, st = call(of, mine, parents, [100, 200, 64])
    assert st == [0] * B
    of[1], of[2] = 3, -2                          # no such prefix
    mine[3], mine[7] = -1, 124                    # a negative length, no room for the tree
    parents[4] = [-1, 0, 2, 1, 0]
    bad, st = call(of, mine, parents, [100, 200, 300])   # prefix 2 longer than the store
    assert st == [0, A.ACESPEC_EBADTREE, A.ACESPEC_EBADTREE, A.ACESPEC_EBADTREE, A.ACESPEC_EBADTREE, 0,
                  A.ACESPEC_EBADTREE, A.ACESPEC_EBADTREE]
    for b in (0, 5):
        assert torch.equal(good[b], bad[b])


def test_malformed_sessions_among_many():
    """More than 64 sessions, some behind prefixes that are none or whose length is wrong: flagged, and
    the others as they are without them."""
    from paper_2609_02514_amd import acespec as A
    B, N, H, Hkv, hd = 90, 1, 4, 1, 64
    shared, _, _ = store(1, [100, 2400, 64, 2300], Hkv, hd, "bf16", 1)
    k, v = random_cache(1, B, Hkv, 64, hd, "bf16", 2)
    q = torch.randn(B, N + 1, H, hd, device="cuda").to(torch.bfloat16)
    of = [b % 4 for b in range(B)]
    ver, parents, mine = verifier(1, B, H, Hkv, hd, "bf16", N), i32([[-1, 0]] * B), i32([b % 7 for b in range(B)])

    def call(of, lens):
        shared.len = i32(lens)
        out, status = torch.zeros_like(q), i32([9] * B)
        ver.attention_shared(shared, i32(of), k, v, 64, mine, 0, q, parents, out, status)
        torch.cuda.synchronize()
        return out, status.tolist()

    good, st = call(of, [100, 2400, 64, 2300])
    assert st == [0] * B
    odd = list(of)
    odd[3], odd[5], odd[40] = 4, -2, 7
    bad, st = call(odd, [100, 2400, 3000, 2300])      # prefix 2 longer than the store
    for b in range(B):
        wrong = odd[b] == 2 or odd[b] not in range(4)
        assert st[b] == (A.ACESPEC_EBADTREE if wrong else 0)
    worst = max(float((good[b].float() - bad[b].float()).abs().max()) for b in range(B) if st[b] == 0)
    assert worst <= 2.0 ** -7 * float(good.float().abs().max())   # (cut elsewhere: parts round apart)
    ver.close()


def test_large_scores_and_far_apart_references():
    """Scores of several hundred that grow along the prefix, so that the reference of the exponents
    moves again and again, and rows whose own slots outweigh the prefix or are outweighed by it."""
    hd, H, Hkv, n, N = 128, 8, 2, 1000, 3

    def poison(shared, sk, sv, k, v, parents):
        sk *= torch.linspace(-3, 3, sk.shape[3], device="cuda").view(1, 1, 1, -1, 1).to(sk.dtype) * 8
        rec = sr.records(sk, sv, True)
        shared.blocks[:, :, :, :rec.shape[3]] = rec
        k[:, 0] *= 30
        k[:, 1] *= 0.01
    for scap in (0, LARGE):
        check_attention("bf16", hd, H, Hkv, [n], [0, 0, 0], [10, 64, 0], N, seed=21, poison=poison, reach=1, scap=scap)


def test_offsets_beyond_32_bits():
    """A store of 5 GB and an own cache of 4.3 GB, the last prefix and session in use.  Keys are 0, so
    that every slot weighs the same; the output is the values' mean."""
    from paper_2609_02514_amd.acespec import SharedPrefix
    P, Hkv, hd, scap, B, cap = 20, 2, 128, 2 ** 18, 17, 2 ** 18
    shared = SharedPrefix.alloc(1, P, Hkv, hd, scap, "bf16")
    shared.blocks[0, P - 1, :, :, 64 * hd:] = 1
    shared.blocks[0, P - 1, :, scap // 128:, 64 * hd:] = 3
    shared.len = i32([0] * (P - 1) + [scap])
    k = torch.zeros(1, B, Hkv, cap, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(1, B, Hkv, hd, cap, dtype=torch.bfloat16, device="cuda")
    v[0, B - 1] = 5
    own = cap - 1
    ver = verifier(1, B, Hkv, Hkv, hd, "bf16", 0)
    q, out = (torch.ones(B, 1, Hkv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = i32([9] * B)
    of = i32([-1] * (B - 1) + [P - 1])
    ver.attention_shared(shared, of, k, v, cap, i32([0] * (B - 1) + [own]), 0, q, i32([[-1]] * B), out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * B and not bool(out[:-1].any())
    want = (2.0 * scap + 5.0 * cap) / (scap + cap)   # (weights are 1, sums exact: joins and the output round)
    assert bool(((out[-1].double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -20)).all()), out[-1]
    new = i32([0] * P)
    ver.share_prefix(k, v, cap, i32([0] * (B - 1) + [cap]), i32([-1] * (P - 1) + [B - 1]), shared, new)
    torch.cuda.synchronize()
    assert new.tolist() == [0] * (P - 1) + [cap]
    assert bool((shared.blocks[0, P - 1, :, :, 64 * hd:] == 5).all()) and not bool(shared.blocks[0, :P - 1].any())
    dk, dv, new = torch.ones_like(k), torch.ones_like(v), i32([0] * B)
    lens = i32([0] * (B - 1) + [cap])
    ver.fork_kv(k, v, cap, lens, dk, dv, cap, lens, i32([-1] * (B - 1) + [B - 1]), new, i32([3] * B))
    torch.cuda.synchronize()
    assert new.tolist() == [0] * (B - 1) + [cap - 3]
    assert bool((dv[0, B - 1, :, :, :cap - 3] == 5).all()) and bool((dv[0, B - 1, :, :, cap - 3:] == 1).all())
    assert bool((dk[0, :B - 1] == 1).all()) and not bool(dk[0, B - 1, :, :cap - 3].any())
    del k, v, dk, dv, shared
    torch.cuda.empty_cache()


# ---- norms and rotation ---------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H, Hkv, B, N, held, norm", [
    (4, 4, 1, 0, [100], "qk"), (8, 2, 3, 16, [1000, 7], "qk"), (7, 1, 5, 64, None, "qk"),
    (64, 8, 2, 8, [16384], "q"), (8, 8, 2, 33, [3], "k"), (2, 1, 4, 15, None, "")])
def test_normed_rotation_against_64_bits(dtype, hd, H, Hkv, B, N, held, norm):
    """Sums of hd squares and the products around them are in fp32: an element is off by at most
    (hd / 2 + 16) 2^-24 of the magnitudes of its two terms, and by the output's rounding."""
    r, n1, L, layer = random.Random(N), N + 1, 2, 1
    from paper_2609_02514_amd.acespec import SharedPrefix
    mine = [r.randint(0, 150) for _ in range(B)]
    cap = up64(max(mine) + n1)
    of = [b % (len(held) + 1) - 1 for b in range(B)] if held else None
    shared = None
    if held:
        shared = SharedPrefix.alloc(L, len(held), Hkv, hd, max(held), dtype)
        shared.len = i32(held)
    k, v = random_cache(L, B, Hkv, cap, hd, dtype, 4)
    k0, v0 = k.clone(), v.clone()
    g = torch.Generator().manual_seed(N)
    qkv = (torch.randn(B, n1, H + 2 * Hkv, hd, generator=g) * torch.exp2(torch.randn(B, n1, H + 2 * Hkv, 1, generator=g) * 4))
    qkv[0, 0, 0] = 0                              # a head of zeros stays zero
    qkv = qkv.to(DT[dtype]).cuda()
    gq, gk = ((torch.rand(hd, generator=g) * 2 - 0.5).to(DT[dtype]).cuda() for _ in range(2))
    gq, gk = gq if "q" in norm else None, gk if "k" in norm else None
    parents = [random_parents(r, N) for _ in range(B)]
    ver = verifier(L, B, H, Hkv, hd, dtype, N)
    q, status = torch.full((B, n1, H, hd), 99.0, device="cuda").to(DT[dtype]), i32([9] * B)
    ver.qk_norm_rope(qkv.view(B, n1, -1), gq, gk, k, v, cap, i32(mine), layer, i32(parents), q, status,
                     shared, i32(of) if held else None)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * B
    for b, m in enumerate(mine):
        front = held[of[b]] if held and of[b] >= 0 else 0
        pos = torch.tensor(om.tree_depths(parents[b]), device="cuda") + front + m
        for got, x, gain in ((q[b], qkv[b, :, :H], gq), (k[layer, b, :, m:m + n1].transpose(0, 1), qkv[b, :, H:H + Hkv], gk)):
            want, mag = sr.normed_rotated(x, gain, pos)
            tol = mag * (hd / 2 + 16) * 2.0 ** -24 + 1e-30
            tol = tol + (want.abs() + tol) * torch.finfo(DT[dtype]).eps / 2
            err = ((got.double() - want).abs() / tol).max()
            assert err <= 1.0, (b, float(err))
        assert torch.equal(v[layer, b, :, :, m:m + n1], qkv[b, :, H + Hkv:].permute(1, 2, 0))
        k[layer, b, :, m:m + n1], v[layer, b, :, :, m:m + n1] = k0[layer, b, :, m:m + n1], v0[layer, b, :, :, m:m + n1]
    assert torch.equal(k, k0) and torch.equal(v, v0)     # and nothing else was written
    ver.close()


def test_rotation_of_malformed_sessions_writes_nothing():
    from paper_2609_02514_amd import acespec as A
    B, N, H, Hkv, hd = 6, 2, 4, 2, 128
    shared, _, _ = store(1, [10, 20], Hkv, hd, "bf16", 1)
    k, v = random_cache(1, B, Hkv, 64, hd, "bf16", 2)
    k0, v0 = k.clone(), v.clone()
    ver = verifier(1, B, H, Hkv, hd, "bf16", N)
    qkv = torch.randn(B, N + 1, (H + 2 * Hkv) * hd, device="cuda").to(torch.bfloat16)
    q, status = torch.full((B, N + 1, H, hd), 7.0, device="cuda").to(torch.bfloat16), i32([9] * B)
    parents = [[-1, 0, 1], [-1, 0, 2], [0, 0, 1], [-1, 0, 0], [-1, 0, 0], [-1, 0, 0]]
    ver.qk_norm_rope(qkv, None, None, k, v, 64, i32([61, 0, 0, 62, -1, 0]), 0, i32(parents), q, status, shared,
                     i32([0, 0, 0, 0, 0, 2]))
    torch.cuda.synchronize()
    assert status.tolist() == [0] + [A.ACESPEC_EBADTREE] * 5
    assert bool((q[1:] == 7).all()) and torch.equal(k[:, 1:], k0[:, 1:]) and torch.equal(v[:, 1:], v0[:, 1:])
    assert not torch.equal(k[:, 0], k0[:, 0])
    ver.close()


# ---- forks ----------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens, frm, first, dcap", [
    ([70, 0, 513, 1], [2, 0, -1, 2, 3, 1, 2, 0], [0, 0, 0, 0, 0, 0, 0, 0], 576),
    ([70, 0, 513, 1], [2, 2, 2, 2, 0, 0, 3, 2], [1, 7, 8, 256, 69, 70, 1, 513], 1024),
    ([300], [0, 0], None, 320)])
def test_sessions_take_over_slots(dtype, hd, lens, frm, first, dcap):
    L, Hkv, Bs, Bd = 2, 3, len(lens), len(frm)
    cap = up64(max(lens))
    k, v = random_cache(L, Bs, Hkv, cap, hd, dtype, 1)
    dk, dv = random_cache(L, Bd, Hkv, dcap, hd, dtype, 2)
    wk, wv, want = dk.clone(), dv.clone(), []
    dlen = [5 + b for b in range(Bd)]
    for b, s in enumerate(frm):
        f = first[b] if first else 0
        want.append(dlen[b] if s < 0 else lens[s] - f)
        if s >= 0:
            wk[:, b, :, :want[b]] = k[:, s, :, f:lens[s]]
            wv[:, b, :, :, :want[b]] = v[:, s, :, :, f:lens[s]]
    ver, new = verifier(L, max(Bs, Bd), Hkv, Hkv, hd, dtype, 0), i32([9] * Bd)
    ver.fork_kv(k, v, cap, i32(lens), dk, dv, dcap, i32(dlen), i32(frm), new, None if first is None else i32(first))
    torch.cuda.synchronize()
    assert new.tolist() == want and torch.equal(dk, wk) and torch.equal(dv, wv)
    ver.close()


@pytest.mark.parametrize("dtype, hd", [("bf16", 128), ("f32", 64)])
def test_a_batch_closes_its_gaps_in_place(dtype, hd):
    """Sessions 4 and 5 move to rows 1 and 0 (5 without its first 3 slots); 2 is its own source; 3's
    source receives itself and is refused."""
    lens, frm, first = [10, 20, 30, 40, 300, 65], [5, 4, 2, 1, -1, -1], [3, 0, 0, 0, 0, 0]
    k, v = random_cache(2, 6, 2, 320, hd, dtype, 1)
    wk, wv = k.clone(), v.clone()
    wk[:, 0, :, :62], wv[:, 0, :, :, :62] = k[:, 5, :, 3:65], v[:, 5, :, :, 3:65]
    wk[:, 1, :, :300], wv[:, 1, :, :, :300] = k[:, 4, :, :300], v[:, 4, :, :, :300]
    ver, new, n = verifier(2, 6, 2, 2, hd, dtype, 0), i32([9] * 6), i32(lens)
    ver.fork_kv(k, v, 320, n, k, v, 320, n, i32(frm), new, i32(first))
    torch.cuda.synchronize()
    assert new.tolist() == [62, 300, 30, -1, 300, 65]
    assert torch.equal(k, wk) and torch.equal(v, wv)
    ver.close()


def test_forks_that_are_refused_on_the_device_write_nothing():
    k, v = random_cache(1, 3, 2, 128, 64, "bf16", 1)
    dk, dv = random_cache(1, 7, 2, 64, 64, "bf16", 2)
    wk, wv = dk.clone(), dv.clone()
    ver, new = verifier(1, 7, 2, 2, 64, "bf16", 0), i32([9] * 7)
    # no such session twice, no room, first out of range twice, a length beyond the cache, and one that is fine
    ver.fork_kv(k, v, 128, i32([65, 20, 129]), dk, dv, 64, i32([0] * 7), i32([3, -2, 0, 1, 1, 2, 0]), new,
                i32([0, 0, 0, 21, -1, 66, 1]))
    torch.cuda.synchronize()
    wk[:, 6], wv[:, 6] = k[:, 0, :, 1:65], v[:, 0, :, :, 1:65]
    assert new.tolist() == [-1] * 6 + [64] and torch.equal(dk, wk) and torch.equal(dv, wv)
    ver.close()


# ---- together -------------------------------------------------------------------------------


def workload(dtype, **kw):
    base = dict(name="shared", dtype=dtype, L=2, d=256, H=4, Hkv=2, hd=64, F=512, V=2048, B=4, S=150,
                tree="widths_2455", depth=4, q_std=2.5, q_T=0.8, T=0.8, top_p=0.9, top_k=16, ragged=True,
                seed_base=91)
    return synth.Workload(**dict(base, **kw))


def gains(w, seed=3):
    g = torch.Generator().manual_seed(seed)
    return [tuple((torch.rand(w.hd, generator=g) + 0.5).to(DT[w.dtype]).cuda() for _ in range(2)) for _ in range(w.L)]


def start(w, cut, max_nodes=None):
    """A batch whose first cut[b] slots become session b's shared prefix: the store, prefix_of, and
    the sessions' own caches with what is left, made by the framework's calls."""
    from paper_2609_02514_amd.acespec import SharedPrefix, Verifier
    batch = synth.make_batch(w, "cuda")
    ver = Verifier.for_workload(w)
    n1 = batch.tokens.shape[1]
    lens = batch.prefix_len.tolist()
    frm = [b for b in range(w.B) if cut[b] > 0]
    shared = SharedPrefix.alloc(w.L, max(1, len(frm)), w.Hkv, w.hd, max(cut + [1]), w.dtype)
    new = i32([0] * shared.prefixes)
    ver.share_prefix(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, i32(frm or [-1]), shared, new,
                     i32([cut[b] for b in frm] or [0]))
    shared.len = new
    of = [frm.index(b) if b in frm else -1 for b in range(w.B)]
    cap = up64(max(n - c for n, c in zip(lens, cut)) + 4 * n1)
    k, v = (torch.zeros(s, dtype=DT[w.dtype], device="cuda") for s in
            ((w.L, w.B, w.Hkv, cap, w.hd), (w.L, w.B, w.Hkv, w.hd, cap)))
    own = i32([0] * w.B)
    ver.fork_kv(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, k, v, cap, i32([0] * w.B),
                i32(list(range(w.B))), own, i32(cut))
    return batch, ver, shared, i32(of), k, v, cap, own


@pytest.mark.parametrize("dtype, kw, normed", [
    ("f32", {}, True), ("f32", dict(hd=128, d=512), False), ("bf16", {}, False), ("bf16", {}, True),
    ("bf16", dict(hd=128, d=512, H=8, Hkv=2), True), ("bf16", dict(B=40, S=90, H=8, Hkv=1), True),
    ("bf16", dict(tree="chain_sib", depth=8, sib=7, H=8, Hkv=1), False)])
def test_take_over_fork_verify_commit_and_verify(dtype, kw, normed):
    """The operators as they are used: sessions' fronts become shared prefixes, what is left of them
    their own caches; a verify step behind the prefixes, the commit of its path, the next step.
    Logits against the 64-bit decoder over (prefix, own slots): within 1e-4 (fp32 model) and 2e-2
    (bf16) of their largest, the bounds that the verify step's own tests use."""
    w = workload(dtype, **kw)
    W = synth.make_weights(w, "cuda")
    r = random.Random(1)
    lens = synth.make_batch(w, "cuda").prefix_len.tolist()
    cut = [0 if b % 4 == 3 else r.randint(1, lens[b]) for b in range(w.B)]
    batch, ver, shared, of, k, v, cap, own = start(w, cut)
    norms = gains(w) if normed else None
    n1 = batch.tokens.shape[1]
    outs = ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True)
    ws, parents, F64, dims = ver.weights_struct(W), batch.parents.tolist(), om.F64Weights(W), om.dims_of(w)
    n64 = [tuple(om.to_f64(x) for x in pair) for pair in norms] if normed else None
    tokens, sample = batch.tokens, range(w.B) if w.B < 10 else [0, 3, 17, w.B - 1]
    # the 64-bit decoder's own cache
    ref = {b: [[om.to_f64(batch.kv_k[l, b, :, :lens[b]]), om.to_f64(batch.kv_v[l, b, :, :, :lens[b]]).transpose(0, 2, 1)]
               for l in range(w.L)] for b in sample}
    for step in range(2):
        hz.log(f"verify_tree_shared {dtype} step {step} cut={cut[:8]} own={own.tolist()[:8]}")
        ver.verify_tree_shared(ws, shared, of, k, v, cap, own, tokens, batch.parents, batch.q, batch.u, w.T,
                               w.top_p, w.top_k, outs, norms)
        torch.cuda.synchronize()
        assert outs["status"].tolist() == [0] * w.B
        chain, at = [], 0
        while [j for j in range(1, n1) if parents[0][j] == at]:   # the deepest chain is committed
            at = [j for j in range(1, n1) if parents[0][j] == at][-1]
            chain.append(at)
        for b in sample:
            z, rows = sr.forward(F64, dims, [x[0] for x in ref[b]], [x[1] for x in ref[b]], tokens[b].tolist(),
                                 parents[b], ref[b][0][0].shape[1], n64)
            got = outs["logits_out"].view(w.B, n1, w.V)[b].double().cpu().numpy()
            err = np.abs(got - z).max() / np.abs(z).max()
            hz.log(f"  session {b}: logits off by {err:.2e} of the largest")
            assert err < (1e-4 if dtype == "f32" else 2e-2)
            for l, (rk, rv) in enumerate(rows):
                keep = [0] + chain
                ref[b][l][0] = np.concatenate([ref[b][l][0], rk[keep].transpose(1, 0, 2)], 1)
                ref[b][l][1] = np.concatenate([ref[b][l][1], rv[keep].transpose(1, 0, 2)], 1)
        path = torch.full((w.B, n1), -1, dtype=torch.int32)
        path[:, :len(chain)] = torch.tensor(chain, dtype=torch.int32)
        new = i32([0] * w.B)
        ver.commit_kv(k, v, cap, own, path.cuda(), i32([len(chain)] * w.B), outs["status"], new)
        torch.cuda.synchronize()
        assert new.tolist() == [n + 1 + len(chain) for n in own.tolist()]
        own, tokens = new, torch.roll(tokens, 1, 1)
    ver.close()


def test_without_prefixes_and_norms_it_is_the_verify_step():
    for dtype in ("bf16", "f32"):
        w = workload(dtype)
        W, batch = synth.make_weights(w, "cuda"), synth.make_batch(w, "cuda")
        from paper_2609_02514_amd.acespec import Verifier
        ver = Verifier.for_workload(w)
        n1 = batch.tokens.shape[1]
        a, b = (ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True) for _ in range(2))
        ws = ver.weights_struct(W)
        head = (batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, batch.tokens, batch.parents, batch.q, batch.u,
                w.T, w.top_p, w.top_k)
        ver.verify_tree(ws, *head, a)
        ver.verify_tree_shared(ws, None, None, *head, b)
        torch.cuda.synchronize()
        for key in a:
            assert torch.equal(a[key], b[key]), key
        q_hat = torch.rand(w.B, n1, device="cuda")
        args = head[:6] + (q_hat,) + head[7:]
        ver.verify_tree_scalar_q(ws, *args, a)
        ver.verify_tree_shared(ws, None, None, *args, b, scalar=True)
        torch.cuda.synchronize()
        for key in a:
            assert torch.equal(a[key], b[key]), key
        ver.close()


def test_one_layers_calls_are_the_steps():
    """qk_norm_rope and attention_shared, one after the other over one layer's projection."""
    B, N, H, Hkv, hd, L = 3, 6, 8, 2, 128, 2
    for dtype in ("bf16", "f32"):
        held, of, mine = [200, 33], [1, 0, 1], [9, 0, 70]
        shared, sk, sv = store(L, held, Hkv, hd, dtype, 1)
        cap = up64(max(mine) + N + 1)
        k, v = random_cache(L, B, Hkv, cap, hd, dtype, 2)
        g = torch.Generator().manual_seed(3)
        qkv = torch.randn(B, N + 1, (H + 2 * Hkv) * hd, generator=g).to(DT[dtype]).cuda()
        gq, gk = ((torch.rand(hd, generator=g) + 0.5).to(DT[dtype]).cuda() for _ in range(2))
        r = random.Random(4)
        parents = [random_parents(r, N) for _ in range(B)]
        ver = verifier(L, B, H, Hkv, hd, dtype, N)
        q, out = (torch.zeros(B, N + 1, H, hd, dtype=DT[dtype], device="cuda") for _ in range(2))
        status = i32([9] * B)
        ver.qk_norm_rope(qkv, gq, gk, k, v, cap, i32(mine), 1, i32(parents), q, status, shared, i32(of))
        ver.attention_shared(shared, i32(of), k, v, cap, i32(mine), 1, q, i32(parents), out, status)
        torch.cuda.synchronize()
        assert status.tolist() == [0] * B
        for b, m in enumerate(mine):
            n, p = held[of[b]], of[b]
            want, mag, big = sr.attend(q[b], (sk[1, p, :, :n], sv[1, p, :, :, :n].transpose(1, 2)),
                                       k[1, b, :, :m + N + 1], v[1, b, :, :, :m + N + 1], m, parents[b])
            assert bool(((out[b].double() - want).abs() <= bound(dtype, want, mag, big, hd)).all())
        ver.close()


def test_a_step_by_tiles_decides_as_one_session_by_session():
    """The same step behind a store so large that prefixes are read in tiles: logits differ by the
    rounding of weights and outputs to fp16, through two layers."""
    for kw in (dict(H=8, Hkv=2, hd=128, d=512), dict(H=4, Hkv=2, hd=64, tree="chain_sib", depth=8, sib=7)):
        w = workload("bf16", **kw)
        W = synth.make_weights(w, "cuda")
        logits = []
        for cap in (0, LARGE):
            batch, ver, shared, of, k, v, ocap, own = start(w, [100, 40, 0, 70])
            if cap:
                from paper_2609_02514_amd.acespec import SharedPrefix
                wide = SharedPrefix.alloc(w.L, shared.prefixes, w.Hkv, w.hd, cap, "bf16")
                wide.blocks[:, :, :, :shared.blocks.shape[3]] = shared.blocks
                wide.len = shared.len
                shared = wide
            n1 = batch.tokens.shape[1]
            outs = ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True)
            ver.verify_tree_shared(ver.weights_struct(W), shared, of, k, v, ocap, own, batch.tokens, batch.parents, batch.q,
                                   batch.u, w.T, w.top_p, w.top_k, outs)
            torch.cuda.synchronize()
            assert outs["status"].tolist() == [0] * w.B
            logits.append(outs["logits_out"].double())
            ver.close()
        # an activation of a layer is off by a few roundings to fp16 (2^-11 each), of which a logit's
        # sum of d products keeps its share of their root sum of squares
        err = (logits[0] - logits[1]).norm() / logits[0].norm()
        hz.log(f"tiles against session by session: {float(err):.2e}")
        assert 0 < err < 8 * 2.0 ** -11


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_alone_and_the_scalar_uplink(dtype):
    """Norms without any prefix decide as norms with a store that nobody stands behind, up to the
    rounding of another attention kernel; q_hat in q's place changes nothing of the forward pass."""
    w = workload(dtype, H=8, Hkv=2, hd=128, d=512)
    W, norms = synth.make_weights(w, "cuda"), gains(w)
    batch, ver, shared, of, k, v, cap, own = start(w, [0, 0, 0, 0])
    behind = start(w, [100, 40, 0, 70])
    n1, ws = batch.tokens.shape[1], ver.weights_struct(W)
    head = (batch.tokens, batch.parents, batch.q, batch.u, w.T, w.top_p, w.top_k)
    q_hat = torch.rand(w.B, n1, generator=torch.Generator().manual_seed(1)).cuda()
    outs = [ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True) for _ in range(4)]
    ver.verify_tree_shared(ws, None, None, k, v, cap, own, *head, outs[0], norms)
    ver.verify_tree_shared(ws, shared, i32([-1] * w.B), k, v, cap, own, *head, outs[1], norms)
    for o, scalar, q in ((outs[2], False, batch.q), (outs[3], True, q_hat)):
        behind[1].verify_tree_shared(ws, *behind[2:], *head[:2], q, *head[3:], o, norms, scalar=scalar)
    torch.cuda.synchronize()
    for o in outs:
        assert o["status"].tolist() == [0] * w.B
    a, b = (o["logits_out"].double() for o in outs[:2])
    err = float((a - b).norm() / a.norm())
    hz.log(f"norms alone {dtype}: {err:.2e}")
    assert err < (8 * 2.0 ** -11 if dtype == "bf16" else 512 * 2.0 ** -24)
    for key in ("logits_out", "topk_ids", "topk_probs"):
        assert torch.equal(outs[2][key], outs[3][key]), key
    assert outs[3]["next_token"].tolist() == [-1] * w.B and bool((outs[3]["resample_token"] == -1).all())
    ver.close()
    behind[1].close()


def test_a_nonfinite_shared_value_flags_the_sessions_behind_it():
    from paper_2609_02514_amd import acespec as A
    w = workload("bf16")
    W = synth.make_weights(w, "cuda")
    batch, ver, shared, of, k, v, cap, own = start(w, [20, 30, 0, 40])
    _, at_v = sr.places(w.hd, True)
    shared.blocks[1, 1, 0, 0, at_v[5, 7]] = math.inf      # session 1's prefix, slot 7
    n1 = batch.tokens.shape[1]
    outs = ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True)
    ver.verify_tree_shared(ver.weights_struct(W), shared, of, k, v, cap, own, batch.tokens, batch.parents, batch.q,
                           batch.u, w.T, w.top_p, w.top_k, outs)
    torch.cuda.synchronize()
    assert outs["status"].tolist() == [0, A.ACESPEC_ENONFINITE, 0, 0]
    ver.close()


def test_a_captured_run_replays_between_other_calls():
    """Take-over, fork, verify step and commit in one graph; a layer's attention in another; both
    replayed between eager calls on the same context and a stream of their own."""
    w = workload("bf16", H=8, Hkv=2, hd=128, d=512)
    W = synth.make_weights(w, "cuda")
    cut = [100, 40, 0, 70]
    batch, ver, shared, of, k, v, cap, own = start(w, cut)
    n1 = batch.tokens.shape[1]
    ws, norms = ver.weights_struct(W), gains(w)
    outs = ver.alloc_outputs(w.B * n1, w.B, n1, w.top_k, w.V, "cuda", True)
    new, held, first = i32([0] * w.B), i32([0] * shared.prefixes), i32(cut)
    path, plen = i32([[1, 3] + [-1] * (n1 - 2)] * w.B), i32([2] * w.B)
    frm, every, none = i32([0, 1, 3]), i32(list(range(w.B))), i32([0] * w.B)
    count = i32([c for c in cut if c])
    g = torch.Generator().manual_seed(8)
    qs = [torch.randn(w.B, n1, w.H, w.hd, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    att, st = [torch.zeros_like(q) for q in qs], [i32([9] * w.B) for _ in qs]

    def run():
        ver.share_prefix(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, frm, shared, held, count)
        ver.fork_kv(batch.kv_k, batch.kv_v, batch.cap, batch.prefix_len, k, v, cap, none, every, new, first)
        ver.verify_tree_shared(ws, shared, of, k, v, cap, own, batch.tokens, batch.parents, batch.q, batch.u, w.T,
                               w.top_p, w.top_k, outs, norms)
        ver.commit_kv(k, v, cap, own, path, plen, outs["status"], new)

    def layer(i):
        ver.attention_shared(shared, of, k, v, cap, own, i, qs[i], batch.parents, att[i], st[i])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        layer(0)
        layer(1)
        side.synchronize()
        seen = [*outs.values(), new, held, k, v, shared.blocks, *att, *st]
        want = [t.clone() for t in seen]
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        with torch.cuda.graph(graphs[0], stream=side):
            run()
        with torch.cuda.graph(graphs[1], stream=side):
            layer(0)
        for i in range(4):
            for t in [*outs.values(), new, held, *att, *st, shared.blocks]:
                t.zero_()
            graphs[0].replay()
            layer(1)
            graphs[1].replay()
            side.synchronize()
            for j, (a, b) in enumerate(zip(seen, want)):
                assert torch.equal(a.nan_to_num(), b.nan_to_num()), (i, j)
    ver.close()


@pytest.mark.parametrize("hd, N", [(128, 16), (128, 0), (64, 3)])
def test_captured_attention_by_tiles_and_session_by_session(hd, N):
    """Two graphs on one context, whose workspace they share, replayed in both orders between eager calls."""
    B, H, Hkv, L = 3, 8, 2, 1
    small, _, _ = store(L, [200, 70], Hkv, hd, "bf16", 1)
    wide, _, _ = store(L, [150, 33], Hkv, hd, "bf16", 2, LARGE)
    k, v = random_cache(L, B, Hkv, 128, hd, "bf16", 3)
    ver, of, mine = verifier(L, B, H, Hkv, hd, "bf16", N), i32([1, 0, 1]), i32([5, 64, 0])
    r, g = random.Random(5), torch.Generator().manual_seed(6)
    par = i32([random_parents(r, N) for _ in range(B)])
    q = torch.randn(B, N + 1, H, hd, generator=g).to(torch.bfloat16).cuda()
    outs, status = [torch.zeros_like(q) for _ in range(2)], [i32([9] * B) for _ in range(2)]

    def call(i):
        ver.attention_shared((small, wide)[i], of, k, v, 128, mine, 0, q, par, outs[i], status[i])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(2):
            call(i)
        side.synchronize()
        want, graphs = [o.clone() for o in outs], [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for i in range(2):
            with torch.cuda.graph(graphs[i], stream=side):
                call(i)
        for order in ((0, 1), (1, 0), (1, 1, 0), (0, 0, 1)):
            for t in outs + status:
                t.fill_(9)
            for i in order:
                graphs[i].replay()
            side.synchronize()
            assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
            assert status[0].tolist() == status[1].tolist() == [0] * B
            call(order[0])
    torch.cuda.synchronize()
    ver.close()


def test_a_call_repeats_bit_for_bit():
    for scap in (0, LARGE):
        args = ("bf16", 128, 16, 2, [1000, 300], [0, 1, 0, 0, 1, 0, 0], [5, 9, 100, 3, 0, 7, 64], 16)
        assert torch.equal(check_attention(*args, seed=2, scap=scap), check_attention(*args, seed=2, scap=scap))


def test_wrong_tensors_are_refused():
    from paper_2609_02514_amd.acespec import SharedPrefix, Verifier
    B, N, H, Hkv, hd, L = 2, 3, 4, 2, 64, 2
    ver = verifier(L, B, H, Hkv, hd, "bf16", N)
    shared, _, _ = store(L, [70], Hkv, hd, "bf16", 1)
    other, _, _ = store(1, [70], Hkv, hd, "bf16", 1)
    f32, _, _ = store(L, [70], Hkv, hd, "f32", 1)
    k, v = random_cache(L, B, Hkv, 128, hd, "bf16", 2)
    par, own, of, st = i32([[-1, 0, 1, 2]] * B), i32([1, 2]), i32([0, 0]), i32([0, 0])
    q = torch.zeros(B, N + 1, H, hd, dtype=torch.bfloat16, device="cuda")
    good = dict(shared=shared, prefix_of=of, kv_k=k, kv_v=v, capacity=128, prefix_len=own, layer=0, q=q, parents=par,
                out=torch.zeros_like(q), status=st)
    ver.attention_shared(**good)
    for bad in (dict(shared=other), dict(shared=f32), dict(prefix_of=of.long()), dict(prefix_of=i32([0])),
                dict(prefix_of=None), dict(kv_k=v), dict(kv_v=k), dict(capacity=64), dict(prefix_len=i32([1, 2, 3])),
                dict(prefix_len=own.cpu()), dict(q=q.float()), dict(q=q.transpose(1, 2)), dict(out=q[:1]),
                dict(parents=par.long()), dict(status=i32([0])), dict(kv_k=k[:1]), dict(q=None), dict(out=None),
                dict(status=None), dict(kv_v=None)):
        with pytest.raises(ValueError):
            ver.attention_shared(**dict(good, **bad))
    with pytest.raises(ValueError, match="moved"):
        gone, _, _ = store(L, [70], Hkv, hd, "bf16", 1)
        gone.blocks.set_(gone.blocks.clone())
        ver.attention_shared(**dict(good, shared=gone))
    with pytest.raises(ValueError):
        SharedPrefix(shared.blocks, 64, shared.len)          # 128 slots
    with pytest.raises(ValueError):
        SharedPrefix(shared.blocks.to(torch.bfloat16), 128, shared.len)
    with pytest.raises(ValueError):
        shared.len = i32([1, 2])
    qkv = torch.zeros(B, N + 1, (H + 2 * Hkv) * hd, dtype=torch.bfloat16, device="cuda")
    gain = torch.ones(hd, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(qkv=qkv[..., 8:]), dict(q_gain=gain.float()), dict(k_gain=gain[:32]), dict(shared=None),
                dict(q_out=q.float())):
        with pytest.raises(ValueError):
            ver.qk_norm_rope(**dict(dict(qkv=qkv, q_gain=gain, k_gain=gain, kv_k=k, kv_v=v, capacity=64, prefix_len=own,
                                         layer=0, parents=par, q_out=q, status=st, shared=shared, prefix_of=of), **bad))
    with pytest.raises(ValueError):
        ver.share_prefix(k, v, 128, own, i32([0, 0]), shared, i32([0]))
    with pytest.raises(ValueError):
        ver.fork_kv(k, v, 128, own, k, v, 128, own, i32([0, 0]), i32([0]))
    ver.close()
