"""Plain 64-bit forms of the 4-bit KV cache's operators, for the tests alone: the cache's values
from their definition (a search over the grid), the attention as a loop over sessions and rows,
and a decoder forward pass whose tree attention has a window.  Nothing here knows the records'
inner order or the kernels' blocks."""
import math

import numpy as np
import torch

from oracle import model as om

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]   # codes 0 .. 7: odd codes have an odd mantissa


def held(x):
    """What groups x [..., 32] are held as, in float64."""
    x = x.double()
    a = x.abs()
    top = a.amax(-1, keepdim=True)
    bad = ~torch.isfinite(x).all(-1, keepdim=True) | (torch.nan_to_num(top, nan=math.inf) >= 57344.0)
    safe = torch.where(bad, torch.ones_like(top), top.clamp_min(2.0 ** -60))
    floor = torch.floor(torch.log2(safe))
    floor = torch.where(torch.exp2(floor) > safe, floor - 1, floor)
    floor = torch.where(torch.exp2(floor + 1) <= safe, floor + 1, floor)
    e = floor - 2 + (safe >= 1.75 * torch.exp2(floor)).double()
    scale = torch.exp2(e.clamp_min(-13))
    y = torch.nan_to_num(a, nan=0.0, posinf=0.0) / scale
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    dist = (y.unsqueeze(-1) - grid).abs()
    # of two equally near values the one with the even code (a hair nearer)
    code = (dist * 2 + torch.tensor([0, 1] * 4, device=x.device) * 1e-12).argmin(-1)
    out = grid[code] * scale * torch.sign(torch.nan_to_num(x, nan=0.0))
    return torch.where(bad, torch.full_like(out, math.nan), out)


def held_keys(k):
    """Keys [..., slots, hd], whole blocks."""
    return held(k.reshape(*k.shape[:-1], k.shape[-1] // 32, 32)).reshape(k.shape)


def held_values(v):
    """Values [..., hd, slots], whole blocks."""
    return held(v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32)).reshape(v.shape)


def lines(parents):
    """Each row's ancestors and itself, root first."""
    out = [[0]]
    for r in range(1, len(parents)):
        out.append(out[parents[r]] + [r])
    return out


def sees(P, parents, window, sinks):
    """[n1, P + n1] bool: which prefix slots and tree rows each row attends to."""
    line, n1 = lines(parents), len(parents)
    m = torch.zeros((n1, P + n1), dtype=torch.bool)
    for r in range(n1):
        pos = P + len(line[r]) - 1
        for s in range(P):
            m[r, s] = window == 0 or pos - s < window or s < sinks
        for j in line[r]:
            pj = P + len(line[j]) - 1
            m[r, P + j] = window == 0 or pos - pj < window or pj < sinks
    return m


def attend(q, k, v, P, parents, window=0, sinks=0):
    """One session: q [n1, H, hd], k, v [Hkv, P + n1, hd]; (out, the same with |v|, largest sum
    of |q k| / sqrt(hd) over a row's slots), float64.  Slots a row does not see play no part,
    whatever they hold."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    n1, H, hd = q.shape
    G = H // k.shape[0]
    m = sees(P, parents, window, sinks)
    out, mag, big = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(n1, H, 1, dtype=torch.float64)
    for h in range(H):
        for r in range(n1):
            at = m[r].nonzero().squeeze(1)
            kk, vv = k[h // G, at], v[h // G, at]
            z = (kk @ q[r, h]) / math.sqrt(hd)
            p = torch.softmax(z, 0)
            out[r, h], mag[r, h] = p @ vv, p @ vv.abs()
            big[r, h] = (kk.abs() @ q[r, h].abs()).max() / math.sqrt(hd)
    return out, mag, big


def forward_windowed(W, dims, kpre, vpre, tokens, parents, P, window, sinks):
    """Logits of a session's tree rows (float64): the oracle's decoder with a window in its
    mask.  kpre, vpre: per layer [Hkv, P, hd]."""
    depth = np.array(om.tree_depths(parents))
    vis = sees(P, parents, window, sinks).numpy()
    cos, sin = om.rope_cos_sin(P + depth, dims.hd, dims.rope_base)
    x = W.embed_rows(tokens)
    H, Hkv, hd, n = dims.H, dims.Hkv, dims.hd, len(parents)
    for l in range(dims.L):
        a = om.rms_norm(x, W.get("attn_norm", l), dims.rms_eps)
        qkv = a @ W.get("wqkv", l).T
        q = om.apply_rope(qkv[:, :H * hd].reshape(n, H, hd), cos, sin)
        k = om.apply_rope(qkv[:, H * hd:(H + Hkv) * hd].reshape(n, Hkv, hd), cos, sin)
        v = qkv[:, (H + Hkv) * hd:].reshape(n, Hkv, hd)
        o = np.zeros((n, H, hd))
        for h in range(H):
            g = h // (H // Hkv)
            keys, vals = np.concatenate([kpre[l][g], k[:, g]]), np.concatenate([vpre[l][g], v[:, g]])
            s = np.where(vis, q[:, h] @ keys.T / np.sqrt(hd), -np.inf)
            o[:, h] = om.softmax_rows(s) @ vals
        x = x + o.reshape(n, H * hd) @ W.get("wo", l).T
        b = om.rms_norm(x, W.get("mlp_norm", l), dims.rms_eps)
        gu = b @ W.get("w_gate_up", l).T
        x = x + (om.silu(gu[:, :dims.F]) * gu[:, dims.F:]) @ W.get("w_down", l).T
    return om.final_logits(W, dims, x)
