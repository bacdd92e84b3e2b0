"""Sessions behind shared prefixes in 64 bits, from the definitions: where a record keeps a slot,
attention over (prefix, own slots, tree), the heads' norms with the rotation, and the decoder."""
import math

import numpy as np
import torch

from oracle import model as om


def places(hd, packed):
    """Where a record of 64 slots keeps slot i's head dim d: keys [64, hd], values [hd, 64]."""
    i, d = torch.arange(64).view(-1, 1), torch.arange(hd).view(1, -1)
    if not packed:
        return i * hd + d, 64 * hd + d.t() * 64 + i.t()
    r = (i // 16 % 2) * 16 + (i // 4 % 2) * 8 + (i // 8 % 2) * 4 + i % 4   # row of a 32-row operand
    k = ((i // 32) * (hd // 16) + d // 16) * 512 + ((d // 8 % 2) * 32 + r) * 8 + d % 8
    i, d = i.t(), d.t()
    v = ((i // 16) * (hd // 32) + d // 32) * 512 + ((i // 8 % 2) * 32 + d % 32) * 8 + i % 8
    return k, 64 * hd + v


def records(k, v, packed):
    """[.., slots / 64, 128 hd] of keys [.., slots, hd] and values [.., hd, slots]."""
    *lead, slots, hd = k.shape
    at_k, at_v = (p.flatten().to(k.device) for p in places(hd, packed))
    out = torch.zeros(*lead, slots // 64, 128 * hd, dtype=torch.float16 if packed else k.dtype, device=k.device)
    out[..., at_k] = k.reshape(*lead, slots // 64, 64 * hd).to(out.dtype)
    out[..., at_v] = v.unflatten(-1, (slots // 64, 64)).transpose(-3, -2).flatten(-2).to(out.dtype)
    return out


def sees(parents):
    return torch.from_numpy(om.ancestor_matrix(parents))


def attend(q, front, k, v, P, parents):
    """One session: q [n1, H, hd]; front (keys [Hkv, n, hd], values [Hkv, n, hd]); own slots k
    [Hkv, P + n1, hd], v [Hkv, hd, P + n1].  (out, the same with |v|, largest sum of |q k| / sqrt(hd)
    of a row), float64.  Slots that a row does not see play no part, whatever they hold."""
    n1, H, hd = q.shape
    q, fk, fv, k, v = (x.double() for x in (q, *front, k, v.transpose(1, 2)))
    G, n = H // k.shape[0], fk.shape[1]
    vis = torch.ones(n1, n + P + n1, dtype=torch.bool)
    vis[:, n + P:] = sees(parents)
    vis = vis.to(q.device)
    kk, vv = torch.cat([fk, k], 1), torch.cat([fv, v], 1)
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    big = torch.zeros(n1, H, 1, dtype=torch.float64, device=q.device)
    for h in range(H):
        kh, vh = kk[h // G], vv[h // G]
        for rows in ([slice(None)] if bool(kh.isfinite().all() & vh.isfinite().all()) else range(n1)):
            rows = rows if isinstance(rows, slice) else slice(rows, rows + 1)
            at = vis[rows].any(0).nonzero().squeeze(1)
            z = (q[rows, h] @ kh[at].t()) / math.sqrt(hd)
            p = torch.softmax(z.masked_fill(~vis[rows][:, at], -math.inf), -1)
            out[rows, h], mag[rows, h] = p @ vh[at], p @ vh[at].abs()
            big[rows, h] = (q[rows, h].abs() @ kh[at].abs().t()).amax(-1, keepdim=True) / math.sqrt(hd)
    return out, mag, big


def normed_rotated(x, gain, pos, base=10000.0, eps=1e-5):
    """x [rows, heads, hd] normalised (gain [hd] or None) and rotated to pos [rows]; and the sum of
    the magnitudes of the rotation's two terms."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    h = x.shape[-1] // 2
    ang = pos.double().view(-1, 1, 1) * base ** (-2 * torch.arange(h, device=x.device, dtype=torch.float64) / (2 * h))
    c, s, a, b = ang.cos(), ang.sin(), x[..., :h], x[..., h:]
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1), mag


def forward(W, dims, kpre, vpre, tokens, parents, P, norms=None):
    """Logits of a session's tree rows (float64) and per layer its rows' keys and values: the oracle's
    decoder over a prefix of P positions (kpre, vpre: per layer [Hkv, P, hd]) with norms, a
    (q gain, k gain) pair of numpy arrays or None a layer."""
    n, H, Hkv, hd = len(parents), dims.H, dims.Hkv, dims.hd
    pos = P + np.array(om.tree_depths(parents))
    vis = np.concatenate([np.ones((n, P), dtype=bool), om.ancestor_matrix(parents)], 1)
    cos, sin = om.rope_cos_sin(pos, hd, dims.rope_base)
    x, rows = W.embed_rows(tokens), []
    for l in range(dims.L):
        qkv = om.rms_norm(x, W.get("attn_norm", l), dims.rms_eps) @ W.get("wqkv", l).T
        q, k, v = (a.reshape(n, -1, hd) for a in np.split(qkv, [H * hd, (H + Hkv) * hd], 1))
        if norms:
            q, k = (a if w is None else om.rms_norm(a, w, dims.rms_eps) for a, w in zip((q, k), norms[l]))
        q, k = om.apply_rope(q, cos, sin), om.apply_rope(k, cos, sin)
        rows.append((k, v))
        o = np.zeros((n, H, hd))
        for h in range(H):
            g = h // (H // Hkv)
            s = q[:, h] @ np.concatenate([kpre[l][g], k[:, g]]).T / np.sqrt(hd)
            o[:, h] = om.softmax_rows(np.where(vis, s, -np.inf)) @ np.concatenate([vpre[l][g], v[:, g]])
        x = x + o.reshape(n, H * hd) @ W.get("wo", l).T
        gu = om.rms_norm(x, W.get("mlp_norm", l), dims.rms_eps) @ W.get("w_gate_up", l).T
        x = x + (om.silu(gu[:, :dims.F]) * gu[:, dims.F:]) @ W.get("w_down", l).T
    return om.final_logits(W, dims, x), rows
