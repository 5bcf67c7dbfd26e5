"""fp64 oracle of what a layer does around its attention, in plain NumPy: rotary positions with several axes, layer
norm, attention in a window with first tokens that stay visible, and their gradients."""
from __future__ import annotations

import numpy as np


# ---- rotary positions ---------------------------------------------------------------------------------------
def grid_positions(N, grid, start=None):
    """int64 [N, axes]: positions of a row-major grid's tokens, -1 behind them."""
    start = (0,) * len(grid) if start is None else start
    pos = np.full((N, len(grid)), -1, dtype=np.int64)
    cells = np.stack(np.meshgrid(*[np.arange(g) + s for g, s in zip(grid, start)], indexing="ij"), -1).reshape(-1, len(grid))
    pos[: len(cells)] = cells
    return pos


def rope(x, pos, dims, lengths, theta=10000.0, scale=None, interleaved=True, inverse=False):
    """x [B, H, N, D], pos [N, axes] or [B, N, axes] -> fp64 [B, H, N, D]."""
    x = np.asarray(x, dtype=np.float64)
    B, _, N, _ = x.shape
    pos = np.broadcast_to(np.asarray(pos), (B, N, len(dims)))
    angles = []
    for a, d in enumerate(dims):
        p = pos[..., a].astype(np.float64)
        f = np.array([theta ** (-2.0 * i / d) for i in range(d // 2)])
        ang = np.where(p < 0, 0.0, p * (1.0 if scale is None else scale[a]))[..., None] * f
        angles.append(np.where((p >= lengths[a])[..., None], np.nan, ang))
    ang = np.concatenate(angles, -1)[:, None]  # [B, 1, N, P]
    c, s = np.cos(ang), np.sin(ang) * (-1.0 if inverse else 1.0)
    P = ang.shape[-1]
    first, second = (np.arange(0, 2 * P, 2), np.arange(1, 2 * P, 2)) if interleaved else (np.arange(P), np.arange(P, 2 * P))
    out = x.copy()
    u, v = x[..., first], x[..., second]
    out[..., first], out[..., second] = u * c - v * s, u * s + v * c
    return out


# ---- layer norm ---------------------------------------------------------------------------------------------
def layer_norm(x, weight=None, bias=None, eps=1e-6, center=True):
    x = np.asarray(x, dtype=np.float64)
    d = x - x.mean(-1, keepdims=True) if center else x
    h = d / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return h * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)


def layer_norm_grads(dy, x, weight=None, eps=1e-6, center=True):
    """(dx, dweight, dbias)"""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    d = x - x.mean(-1, keepdims=True) if center else x
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    h, g = d * r, dy * (1.0 if weight is None else weight)
    dx = r * (g - h * (g * h).mean(-1, keepdims=True) - (g.mean(-1, keepdims=True) if center else 0.0))
    rows = tuple(range(x.ndim - 1))
    return dx, (dy * h).sum(rows), dy.sum(rows)


# ---- attention in a window ----------------------------------------------------------------------------------
def window_visible(Nq, Nk, left, right, sinks, frame, start, q_len=None, k_len=None):
    """bool [Nq, Nk] of one batch entry whose query 0 is at position ``start``."""
    p = start + np.arange(Nq, dtype=np.int64)
    f = np.floor_divide(p, frame)
    j = np.arange(Nk, dtype=np.int64)
    k_len = Nk if k_len is None else min(max(int(k_len), 0), Nk)
    q_len = Nq if q_len is None else min(max(int(q_len), 0), Nq)
    lo = (f - left) * frame if left >= 0 else np.zeros(Nq, dtype=np.int64)
    hi = np.minimum((f + right + 1) * frame, k_len) if right >= 0 else np.full(Nq, k_len, dtype=np.int64)
    seen = (j < hi[:, None]) & ((j >= lo[:, None]) | (j < sinks))
    seen[q_len:] = False
    return seen


def window_attention(q, k, v, visible, scale):
    """q [B, Hq, Nq, D], k, v [B, Hkv, Nk, D], visible bool [B, Nq, Nk] -> (out, lse), zeros and -inf for empty rows."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    G = q.shape[1] // k.shape[1]
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    for b in range(q.shape[0]):
        see = visible[b]
        some = see.any(-1)
        keys = see.any(0)
        for h in range(q.shape[1]):
            kk, vv = np.where(keys[:, None], k[b, h // G], 0.0), np.where(keys[:, None], v[b, h // G], 0.0)
            s = np.where(see, q[b, h] @ kk.T * scale, -np.inf)[some]
            if s.size == 0:
                continue
            m = s.max(-1, keepdims=True)
            e = np.exp(s - m)
            t = e.sum(-1, keepdims=True)
            out[b, h, some] = e / t @ vv
            lse[b, h, some] = (m + np.log(t))[:, 0]
    return out, lse


def window_attention_grads(dout, q, k, v, visible, scale):
    """(dq, dk, dv)"""
    dout, q, k, v = (np.asarray(t, dtype=np.float64) for t in (dout, q, k, v))
    G = q.shape[1] // k.shape[1]
    out, lse = window_attention(q, k, v, visible, scale)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(q.shape[0]):
        see = visible[b]
        some, keys = see.any(-1), see.any(0)
        for h in range(q.shape[1]):
            kk, vv = np.where(keys[:, None], k[b, h // G], 0.0), np.where(keys[:, None], v[b, h // G], 0.0)
            qq, do = np.where(some[:, None], q[b, h], 0.0), np.where(some[:, None], dout[b, h], 0.0)
            p = np.where(see, np.exp(np.where(see, qq @ kk.T * scale, 0.0) - np.where(some, lse[b, h], 0.0)[:, None]), 0.0)
            ds = p * (do @ vv.T - (do * out[b, h]).sum(-1, keepdims=True)) * scale
            dq[b, h] = ds @ kk
            dk[b, h // G] += ds.T @ qq
            dv[b, h // G] += p.T @ do
    return dq, dk, dv
