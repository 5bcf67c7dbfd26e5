"""Positions, normalisation and windowed attention of a video transformer's layers, as timed cases.

Around the attention of a layer its queries and keys are normalised, turned by their positions in time, height and
width, and, in long or streamed videos, attend to a window of frames and a few first tokens.  The cases below are
these operators at the token grids of the repository's benchmark and at generic sizes: the smallest calls, where
latency counts, up to whole layers, forwards and gradients.  Where ``own`` is true ``run`` makes the library's calls,
otherwise it computes the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

ROPE, NORM, STEP, WINDOW = "rope", "norm", "step", "window"
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# rope    frames x rows x cols tokens on a grid, `text` tokens without a position behind them; H query heads, Hkv key heads
#         of D channels, q and k rotated together; layout as below; halves: pairs (i, i + D/2) instead of (2i, 2i+1);
#         listed_positions: positions come as a tensor and not as a grid; inverse: the gradient's rotation
# norm    `tokens` rows of `width` channels, or of every head of a [B, tokens, H, D] tensor (heads > 0); train: the
#         gradients of input, weight and bias for a given gradient of the output, else the normalised rows
# step, window  attention of Nq queries over Nk keys in a window of `left` frames before and `right` behind a query's own
#         (-1: all of them) and the first `sinks` keys; frame: tokens per frame; ragged: lengths differ over the batch
#         (see _lengths), with an empty sequence among them; train: outputs and gradients of one training pass
_ROPE = dict(kind=ROPE, B=1, H=40, Hkv=40, D=128, frames=21, rows=30, cols=52, text=0, dtype="bf16", layout="packed",
             halves=False, listed_positions=False, inverse=False)
_NORM = dict(kind=NORM, tokens=32760, heads=0, width=5120, dtype="bf16", weights="f32", affine=True, center=True, train=False)
_ATT = dict(kind=WINDOW, B=1, H=12, Hkv=12, Nq=8190, Nk=8190, D=128, left=2, right=0, sinks=0, frame=1, ragged=False,
            dtype="bf16", layout="bnhd", train=False)


def listed():
    return [
        # one 32 x 32 frame of two heads: launch and latency
        dict(_ROPE, name="rope_tiny", H=2, Hkv=2, D=64, frames=1, rows=32, cols=32),
        # q and k of a 480p layer as slices of its fused projection
        dict(_ROPE, name="rope_480p_fused", layout="fused"),
        # gradients of a joint text/video layer: positions as a tensor, pairs in halves, half precision, shared key heads
        dict(_ROPE, name="rope_joint_grad_f16", B=2, H=24, Hkv=8, D=128, frames=13, rows=30, cols=41, text=77, dtype="f16",
             layout="bnhd", halves=True, listed_positions=True, inverse=True),
        # every head of q by itself, root mean square, as it stands in front of the rotation
        dict(_NORM, name="norm_heads_480p", heads=40, width=128, center=False),
        # the gradients of a 480p layer's input norm, all 40 heads wide
        dict(_NORM, name="norm_480p_train", train=True),
        # a small odd-sized layer norm in single precision
        dict(_NORM, name="norm_odd_f32_train", tokens=333, width=1001, dtype="f32", train=True),
        # one token of one short stream
        dict(_ATT, name="step_short", kind=STEP, H=8, Hkv=2, Nq=1, Nk=700, D=64, left=256, sinks=4),
        # single tokens of a batch of streams of different lengths over long caches, shared key heads
        dict(_ATT, name="step_batch_long", kind=STEP, B=16, H=32, Hkv=8, Nq=1, Nk=65536, left=16383, sinks=64, ragged=True),
        # a padded batch in half precision with odd lengths and token windows to both sides
        dict(_ATT, name="window_ragged_f16", B=3, H=6, Hkv=3, Nq=1531, Nk=1531, D=64, left=400, right=37, sinks=5,
             ragged=True, dtype="f16"),
        # four heads of a 480p clip: a frame sees itself, four before it and the first
        dict(_ATT, name="window_480p", H=4, Hkv=4, Nq=32760, Nk=32760, left=4, sinks=1560, frame=1560),
        # a training pass of a low-resolution clip's layer, windows of whole frames
        dict(_ATT, name="window_8k_train", sinks=390, frame=390, train=True),
        # a training pass over sixteen thousand tokens, frames to both sides, two query heads to a key head
        dict(_ATT, name="window_16k_train", H=8, Hkv=4, Nq=16380, Nk=16380, left=6, right=2, sinks=780, frame=780, train=True),
    ]


def _spread(rng, lo, hi):
    """Log-uniform integer in [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice([ROPE, ROPE, NORM, NORM, STEP, STEP, WINDOW, WINDOW, WINDOW, WINDOW])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    while True:
        if kind == ROPE:
            hkv = _spread(rng, 1, 40)
            c = dict(_ROPE, B=rng.choice([1, 1, 2]), H=hkv * rng.choice([1, 1, 2, 4]), Hkv=hkv, D=rng.choice([64, 128, 128]),
                     frames=_spread(rng, 1, 28), rows=rng.randint(7, 45), cols=rng.randint(9, 80),
                     text=rng.choice([0, rng.randint(1, 256)]), dtype=rng.choice([dtype, dtype, "f32"]),
                     layout=rng.choice(["packed", "bnhd", "fused"]), halves=rng.random() < 0.4,
                     listed_positions=rng.random() < 0.4, inverse=rng.random() < 0.4)
            if c["layout"] == "fused":
                c["Hkv"] = c["H"]
        elif kind == NORM:
            heads = rng.choice([0, 0, _spread(rng, 1, 40)])
            dtype = rng.choice([dtype, dtype, "f32"])
            width = rng.choice([64, 128]) if heads else rng.choice([_spread(rng, 5, 8192), 8 * _spread(rng, 8, 1024)])
            c = dict(_NORM, tokens=_spread(rng, 1, 40000), heads=heads, width=width, dtype=dtype,
                     weights=rng.choice([dtype, "f32"]), affine=rng.random() < 0.8, center=rng.random() < 0.6,
                     train=rng.random() < 0.6)
        elif kind == STEP:
            hkv = _spread(rng, 1, 16)
            c = dict(_ATT, kind=STEP, B=_spread(rng, 1, 24), H=hkv * rng.choice([1, 2, 4, 8]), Hkv=hkv,
                     Nq=rng.choice([1, 1, 1, rng.randint(2, 4)]), Nk=_spread(rng, 40, 65536), D=rng.choice([64, 128, 128]),
                     sinks=rng.choice([0, rng.randint(1, 64)]), ragged=rng.random() < 0.6, dtype=dtype)
            c["left"] = rng.choice([-1, _spread(rng, 1, c["Nk"])])
        else:
            hkv = _spread(rng, 1, 12)
            n = _spread(rng, 200, 16380)
            c = dict(_ATT, B=rng.choice([1, 1, 2, 3]), H=hkv * rng.choice([1, 1, 2, 4]), Hkv=hkv, Nq=n, Nk=n,
                     D=rng.choice([64, 128, 128]), frame=rng.choice([1, rng.randint(2, max(3, n // 6))]),
                     right=rng.choice([0, 0, -1, 1, 2]), ragged=rng.random() < 0.4, dtype=dtype,
                     layout=rng.choice(["packed", "bnhd", "fused"]), train=rng.random() < 0.5)
            c["left"] = rng.choice([-1, _spread(rng, 1, max(2, n // (2 * c["frame"])))])
            c["sinks"] = rng.choice([0, rng.randint(1, 64), c["frame"]])
            if rng.random() < 0.3 and not c["train"]:  # a chunk of new tokens behind the ones that are there
                c["Nq"] = max(1, n // rng.randint(2, 20))
            if c["layout"] == "fused":
                c["Hkv"], c["Nq"] = c["H"], c["Nk"]
        w = work(c)
        scores = c.get("B", 1) * c.get("H", 0) * c["Nq"] * c["Nk"] if kind in (STEP, WINDOW) else 0
        cache = c["B"] * c["Hkv"] * c["Nk"] * c["D"] if kind in (STEP, WINDOW) else 0
        if w["bytes"] <= 1.3e9 and w["flops"] <= 6e11 and scores <= 2.2e9 and cache <= 1.1e9:
            return c


# ---- which key a query sees ---------------------------------------------------------------------------------
def _lengths(c):
    """(q_start, q_len, k_len) of every batch entry: the queries are the last ones of the keys, and with `ragged` entry b
    lacks the last b/B of its keys, less an odd number, and entry 1 has none at all."""
    start, nq, nk = [], [], []
    for b in range(c["B"]):
        k = c["Nk"] - (b * (c["Nk"] // c["B"]) - 3 * b if b != 1 else c["Nk"]) if c["ragged"] else c["Nk"]
        k = max(0, min(c["Nk"], k))
        q = min(c["Nq"], k)
        start.append(k - q)
        nq.append(q)
        nk.append(k)
    return start, nq, nk


def _bounds(c, p, k_len):
    """[lo, hi) and the sinks' end of queries at positions p (numpy or torch, 64 bits)."""
    f = p // c["frame"]
    lo = (f - c["left"]) * c["frame"] if c["left"] >= 0 else 0 * p
    hi = (f + c["right"] + 1) * c["frame"] if c["right"] >= 0 else 0 * p + k_len
    return lo.clip(0, None), (hi - (hi - k_len).clip(0, None)).clip(0, None)


def _pairs(c):
    """(visible pairs, keys that some query sees) of one head over the batch."""
    pairs = keys = 0
    for start, nq, nk in zip(*_lengths(c)):
        lo, hi = _bounds(c, start + np.arange(nq, dtype=np.int64), nk)
        window = np.maximum(hi - lo, 0)
        sinks = np.minimum(np.minimum(c["sinks"], lo), hi)
        pairs += int((window + sinks).sum())
        if nq and hi[-1] > 0:
            keys += int(hi[-1] - lo[0] + min(c["sinks"], lo[0], hi[-1]))
    return pairs, keys


def work(case):
    c, size = case, 2 if case["dtype"] != "f32" else 4
    if c["kind"] == ROPE:
        n = c["B"] * (c["frames"] * c["rows"] * c["cols"] + c["text"]) * (c["H"] + c["Hkv"]) * c["D"]
        return {"bytes": 2 * n * size, "flops": 3 * n}
    if c["kind"] == NORM:
        n = c["tokens"] * max(c["heads"], 1) * c["width"]
        w = (4 if c["weights"] == "f32" else size) * c["width"] if c["affine"] else 0
        return {"bytes": (3 if c["train"] else 2) * n * size + (3 if c["train"] else 2) * w, "flops": (14 if c["train"] else 7) * n}
    pairs, keys = _pairs(c)
    nq = c["B"] * c["H"] * c["Nq"]
    times = 2 if c["train"] else 1
    data = times * (2 * nq * c["D"] * size + 2 * c["Hkv"] * keys * c["D"] * size) + 4 * nq
    return {"bytes": data, "flops": (14 if c["train"] else 4) * c["D"] * pairs * c["H"]}


# ---- inputs ------------------------------------------------------------------------------------------------
def _heads(gen, B, N, H, D, dtype, layout, n=1):
    """n tensors of logical shape [B, H, N, D]."""
    if layout == "fused":
        whole = torch.randn((B, N, 3, H, D), device="cuda", generator=gen).to(dtype)
        return [whole[:, :, i].transpose(1, 2) for i in range(n)]
    if layout == "bnhd":
        return [torch.randn((B, N, H, D), device="cuda", generator=gen).to(dtype).transpose(1, 2) for _ in range(n)]
    return [torch.randn((B, H, N, D), device="cuda", generator=gen).to(dtype) for _ in range(n)]


def _rope_dims(c):
    """Channels of the three axes: the space axes alike, time the rest."""
    side = c["D"] // 3 // 2 * 2
    return (c["D"] - 2 * side, side, side)


def prepare(case, seed):
    c, dtype = case, _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": c}
    if c["kind"] == ROPE:
        n_video = c["frames"] * c["rows"] * c["cols"]
        N = n_video + c["text"]
        if c["layout"] == "fused":
            state["q"], state["k"] = _heads(gen, c["B"], N, c["H"], c["D"], dtype, "fused", 2)
        else:
            (state["q"],) = _heads(gen, c["B"], N, c["H"], c["D"], dtype, c["layout"])
            (state["k"],) = _heads(gen, c["B"], N, c["Hkv"], c["D"], dtype, c["layout"])
        if c["listed_positions"]:
            t = torch.arange(N, device="cuda")
            grid = torch.stack([t // (c["rows"] * c["cols"]), t // c["cols"] % c["rows"], t % c["cols"]], 1)
            grid[n_video:] = -1
            state["positions"] = grid.to(torch.int32)
        # cosines and sines of every position of an axis, made once for all layers
        state["tables"] = []
        for dims, length in zip(_rope_dims(c), (c["frames"], c["rows"], c["cols"])):
            i = torch.arange(dims // 2, dtype=torch.float64, device="cuda")
            angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-2.0 * i / dims)
            state["tables"].append(torch.stack([torch.cos(angle), torch.sin(angle)]).float())
        if own:
            import paper_2603_05503_amd as pkg

            state["rope"] = pkg.RotaryAxes(_rope_dims(c), (c["frames"], c["rows"], c["cols"]), interleaved=not c["halves"])
        return state
    if c["kind"] == NORM:
        shape = (c["tokens"], c["heads"], c["width"]) if c["heads"] else (c["tokens"], c["width"])
        state["x"] = (torch.randn(shape, device="cuda", generator=gen) * 1.5 + 0.3).to(dtype)
        state["weight"] = state["bias"] = None
        if c["affine"]:
            wtype = _TYPES[c["weights"]]
            state["weight"] = (1.0 + 0.2 * torch.randn(c["width"], device="cuda", generator=gen)).to(wtype)
            state["bias"] = (0.2 * torch.randn(c["width"], device="cuda", generator=gen)).to(wtype)
        if c["train"]:
            state["dy"] = torch.randn(shape, device="cuda", generator=gen).to(dtype)
        return state
    if c["layout"] == "fused":
        state["q"], state["k"], state["v"] = _heads(gen, c["B"], c["Nk"], c["H"], c["D"], dtype, "fused", 3)
    else:
        (state["q"],) = _heads(gen, c["B"], c["Nq"], c["H"], c["D"], dtype, c["layout"])
        state["k"], state["v"] = _heads(gen, c["B"], c["Nk"], c["Hkv"], c["D"], dtype, c["layout"], 2)
    if c["train"]:
        (state["dout"],) = _heads(gen, c["B"], c["Nq"], c["H"], c["D"], dtype, "packed")
    state["lengths"] = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in _lengths(c)]
    if own:
        import paper_2603_05503_amd as pkg

        state["window"] = pkg.Window(left=c["left"], right=c["right"], sinks=c["sinks"], frame=c["frame"],
                                     offset=c["Nk"] - c["Nq"])
    return state


# ---- the operators in their plain form ---------------------------------------------------------------------
def _plain_rope(s):
    c, q = s["case"], s["q"]
    N, S = q.shape[2], sum(_rope_dims(c)) // 2
    t = torch.arange(N, device=q.device)
    if c["listed_positions"]:
        pos = s["positions"].long()
    else:
        pos = torch.stack([t // (c["rows"] * c["cols"]), t // c["cols"] % c["rows"], t % c["cols"]], 1)
    has = (t < N - c["text"])[:, None]
    turn = torch.cat([tab[:, pos[:, a].clamp(0, tab.shape[1] - 1)] for a, tab in enumerate(s["tables"])], 2)
    cos, sin = torch.where(has, turn[0], 1.0), torch.where(has, turn[1], 0.0)
    if c["inverse"]:
        sin = -sin

    def rotated(x):
        x = x.float()
        a, b = (x[..., :S], x[..., S:]) if c["halves"] else (x[..., 0::2], x[..., 1::2])
        u, v = a * cos - b * sin, a * sin + b * cos
        return (torch.cat([u, v], -1) if c["halves"] else torch.stack([u, v], -1).flatten(-2)).to(q.dtype)

    return {"q": rotated(q), "k": rotated(s["k"])}


def _plain_norm(s, eps=1e-6):
    c, x = s["case"], s["x"].float()
    if c["center"]:
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    h = x * r
    if not c["train"]:
        y = h * s["weight"].float() + s["bias"].float() if c["affine"] else h
        return {"y": y.to(s["x"].dtype)}
    dy = s["dy"].float()
    g = dy * s["weight"].float() if c["affine"] else dy
    d = g - h * (g * h).mean(-1, keepdim=True)
    if c["center"]:
        d = d - g.mean(-1, keepdim=True)
    out = {"dx": (d * r).to(s["x"].dtype)}
    if c["affine"]:
        rows = tuple(range(x.dim() - 1))
        out["dweight"] = (dy * h).sum(rows).to(s["weight"].dtype)
        out["dbias"] = dy.sum(rows).to(s["weight"].dtype)
    return out


def _visible(c, lengths, device):
    """Truth values [B, Nq, Nk]."""
    start, nq, nk = (x.long()[:, None] for x in lengths)
    i, j = torch.arange(c["Nq"], device=device)[None], torch.arange(c["Nk"], device=device)
    lo, hi = _bounds(c, start + i, nk)
    return (j < hi[..., None]) & ((j >= lo[..., None]) | (j < c["sinks"])) & (i < nq)[..., None]


def _plain_attention(s):
    c = s["case"]
    B, H, Hkv, Nq, D, G = c["B"], c["H"], c["Hkv"], c["Nq"], c["D"], c["H"] // c["Hkv"]
    scale = 1.0 / math.sqrt(D)
    q = s["q"].float().reshape(B, Hkv, G * Nq, D)
    k, v = s["k"].float().contiguous(), s["v"].float().contiguous()
    seen = _visible(c, s["lengths"], q.device)[:, None, None]
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(B, Hkv, G, Nq, c["Nk"])
    p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True).clamp_(min=-1e30)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total.clamp(min=1e-30))
    p = p.view(B, Hkv, G * Nq, c["Nk"])
    out = torch.matmul(p, v)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf).view(B, H, Nq)
    res = {"out": out.view(B, H, Nq, D).to(s["q"].dtype), "lse": lse}
    if c["train"]:
        do = s["dout"].float().reshape(B, Hkv, G * Nq, D)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
        ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        del p
        res["dq"] = torch.matmul(ds, k).view(B, H, Nq, D).to(s["q"].dtype)
        res["dk"] = torch.matmul(ds.transpose(2, 3).contiguous(), q).to(s["q"].dtype)
        res["dv"] = dv.to(s["q"].dtype)
    return res


# ---- the library's calls -----------------------------------------------------------------------------------
def _own(s):
    import paper_2603_05503_amd as pkg

    c = s["case"]
    if c["kind"] == ROPE:
        where = dict(positions=s["positions"]) if c["listed_positions"] else dict(grid=(c["frames"], c["rows"], c["cols"]))
        q, k = pkg.rope_axes(s["q"], s["k"], s["rope"], inverse=c["inverse"], **where)
        return {"q": q, "k": k}
    if c["kind"] == NORM:
        if not c["train"]:
            return {"y": pkg.layer_norm_fwd(s["x"], s["weight"], s["bias"], eps=1e-6, center=c["center"])}
        dx, dw, db = pkg.layer_norm_bwd(s["dy"], s["x"], s["weight"], s["bias"], eps=1e-6, center=c["center"])
        return {"dx": dx, "dweight": dw, "dbias": db} if c["affine"] else {"dx": dx}
    scale = 1.0 / math.sqrt(c["D"])
    lengths = dict(zip(("q_start", "q_len", "k_len"), s["lengths"])) if c["ragged"] else {}
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=s["q"].device)
    pkg.window_attn_fwd(s["q"], s["k"], s["v"], out, s["window"], scale, lse=lse, **lengths)
    res = {"out": out, "lse": lse}
    if c["train"]:
        res["dq"], res["dk"], res["dv"] = pkg.window_attn_bwd(s["dout"], s["q"], s["k"], s["v"], out, lse, s["window"], scale,
                                                              **lengths)
    return res


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return _plain_rope(state) if kind == ROPE else _plain_norm(state) if kind == NORM else _plain_attention(state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def _exact_rope(c, s):
    q = s["q"]
    N, n_video, D = q.shape[2], q.shape[2] - c["text"], c["D"]
    angle = torch.zeros((N, D // 2), dtype=torch.float64, device=q.device)
    n = torch.arange(n_video, device=q.device)
    place = (torch.div(n, c["rows"] * c["cols"], rounding_mode="floor"),
             torch.div(n, c["cols"], rounding_mode="floor").remainder(c["rows"]), n.remainder(c["cols"]))
    at = 0
    for dims, pos in zip(_rope_dims(c), place):
        for i in range(dims // 2):
            angle[:n_video, at + i] = pos.double() / 10000.0 ** (2.0 * i / dims)
        at += dims // 2
    turn = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)

    def rotated(x):
        out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        for h in range(x.shape[1]):
            y = x[:, h].double()
            z = torch.complex(y[..., : D // 2], y[..., D // 2:]) if c["halves"] else torch.view_as_complex(
                y.reshape(y.shape[0], N, D // 2, 2).contiguous())
            z = z * turn
            out[:, h] = torch.cat([z.real, z.imag], -1) if c["halves"] else torch.view_as_real(z).reshape(y.shape)
        return out

    return {"q": rotated(q), "k": rotated(s["k"])}


def _exact_norm(c, s, eps=1e-6):
    x = s["x"].double().reshape(-1, c["width"])
    mean = x.mean(1) if c["center"] else torch.zeros_like(x[:, 0])
    var = ((x - mean[:, None]) ** 2).sum(1) / c["width"]
    std = (var + eps).sqrt()
    h = (x - mean[:, None]) / std[:, None]
    w = s["weight"].double() if c["affine"] else torch.ones(c["width"], dtype=torch.float64, device=x.device)
    if not c["train"]:
        y = h * w
        if c["affine"]:
            y += s["bias"].double()
        return {"y": y.reshape(s["x"].shape)}
    dy = s["dy"].double().reshape(-1, c["width"])
    g = dy * w
    # the jacobian's three terms: of the row itself, of its mean, of its deviation
    dx = g / std[:, None] - h * ((g * h).sum(1) / c["width"] / std)[:, None]
    if c["center"]:
        dx -= (g.sum(1) / c["width"] / std)[:, None]
    out = {"dx": dx.reshape(s["x"].shape)}
    if c["affine"]:
        out["dweight"] = (dy * h).sum(0)
        out["dbias"] = dy.sum(0)
    return out


def _exact_attention(c, s):
    """Head by head and query rows in pieces, so that 64-bit scores stay small."""
    dev, D, G, scale = s["q"].device, c["D"], c["H"] // c["Hkv"], 1.0 / math.sqrt(c["D"])
    f64 = dict(dtype=torch.float64, device=dev)
    out, dq = torch.zeros(s["q"].shape, **f64), torch.zeros(s["q"].shape, **f64)
    dk, dv = torch.zeros(s["k"].shape, **f64), torch.zeros(s["k"].shape, **f64)
    lse = torch.full(s["q"].shape[:3], -math.inf, **f64)
    for b, (start, nq, nk) in enumerate(zip(*_lengths(c))):
        if nq == 0:
            continue
        j = torch.arange(nk, device=dev)
        step = max(1, (1 << 27) // max(nk, 1))
        for i0 in range(0, nq, step):
            i1 = min(nq, i0 + step)
            frame = torch.div(start + torch.arange(i0, i1, device=dev), c["frame"], rounding_mode="floor")[:, None]
            near = torch.ones((i1 - i0, nk), dtype=torch.bool, device=dev)
            of = torch.div(j, c["frame"], rounding_mode="floor")
            if c["left"] >= 0:
                near &= of >= frame - c["left"]
            if c["sinks"] > 0:
                near |= j < c["sinks"]
            if c["right"] >= 0:
                near &= of <= frame + c["right"]
            for h in range(c["H"]):
                k, v, q = s["k"][b, h // G, :nk].double(), s["v"][b, h // G, :nk].double(), s["q"][b, h, i0:i1].double()
                logits = torch.where(near, (q @ k.T) * scale, -math.inf)
                z = torch.logsumexp(logits, 1)
                p = torch.where(near, torch.exp(logits - z[:, None]), 0.0)
                o = p @ v
                lse[b, h, i0:i1], out[b, h, i0:i1] = z, o
                if c["train"]:
                    do = s["dout"][b, h, i0:i1].double()
                    ds = p * (do @ v.T - (do * o).sum(1, keepdim=True)) * scale
                    dq[b, h, i0:i1] = ds @ k
                    dk[b, h // G, :nk] += ds.T @ q
                    dv[b, h // G, :nk] += p.T @ do
    res = {"out": out, "lse": lse}
    return dict(res, dq=dq, dk=dk, dv=dv) if c["train"] else res


def exact(case, seed):
    c = case
    if c["kind"] in (STEP, WINDOW) and c["B"] * c["H"] * c["Nq"] * c["Nk"] * (3 if c["train"] else 1) > 8e9:
        return None
    s = prepare(c, seed)
    return _exact_rope(c, s) if c["kind"] == ROPE else _exact_norm(c, s) if c["kind"] == NORM else _exact_attention(c, s)
