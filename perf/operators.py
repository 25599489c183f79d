"""The learned operators on ragged birds, as a program that uses them asks for them.

A per-bird encoder takes the detections of a batch of frames (or the tracks of
a batch of birds) and runs, on the library's CSR layout:

  norm       layer norm of every bird's features, with the residual sum, and
             its backward pass with the weights' gradients
  rotary     rotary positions of queries and keys from time, y and x
  attention  attention within each frame (or track): capped scores, a bias
             that falls with the squared distance between birds, hidden birds,
             order with a prefix; its backward pass; one query over a long
             history

  listed()   the cases that are always timed
  draw(rng)  another case of the same ranges
  prepare    what the program has in hand before the call
  run        one pass: plain torch in 32 bits, or the library's entry points
             where own is true
  work       bytes and flops that a pass cannot do without
  exact      the outputs in 64 bits, from the definitions

Inputs are synthetic and made on the GPU from the seed alone: unit normal
features, birds in Gaussian groups over a uniform background.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

QUANTA = 16  # positions are in 1/16 px

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _norm(rows, width, **more):
    case = {"kind": "norm", "rows": rows, "width": width, "dtype": "bfloat16",
            "residual": False,  # add the block's input first, and return the sum
            "train": False,     # backward too
            "eps": 1e-5}
    case.update(more)
    return case


def _rotary(birds, frames, **more):
    case = {"kind": "rotary", "birds": birds, "frames": frames, "dtype": "bfloat16",
            "q_heads": 8, "k_heads": 8, "head_dim": 64,
            "t_pairs": 8, "y_pairs": 12, "x_pairs": 12,   # pairs of dimensions turned by time, y and x
            "width": 1920, "height": 1080,
            "fused": True,          # queries, keys and values are slices of one projection
            "interleaved": False,   # pairs (2j, 2j + 1), else (j, j + pairs)
            "inverse": False}       # turned back: the gradient's direction
    case.update(more)
    return case


def _attention(frames, birds, **more):
    case = {"kind": "attention", "frames": frames, "birds": birds, "dtype": "bfloat16",
            "counts": "even",       # "even", "poisson" around birds, or "tracks" of 1 to birds
            "queries": 0,           # queries per frame, 0: the birds themselves
            "q_heads": 8, "kv_heads": 8, "head_dim": 64,
            "width": 1920, "height": 1080, "groups": 6, "uniform": 0.1,
            "distance": True,       # scores fall with the squared distance
            "cap": 0.0,             # scores capped by cap * tanh(s / cap)
            "hidden": 0.0,          # share of the keys that take no part
            "causal": False,        # a key is seen by itself and later ones ...
            "prefix": 0,            # ... or, among the first `prefix`, by all
            "fused": True, "train": False}
    case.update(more)
    return case


def listed():
    return [
        # one live frame of 500 birds: the encoder's norm, where latency counts
        dict(_norm(500, 512), name="norm 500x512"),
        # a training step's norm with the residual sum, two seconds of video
        dict(_norm(128000, 512, residual=True, train=True), name="norm train 128000x512"),
        # master-precision features of an odd width, a whole house in one frame
        dict(_norm(30000, 333, dtype="float32", train=True), name="norm train 30000x333 f32"),
        # one live frame
        dict(_rotary(500, 1), name="rotary 500"),
        # two seconds of video, queries and keys in the fused projection
        dict(_rotary(128000, 64), name="rotary 128000"),
        # the gradient's direction, in single precision, few key heads
        dict(_rotary(30000, 1, dtype="float32", q_heads=6, k_heads=2, head_dim=96, t_pairs=0, y_pairs=21, x_pairs=21, width=3840,
                     height=2160, fused=False, interleaved=True, inverse=True), name="rotary back 30000 f32"),
        # one live frame
        dict(_attention(1, 500, uniform=1.0), name="attention 1x500"),
        # two seconds of video, inference with capped scores
        dict(_attention(64, 2000, cap=30.0, dtype="float16"), name="attention 64x2000 cap"),
        # 4K frames of ragged counts, wide heads shared by four queries each, some birds hidden
        dict(_attention(24, 8000, counts="poisson", kv_heads=2, head_dim=128, width=3840, height=2160, groups=12,
                        hidden=0.1), name="attention 24x8000 shared"),
        # a training step on two seconds of video
        dict(_attention(64, 2000, train=True), name="attention train 64x2000"),
        # a training step on tracks: what a bird did before, a few frames of context seen by all
        dict(_attention(96, 4500, counts="tracks", distance=False, causal=True, prefix=30, kv_heads=4, train=True,
                        dtype="float16"), name="attention train 96 tracks"),
        # one query per camera over some minutes of history
        dict(_attention(256, 8000, counts="poisson", queries=1, kv_heads=2, head_dim=128, fused=False),
             name="attention token 256x8000"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["norm", "norm", "rotary", "rotary", "attention", "attention", "attention", "attention"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if kind == "norm":
        width = rng.choice([_log(rng, 16, 4096), 64 * _log(rng, 1, 32), 8 * _log(rng, 4, 200)])
        rows = _log(rng, 1, max(2, 128000 * 512 // width))
        return _norm(rows, width, dtype=dtype, residual=rng.random() < 0.5, train=rng.random() < 0.6,
                     eps=rng.choice([1e-5, 1e-6, 1e-3]))
    if kind == "rotary":
        dim = rng.choice([32, 64, 64, 96, 128, 128])
        kv = rng.choice([1, 2, 4, 6, 8])
        group = rng.choice([1, 1, 2, 4])
        half = dim // 2
        nt = rng.randrange(0, half // 2)
        ny = rng.randrange(0, (half - nt) // 2 + 1)
        nx = half - nt - ny if rng.random() < 0.5 else rng.randrange(0, half - nt - ny + 1)
        if nt + ny + nx == 0:
            nx = 1
        frames = _log(rng, 1, 64)
        birds = max(frames, _log(rng, 1, 128000 * 1024 // ((kv * group + kv) * dim)))
        return _rotary(min(birds, 300000), frames, dtype=dtype, q_heads=kv * group, k_heads=kv, head_dim=dim,
                       t_pairs=nt, y_pairs=ny, x_pairs=nx, fused=rng.random() < 0.5, interleaved=rng.random() < 0.3,
                       inverse=rng.random() < 0.3)
    dtype = rng.choice(["bfloat16", "float16"])
    dim = rng.choice([32, 64, 64, 64, 96, 128, 128, 40, 80])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 1, 2, 4, 8])
    form = rng.choice(["infer", "infer", "train", "train", "token"])
    more = dict(dtype=dtype, q_heads=kv * group, kv_heads=kv, head_dim=dim, train=form == "train",
                distance=rng.random() < 0.6, cap=rng.choice([0.0, 0.0, 15.0, 50.0]),
                hidden=rng.choice([0.0, 0.0, 0.1, 0.6]), counts=rng.choice(["even", "poisson", "tracks"]),
                fused=rng.random() < 0.5)
    if form == "token":
        return _attention(_log(rng, 1, 256), _log(rng, 1, 16000), queries=rng.choice([1, 1, 1, 2, 5]),
                          causal=rng.random() < 0.3, **dict(more, train=False, fused=False))
    if rng.random() < 0.4:
        more.update(causal=True, prefix=rng.choice([0, 0, 7, 100]))
    return _attention(_log(rng, 1, 200), _log(rng, 1, 16000), **more)


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    most_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw_once(rng)
        w = work(case)
        if case["kind"] != "attention" or (w["flops"] <= 0.5 * most and w["bytes"] <= most_bytes
                                           and case["frames"] * case["birds"] * case["q_heads"] <= 20_000_000):
            return case


# ---------------------------------------------------------------------------
# What the case says about sizes
# ---------------------------------------------------------------------------

def _key_counts(case):
    """Keys per frame, from the case alone."""
    F, n = case["frames"], case["birds"]
    if case["counts"] == "even":
        return [n] * F
    rng = random.Random(7919 * F + n)
    if case["counts"] == "poisson":
        return [max(0, int(round(rng.gauss(n, math.sqrt(n))))) for _ in range(F)]
    return [1 + rng.randrange(n) for _ in range(F)]


def _query_counts(case):
    return [case["queries"]] * case["frames"] if case["queries"] else _key_counts(case)


def _seen_pairs(case):
    """(query, key) pairs within the frames and the order (hidden keys count)."""
    pairs = 0
    for nq, nk in zip(_query_counts(case), _key_counts(case)):
        if not case["causal"]:
            pairs += nq * nk
            continue
        pre = min(case["prefix"], nk)
        last = np.clip(np.arange(nq, dtype=np.int64) + (nk - nq) + 1, 0, nk)
        pairs += int(np.maximum(last, pre).sum())
    return pairs


def _pairs(case):
    return case["t_pairs"], case["y_pairs"], case["x_pairs"]


def work(case):
    b = SIZE[case["dtype"]]
    if case["kind"] == "norm":
        cells = case["rows"] * case["width"]
        moved = 2 + 2 * case["residual"]
        flops = 8 * cells
        if case["train"]:
            # the gradient of the output (and of the sum), the normalised input again, the input's gradient
            moved += 3 + case["residual"]
            flops += 14 * cells
        return {"bytes": moved * cells * b + (8 + 8 * case["train"]) * case["width"], "flops": flops}
    if case["kind"] == "rotary":
        heads = case["q_heads"] + case["k_heads"]
        cells = case["birds"] * heads * case["head_dim"]
        turned = case["birds"] * heads * 2 * sum(_pairs(case))
        return {"bytes": 2 * cells * b + 12 * case["birds"], "flops": 3 * turned}
    tq, tk = sum(_query_counts(case)), sum(_key_counts(case))
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    q_bytes, k_bytes = tq * Hq * D * b, tk * Hk * D * b
    total = 2 * q_bytes + 2 * k_bytes
    flops = 4 * _seen_pairs(case) * Hq * D
    if case["train"]:
        total += 2 * q_bytes + 2 * k_bytes
        flops += 10 * _seen_pairs(case) * Hq * D
    total += (8 * (tq + tk) if case["distance"] else 0) + (tk if case["hidden"] else 0)
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _places(total, case, gen):
    """int32 [total, 2] in 1/16 px: Gaussian groups over a uniform background."""
    w, h = case["width"], case["height"]
    size = torch.tensor([w, h], dtype=torch.float32, device="cuda")
    spots = torch.rand(total, 2, device="cuda", generator=gen) * size
    groups = case.get("groups", 6)
    if groups:
        means = torch.rand(groups, 2, device="cuda", generator=gen) * size
        std = 80 + 120 * torch.rand(groups, 1, device="cuda", generator=gen)
        which = torch.randint(0, groups, (total,), device="cuda", generator=gen)
        near = means[which] + std[which] * torch.randn(total, 2, device="cuda", generator=gen)
        alone = torch.rand(total, 1, device="cuda", generator=gen) < case.get("uniform", 0.1)
        spots = torch.where(alone, spots, near)
    q = (spots * QUANTA).to(torch.int32)
    top = torch.tensor([QUANTA * w - 1, QUANTA * h - 1], dtype=torch.int32, device="cuda")
    return torch.minimum(q.clamp_min(0), top).contiguous()


def _offsets(counts):
    return torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")


def _frequencies(case):
    """Radians per frame for the time pairs, per px for the y and x pairs:
    wavelengths from 16 frames to 9000 (five minutes), 32 px to 8192 px."""
    nt, ny, nx = _pairs(case)
    def axis(n, short, long):
        return [2 * math.pi / (short * (long / short) ** (j / max(n - 1, 1))) for j in range(n)]
    return axis(nt, 16.0, 9000.0), axis(ny, 32.0, 8192.0), axis(nx, 32.0, 8192.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    state = dict(case)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(dtype)

    if case["kind"] == "norm":
        n, w = case["rows"], case["width"]
        state["x"] = normal(n, w) + 0.5
        state["weight"] = 1 + 0.1 * torch.randn(w, device="cuda", generator=gen)
        state["bias"] = 0.1 * torch.randn(w, device="cuda", generator=gen)
        state["r"] = normal(n, w) if case["residual"] else None
        state["grad_y"] = normal(n, w) if case["train"] else None
        state["grad_sum"] = normal(n, w) if case["train"] and case["residual"] else None
        return state
    if case["kind"] == "rotary":
        n, Hq, Hk, D = case["birds"], case["q_heads"], case["k_heads"], case["head_dim"]
        if case["fused"]:
            qkv = normal(n, Hq + 2 * Hk, D)
            state["q"], state["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        else:
            state["q"], state["k"] = normal(n, Hq, D), normal(n, Hk, D)
        state["xy"] = _places(n, case, gen)
        state["time"] = (torch.arange(n, device="cuda", dtype=torch.int64) * case["frames"] // n).to(torch.int32) \
            + int(torch.randint(0, 9000, (1,), generator=torch.Generator().manual_seed(seed)))
        freq_t, freq_y, freq_x = _frequencies(case)
        if own:
            import paper_2512_07009_amd as flock
            state["axes"] = flock.RotaryAxes(freq_t, freq_y, freq_x)
        else:
            # turns per frame and per 1/16 px in 2^-64 turns: integer products give the phase without error
            per = [f / (2 * math.pi) for f in freq_t] + [f / (2 * math.pi * QUANTA) for f in freq_y + freq_x]
            steps = [int(p * 2.0 ** 64) % (1 << 64) for p in per]
            state["steps"] = torch.tensor([s - (1 << 64) if s >> 63 else s for s in steps], dtype=torch.int64,
                                          device="cuda")
        return state
    Hq, Hk, D = case["q_heads"], case["kv_heads"], case["head_dim"]
    state["k_counts"], state["q_counts"] = _key_counts(case), _query_counts(case)
    tk, tq = sum(state["k_counts"]), sum(state["q_counts"])
    if case["fused"] and not case["queries"]:
        qkv = normal(tk, Hq + 2 * Hk, D)
        state["q"], state["k"], state["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        state["q"], state["k"], state["v"] = normal(tq, Hq, D), normal(tk, Hk, D), normal(tk, Hk, D)
    state["k_offsets"] = _offsets(state["k_counts"])
    state["q_offsets"] = _offsets(state["q_counts"]) if case["queries"] else state["k_offsets"]
    state["k_xy"] = state["q_xy"] = state["slopes"] = None
    if case["distance"]:
        state["k_xy"] = _places(tk, case, gen)
        state["q_xy"] = _places(tq, case, gen) if case["queries"] else state["k_xy"]
        # heads look from 30 px to the whole frame: slope = 1 / (2 sigma^2)
        sigma = 30.0 * 32.0 ** (torch.arange(Hq, device="cuda", dtype=torch.float32) / max(Hq - 1, 1))
        state["slopes"] = 0.5 / (sigma * sigma)
    state["keep"] = (torch.rand(tk, device="cuda", generator=gen) >= case["hidden"]).to(torch.uint8) \
        if case["hidden"] else None
    state["prefix_lengths"] = torch.full((case["frames"],), case["prefix"], dtype=torch.int32, device="cuda") \
        if case["causal"] and case["prefix"] else None
    state["scale"] = D ** -0.5
    state["grad_out"] = normal(tq, Hq, D) if case["train"] else None
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    kind = state["kind"]
    if own:
        return {"norm": _own_norm, "rotary": _own_rotary, "attention": _own_attention}[kind](state)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "attention": _plain_attention}[kind](state)


def _own_norm(s):
    import paper_2512_07009_amd as flock
    y, h, mean, rstd = flock.layer_norm_rows(s["x"], s["weight"], s["bias"], s["eps"], residual=s["r"])
    out = {"y": y}
    if s["residual"]:
        out["sum"] = h
    if s["train"]:
        out["dx"], out["dw"], out["db"] = flock.layer_norm_rows_backward(s["grad_y"], h, s["weight"], mean, rstd,
                                                                         grad_sum=s["grad_sum"])
    return out


def _own_rotary(s):
    import paper_2512_07009_amd as flock
    q, k = flock.rotary_frames(s["q"], s["k"], s["xy"], s["axes"], time=s["time"], interleaved=s["interleaved"],
                               inverse=s["inverse"])
    return {"q": q, "k": k}


def _own_attention(s):
    import paper_2512_07009_amd as flock
    more = dict(k_offsets=s["k_offsets"], q_xy=s["q_xy"], k_xy=s["k_xy"], slopes=s["slopes"], scale=s["scale"],
                cap=s["cap"], keep=s["keep"], causal=s["causal"], prefix=s["prefix_lengths"])
    if not s["train"]:
        return {"out": flock.attention_frames(s["q"], s["k"], s["v"], s["q_offsets"], **more)}
    out, lse = flock.attention_frames(s["q"], s["k"], s["v"], s["q_offsets"], return_lse=True, **more)
    dq, dk, dv, ds = flock.attention_frames_backward(s["grad_out"], s["q"], s["k"], s["v"], out, lse, s["q_offsets"],
                                                     **more)
    grads = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if s["distance"]:
        grads["dslopes"] = ds
    return grads


# --- plain forms ---

def _plain_norm(s):
    x = s["x"].float()
    out = {}
    if s["residual"]:
        # the sum is kept in the features' type, and that is what is normalised
        h = (x + s["r"].float()).to(s["x"].dtype)
        out["sum"] = h
        x = h.float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + s["eps"])
    xh = c * rstd
    out["y"] = (xh * s["weight"] + s["bias"]).to(s["x"].dtype)
    if s["train"]:
        gy = s["grad_y"].float()
        g = gy * s["weight"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s["residual"]:
            dx = dx + s["grad_sum"].float()
        out["dx"] = dx.to(s["x"].dtype)
        out["dw"] = (gy * xh).sum(0)
        out["db"] = gy.sum(0)
    return out


def _plain_rotary(s):
    nt, ny, nx = _pairs(s)
    pos = torch.cat([s["time"][:, None].expand(-1, nt), s["xy"][:, 1:2].expand(-1, ny),
                     s["xy"][:, 0:1].expand(-1, nx)], 1).to(torch.int64)
    phase = (pos * s["steps"]) >> 32            # signed 2^-32 turns, whole turns dropped by the overflow
    angle = phase.to(torch.float32) * (2 * math.pi / 2.0 ** 32)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if s["inverse"]:
        sin = -sin
    n = nt + ny + nx

    def turn(t):
        z = t.float()
        if s["interleaved"]:
            a, b = z[..., 0:2 * n:2], z[..., 1:2 * n:2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = z[..., :n], z[..., n:2 * n]
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([turned, z[..., 2 * n:]], -1).to(t.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _frame_groups(s, most):
    """Runs of frames whose padded scores hold at most `most` numbers (or one
    frame), with the query rows taken at a time: (first, past, nq, nk, rows)."""
    F, Hq = len(s["k_counts"]), s["q_heads"]
    f0 = 0
    while f0 < F:
        nq, nk, f1 = s["q_counts"][f0], s["k_counts"][f0], f0 + 1
        while f1 < F:
            a, b = max(nq, s["q_counts"][f1]), max(nk, s["k_counts"][f1])
            if (f1 + 1 - f0) * Hq * a * b > most:
                break
            nq, nk, f1 = a, b, f1 + 1
        if nq > 0:
            yield f0, f1, nq, nk, max(1, min(nq, most // max(1, (f1 - f0) * Hq * nk)))
        f0 = f1


def _plain_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    Hq, Hk, D = s["q_heads"], s["kv_heads"], s["head_dim"]
    G, dev, tq, tk = Hq // Hk, q.device, q.shape[0], k.shape[0]
    qo, ko = s["q_offsets"].long(), s["k_offsets"].long()
    train, cap = s["train"], s["cap"]
    # one more row takes what is written for the padding
    out = torch.zeros(tq + 1, Hq, D, device=dev)
    if train:
        dq = torch.zeros(tq + 1, Hq, D, device=dev)
        dk, dv = torch.zeros(tk + 1, Hk, D, device=dev), torch.zeros(tk + 1, Hk, D, device=dev)
        dslopes = torch.zeros(Hq, device=dev)
    for f0, f1, nq, nk, step in _frame_groups(s, 1 << 29):
        if nk == 0:
            continue
        B = f1 - f0
        kcount = (ko[f0 + 1:f1 + 1] - ko[f0:f1])[:, None]
        qcount = (qo[f0 + 1:f1 + 1] - qo[f0:f1])[:, None]
        kj = torch.arange(nk, device=dev)[None, :]
        kvalid = kj < kcount
        kidx = torch.where(kvalid, ko[f0:f1, None] + kj, 0)
        kk = k[kidx].float().permute(0, 2, 3, 1)                        # [B, Hk, D, nk]
        vv = v[kidx].float().permute(0, 2, 1, 3) * kvalid[:, None, :, None]
        for i0 in range(0, nq, step):
            n = min(step, nq - i0)
            qi = torch.arange(i0, i0 + n, device=dev)[None, :]
            qvalid = qi < qcount
            qidx = torch.where(qvalid, qo[f0:f1, None] + qi, 0)
            qq = q[qidx].float().view(B, n, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, D)
            t = torch.matmul(qq, kk).mul_(s["scale"]).view(B, Hk, G, n, nk)
            if cap:
                t = torch.tanh(t.div_(cap))
                sc = t * cap
            else:
                sc = t
            if s["distance"]:
                qp, kp = s["q_xy"][qidx].float() / QUANTA, s["k_xy"][kidx].float() / QUANTA
                d2 = (qp[:, :, None, 0] - kp[:, None, :, 0]) ** 2 + (qp[:, :, None, 1] - kp[:, None, :, 1]) ** 2
                sc = sc - s["slopes"].view(1, Hk, G, 1, 1) * d2[:, None, None]
            seen = kvalid[:, None, :].expand(B, n, nk)
            if s["keep"] is not None:
                seen = seen & (s["keep"][kidx] != 0)[:, None, :]
            if s["causal"]:
                order = kj[:, None, :] <= qi[:, :, None] + (kcount - qcount)[:, :, None]
                if s["prefix_lengths"] is not None:
                    order = order | (kj < s["prefix_lengths"][f0:f1, None])[:, None, :]
                seen = seen & order
            sc = sc.masked_fill(~seen[:, None, None], -math.inf)
            top = sc.amax(-1, keepdim=True)
            p = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
            del sc
            total = p.sum(-1, keepdim=True)
            p = p.div_(torch.where(total == 0, 1.0, total)).view(B, Hk, G * n, nk)
            o = torch.matmul(p, vv)
            to = torch.where(qvalid, qidx, tq).flatten()
            rows = lambda z: z.view(B, Hk, G, n, D).permute(0, 3, 1, 2, 4).reshape(B * n, Hq, D)  # noqa: E731
            out[to] = rows(o)
            if not train:
                continue
            go = (s["grad_out"][qidx].float() * qvalid[:, :, None, None]).view(B, n, Hk, G, D)
            go = go.permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, D)
            dv_part = torch.matmul(p.transpose(2, 3), go)
            dp = torch.matmul(go, vv.transpose(2, 3))
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            del dp, p
            if s["distance"]:
                dslopes -= (ds.view(B, Hk, G, n, nk) * d2[:, None, None]).sum((0, 3, 4)).view(Hq)
            if cap:
                ds = ds * (1 - t * t).view(B, Hk, G * n, nk)
            dq[to] = rows(torch.matmul(ds, kk.transpose(2, 3)) * s["scale"])
            dk_part = torch.matmul(ds.transpose(2, 3), qq) * s["scale"]
            kto = torch.where(kvalid, kidx, tk).flatten()
            dk.index_add_(0, kto, dk_part.permute(0, 2, 1, 3).reshape(B * nk, Hk, D))
            dv.index_add_(0, kto, dv_part.permute(0, 2, 1, 3).reshape(B * nk, Hk, D))
    result = {"out": out[:tq].to(q.dtype)}
    if train:
        result.update(dq=dq[:tq].to(q.dtype), dk=dk[:tk].to(q.dtype), dv=dv[:tk].to(q.dtype))
        if s["distance"]:
            result["dslopes"] = dslopes
    return result


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "attention": _exact_attention}[case["kind"]](s)


def _exact_norm(s):
    out = {"y": None}
    x = s["x"].double()
    if s["residual"]:
        out["sum"] = s["x"].double() + s["r"].double()
        x = out["sum"].to(s["x"].dtype).double()     # normalised as it is kept
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    xh = (x - mean) / torch.sqrt(var + s["eps"])
    w = s["weight"].double()
    out["y"] = xh * w + s["bias"].double()
    if s["train"]:
        gy, n = s["grad_y"].double(), s["width"]
        out["dw"], out["db"] = torch.sum(gy * xh, 0), torch.sum(gy, 0)
        gh = gy * w
        # the row's Jacobian: (I - 1 1^T / n - xh xh^T / n) / sqrt(var + eps)
        dx = gh - gh.sum(1, keepdim=True) / n - xh * ((xh * gh).sum(1, keepdim=True) / n)
        out["dx"] = dx / torch.sqrt(var + s["eps"])
        if s["residual"]:
            out["dx"] = out["dx"] + s["grad_sum"].double()
    return out


def _exact_rotary(s):
    ft, fy, fx = _frequencies(s)
    place = s["xy"].double() / QUANTA
    angles = [s["time"].double() * f for f in ft] + [place[:, 1] * f for f in fy] + [place[:, 0] * f for f in fx]
    sign = -1.0 if s["inverse"] else 1.0
    n = len(angles)
    result = {}
    for name in ("q", "k"):
        z = s[name].double()
        w = z.clone()
        for p, angle in enumerate(angles):
            a, b = (2 * p, 2 * p + 1) if s["interleaved"] else (p, p + n)
            turn = torch.polar(torch.ones_like(angle), sign * angle)[:, None]
            r = torch.complex(z[:, :, a].contiguous(), z[:, :, b].contiguous()) * turn
            w[:, :, a], w[:, :, b] = r.real, r.imag
        result[name] = w
    return result


def _exact_attention(s):
    """One frame and one head at a time, a block of queries after the other."""
    if work({k: s[k] for k in _attention(1, 1)})["flops"] > 2e13:
        return None
    Hq, G, scale, cap = s["q_heads"], s["q_heads"] // s["kv_heads"], s["scale"], s["cap"]
    q, k, v = s["q"], s["k"], s["v"]
    f64 = dict(dtype=torch.float64, device="cuda")
    out = torch.zeros(q.shape, **f64)
    train = s["train"]
    if train:
        dq, dk, dv = torch.zeros(q.shape, **f64), torch.zeros(k.shape, **f64), torch.zeros(v.shape, **f64)
        dslopes = torch.zeros(Hq, **f64)
    q0 = k0 = 0
    for f, (nq, nk) in enumerate(zip(s["q_counts"], s["k_counts"])):
        sel_k = slice(k0, k0 + nk)
        block = max(1, min(nq, (1 << 27) // max(1, nk * Hq)))
        for i in range(0, nq if nk else 0, max(block, 1)):
            sel = slice(q0 + i, q0 + min(nq, i + block))
            m = sel.stop - sel.start
            hide = torch.zeros(m, nk, dtype=torch.bool, device="cuda")
            if s["causal"]:
                late = torch.arange(nk, device="cuda")[None, :] - torch.arange(i, i + m, device="cuda")[:, None]
                hide = late > nk - nq
                if s["prefix_lengths"] is not None:
                    hide[:, :s["prefix"]] = False
            if s["keep"] is not None:
                hide = hide | (s["keep"][sel_k] == 0)[None, :]
            if s["distance"]:
                gap = (s["q_xy"][sel].double()[:, None] - s["k_xy"][sel_k].double()[None]) / QUANTA
                dist = gap.pow(2).sum(-1)
            # all heads at once: [Hq, m, nk]
            qh = q[sel].double().transpose(0, 1).contiguous()
            kh = k[sel_k].double().transpose(0, 1).contiguous().repeat_interleave(G, 0)
            vh = v[sel_k].double().transpose(0, 1).contiguous().repeat_interleave(G, 0)
            z = scale * (qh @ kh.transpose(1, 2).contiguous())
            if cap:
                th = torch.tanh(z / cap)
                z = cap * th
            if s["distance"]:
                z = z - s["slopes"].double()[:, None, None] * dist
            z[:, hide] = -math.inf
            w = torch.nan_to_num(torch.softmax(z, -1), nan=0.0)   # a query that sees no key gives zeros
            del z
            out[sel] = (w @ vh).transpose(0, 1)
            if train:
                g = s["grad_out"][sel].double().transpose(0, 1).contiguous()
                gw = g @ vh.transpose(1, 2).contiguous()
                per_kv = lambda t: t.view(Hq // G, G, nk, -1).sum(1).transpose(0, 1)  # noqa: E731
                dv[sel_k] += per_kv(w.transpose(1, 2).contiguous() @ g)
                gz = w * gw
                gz = gz - w * gz.sum(-1, keepdim=True)
                del gw, w
                if s["distance"]:
                    dslopes -= (gz * dist).sum((1, 2))
                if cap:
                    gz = gz * (1 - th * th)
                dq[sel] = (scale * (gz @ kh)).transpose(0, 1)
                dk[sel_k] += scale * per_kv(gz.transpose(1, 2).contiguous() @ qh)
        q0, k0 = q0 + nq, k0 + nk
    result = {"out": out}
    if train:
        result.update(dq=dq, dk=dk, dv=dv)
        if s["distance"]:
            result["dslopes"] = dslopes
    return result
