"""attention_frames and its backward pass against the 64-bit reference: sizes
around the tiles, ragged and empty frames, shared heads, all head widths,
distances, caps, hidden keys, order with prefixes, single queries, strides,
far offsets, streams and graphs; gradients also against differences."""

import math

import pytest
import torch

import paper_2512_07009_amd as flock
from tests import encoder_reference as ref

pytestmark = pytest.mark.gpu


def offsets(counts):
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    return off


def make(seed, q_counts, k_counts, Hq, Hk, D, dtype, distance=False, hidden=0.0, causal=False, prefix=None, cap=0.0,
         far=0, sigma=(20.0, 300.0), spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    tq, tk = sum(q_counts), sum(k_counts)
    own = q_counts is k_counts
    rnd = lambda *s: (spread * torch.randn(*s, generator=gen)).to(dtype)  # noqa: E731
    c = dict(q=rnd(tq, Hq, D), k=rnd(tk, Hk, D), v=rnd(tk, Hk, D), q_off=offsets(q_counts), k_off=offsets(k_counts),
             scale=D ** -0.5, cap=cap, causal=causal)
    c["grad"] = rnd(tq, Hq, D)
    if distance:
        c["k_xy"] = (torch.rand(tk, 2, generator=gen) * 16 * 400).int() + far
        c["q_xy"] = c["k_xy"] if own else (torch.rand(tq, 2, generator=gen) * 16 * 400).int() + far
        sig = sigma[0] * (sigma[1] / sigma[0]) ** (torch.arange(Hq) / max(Hq - 1, 1))
        c["slopes"] = (0.5 / sig ** 2).float()
    if hidden:
        c["keep"] = (torch.rand(tk, generator=gen) >= hidden).to(torch.uint8)
    if prefix is not None:
        c["prefix"] = torch.tensor(prefix, dtype=torch.int32)
    return c


def call(c, train=True, stream=None):
    d = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in c.items()}
    qo = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    ko = torch.tensor(c["k_off"], dtype=torch.int32).cuda()
    more = dict(k_offsets=ko, q_xy=d.get("q_xy"), k_xy=d.get("k_xy"), slopes=d.get("slopes"), scale=c["scale"],
                cap=c["cap"], keep=d.get("keep"), causal=c["causal"], prefix=d.get("prefix"))
    out, lse = flock.attention_frames(d["q"], d["k"], d["v"], qo, return_lse=True, **more)
    r = {"out": out, "lse": lse}
    if train:
        r["dq"], r["dk"], r["dv"], r["ds"] = flock.attention_frames_backward(d["grad"], d["q"], d["k"], d["v"], out,
                                                                            lse, qo, **more)
    torch.cuda.synchronize()
    return r


def reference(c, train=True):
    return ref.attention(c["q"], c["k"], c["v"], c["q_off"], c["k_off"], c["scale"], c["cap"], c.get("q_xy"),
                         c.get("k_xy"), c.get("slopes"), c.get("keep"), c["causal"], c.get("prefix"),
                         c["grad"] if train else None)


def compare(c, train=True):
    got = call(c, train)
    want, bound = reference(c, train)
    for n in want:
        if n == "ds" and got[n] is None:
            continue
        ref.check(got[n], want[n], bound[n], n)
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 300])
def test_one_frame(n, dtype):
    compare(make(n, [n], [n], 2, 2, 64, dtype, distance=True))


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 64, 80, 96, 104, 128])
@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (4, 2), (6, 1), (8, 8)])
def test_widths_and_heads(dim, heads):
    counts = [70, 0, 5, 131]
    compare(make(dim, counts, counts, *heads, dim, torch.bfloat16, distance=dim % 16 == 0, cap=5.0 if dim > 64 else 0.0))


@pytest.mark.parametrize("flags", [dict(), dict(distance=True), dict(cap=2.0), dict(distance=True, cap=2.0),
                                   dict(hidden=0.3), dict(hidden=0.9, distance=True), dict(causal=True),
                                   dict(causal=True, hidden=0.5, cap=3.0), dict(causal=True, distance=True),
                                   dict(causal=True, prefix=[0, 40, 3, 1000, 1])])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_masks_and_scores(flags, dtype):
    counts = [100, 77, 0, 258, 1]
    compare(make(7, counts, counts, 4, 2, 64, dtype, **flags))


# enough rows for 128-row tiles (more tiles than twice the card's compute units)
@pytest.mark.parametrize("flags", [dict(distance=True), dict(causal=True, prefix=[5] * 90), dict(hidden=0.4, cap=4.0),
                                   dict(causal=True, hidden=0.2, distance=True)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_many_frames(flags, dim):
    counts = [(37 * f) % 190 for f in range(90)]
    compare(make(dim, counts, counts, 8, 8, dim, torch.bfloat16, **flags))


@pytest.mark.parametrize("queries", [1, 2, 5, 17])
@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (6, 6)])
@pytest.mark.parametrize("flags", [dict(), dict(distance=True, hidden=0.2), dict(causal=True), dict(cap=10.0)])
def test_few_queries_over_long_histories(queries, heads, flags):
    k_counts = [1500, 0, 3, 1, 700, 129]
    c = make(queries, [queries] * 6, k_counts, *heads, 64 if heads[0] != 6 else 128, torch.bfloat16, **flags)
    compare(c)


@pytest.mark.parametrize("n", [4097, 9000])
def test_long_history(n):
    compare(make(n, [1], [n], 8, 1, 64, torch.float16, distance=True))
    compare(make(n, [3], [n], 2, 2, 40, torch.bfloat16, causal=True))


def test_queries_beyond_the_keys_of_an_ordered_frame():
    """More queries than keys: the first ones see nothing."""
    c = make(3, [9, 70], [4, 30], 2, 1, 64, torch.bfloat16, causal=True)
    got = compare(c)
    assert (got["out"][:5] == 0).all() and (got["lse"][:5] == -math.inf).all() and (got["dq"][:5] == 0).all()


def test_frames_whose_keys_are_all_hidden():
    c = make(4, [40, 200, 33], [40, 200, 33], 4, 4, 64, torch.bfloat16, distance=True, hidden=0.1)
    c["keep"][40:240] = 0
    got = compare(c)
    assert (got["out"][40:240] == 0).all() and (got["lse"][40:240] == -math.inf).all()
    assert (got["dk"][40:240] == 0).all() and (got["dv"][40:240] == 0).all() and (got["dq"][40:240] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("causal", [False, True])
def test_hidden_keys_are_not_read(bad, causal):
    c = make(5, [150], [150], 2, 2, 64, torch.bfloat16, distance=True, hidden=0.3, causal=causal)
    gone = c["keep"] == 0
    c["k"][gone] = bad
    c["v"][gone] = bad
    compare(c)


def test_lowest_and_largest_scores():
    """Scores far beyond exp's range, and many that underflow."""
    c = make(6, [130], [130], 2, 2, 64, torch.bfloat16, distance=True, sigma=(0.05, 2.0))
    compare(c)
    c = make(8, [64], [64], 2, 2, 64, torch.bfloat16)
    c["q"] = c["q"] * 32
    # scores of some thousand: their 32-bit rounding alone moves the weights, so only the winner is checked
    got = call(c, train=False)
    want, _ = reference(c, train=False)
    assert torch.isfinite(got["out"].float()).all()
    assert (got["lse"].cpu().double() - want["lse"]).abs().max() <= 1e-5 * want["lse"].abs().max()


def test_birds_far_from_the_origin():
    """Distances come from exact differences, wherever the birds are."""
    compare(make(9, [200], [200], 4, 4, 64, torch.bfloat16, distance=True, far=(1 << 24) - 16 * 400 - 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cap", [0.0, 6.0])
@pytest.mark.parametrize("heads", [(2, 2), (4, 1)])
def test_groups_of_birds_far_apart(heads, cap, dtype):
    """Tiles whose birds are near each other and tiles that are not: distances
    by matrix products and by differences in one frame (enough rows for tiles
    of 128)."""
    counts = [190] * 100
    c = make(17, counts, counts, *heads, 32, dtype, distance=True, cap=cap, hidden=0.1, sigma=(15.0, 60.0))
    place = torch.arange(sum(counts))
    # a third of the birds 20000 px away, in runs of two tiles of keys and mixed with the others
    far = ((place // 128) % 3 == 1) | (place % 7 == 0)
    c["k_xy"][:, 0] += far.int() * 16 * 20000
    compare(c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("flags", [dict(), dict(cap=5.0), dict(hidden=0.3), dict(causal=True)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_outputs_without_lse(dim, flags, dtype):
    """Inference, with sharp and wide heads, two query heads a key head."""
    counts = [(53 * f) % 260 for f in range(80)]
    c = make(19 + dim, counts, counts, 8, 4, dim, dtype, distance=True, sigma=(10.0, 300.0), **flags)
    d = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in c.items()}
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    got = flock.attention_frames(d["q"], d["k"], d["v"], off, q_xy=d["q_xy"], slopes=d["slopes"], scale=c["scale"],
                                 cap=c["cap"], keep=d.get("keep"), causal=c["causal"])
    want, bound = reference(c, train=False)
    ref.check(got, want["out"], bound["out"], "out")


def test_steep_flat_and_rising_slopes():
    """Slopes of zero, below zero and many times a frame's size."""
    c = make(18, [150, 90], [150, 90], 4, 4, 64, torch.bfloat16, distance=True)
    c["slopes"] = torch.tensor([0.0, -1e-5, 1e-3, 0.5])
    compare(c)


def test_slices_of_one_projection():
    c = make(10, [90, 45], [90, 45], 4, 2, 64, torch.bfloat16, distance=True)
    n = 135
    qkv = torch.zeros(n, 8, 64, dtype=torch.bfloat16, device="cuda")
    qkv[:, :4], qkv[:, 4:6], qkv[:, 6:] = c["q"].cuda(), c["k"].cuda(), c["v"].cuda()
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    xy, sl = c["q_xy"].cuda(), c["slopes"].cuda()
    a = flock.attention_frames(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], off, q_xy=xy, slopes=sl, return_lse=True)
    b = flock.attention_frames(c["q"].cuda(), c["k"].cuda(), c["v"].cuda(), off, q_xy=xy, slopes=sl, return_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # every frame attends to the same row of keys (stride 0)
    one_k, one_v = c["k"][:1].cuda().expand(n, 2, 64), c["v"][:1].cuda().expand(n, 2, 64)
    got = flock.attention_frames(qkv[:, :4], one_k, one_v, off)
    assert torch.allclose(got.float(), c["v"][0].cuda().repeat_interleave(2, 0).float().expand(n, 4, 64), rtol=2 ** -7)


def test_offsets_beyond_32_bits():
    """Rows that begin more than 2^32 elements into their tensor."""
    n, stride = 600, 1 << 23
    big = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    c = make(11, [1, 40], [n - 60, 60], 2, 1, 64, torch.bfloat16)
    k, v = big.as_strided((n, 1, 64), (stride, 64, 1)), big.as_strided((n, 1, 64), (stride, 64, 1), 128)
    k.copy_(c["k"].cuda())
    v.copy_(c["v"].cuda())
    q, go = c["q"].cuda(), c["grad"].cuda()
    qo, ko = (torch.tensor(c[x], dtype=torch.int32).cuda() for x in ("q_off", "k_off"))
    out, lse = flock.attention_frames(q, k, v, qo, k_offsets=ko, return_lse=True)
    dq, dk, dv, _ = flock.attention_frames_backward(go, q, k, v, out, lse, qo, k_offsets=ko)
    want, bound = reference(c)
    for name, got in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(got, want[name], bound[name], name)


def test_same_bits_again_and_in_any_batch():
    c = make(12, [260, 129, 64], [260, 129, 64], 4, 2, 64, torch.bfloat16, distance=True)
    a, b = call(c), call(c)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_gradients_against_differences():
    """Directional derivatives of the 64-bit forward pass."""
    c = make(13, [20, 13], [20, 13], 2, 1, 16, torch.bfloat16, distance=True, cap=4.0, causal=True, prefix=[3, 0])
    got = call(c)
    _, bound = reference(c)
    gen = torch.Generator().manual_seed(99)
    eps = 1e-4

    def loss(moved):
        class Wide(torch.Tensor):
            pass
        d = {n: (c[n].double() if n in ("q", "k", "v") else c[n]) for n in c}
        for n, t in moved.items():
            d[n] = (d[n].double() if n != "slopes" else d[n].double()) + t
        ref.UNIT[torch.float64] = 0.0
        ref.TINY[torch.float64] = 0.0
        r, _ = ref.attention(d["q"], d["k"], d["v"], d["q_off"], d["k_off"], d["scale"], d["cap"], d["q_xy"], d["k_xy"],
                             d["slopes"], None, True, d["prefix"])
        return (r["out"] * c["grad"].double()).sum()

    for name, g in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("slopes", "ds")):
        step = torch.randn(c[name].shape, generator=gen, dtype=torch.float64)
        if name == "slopes":
            step = step * c["slopes"].double()
        diff = (loss({name: eps * step}) - loss({name: -eps * step})) / (2 * eps)
        mine = (got[g].cpu().double() * step).sum()
        room = (bound[g] * step.abs()).sum() + 1e-5 * (1 + diff.abs())
        assert (mine - diff).abs() <= room, (name, float(mine), float(diff), float(room))


def test_on_another_stream():
    c = make(14, [300], [300], 2, 2, 64, torch.bfloat16)
    want = call(c, train=False)["out"]
    d = {n: c[n].cuda() for n in ("q", "k", "v")}
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = flock.attention_frames(d["q"], d["k"], d["v"], off, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_in_a_graph():
    """Replays equal the eager call, with other work between them."""
    c = make(15, [1], [5000], 8, 2, 64, torch.bfloat16, distance=True)
    d = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in c.items()}
    qo, ko = (torch.tensor(c[x], dtype=torch.int32).cuda() for x in ("q_off", "k_off"))

    def step():
        o, l = flock.attention_frames(d["q"], d["k"], d["v"], qo, k_offsets=ko, q_xy=d["q_xy"], k_xy=d["k_xy"],
                                      slopes=d["slopes"], return_lse=True)
        return (o, l) + flock.attention_frames_backward(d["grad"], d["q"], d["k"], d["v"], o, l, qo, k_offsets=ko,
                                                        q_xy=d["q_xy"], k_xy=d["k_xy"], slopes=d["slopes"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        d["q"].mul_(-1 if turn else 1)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)


def test_inconsistent_offsets_leave_their_outputs():
    """A frame whose offsets run backwards or past the end is not read."""
    c = make(16, [50, 50, 50], [50, 50, 50], 2, 2, 64, torch.bfloat16)
    q, k, v = (c[n].cuda() for n in "qkv")
    for off in ([0, 50, 400, 150], [0, 90, 50, 150], [-5, 50, 100, 150]):
        o = torch.tensor(off, dtype=torch.int32).cuda()
        out = torch.full_like(q, 7.0)
        flock.attention_frames(q, k, v, o, out=out)
        torch.cuda.synchronize()
        bad = [not (0 <= off[f] <= off[f + 1] <= 150) for f in range(3)]
        if off[0] == -5:
            assert (out[:50] == 7).all()
            assert (out[50:] != 7).any()
        assert any(bad)


def test_empty_calls():
    z = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    off0 = torch.zeros(1, dtype=torch.int32, device="cuda")
    off2 = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert flock.attention_frames(z, z, z, off0).shape == (0, 2, 64)
    assert flock.attention_frames(z, z, z, off2).shape == (0, 2, 64)
    q = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    qo = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    out, lse = flock.attention_frames(q, z, z, qo, k_offsets=off2, return_lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()
    dq, dk, dv, _ = flock.attention_frames_backward(q, q, z, z, out, lse, qo, k_offsets=off2)
    assert (dq == 0).all() and dk.shape == (0, 2, 64)
    dq, dk, dv, _ = flock.attention_frames_backward(z, z, q, q, z, lse[:0], off2, k_offsets=qo)
    assert (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("frames,n_q,n_k", [(0, 0, 0), (2, 0, 0), (2, 0, 3), (2, 3, 0)])
def test_slopes_without_pairs(frames, n_q, n_k):
    q, k = (torch.ones(n, 2, 64, dtype=torch.bfloat16, device="cuda") for n in (n_q, n_k))
    qo, ko = (torch.tensor([0, 1, n][:frames + 1] if n else [0] * (frames + 1), dtype=torch.int32, device="cuda")
              for n in (n_q, n_k))
    more = dict(k_offsets=ko, slopes=torch.ones(2, device="cuda"), q_xy=torch.ones(n_q, 2, dtype=torch.int32, device="cuda"),
                k_xy=torch.ones(n_k, 2, dtype=torch.int32, device="cuda"))
    out, lse = flock.attention_frames(q, k, k, qo, return_lse=True, **more)
    assert (out == 0).all() and (lse == -math.inf).all()
    dirty = torch.full((1 << 16,), math.nan, device="cuda")  # what the gradients' memory may hold
    del dirty
    dq, dk, dv, ds = flock.attention_frames_backward(q, q, k, k, out, lse, qo, **more)
    assert (ds == 0).all() and (dq == 0).all() and (dk == 0).all() and (dv == 0).all()


def test_python_refusals():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="dtype"):
        flock.attention_frames(q.float(), q.float(), q.float(), off)
    with pytest.raises(ValueError, match="multiple of 8"):
        flock.attention_frames(q[..., :60].contiguous(), q[..., :60].contiguous(), q[..., :60].contiguous(), off)
    with pytest.raises(ValueError, match="type and device"):
        flock.attention_frames(q, q.half(), q.half(), off)
    with pytest.raises(ValueError, match="contiguous rows"):
        flock.attention_frames(q[..., ::2], q[..., ::2], q[..., ::2], off)
    with pytest.raises(ValueError, match="q_offsets"):
        flock.attention_frames(q, q, q, off.long())
    with pytest.raises(ValueError, match="q_xy"):
        flock.attention_frames(q, q, q, off, slopes=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError, match="keep"):
        flock.attention_frames(q, q, q, off, keep=torch.ones(4, dtype=torch.bool, device="cuda"))
    with pytest.raises(ValueError, match="16-byte"):
        z = torch.zeros(4 * 2 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 2, 64)
        flock.attention_frames(z, q, q, off)
    with pytest.raises(ValueError, match="cap"):
        flock.attention_frames(q, q, q, off, cap=-1.0)


@pytest.mark.parametrize("dim", [32, 64, 72, 80, 96, 128])
def test_rows_as_far_apart_as_they_may_be(dim):
    """Strides up to the largest, in a tensor of NaN: hidden keys and what lies
    beyond a head's dimensions are not read, wherever the tile's rows are."""
    n, stride = 150, (1 << 24) - 8
    big = torch.full((n * stride,), math.nan, dtype=torch.bfloat16, device="cuda")
    c = make(20 + dim, [2], [n], 2, 1, dim, torch.bfloat16, hidden=0.2)
    k, v = big.as_strided((n, 1, dim), (stride, dim, 1)), big.as_strided((n, 1, dim), (stride, dim, 1), 1024)
    kept = c["keep"].bool().cuda()
    k[kept], v[kept] = c["k"].cuda()[kept], c["v"].cuda()[kept]
    q, go, keep = c["q"].cuda(), c["grad"].cuda(), c["keep"].cuda()
    qo, ko = (torch.tensor(c[x], dtype=torch.int32).cuda() for x in ("q_off", "k_off"))
    out, lse = flock.attention_frames(q, k, v, qo, k_offsets=ko, keep=keep, return_lse=True)
    dq, dk, dv, _ = flock.attention_frames_backward(go, q, k, v, out, lse, qo, k_offsets=ko, keep=keep)
    want, bound = reference(c)
    for name, got in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(got, want[name], bound[name], name)


def test_places_and_lse_of_another_shape_are_refused():
    """As many values in another order would be read as other places."""
    q = torch.zeros(6, 2, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    xy = torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    slopes = torch.ones(2, device="cuda")
    for wrong in (xy.t().contiguous(), xy.flatten(), xy[:, None].contiguous()):
        with pytest.raises(ValueError, match="q_xy"):
            flock.attention_frames(q, q, q, off, slopes=slopes, q_xy=wrong)
        with pytest.raises(ValueError, match="k_xy"):
            flock.attention_frames(q, q, q, off, slopes=slopes, q_xy=xy, k_xy=wrong)
    out, lse = flock.attention_frames(q, q, q, off, return_lse=True)
    for wrong in (lse.t().contiguous(), lse.flatten()):
        with pytest.raises(ValueError, match="lse"):
            flock.attention_frames_backward(q, q, q, q, out, wrong, off)


CAPS = [30.0, 64.0, 65.0, 1e3, 1e4, 1e5, 1e6, 1e9, 1e28, 3e38]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("distance", [False, True])
@pytest.mark.parametrize("cap", CAPS)
def test_caps_of_any_size(cap, distance, dtype):
    """Scores far below their cap keep their digits (lse shows them)."""
    counts = [300, 5]
    compare(make(31, counts, counts, 2, 2, 64, dtype, distance=distance, cap=cap))


@pytest.mark.parametrize("dim", [32, 96, 128])
@pytest.mark.parametrize("cap", [100.0, 1e5])
def test_high_caps_that_bite(cap, dim):
    """Scores on both sides of half their cap, in every width."""
    c = make(32 + dim, [150, 40], [150, 40], 4, 2, dim, torch.bfloat16, distance=dim != 96, cap=cap)
    c["q"] = c["q"] / 8
    c["scale"] = c["scale"] * cap  # scores around cap / 8, a few above half of it: the winner takes all
    got = call(c)
    want, bound = reference(c)
    for n in ("out", "dq", "dk", "dv"):
        assert torch.isfinite(got[n].float()).all(), n
    # 32-bit scores: products off by 64 roundings of 2^-24 at most, tanh by 5
    assert (got["lse"].cpu().double() - want["lse"]).abs().max() <= 2.0 ** -18 * cap


@pytest.mark.parametrize("cap", CAPS)
def test_caps_of_any_size_without_lse(cap):
    """Inference on rows enough for tiles of 128, with distances."""
    counts = [(53 * f) % 260 for f in range(80)]
    c = make(34, counts, counts, 8, 4, 64, torch.float16, distance=True, sigma=(10.0, 300.0), cap=cap)
    d = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in c.items()}
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    got = flock.attention_frames(d["q"], d["k"], d["v"], off, q_xy=d["q_xy"], slopes=d["slopes"], cap=cap)
    want, bound = reference(c, train=False)
    ref.check(got, want["out"], bound["out"], "out")


def check_norms(got, want, dtype, names=("out", "dq", "dk", "dv")):
    """Errors as norms: an output's own rounding, its factor's of 16 bits and its
    other factors' (delta, weights) are three of one size at most, each on its
    own: sqrt(3) of one, below 2."""
    for n in names:
        x = got[n].cpu().double()
        assert torch.isfinite(x).all(), n
        own = (want[n].to(dtype).double() - want[n]).norm()
        error = (x - want[n]).norm()
        assert error <= 2 * own, f"{n}: error {error / want[n].norm():.2e} of its norm, its rounding {own / want[n].norm():.2e}"


@pytest.mark.parametrize("size", [1e3, 1.0, 1e-1, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("flags", [dict(), dict(distance=True), dict(causal=True, prefix=[4]), dict(cap=5.0, hidden=0.2)])
def test_float16_gradients_of_any_size(size, flags):
    """dS over 2000 keys is far below the type's normal numbers."""
    c = make(33, [2000], [2000], 2, 1, 64, torch.float16, **flags)
    c["grad"] = (c["grad"].double() * size).half()
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, torch.float16)


def float16_factors_beyond_the_type(dim, distance):
    """dS above 65504 in gradients that are not, and values that grow by 2^20
    along the keys: each sum's scale comes down on its way."""
    c = make(35, [3, 5], [3, 5], 2, 2, dim, torch.float16, distance=distance)
    c["grad"] = (c["grad"].float() * 8000).half()
    c["q"], c["k"] = c["q"] / 64, c["k"] / 64
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, torch.float16)
    c = make(36, [500], [500], 1, 1, dim, torch.float16, distance=distance)
    c["v"] = (c["v"].double() * 2.0 ** (20.0 * torch.arange(500)[:, None, None] / 500 - 12)).half()
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, torch.float16, ("out", "dq", "dv"))
    c = make(37, [500], [500], 1, 1, dim, torch.float16, distance=distance)
    c["grad"] = (c["grad"].double() * 2.0 ** (20.0 * torch.arange(500)[:, None, None] / 500 - 12)).half()
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, torch.float16, ("out", "dk", "dv"))


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_float16_factors_beyond_the_type(dim):
    float16_factors_beyond_the_type(dim, distance=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("flags", [dict(), dict(distance=True), dict(cap=20.0, causal=True), dict(hidden=0.3)])
@pytest.mark.parametrize("sharp", [1, 2, 4, 8])
def test_errors_of_flat_and_sharp_weights(dtype, dim, flags, sharp):
    """Gradients keep their digits however sharp the weights are, with and
    without distances (delta as the rounded output gives it is not enough)."""
    counts = [300, 3, 40]
    c = make(32, counts, counts, 4, 2, dim, dtype, **flags)
    c["q"] = c["q"] * sharp
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, dtype)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_float16_factors_beyond_the_type_with_distances(dim):
    """(So few birds that the weights are sharp.)"""
    float16_factors_beyond_the_type(dim, distance=True)


@pytest.mark.parametrize("dim", [96, 128])
def test_workgroups_with_and_without_sharp_rows(dim):
    """One sharp row sends a workgroup of wide heads over its keys again, the
    others of its rows and other workgroups being flat."""
    c = make(38, [700], [700], 2, 2, dim, torch.float16)
    c["q"][200] = c["q"][200] * 30
    got = call(c)
    want, _ = reference(c)
    check_norms(got, want, torch.float16)
    row = (got["dq"][200].cpu().double() - want["dq"][200]).norm()
    # three errors of at most 2^-11 of the row's size (its own, its factor's, its weights')
    assert row <= 3 * 2.0 ** -11 * want["dq"][200].norm()


@pytest.mark.parametrize("dtype,limit", [(torch.bfloat16, 4096), (torch.float16, 1536)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("share", [0.5, 0.95, 1.05])
def test_distances_at_the_limit_of_products(dtype, limit, cap, share):
    """Birds of two far spots, with slopes that make the products of the distances
    as large as they may be (and just larger, where differences are taken): what
    they leave a weight off by stays below what rounding costs."""
    counts = [200 - f % 7 for f in range(80)]
    c = make(39, counts, counts, 8, 4, 64, dtype, distance=True, cap=cap)
    gen = torch.Generator().manual_seed(40)
    n = sum(counts)
    sigma = 8.0
    c["slopes"] = torch.full((8,), 0.5 / sigma ** 2)
    reach = math.sqrt(share * limit / (float(c["slopes"][0]) * math.log2(math.e)))  # px
    spot = (torch.arange(n) % 2)[:, None] * torch.tensor([2 * reach, 0.0])
    c["q_xy"] = c["k_xy"] = ((spot + 40 + sigma * torch.randn(n, 2, generator=gen)) * 16).int()
    want, _ = reference(c)
    check_norms(call(c), want, dtype, ("out", "dq", "dk", "dv"))
    d = {k: (t.cuda() if torch.is_tensor(t) else t) for k, t in c.items()}
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    out = flock.attention_frames(d["q"], d["k"], d["v"], off, q_xy=d["q_xy"], slopes=d["slopes"], cap=cap)
    check_norms({"out": out}, want, dtype, ("out",))


def test_offsets_are_checked_on_request(monkeypatch):
    monkeypatch.setenv("FLOCK_VALIDATE", "1")
    q = torch.randn(20, 2, 64, device="cuda").to(torch.bfloat16)
    good = torch.tensor([0, 7, 20], dtype=torch.int32, device="cuda")
    out, lse = flock.attention_frames(q, q, q, good, return_lse=True)
    flock.attention_frames_backward(q, q, q, q, out, lse, good)
    for bad, text in (([1, 7, 20], r"q_offsets\[0\]"), ([0, 9, 7, 20], "decrease at frame 1"), ([0, 7, 19], "its total is 20")):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        held = torch.full_like(q, 7.0)
        with pytest.raises(ValueError, match=text):
            flock.attention_frames(q, q, q, off, out=held)
        assert (held == 7).all()
        with pytest.raises(ValueError, match=text):
            flock.attention_frames_backward(q, q, q, q, out, lse, off)
        if len(bad) == 3:
            with pytest.raises(ValueError, match=text.replace("q_", "k_")):
                flock.attention_frames(q, q, q, good, k_offsets=off)


def test_frame_alone_and_in_a_batch():
    """A frame's results do not depend on the others where the batch takes the
    same kernel and shares of the keys: few rows a frame, histories below two
    shares."""
    counts = [[1, 60, 33], [200, 250, 129]]
    c = make(41, counts[0], counts[1], 4, 2, 64, torch.bfloat16, distance=True, hidden=0.1)
    all_of = call(c)
    for f in range(3):
        qs, ks = slice(c["q_off"][f], c["q_off"][f + 1]), slice(c["k_off"][f], c["k_off"][f + 1])
        one = dict(c, q=c["q"][qs], grad=c["grad"][qs], q_xy=c["q_xy"][qs], k=c["k"][ks], v=c["v"][ks], k_xy=c["k_xy"][ks],
                   keep=c["keep"][ks], q_off=[0, counts[0][f]], k_off=[0, counts[1][f]])
        got = call(one)
        for n, rows in (("out", qs), ("lse", qs), ("dq", qs), ("dk", ks), ("dv", ks)):
            assert torch.equal(got[n], all_of[n][rows]), (f, n)


def bad_frames(off, total):
    return [not (0 <= off[f] <= off[f + 1] <= total) for f in range(len(off) - 1)]


@pytest.mark.parametrize("form", ["few rows", "shares of the keys", "many rows"])
@pytest.mark.parametrize("bad", ["past the end", "backwards", "negative"])
def test_inconsistent_frames(form, bad):
    """A frame whose offsets run backwards or past the end is not read, and rows
    that no consistent frame holds are left alone in every output.  What a
    consistent frame gets is not defined (tiles are numbered by the offsets), but
    where one launch makes it, it is right or left alone."""
    frames, n = (200, 60) if form == "many rows" else (4, 60)
    heads = (8, 8) if form == "many rows" else (2, 1)
    total, n_k = frames * n, 3000 if form == "shares of the keys" else n
    c = make(42, [n] * frames, [n_k] * frames, *heads, 64, torch.bfloat16)
    want, bound = reference(c)
    q_off = list(c["q_off"])
    if bad == "past the end":       # frames 1 and 2 are bad
        q_off[2] = total + 100
    elif bad == "backwards":        # frame 1 is bad, frame 2 begins where frame 1 did
        q_off[2] = q_off[1] - 1 if form == "few rows" else q_off[1] - 7
    else:                           # frame 0 is bad
        q_off[0] = -5
    ok = [not x for x in bad_frames(q_off, total)]
    d = {k: (t.cuda() if torch.is_tensor(t) else t) for k, t in c.items()}
    qo = torch.tensor(q_off, dtype=torch.int32).cuda()
    ko = torch.tensor(c["k_off"], dtype=torch.int32).cuda()
    out = torch.full_like(d["q"], 7.0)
    _, lse = flock.attention_frames(d["q"], d["k"], d["v"], qo, k_offsets=ko, out=out, return_lse=True)
    # rows that only their own, consistent frame holds, and rows of none
    holders = [[f for f in range(frames) if ok[f] and q_off[f] <= i < q_off[f + 1]] for i in range(total)]
    right = torch.tensor([h == [i // n] and q_off[h[0]] == c["q_off"][h[0]] and q_off[h[0] + 1] == c["q_off"][h[0] + 1]
                          for i, h in enumerate(holders)])
    free = torch.tensor([not h for h in holders])
    assert right.any() and (free.any() or bad == "backwards")
    written = right & (out.cpu() != 7).flatten(1).any(1)
    if form != "shares of the keys":
        ref.check(out.cpu()[written], want["out"][written], bound["out"][written], "out")
    assert (out.cpu()[free] == 7).all()
    # the backward pass by the C ABI, into gradients that hold something
    dq, dk, dv = (torch.full_like(d[x], 7.0) for x in "qkv")
    full, full_lse = flock.attention_frames(d["q"], d["k"], d["v"], torch.tensor(c["q_off"], dtype=torch.int32).cuda(),
                                            k_offsets=ko, return_lse=True)
    lib = flock.lib()
    tq, tk, hq, hk, dim = total, frames * n_k, *heads, 64
    st = lib.attention_frames_backward(2, d["grad"].data_ptr(), hq * dim, d["q"].data_ptr(), hq * dim, d["k"].data_ptr(),
                                       hk * dim, d["v"].data_ptr(), hk * dim, full.data_ptr(), hq * dim, full_lse.data_ptr(),
                                       qo.data_ptr(), ko.data_ptr(), frames, tq, tk, hq, hk, dim, None, None, None, None, 0,
                                       None, c["scale"], 0.0, dq.data_ptr(), hq * dim, dk.data_ptr(), hk * dim, dv.data_ptr(),
                                       hk * dim, None, None, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0
    written = right & (dq.cpu() != 7).flatten(1).any(1)
    ref.check(dq.cpu()[written], want["dq"][written], bound["dq"][written], "dq")
    assert (dq.cpu()[free] == 7).all()
    for f in range(frames):
        if not ok[f]:
            keys = slice(f * n_k, (f + 1) * n_k)
            assert (dk[keys] == 7).all() and (dv[keys] == 7).all(), f


@pytest.mark.parametrize("cap", [1e-30, 1e-37, 1e-38, 1e-40, 1e-45])
def test_tiny_caps(cap):
    """Down to the smallest number: the products no longer matter, and hidden
    keys stay hidden."""
    compare(make(50, [130, 20], [130, 20], 2, 2, 64, torch.bfloat16, cap=cap, hidden=0.3, distance=True))


@pytest.mark.parametrize("scale", [1e-10, 1e-30, 1e-36, 1e-38, 1e-40])
@pytest.mark.parametrize("cap", [0.0, 5.0, 100.0])
def test_tiny_scales(scale, cap):
    """Distances alone make the scores, with lse and without."""
    counts = [(53 * f) % 260 for f in range(80)]
    c = make(51, counts, counts, 8, 4, 64, torch.bfloat16, distance=True, sigma=(10.0, 300.0), cap=cap)
    c["scale"] = scale
    got = call(c)
    want, bound = reference(c)
    for n in want:
        ref.check(got[n], want[n], bound[n], n)
    d = {n: (t.cuda() if torch.is_tensor(t) else t) for n, t in c.items()}
    off = torch.tensor(c["q_off"], dtype=torch.int32).cuda()
    out = flock.attention_frames(d["q"], d["k"], d["v"], off, q_xy=d["q_xy"], slopes=d["slopes"], scale=scale, cap=cap)
    ref.check(out, want["out"], bound["out"], "out")
