"""attention_tracks keeps the digits of values beside pages of far larger ones:
pages that a row gives no weight or does not see, before, among and after those
that it does, in each of its kernels; and those of weights far below the largest."""

import math

import pytest
import torch

import paper_2512_07009_amd as flock
from tests import serving_reference as ref
from tests.encoder_reference import TINY, UNIT
from tests.test_tracks_gpu import cuda, int32, offsets_of, pool, table_of

pytestmark = pytest.mark.gpu

PAGE, E32 = 64, ref.E32
# Weights in float16 are off by 2^-11 of themselves, or by 2^-25 of what they are relative to: 2^-7 of the row's largest at
# the time, over 2^-4 at least where the page's scale of values is in them.
LEAST = 2.0 ** -28


def reference(q, cache, offsets, table, lengths, scale, cap=0.0, window=0):
    """Outputs in 64 bits and what rounding may cost: no token costs more than its own weight and value allow."""
    k8, v8, k_scale, v_scale = cache
    u = UNIT[q.dtype]
    Hq, D = q.shape[1:]
    G = Hq // k_scale.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    for t in range(len(lengths)):
        n, length = offsets[t + 1] - offsets[t], lengths[t]
        if n <= 0 or length <= 0:
            continue
        ids = table[t, :(length + PAGE - 1) // PAGE].long()
        j, i = torch.arange(length)[None], torch.arange(length - n, length)[:, None]
        seen = j <= i
        if window:
            seen &= j > i - window
        rows = slice(offsets[t], offsets[t + 1])
        for h in range(Hq):
            K = (k8[ids, h // G].double() * k_scale[ids, h // G].double()[:, None, None]).reshape(-1, D)[:length]
            V = (ref.in_order(v8[ids, h // G]).double() * v_scale[ids, h // G].double()[:, None, None]).reshape(-1, D)[:length]
            Q = q[rows, h].double()
            s = scale * (Q @ K.T)
            ds = scale * (E32 * (8 + D ** 0.5) * (Q.abs() @ K.abs().T) + Q.abs().amax(1, keepdim=True) / 65024 * K.abs().sum(1))
            if cap:
                s = cap * torch.tanh(s / cap)
                ds = ds + 4e-7 * (s.abs() if cap > 64 else torch.full_like(s, cap))
            s = torch.where(seen, s, -math.inf)
            some = seen.any(1, keepdim=True)
            m = torch.where(some, s.amax(1, keepdim=True), 0.0)
            p = torch.exp(s - m)
            # the score and its difference from the shift, in units of log 2, are rounded
            ds = torch.where(seen, ds + 4 * E32 * (s.abs() + m.abs()), 0.0)
            total = torch.where(some, p.sum(1, keepdim=True), 1.0)
            o = (p @ V) / total
            size = (p @ V.abs()) / total
            b = (2.0 ** -11 + (64 + len(ids)) * E32) * size
            b = b + 1.1 * ((p * ds) @ V.abs() + o.abs() * (p * ds).sum(1, keepdim=True)) / total
            b = b + 1.1 * (p.clamp_max(LEAST) @ V.abs()) / total
            out[rows, h], bound[rows, h] = o, u * (o.abs() + b) + b + TINY[q.dtype] + 1e-30
    return out, bound


def attend(seed, lengths, queries, change, q_heads=4, kv_heads=2, dim=64, dtype=torch.bfloat16, cap=0.0, window=0):
    gen = torch.Generator().manual_seed(seed)
    pages = sum((n + PAGE - 1) // PAGE for n in lengths)
    c = pool(gen, pages, kv_heads, dim)
    table = table_of(gen, lengths, pages)
    offsets = offsets_of(queries)
    q = torch.randn(offsets[-1], q_heads, dim, generator=gen)
    q[:, :, 0] = 8.0
    q = q.to(dtype)
    scale = dim ** -0.5
    for t, n in enumerate(lengths):
        change(c, table[t, :(n + PAGE - 1) // PAGE].long(), scale)
    got = flock.attention_tracks(q.cuda(), cuda(c), int32(offsets), table.cuda(), int32(lengths), scale=scale, cap=cap,
                                 window=window)
    torch.cuda.synchronize()
    want, bound = reference(q, c, offsets, table, lengths, scale, cap, window)
    got, most = got.cpu().double(), torch.finfo(dtype).max
    err = (got - want).abs()
    # infinity is right where a value that the bound allows is beyond the type (values of 2^40 in float16)
    far = got.isinf() & (want * got.sign() + bound > most)
    over = ~(err <= bound) & ~far
    assert not over.any(), f"{over.sum()} of {err.numel()} above their bound, off by up to " \
                           f"{(err[over] / want.abs()[over].clamp_min(1e-300)).max():.3e} of themselves"


def large(power, at, hidden=True):
    """Every track's page `at` (of its pages, as a fraction) holds values 2^power times the others'; its keys all lie 60
    against every query where hidden."""
    def change(c, ids, scale):
        k, v, k_scale, v_scale = c
        page = ids[min(int(at * len(ids)), len(ids) - 1)]
        v_scale[page] *= 2.0 ** power
        if hidden:
            k[page] = 0
            k[page, :, :, 0] = -127
            k_scale[page] = 60 / (scale * 8 * 127)
    return change


def uneven(power):
    """Scales of values over 2^-power to 2^power, in no order."""
    def change(c, ids, scale):
        gen = torch.Generator().manual_seed(len(ids))
        c[3][ids] = 2.0 ** (power * (2 * torch.rand(len(ids), c[3].shape[1], generator=gen) - 1))
    return change


FEW = ([300, 70, 700], [1, 1, 2])
SHARED = ([9000, 4000], [1, 1])                 # several workgroups share a track's pages
RUNS = ([260 + 5 * i for i in range(40)], [150] * 40)


@pytest.mark.parametrize("power", [10, 18, 25, 45, 90])
@pytest.mark.parametrize("at", [0.0, 0.4, 1.0])
def test_pages_without_weight(power, at):
    attend(1, *FEW, large(power, at))
    attend(2, *FEW, large(power, at), dim=128, dtype=torch.float16)
    attend(3, *SHARED, large(power, at), cap=100.0)


@pytest.mark.parametrize("power", [12, 25, 90])
def test_pages_without_weight_of_many_rows(power):
    for at in (0.0, 0.3):
        attend(4, *RUNS, large(power, at), q_heads=16, kv_heads=8, dim=32)
    attend(5, *RUNS, large(power, 0.0), q_heads=16, kv_heads=8, dim=128, dtype=torch.float16, cap=100.0)


@pytest.mark.parametrize("power", [14, 30, 90])
def test_pages_out_of_the_window(power):
    """The rows of a tile that see the large page are beside those that do not."""
    attend(6, [300, 200], [40, 60], large(power, 0.5, hidden=False), window=50)
    attend(7, *RUNS, large(power, 0.5, hidden=False), q_heads=16, kv_heads=8, window=70)
    attend(8, *RUNS, large(power, 0.5, hidden=False), q_heads=16, kv_heads=8, dim=96, dtype=torch.float16, window=30)


def test_many_short_tracks():
    """A wave a workgroup."""
    gen = torch.Generator().manual_seed(9)
    lengths = torch.randint(1, 300, (1600,), generator=gen).tolist()
    attend(9, lengths, [1] * 1600, large(25, 0.0), q_heads=2, dim=32)
    attend(10, lengths, [1] * 1600, uneven(40), q_heads=2, dim=16, dtype=torch.float16)


@pytest.mark.parametrize("power", [3, 8, 20, 60])
def test_uneven_scales(power):
    attend(11, *FEW, uneven(power))
    attend(12, *SHARED, uneven(power), dim=128)
    attend(13, *RUNS, uneven(power), q_heads=16, kv_heads=8)


def small(power):
    """A track's first token gets 2^power times the weight of any other, and its values are zeros."""
    def change(c, ids, scale):
        k, v, k_scale, v_scale = c
        k[ids] = 0
        k[ids[0], :, 0, 0] = 127
        k_scale[ids[0]] = power * math.log(2) / (scale * 8 * 127)
        v[ids[0], :, :, ref.place(0)] = 0
    return change


@pytest.mark.parametrize("power", [10, 14, 17, 20, 24, 27])
def test_small_weights(power):
    attend(14, [64, 3, 40], [1, 1, 2], small(power))
    attend(15, *RUNS, small(power), q_heads=16, kv_heads=8)
    attend(16, *RUNS, small(power), q_heads=16, kv_heads=8, dim=128, dtype=torch.float16)


@pytest.mark.parametrize("lengths,queries,heads,at", [([500, 70], [400, 20], 1, 0), ([420, 700], [1, 1], 1, 5),
                                                      ([9000], [1], 1, 100), ([300] * 40, [150] * 40, 8, 2),
                                                      ([490] * 3200, [1] * 3200, 1, 6)])
@pytest.mark.parametrize("window", [0, 64, 128])
def test_pages_that_are_not_finite_and_far_below(lengths, queries, heads, at, window):
    """A page with a scale of NaN is NaN for the rows that see it, even where its weights are nothing in 32 bits."""
    gen = torch.Generator().manual_seed(17)
    each = [(n + PAGE - 1) // PAGE for n in lengths]
    c = pool(gen, max(each), heads, 64)
    table = torch.full((len(each), max(each)), -1, dtype=torch.int32)
    for t, n in enumerate(each):
        table[t, :n] = torch.arange(n)      # (all tracks read the same pages)
    offsets = offsets_of(queries)
    q = torch.randn(offsets[-1], 2 * heads, 64, generator=gen)
    q[:, :, 0] = 8.0
    c[0][at] = 0
    c[0][at, :, :, 0] = -127
    c[2][at] = 120 / 127      # scores of 120 below
    c[3][at] = math.nan
    places = torch.cat([torch.arange(n - m, n) for n, m in zip(lengths, queries)])
    seen = places >= at * PAGE
    if window:
        seen &= places - window < at * PAGE + PAGE - 1
    got = flock.attention_tracks(q.bfloat16().cuda(), cuda(c), int32(offsets), table.cuda(), int32(lengths), window=window).cpu()
    assert got[seen].isnan().all() and got[~seen].isfinite().all()


@pytest.mark.parametrize("power", [20, 23, 25, 27, 30, 40, 90])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lengths,queries,heads,dim", [([300, 70], [3, 20], 1, 64), ([9000], [1], 2, 128), ([300] * 40, [150] * 40, 8, 64),
                                                       ([280] * 40, [200] * 40, 8, 128), ([70] * 3200, [1] * 3200, 1, 32)])
@pytest.mark.parametrize("cap", [0.0, 2.0 ** 95])
def test_scores_far_beyond_whole_numbers(power, sign, lengths, queries, heads, dim, cap):
    """Scores of up to 2^power, whose steps in 32 bits are far above 1: the largest takes all the weight, and nothing else comes."""
    gen = torch.Generator().manual_seed(18)
    each = [(n + PAGE - 1) // PAGE for n in lengths]
    c = pool(gen, max(each), heads, dim)
    c[0].zero_()
    # every token in turn has a largest before it, or is one: others are 2^power / 64 below
    k = torch.randint(-60, 60, (heads, max(each) * PAGE), generator=gen)
    for at, most in ((0, 64), (40, 70), (100, 84), (250, 100), (8000, 126)):
        k[:, at:at + 1] = most
    c[0][:, :, :, 0] = (sign * k).view(heads, max(each), PAGE).transpose(0, 1)
    c[2].fill_(1.0)
    table = torch.full((len(each), max(each)), -1, dtype=torch.int32)
    for t, n in enumerate(each):
        table[t, :n] = torch.arange(n)      # (all tracks read the same pages)
    offsets = offsets_of(queries)
    q = torch.zeros(offsets[-1], 2 * heads, dim)
    q[:, :, 0] = sign
    got = flock.attention_tracks(q.bfloat16().cuda(), cuda(c), int32(offsets), table.cuda(), int32(lengths), scale=2.0 ** power / 127,
                                 cap=cap)
    v = (ref.in_order(c[1]).double() * c[3].double()[:, :, None, None]).transpose(0, 1).reshape(heads, -1, dim)
    best = k.cummax(1).indices
    rows = [n - m + i for n, m in zip(lengths, queries) for i in range(m)]
    want = v[torch.arange(heads)[None], best[:, rows].T].repeat_interleave(2, 1)
    # its weight is the total, both from the same 32 bits, and 2^-11 in float16
    assert ((got.cpu().double() - want).abs() <= (UNIT[torch.bfloat16] + 2.0 ** -10) * want.abs()).all()
