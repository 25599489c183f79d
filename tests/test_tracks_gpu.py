"""append_tracks and attention_tracks against 64 bits: pages that begin, end and
fill within a call, scales that grow, heads and types, rows without tokens,
windows, tables with no page, values that are not finite, tracks out of range."""

import math

import pytest
import torch

import paper_2512_07009_amd as flock
from tests import serving_reference as ref

pytestmark = pytest.mark.gpu

PAGE = 64


def pool(gen, pages, heads, dim):
    """A pool whose pages hold something already, junk in places of tokens to come among it."""
    whole = lambda *s: torch.randint(-127, 128, s, generator=gen, dtype=torch.int8)  # noqa: E731
    scale = lambda: 0.02 * (0.5 + torch.rand(pages, heads, generator=gen))           # noqa: E731
    return whole(pages, heads, PAGE, dim), whole(pages, heads, dim, PAGE), scale(), scale()


def table_of(gen, lengths, pages, columns=None):
    each = [max(0, (n + PAGE - 1) // PAGE) for n in lengths]
    columns = max([1, *each]) if columns is None else columns
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32)
    order = torch.randperm(pages, generator=gen).int()
    at = 0
    for t, n in enumerate(each):
        table[t, :n] = order[at:at + n]
        at += n
    assert at <= pages
    return table


def offsets_of(counts):
    return [0, *torch.tensor(counts, dtype=torch.int64).cumsum(0).tolist()]


def cuda(c):
    return flock.TrackCache(*(t.cuda() for t in c))


def back(cache):
    return tuple(t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# --- append ---

def append(seed, before, new, heads=2, dim=64, dtype=torch.bfloat16, counts=(8, 12, 12), interleaved=False, fused=False,
           size=1.0, far=0):
    gen = torch.Generator().manual_seed(seed)
    lengths = [b + n for b, n in zip(before, new)]
    pages = sum((n + PAGE - 1) // PAGE for n in lengths) + 3
    start = pool(gen, pages, heads, dim)
    table = table_of(gen, lengths, pages)
    offsets = offsets_of(new)
    total = offsets[-1]
    rows = (size * torch.randn(total, 2 * heads + 1, dim, generator=gen)).to(dtype)
    d = rows.cuda()
    k, v = d[:, 1:1 + heads], d[:, 1 + heads:]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    nt, ny, nx = counts
    xy = (torch.rand(total, 2, generator=gen) * 16 * 1000).int() + far
    time = torch.randint(-1000, 100000, (total,), generator=gen).int()
    freq = [2 * math.pi / w for w in torch.logspace(0.6, 4, max(sum(counts), 1)).tolist()][:sum(counts)]
    axes = flock.RotaryAxes(freq[:nt], freq[nt:nt + ny], freq[nt + ny:]) if sum(counts) else None
    cache = cuda(start)
    flock.append_tracks(cache, k, v, int32(offsets), table.cuda(), int32(lengths), axes=axes, xy=xy.cuda(), time=time.cuda(),
                        interleaved=interleaved)
    torch.cuda.synchronize()
    turned, slack = ref.rotary(rows[:, 1:1 + heads].float(), xy, time, freq, counts, interleaved, False)
    ref.check_append(start, back(cache), turned, rows[:, 1 + heads:].double(), offsets, table, lengths, slack)
    return cache


@pytest.mark.parametrize("before,new", [
    ([0], [1]), ([1], [1]), ([62], [1]), ([63], [1]), ([64], [1]), ([0], [63]), ([0], [64]), ([0], [65]), ([63], [2]),
    ([10], [200]), ([64], [128]), ([1], [190]), ([5, 0, 64, 130], [1, 1, 1, 1]), ([5, 0, 64, 130], [0, 70, 0, 3]),
    ([0, 0, 0], [0, 0, 2]), ([17] * 70, [1] * 70), (list(range(130)), [1 + i % 3 for i in range(130)]),
])
def test_append_pages(before, new):
    append(len(before), before, new)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,dim,counts", [(1, 16, (1, 2, 3)), (3, 32, (0, 0, 16)), (2, 48, (5, 0, 0)), (1, 80, (0, 7, 9)),
                                              (8, 96, (10, 10, 10)), (4, 128, (20, 22, 22)), (2, 112, (0, 0, 0))])
def test_append_heads(heads, dim, counts, dtype):
    append(7, [3, 60, 128], [2, 9, 66], heads=heads, dim=dim, counts=counts, dtype=dtype, fused=True)


def test_append_interleaved_far_small_and_large():
    append(1, [3, 60], [40, 9], interleaved=True)
    append(2, [3, 60], [40, 9], far=10 ** 8, dtype=torch.float32)
    append(3, [3, 60], [40, 9], size=1e-3)      # the pages' scales stay, the new values are few steps
    append(4, [3, 60], [40, 9], size=1e4)       # what they held goes to zero


def test_append_many_tracks():
    gen = torch.Generator().manual_seed(5)
    before = torch.randint(0, 200, (5000,), generator=gen).tolist()
    new = (torch.rand(5000, generator=gen) < 0.7).int().tolist()
    append(5, before, new, heads=1, dim=16, counts=(2, 2, 2))


def test_append_again_changes_nothing():
    gen = torch.Generator().manual_seed(6)
    start = pool(gen, 4, 2, 64)
    k = torch.randn(30, 2, 64, generator=gen).cuda()
    cache = cuda(start)
    args = (int32([0, 30]), int32([[2, 0]]), int32([70]))
    flock.append_tracks(cache, k, k, *args)
    once = back(cache)
    flock.append_tracks(cache, k, k, *args)
    for a, b in zip(once, back(cache)):
        assert torch.equal(a, b)


def test_append_token_by_token_is_near_all_at_once():
    """Each time a page's scale grows, what it holds is rounded again: off by half a step each time."""
    gen = torch.Generator().manual_seed(8)
    k = torch.randn(100, 2, 64, generator=gen).cuda()
    cache = flock.TrackCache.empty(2, 2, 64)
    table = int32([[1, 0]])
    grown = torch.zeros(2, 2, device="cuda")
    last = torch.zeros(2, 2, device="cuda")
    for n in range(1, 101):
        flock.append_tracks(cache, k[n - 1:n], k[n - 1:n], int32([0, 1]), table, int32([n]))
        now = cache.k_scale.flip(0) * torch.tensor([[1.0], [1.0 if n > 64 else 0.0]], device="cuda")
        grown += (now > last).float()
        last = now
    keys, values = (x[[1, 0]].transpose(1, 2).reshape(128, 2, 64)[:100] for x in cache.values())
    scale = cache.k_scale.flip(0).repeat_interleave(64, 0)[:100, :, None]
    allowed = scale * (0.501 * grown.repeat_interleave(64, 0)[:100, :, None])
    assert ((keys - k).abs() <= allowed).all() and ((values - k).abs() <= allowed).all()


def test_append_values_that_are_not_finite():
    gen = torch.Generator().manual_seed(9)
    for bad in (math.nan, math.inf, -math.inf):
        cache = cuda(pool(gen, 5, 2, 32))
        start = back(cache)
        k = torch.randn(3, 2, 32, generator=gen)
        v = k.clone()
        k[1, 0, 5], v[2, 1, 31] = bad, bad
        flock.append_tracks(cache, k.cuda(), v.cuda(), int32([0, 3]), int32([[4]]), int32([10]))
        got = back(cache)
        assert torch.isnan(got[2][4, 0]) and torch.isnan(got[3][4, 1])
        assert torch.isfinite(got[2][4, 1]) and torch.isfinite(got[3][4, 0])
        assert (got[0][4, 0, :10] == 0).all() and (ref.in_order(got[1])[4, 1, :10] == 0).all()
        for a, b in zip(start, got):
            assert torch.equal(a[:4], b[:4])
        # it stays so with what comes after, until the page begins anew
        flock.append_tracks(cache, torch.ones(1, 2, 32, device="cuda"), torch.ones(1, 2, 32, device="cuda"), int32([0, 1]),
                            int32([[4]]), int32([11]))
        assert torch.isnan(cache.k_scale[4, 0])
        flock.append_tracks(cache, torch.ones(1, 2, 32, device="cuda"), torch.ones(1, 2, 32, device="cuda"), int32([0, 1]),
                            int32([[4]]), int32([1]))
        assert torch.isfinite(cache.k_scale[4]).all() and (cache.k[4, :, 0] == 127).all()


def test_append_zeros_and_tiny_values():
    cache = flock.TrackCache.empty(1, 1, 16)
    one = (int32([0, 1]), int32([[0]]))
    tiny = torch.full((1, 1, 16), 1e-33, device="cuda")
    flock.append_tracks(cache, 0 * tiny, tiny, *one, int32([1]))
    assert (cache.k_scale == 0).all() and (cache.v_scale == 0).all()
    flock.append_tracks(cache, tiny + 1, tiny + 1, *one, int32([2]))
    k, v = cache.values()
    assert (k[0, 0, 0] == 0).all() and (v[0, 0, 0] == 0).all()
    assert ((k[0, 0, 1] - 1).abs() < 1e-6).all() and ((v[0, 0, 1] - 1).abs() < 1e-6).all()


def test_append_passes_over_what_is_out_of_range():
    gen = torch.Generator().manual_seed(10)
    start = pool(gen, 6, 2, 32)
    k = torch.randn(12, 2, 32, generator=gen)

    def check(offsets, table, lengths):
        cache = cuda(start)
        flock.append_tracks(cache, k.cuda(), k.cuda(), int32(offsets), int32(table), int32(lengths))
        torch.cuda.synchronize()
        ref.check_append(start, back(cache), k.double(), k.double(), offsets, torch.tensor(table), lengths, torch.zeros_like(k))

    check([0, 4, 8, 12], [[0, 1], [2, -1], [3, 6]], [4, 66, 70])       # pages that are none
    check([0, 4, 8, 12], [[0], [1], [2]], [3, 65, 12])                 # more rows than tokens; longer than its pages
    check([0, 4, 8, 12], [[0], [1], [2]], [-1, 4, 5])
    check([0, 4, 2, 12], [[0], [1], [2]], [4, 4, 12])                  # offsets that decrease
    check([0, 4, 8, 14], [[0], [1], [2]], [4, 4, 12])                  # ... or end beyond the rows
    check([-2, 4, 8, 12], [[0], [1], [2]], [6, 4, 5])
    check([0, 4, 8, 12], [[2 ** 31 - 1], [-2 ** 31], [2]], [4, 4, 5])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tracks,rows", [(3, 100), (300, 2)])
def test_append_whole_numbers_are_the_rounded_quotients(tracks, rows, dtype):
    """To the bit what divisions in 32 bits round to, numbers at half a step among them (half a page's largest is 63.5)."""
    gen = torch.Generator().manual_seed(11)
    heads, dim = 2, 32
    lengths = [rows + t % 50 for t in range(tracks)]
    pages = sum((n + PAGE - 1) // PAGE for n in lengths)
    start = pool(gen, pages, heads, dim)
    table = table_of(gen, lengths, pages)
    new = 4 * torch.randn(2, tracks * rows, heads, dim, generator=gen).to(dtype)
    new[:, ::2, :, 1] = new[:, ::2].abs().amax(3) / 2
    cache = cuda(start)
    flock.append_tracks(cache, new[0].cuda(), new[1].cuda(), int32(offsets_of([rows] * tracks)), table.cuda(), int32(lengths))
    got = back(cache)
    for i in (0, 1):
        whole, before = (c[0] if i == 0 else ref.in_order(c[1]) for c in (got, start))
        for t, n in enumerate(lengths):
            for p in range((n + PAGE - 1) // PAGE):
                page, first = int(table[t, p]), n - rows - p * PAGE
                s0, s1 = max(first, 0), min(n - p * PAGE, PAGE)
                if s1 <= s0:
                    continue
                x = new[i, t * rows + s0 - first:t * rows + s1 - first].float().transpose(0, 1)
                scale = x.abs().amax((1, 2)) / 127
                if s0:
                    scale = torch.maximum(scale, start[2 + i][page])
                assert torch.equal(got[2 + i][page], scale)
                assert torch.equal(whole[page, :, s0:s1].float(), torch.round(x / scale[:, None, None]))
                # (a whole number times a quotient in 32 bits is exact in 64)
                held = before[page, :, :s0].double() * (start[2 + i][page] / scale).double()[:, None, None]
                assert torch.equal(whole[page, :, :s0].double(), torch.round(held))


# --- attention ---

def attend(seed, lengths, queries, q_heads=4, kv_heads=2, dim=64, dtype=torch.bfloat16, cap=0.0, window=0, scale=None,
           columns=None, size=1.0, spoil=None):
    gen = torch.Generator().manual_seed(seed)
    pages = max(1, sum((n + PAGE - 1) // PAGE for n in lengths))
    c = pool(gen, pages, kv_heads, dim)
    table = table_of(gen, lengths, pages, columns)
    if spoil:
        spoil(table, c)
    offsets = offsets_of(queries)
    q = (size * torch.randn(offsets[-1], q_heads, dim, generator=gen)).to(dtype)
    scale = dim ** -0.5 if scale is None else scale
    got = flock.attention_tracks(q.cuda(), cuda(c), int32(offsets), table.cuda(), int32(lengths), scale=scale, cap=cap,
                                 window=window)
    torch.cuda.synchronize()
    want, bound = ref.attention_tracks(q, c, offsets, table, lengths, scale, cap, window)
    ref.check(got, want, bound, "out")
    return got


@pytest.mark.parametrize("length", [1, 2, 3, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 4096, 5000])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_lengths(length, dim):
    attend(length, [length], [1], dim=dim)
    attend(length, [length, 7, length], [1, 1, 1], dim=dim, dtype=torch.float16)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("q_heads,kv_heads,dim", [(1, 1, 16), (4, 1, 32), (2, 2, 48), (6, 2, 80), (8, 8, 96), (8, 1, 112),
                                                  (12, 4, 128), (16, 1, 64), (17, 1, 32), (40, 2, 64)])
def test_attention_heads(q_heads, kv_heads, dim, dtype):
    attend(3, [70, 200, 33], [1, 2, 1], q_heads, kv_heads, dim, dtype)


@pytest.mark.parametrize("queries", [1, 2, 3, 5, 8, 9, 16, 30, 64, 65, 100])
def test_attention_queries(queries):
    attend(queries, [queries, 100 + queries, 300], [queries, queries, queries])
    attend(queries, [queries + 64, 700], [queries, 1], q_heads=3, kv_heads=1, dtype=torch.float16, cap=20.0)


@pytest.mark.parametrize("window", [1, 2, 10, 63, 64, 65, 100, 1000, 10 ** 6, 2 ** 31 - 1])
def test_attention_window(window):
    attend(window, [1, 64, 65, 200, 500], [1, 1, 1, 3, 40], window=window)
    attend(window, [3000], [1], window=window, cap=30.0)


@pytest.mark.parametrize("cap", [1e-30, 0.5, 30.0, 64.0, 65.0, 500.0, 1e30])
@pytest.mark.parametrize("scale", [0.125, 3.0])
def test_attention_cap_and_scale(cap, scale):
    attend(4, [90, 300], [1, 4], cap=cap, scale=scale)


def test_attention_sharp_and_flat():
    attend(5, [900], [2], scale=5.0, size=3.0)
    attend(5, [900], [2], scale=1e-6)
    attend(6, [400], [2], size=1e-20, scale=1e19)
    attend(6, [400], [2], size=1e25, scale=1e-26)
    attend(7, [400], [2], size=1e-6, scale=1e5, dtype=torch.float16)


def test_attention_tracks_without_tokens_or_rows():
    got = attend(7, [0, 5, 0, 64, 200], [1, 0, 2, 1, 0])
    assert (got[:3] == 0).all()
    attend(7, [3, 5], [5, 9])                      # rows before a track's first token see nothing
    attend(8, [0], [1])
    attend(8, [10, 20], [1, 1], columns=500)       # a table far wider than the tracks


def test_attention_ragged_batch():
    gen = torch.Generator().manual_seed(9)
    lengths = torch.randint(0, 700, (150,), generator=gen).tolist()
    queries = [min(n, int(m)) for n, m in zip(lengths, torch.randint(0, 4, (150,), generator=gen))]
    attend(9, lengths, queries, columns=40)


def test_attention_of_one_long_track_among_short_ones():
    attend(10, [3] * 40 + [20000] + [70] * 40, [1] * 81, q_heads=2, kv_heads=1)


def test_attention_pages_that_are_none():
    def spoil(table, c):
        table[0, 1] = -1
        table[1, 0] = len(c[0])
        table[2, :] = 2 ** 31 - 1
        table[3, 2] = -2 ** 31
    got = attend(11, [200, 130, 90, 192, 70], [1, 2, 3, 1, 1], spoil=spoil)
    assert (got[3:6] == 0).all()
    attend(11, [5000, 130, 90, 192], [1, 2, 3, 1], spoil=spoil)


def test_attention_with_scales_that_are_not_finite():
    """A page with NaN is NaN for the rows that see a token of it, and for no other."""
    def spoil(table, c):
        c[2][int(table[0, 1])] = math.nan
        c[3][int(table[1, 0])] = math.nan
    gen = torch.Generator().manual_seed(12)
    lengths, queries = [100, 130, 64], [60, 1, 1]
    for window in (0, 40):
        c = pool(gen, 6, 2, 64)
        table = table_of(gen, lengths, 6)
        spoil(table, c)
        offsets = offsets_of(queries)
        q = torch.randn(62, 4, 64, generator=gen).bfloat16()
        got = flock.attention_tracks(q.cuda(), cuda(c), int32(offsets), table.cuda(), int32(lengths), window=window).cpu()
        # rows 0..23 of track 0 are tokens 40..63, before the page; the one of track 1 sees page 0 without a window
        assert torch.isfinite(got[:24]).all() and torch.isnan(got[24:60]).all()
        assert torch.isnan(got[60]).all() if not window else torch.isfinite(got[60]).all()
        assert torch.isfinite(got[61]).all()


def test_attention_of_zero_pages_and_zero_scales():
    def spoil(table, c):
        c[3][int(table[0, 0])] = 0
        c[2][int(table[0, 1])] = 0
        c[3][int(table[1, 0])] = 0
    attend(13, [200, 50], [1, 1], spoil=spoil)
    attend(13, [200, 50], [1, 1], spoil=spoil, cap=1e-30)
    def uneven(table, c):
        c[3][:] = torch.logspace(-8, 8, c[3].numel()).reshape(c[3].shape)
    attend(14, [900, 50], [1, 1], spoil=uneven)


def test_attention_leaves_rows_of_no_track():
    gen = torch.Generator().manual_seed(15)
    c = cuda(pool(gen, 8, 2, 64))
    q = torch.randn(12, 4, 64, generator=gen).bfloat16().cuda()
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(4, 2)

    def run(offsets, lengths):
        out = torch.full_like(q, 7)
        flock.attention_tracks(q, c, int32(offsets), table, int32(lengths), out=out)
        return out
    out = run([0, 3, 6, 9, 9], [100, 100, 100, 100])
    assert (out[9:] == 7).all() and not (out[:9] == 7).any()
    out = run([0, 3, 6, 9, 12], [100, -1, 129, 100])
    assert (out[3:9] == 7).all() and not (out[:3] == 7).any() and not (out[9:] == 7).any()
    out = run([0, 3, 2, 9, 14], [100, 100, 100, 100])
    assert (out[9:] == 7).all()


def test_attention_of_pages_that_tracks_share():
    """Two tracks that begin alike read the same pages, one page of a track twice too."""
    def share(table, c):
        table[1, :3] = table[0, :3]
        table[2, 4] = table[2, 1]
    for queries in ([1, 1, 1], [40, 3, 60], [300, 250, 200]):
        attend(60, [500, 430, 700], queries, spoil=share)


@pytest.mark.parametrize("window", [0, 2000])
def test_attention_in_two_graphs(window):
    """Two captured calls that share their pages among workgroups, replayed in turn and beside each other."""
    lengths, queries = [9000, 4000], [1, 2]
    gen = torch.Generator().manual_seed(61)
    pages = sum((n + PAGE - 1) // PAGE for n in lengths)
    c, table = cuda(pool(gen, pages, 2, 64)), table_of(gen, lengths, pages).cuda()
    offsets, n = int32(offsets_of(queries)), int32(lengths)
    qs = [torch.randn(3, 8, 64, generator=gen).bfloat16().cuda() for _ in range(2)]
    want = [flock.attention_tracks(q, c, offsets, table, n, window=window) for q in qs]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in qs]
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(flock.attention_tracks(q, c, offsets, table, n, window=window))
        graphs.append(g)
    for turn in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            if turn % 2:
                with torch.cuda.stream(s):
                    g.replay()
            else:
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"turn {turn}"


def test_attention_strides():
    gen = torch.Generator().manual_seed(16)
    c = cuda(pool(gen, 8, 2, 64))
    rows = torch.randn(6, 8 * 64 + 5, generator=gen).bfloat16().cuda()
    q = rows[:, 3:3 + 4 * 64].unflatten(1, (4, 64))
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(2, 8)[:, :4] % 8
    args = (c, int32([0, 3, 6]), table, int32([200, 250]))
    want = flock.attention_tracks(q.contiguous(), *args)
    room = torch.full((6, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    flock.attention_tracks(q, *args, out=room[:, 1:5])
    assert torch.equal(room[:, 1:5], want) and (room[:, 0] == 7).all() and (room[:, 5] == 7).all()


def test_attention_repeats_bit_for_bit_in_any_company():
    """A track's rows do not depend on the other tracks, and a call repeats to the bit."""
    gen = torch.Generator().manual_seed(17)
    c = cuda(pool(gen, 60, 2, 64))
    lengths = [900, 300, 1500, 40]
    table = table_of(gen, lengths, 60).cuda()
    q = torch.randn(4, 8, 64, generator=gen).bfloat16().cuda()
    args = (int32([0, 1, 2, 3, 4]), table, int32(lengths))
    a, b = flock.attention_tracks(q, c, *args), flock.attention_tracks(q, c, *args)
    assert torch.equal(a, b)


@pytest.mark.parametrize("mine,queries,others,total,columns,heads,dim,dtype", [
    ((900, 3), 3, 7, 20, 40, (8, 2), 64, torch.bfloat16),            # several workgroups share a track's pages
    ((900, 3), 40, 300, 500, 40, (4, 1), 128, torch.float16),
    ((200, 500), 1, 3200, 3202, 8, (2, 1), 64, torch.bfloat16),      # a wave a workgroup
    ((700, 450), 400, 60, 9000, 20, (8, 4), 64, torch.bfloat16),     # 128 rows a workgroup
    ((700, 450), 400, 60, 9000, 20, (8, 4), 96, torch.float16),
])
@pytest.mark.parametrize("cap,window", [(0.0, 0), (30.0, 100)])
def test_attention_of_a_track_in_other_company(mine, queries, others, total, columns, heads, dim, dtype, cap, window):
    """Two tracks' rows to the bit, whatever the lengths, rows, pages and places in the batch of the tracks beside them."""
    gen = torch.Generator().manual_seed(62)
    each = [(n + PAGE - 1) // PAGE for n in mine]
    c = cuda(pool(gen, 100, heads[1], dim))
    pages = [torch.randperm(100, generator=gen)[:n].int() for n in each]
    qs = [torch.randn(queries, heads[0], dim, generator=gen).to(dtype) for _ in mine]
    first = None
    for seed in range(3):
        gen = torch.Generator().manual_seed(seed)
        n = others + len(mine)
        at = torch.randperm(n, generator=gen)[:len(mine)].tolist()
        cut = torch.randint(0, total - queries * len(mine) + 1, (others - 1,), generator=gen).sort().values.tolist()
        rest = [b - a for a, b in zip([0, *cut], [*cut, total - queries * len(mine)])]
        lengths = torch.randint(0, PAGE * columns + 1, (n,), generator=gen).tolist()
        table = torch.randint(-1, 101, (n, columns), generator=gen, dtype=torch.int32)
        q = torch.randn(total, heads[0], dim, generator=gen).to(dtype)
        counts = [0] * n
        for t in range(n):
            counts[t] = queries if t in at else rest.pop()
        offsets = offsets_of(counts)
        for i, t in enumerate(at):
            lengths[t], table[t, :each[i]] = mine[i], pages[i]
            q[offsets[t]:offsets[t + 1]] = qs[i]
        out = flock.attention_tracks(q.cuda(), c, int32(offsets), table.cuda(), int32(lengths), cap=cap, window=window)
        got = torch.cat([out[offsets[t]:offsets[t + 1]] for t in at])
        first = got if first is None else first
        assert got.isfinite().all() and torch.equal(got, first)


def test_refusals():
    c = flock.TrackCache.empty(4, 2, 64)
    k = torch.zeros(3, 2, 64, device="cuda")
    off, table, lengths = int32([0, 3]), int32([[0, 1]]), int32([5])
    with pytest.raises(ValueError, match="k and v must"):
        flock.append_tracks(c, k[:, :1], k[:, :1], off, table, lengths)
    with pytest.raises(ValueError, match="k and v must"):
        flock.append_tracks(c, k, k[:2], off, table, lengths)
    with pytest.raises(ValueError, match="type and device"):
        flock.append_tracks(c, k, k.half(), off, table, lengths)
    with pytest.raises(ValueError, match="offsets"):
        flock.append_tracks(c, k, k, off.long(), table, lengths)
    with pytest.raises(ValueError, match="table"):
        flock.append_tracks(c, k, k, off, table.long(), lengths)
    with pytest.raises(ValueError, match="table"):
        flock.append_tracks(c, k, k, off, table[:, ::2].expand(2, 1), lengths)
    with pytest.raises(ValueError, match="lengths"):
        flock.append_tracks(c, k, k, off, table, int32([5, 5]))
    with pytest.raises(ValueError, match="xy"):
        flock.append_tracks(c, k, k, off, table, lengths, axes=flock.RotaryAxes(x=[1.0]))
    with pytest.raises(ValueError, match="time"):
        flock.append_tracks(c, k, k, off, table, lengths, axes=flock.RotaryAxes(time=[1.0]))
    with pytest.raises(ValueError, match="pairs"):
        flock.append_tracks(c, k, k, off, table, lengths, axes=flock.RotaryAxes(time=[1.0] * 33), time=int32([0, 1, 2]))
    q = k.bfloat16()
    with pytest.raises(ValueError, match="dtype"):
        flock.attention_tracks(k, c, off, table, lengths)
    with pytest.raises(ValueError, match="q must"):
        flock.attention_tracks(q[:, :, :32].contiguous(), c, off, table, lengths)
    with pytest.raises(ValueError, match="window"):
        flock.attention_tracks(q, c, off, table, lengths, window=-1)
    with pytest.raises(ValueError, match="scale"):
        flock.attention_tracks(q, c, off, table, lengths, scale=0.0)
    with pytest.raises(ValueError, match="out must"):
        flock.attention_tracks(q, c, off, table, lengths, out=q[:2])
    with pytest.raises(ValueError, match="multiple"):
        flock.attention_tracks(torch.zeros(3, 3, 64, dtype=torch.float16, device="cuda"), c, off, table, lengths)
    with pytest.raises(ValueError, match="k must"):
        flock.TrackCache(c.k[:, :, :32], c.v, c.k_scale, c.v_scale)
    with pytest.raises(ValueError, match="v must"):
        flock.TrackCache(c.k, c.v[:, :, :32], c.k_scale, c.v_scale)
    with pytest.raises(ValueError, match="k_scale"):
        flock.TrackCache(c.k, c.v, c.k_scale.t(), c.v_scale)
    odd = flock.TrackCache.empty(1, 1, 24)
    with pytest.raises(ValueError, match="head_dim"):
        flock.append_tracks(odd, torch.zeros(1, 1, 24, device="cuda"), torch.zeros(1, 1, 24, device="cuda"), int32([0, 1]),
                            int32([[0]]), int32([1]))


@pytest.mark.parametrize("window", [-1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32 + 5])
def test_windows_beyond_32_bits_are_refused(window):
    """(Five tokens are what the low 32 bits of two of them say.)"""
    c = flock.TrackCache.empty(1, 1, 64)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="window"):
        flock.attention_tracks(q, c, int32([0, 1]), int32([[0]]), int32([1]), window=window)


def test_empty_calls():
    c = flock.TrackCache.empty(2, 1, 64)
    none = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    nothing = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    flock.append_tracks(c, none, none, int32([0]), nothing, int32([]))
    assert flock.attention_tracks(none, c, int32([0]), nothing, int32([])).shape == (0, 1, 64)
    one = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    no_pages = flock.TrackCache.empty(0, 1, 64)
    flock.append_tracks(no_pages, one, one, int32([0, 1]), int32([[0]]), int32([1]))
    assert (flock.attention_tracks(one, no_pages, int32([0, 1]), int32([[0]]), int32([1])) == 0).all()


@pytest.mark.parametrize("dim,cap", [(32, 0.0), (64, 20.0), (128, 0.0)])
def test_attention_of_many_short_tracks(dim, cap):
    """A wave a workgroup: 1600 tracks of two kv heads."""
    gen = torch.Generator().manual_seed(18)
    lengths = torch.randint(0, 200, (1600,), generator=gen).tolist()
    queries = [min(n, int(m)) for n, m in zip(lengths, torch.randint(0, 3, (1600,), generator=gen))]
    attend(18, lengths, queries, dim=dim, cap=cap)


@pytest.mark.parametrize("dim,cap,dtype", [(64, 0.0, torch.bfloat16), (96, 30.0, torch.float16), (128, 100.0, torch.bfloat16)])
def test_attention_of_long_runs_of_queries(dim, cap, dtype):
    """128 rows a workgroup: 150 to 700 rows of each track and kv head."""
    gen = torch.Generator().manual_seed(19)
    lengths = (300 + torch.randint(0, 200, (40,), generator=gen)).tolist()
    queries = (75 + torch.randint(0, 100, (40,), generator=gen)).tolist()
    lengths[3], queries[3] = 100, 140       # rows before the track's first token
    queries[5] = 0
    lengths[7], queries[7] = 360, 350
    attend(19, lengths, queries, q_heads=16, kv_heads=8, dim=dim, cap=cap, dtype=dtype)
    attend(19, lengths, queries, q_heads=16, kv_heads=8, dim=dim, cap=cap, dtype=dtype, window=70)


def test_attention_of_long_runs_with_pages_that_are_none_or_not_finite():
    def spoil(table, c):
        table[0, 1] = -1
        table[1, 0] = len(c[0])
        table[2, :] = 2 ** 31 - 1
        c[3][int(table[4, 0])] = 0
        c[2][int(table[5, 1])] = 0
        c[3][:] *= torch.logspace(-3, 3, c[3].numel()).reshape(c[3].shape)
    lengths, queries = [300] * 40, [150] * 40
    got = attend(20, lengths, queries, q_heads=16, kv_heads=8, spoil=spoil)
    assert (got[300:450] == 0).all()

    gen = torch.Generator().manual_seed(21)
    c = pool(gen, 200, 8, 64)
    table = table_of(gen, lengths, 200)
    c[2][int(table[0, 1]), 3] = math.nan    # tokens 64 .. 127 of track 0: none of its queries is before them
    c[3][int(table[1, 3]), 2] = math.nan    # tokens 192 .. 255 of track 1: seen from its 43rd query on
    q = torch.randn(6000, 16, 64, generator=gen).bfloat16()
    got = flock.attention_tracks(q.cuda(), cuda(c), int32(offsets_of(queries)), table.cuda(), int32(lengths)).cpu()
    bad = torch.zeros(6000, 16, dtype=torch.bool)
    bad[:150, 6:8] = True
    bad[192:300, 4:6] = True
    assert torch.equal(torch.isnan(got).all(2), bad) and torch.equal(torch.isnan(got).any(2), bad)
