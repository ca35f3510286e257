"""The token operators on the GPU against plain implementations in 64 bits on the host: rotary positions, appending to the paged
cache, attention of one token over it, eviction; what goes wrong at edges (empty sequences, pages that end inside a tile, slots
without a page, garbage behind the last token), strides, streams, graphs, and pages beyond 4 GB."""
import copy
import ctypes as C
import math
import pickle

import numpy as np
import pytest
import torch

import paper_1808_05488_amd as cb

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 2.0 ** -24                    # half a unit in the last place of float32, relative
ROUND = {F32: EPS, BF16: 2.0 ** -8}       # half a unit: 24 and 8 significant bits



def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    tol = np.broadcast_to(tol, want.shape)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]!r}, not {want[bad][0]!r} +- {tol[bad][0]:.3g}"


# ---------------------------------------------------------------- rotary
def turned64(x, pos, pairs, base, layout, ladder, sign=1.0):
    """x: tokens x heads x dim, float64."""
    y, n, at = x.copy(), sum(pairs), 0
    for a, m in enumerate(pairs):
        for i in range(m):
            f = base ** -(at / n if ladder == cb.CB_LADDER_SHARED else i / m)
            angle = sign * pos[:, a].astype(np.float64) * f
            u, v = (at, n + at) if layout == cb.CB_PAIRS_HALVES else (2 * at, 2 * at + 1)
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            y[..., u], y[..., v] = x[..., u] * c - x[..., v] * s, x[..., u] * s + x[..., v] * c
            at += 1
    return y


def pair_size(x, pairs, layout):
    """|x| + |y| of the pair that every value belongs to (zero behind the pairs)."""
    n, s = sum(pairs), np.zeros_like(x)
    u, v = (np.arange(n), n + np.arange(n)) if layout == cb.CB_PAIRS_HALVES else (2 * np.arange(n), 2 * np.arange(n) + 1)
    s[..., u] = s[..., v] = np.abs(x[..., u]) + np.abs(x[..., v])
    return s


def rotary_tolerance(want, x, pairs, layout, dtype, angle=0.0):
    # two products, a sum, a sine and a cosine within 2 units in the last place each, an angle rounded to 2^-25 of a turn
    return (8 * EPS + 2 * math.pi * 2.0 ** -25 + angle) * pair_size(x, pairs, layout) + ROUND[dtype] * np.abs(want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [cb.CB_PAIRS_HALVES, cb.CB_PAIRS_ADJACENT])
@pytest.mark.parametrize("ladder", [cb.CB_LADDER_SHARED, cb.CB_LADDER_PER_AXIS])
@pytest.mark.parametrize("dim,pairs,hq,hk,n", [(8, (1,), 1, 1, 1), (16, (1, 0, 2), 3, 1, 5), (64, (8, 12, 12), 4, 2, 77),
                                               (80, (8, 12, 10), 5, 1, 33), (128, (16, 24, 24), 8, 2, 300), (72, (7, 9, 9, 2), 2, 2, 65),
                                               (256, (32, 48, 48), 2, 1, 19), (40, (20,), 3, 3, 4100)])
def test_rotate(dtype, layout, ladder, dim, pairs, hq, hk, n):
    rng = np.random.default_rng([dim, hq, n, layout, ladder])
    q, k = dev(rng.standard_normal((n, hq, dim)), dtype), dev(rng.standard_normal((n, hk, dim)), dtype)
    pos = rng.integers(-5, 2000, (n, len(pairs))).astype(np.int32)
    rot = cb.Rotary(dim, pairs, base=10000.0, layout=layout, ladder=ladder)
    for inverse in (False, True):
        out = rot.rotate(q, dev(pos), k=k, inverse=inverse)
        for name, x, got in (("q", q, out[0]), ("k", k, out[1])):
            x = f64(x)
            want = turned64(x, pos, pairs, 10000.0, layout, ladder, -1.0 if inverse else 1.0)
            within(f64(got), want, rotary_tolerance(want, x, pairs, layout, dtype), f"{name}, inverse = {inverse}")
            rest = 2 * sum(pairs)
            assert np.array_equal(f64(got)[..., rest:], x[..., rest:])
    alone = rot.rotate(q, dev(pos))
    assert torch.equal(alone, rot.rotate(q, dev(pos), k=k)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotate_at_any_position(dtype):
    pairs = (8, 12, 12)
    rng = np.random.default_rng(3)
    pos = np.array([[2**31 - 1, -2**31, 2**30], [2**20, 2**20 - 1, -2**20], [0, 0, 0], [123456789, 987654321, -5]], np.int32)
    q = dev(rng.standard_normal((4, 2, 64)), dtype)
    got = cb.Rotary(64, pairs).rotate(q, dev(pos))
    x = f64(q)
    want = turned64(x, pos, pairs, 10000.0, cb.CB_PAIRS_HALVES, cb.CB_LADDER_SHARED)
    # angles of 2^31 radians: float64 frequencies, here and in the oracle, are off by 2^-53 of them (twice)
    within(f64(got), want, rotary_tolerance(want, x, pairs, cb.CB_PAIRS_HALVES, dtype, angle=2e-6), "far positions")
    assert torch.equal(got[2], q[2])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1, 2, 3])
def test_rotate_strided_unaligned_and_in_place(dtype, off):
    rng = np.random.default_rng([5, off])
    n, dim, pairs = 37, 32, (4, 6, 6)
    flat = dev(rng.standard_normal(n * 7 * (dim + off) + 8), dtype)
    q = flat[off:].as_strided((n, 3, dim), (7 * (dim + off), dim + off, 1), off)
    k = flat.as_strided((n, 2, dim), (7 * (dim + off), 2 * (dim + off), 1), off + 3 * (dim + off))
    # the heads in the opposite order, as a wider tensor's
    pos = rng.integers(0, 500, (n, 3)).astype(np.int32)
    rot = cb.Rotary(dim, pairs)
    x, y, before = f64(q), f64(k), flat.clone()
    out = torch.zeros((3, n, dim), dtype=dtype, device="cuda").transpose(0, 1)
    a, b = rot.rotate(q, dev(pos), k=k, q_out=out)
    for name, src, got in (("q", x, a), ("k", y, b)):
        want = turned64(src, pos, pairs, 10000.0, 0, 0)
        within(f64(got), want, rotary_tolerance(want, src, pairs, 0, dtype), name)
    assert torch.equal(flat, before)
    assert rot.rotate(q, dev(pos), q_out=q) is q
    assert torch.equal(q, a)
    inside = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
    inside.as_strided(q.shape, q.stride(), q.storage_offset()).fill_(True)
    assert torch.equal(flat[~inside], before[~inside])


def test_gradient_of_the_rotation():
    """Against differences: the operator is linear, so that a difference quotient is exact but for rounding."""
    rng = np.random.default_rng(8)
    n, heads, dim, pairs = 9, 2, 24, (3, 4, 5)
    pos = dev(rng.integers(0, 300, (n, 3)).astype(np.int32))
    for layout in (0, 1):
        rot = cb.Rotary(dim, pairs, layout=layout)
        x, g, u = (dev(rng.standard_normal((n, heads, dim)), F32) for _ in range(3))
        grad = f64(rot.rotate(g, pos, inverse=True))
        h = 0.5
        diff = (f64(rot.rotate(x + h * u, pos)) - f64(rot.rotate(x - h * u, pos))) / (2 * h)
        a, b = float((diff * f64(g)).sum()), float((grad * f64(u)).sum())
        # every value of both sums is off by a few units in the last place of values of order 1
        assert abs(a - b) <= 40 * EPS * n * heads * dim
        # and the formula: dL/dx = g_x cos + g_y sin, dL/dy = -g_x sin + g_y cos
        want = turned64(f64(g), pos.cpu().numpy(), pairs, 10000.0, layout, 0, -1.0)
        within(grad, want, rotary_tolerance(want, f64(g), pairs, layout, F32), "gradient")


def test_rotate_nothing():
    rot = cb.Rotary(16, (8,))
    q = torch.empty((0, 3, 16), device="cuda")
    assert rot.rotate(q, torch.empty((0, 1), dtype=torch.int32, device="cuda")).shape == (0, 3, 16)


def test_rotate_more_tokens_than_a_launch_takes():
    """Of more than 2^24 tokens the last ones are turned as the same tokens by themselves."""
    n, dim, pairs = (1 << 24) + 1000, 8, (1, 1, 2)
    q = torch.randn((n, 1, dim), device="cuda").to(BF16)
    pos = torch.randint(0, 1000, (n, 3), device="cuda", dtype=torch.int32)
    rot = cb.Rotary(dim, pairs)
    got = rot.rotate(q, pos, k=q)
    for at in (0, (1 << 24) - 500, n - 700):
        want = rot.rotate(q[at:at + 700], pos[at:at + 700].contiguous())
        for x in got:
            assert torch.equal(x[at:at + 700], want)


# ---------------------------------------------------------------- caches
def make_cache(rng, lengths, heads, dim, page, dtype, capacity=None, spare=3, evictable=True, fill=math.nan):
    """A cache whose pages lie in no order; slots that hold no token are `fill`, and so are pages of nobody."""
    pages = [-(-x // page) for x in lengths]
    width = max(1, max(pages)) if capacity is None else -(-capacity // page)
    own = [width if capacity is not None else p for p in pages]          # (with a capacity every sequence has all its pages)
    n_pages = sum(own) + spare
    order = rng.permutation(n_pages).tolist()
    table = np.full((len(lengths), width), -1, np.int32)
    k = np.full((n_pages, heads, page, dim), fill, np.float32)
    v = k.copy()
    for s, n in enumerate(lengths):
        table[s, :own[s]], order = order[:own[s]], order[own[s]:]
        for j in range(n):
            k[table[s, j // page], :, j % page] = rng.standard_normal((heads, dim))
            v[table[s, j // page], :, j % page] = rng.standard_normal((heads, dim))
    cap = width * page
    weight = rng.random((len(lengths), heads, cap)).astype(np.float32) if evictable else None
    time = rng.integers(0, 50, (len(lengths), heads, cap)).astype(np.int32) if evictable else None
    c = cb.TokenCache(dev(k, dtype), dev(v, dtype), dev(table), dev(np.array(lengths, np.int32)),
                      dev(weight) if evictable else None, dev(time) if evictable else None)
    return c


def rows(c, pages, s, h, n):
    """The first n slots of a sequence and head, float64."""
    page = c.k_pages.shape[2]
    table = c.table.cpu().numpy()
    p = f64(pages)
    if n == 0:
        return np.zeros((0, c.head_dim))
    return np.stack([p[table[s, j // page], h, j % page] for j in range(n)])


def attend64(c, q, lengths, scale, softcap, decay=None, dead=()):
    """out, lse, weight and the tolerances of each; dead: (sequence, page in its table) without a page."""
    b, hq, dim = q.shape
    group, page = hq // c.n_kv_heads, c.k_pages.shape[2]
    q64 = f64(q)
    out, lse, tol, size = np.zeros(q64.shape), np.full((b, hq), -np.inf), np.zeros(q64.shape), np.zeros((b, hq))
    weight = None if c.weight is None else f64(c.weight)
    wtol = None if weight is None else np.zeros(weight.shape)
    for s, n in enumerate(lengths):
        keep = np.array([j for j in range(n) if (s, j // page) not in dead], int)
        for h in range(c.n_kv_heads):
            if n:
                k, v = rows(c, c.k_pages, s, h, n)[keep], rows(c, c.v_pages, s, h, n)[keep]
            wsum = np.zeros(n)
            wt = np.zeros(n)
            for g in range(h * group, (h + 1) * group):
                if len(keep) == 0:
                    continue
                with np.errstate(invalid="ignore"):
                    x = (k * q64[s, g]).sum(1) * scale
                    # a score: products summed in some order, a factor, and the cap's three operations on values up to its size
                    es = (2 * math.sqrt(dim) + 8) * EPS * float(np.nanmax(np.where(np.isfinite(k), np.abs(k * q64[s, g]), 0).sum(1))) * abs(scale)
                if softcap:
                    x = softcap * np.tanh(x / softcap)
                    es += 8 * EPS * softcap
                top = x.max()
                if top == -np.inf:
                    continue
                p = np.exp(x - top)
                z = p.sum()
                p /= z
                out[s, g], lse[s, g] = p @ v, top + math.log(z)
                # e^x of a score that is off by es, and a sum over the tokens in pieces
                rel = 2 * es + (16 + 2 * math.sqrt(len(keep))) * EPS
                tol[s, g] = rel * (p @ np.abs(v)) + ROUND[q.dtype] * np.abs(out[s, g])
                if q.dtype == BF16:
                    tol[s, g] += 2.0 ** -17 * (p @ np.abs(v))          # weights in two bfloat16 terms
                size[s, g] = es + (16 + abs(lse[s, g])) * 4 * EPS
                wsum[keep] += p
                wt[keep] += rel * p
            if weight is not None and decay is not None:
                weight[s, h, :n] = weight[s, h, :n] * decay + wsum
                wtol[s, h, :n] = wt + 4 * EPS * np.abs(weight[s, h, :n])
    return out, lse, weight, tol, size, wtol


def check_attend(c, q, lengths, softcap=0.0, scale=None, accumulate=False, decay=1.0, dead=(), **kw):
    want = attend64(c, q, lengths, c.head_dim ** -0.5 if scale is None else scale, softcap, decay if accumulate else None, dead)
    out, lse = c.attend(q, softcap=softcap, scale=scale, accumulate=accumulate, decay=decay, **kw)
    within(f64(out), want[0], want[3], "out")
    got = f64(lse)
    assert np.array_equal(np.isneginf(got), np.isneginf(want[1]))
    fine = np.isfinite(want[1])
    within(got[fine], want[1][fine], want[4][fine], "lse")
    if accumulate:
        within(f64(c.weight), want[2], want[5], "weight")
    return out


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (2, 4, 128), (3, 3, 40)])
def test_attend_at_the_edges_of_tiles_and_pages(dtype, page, heads, group, dim):
    rng = np.random.default_rng([1, page, dim])
    c = make_cache(rng, EDGES, heads, dim, page, dtype)
    q = dev(rng.standard_normal((len(EDGES), heads * group, dim)) * 2, dtype)
    check_attend(c, q, EDGES, accumulate=True, decay=0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [8, 16, 24, 32, 64, 72, 80, 96, 128, 136, 192, 256])
@pytest.mark.parametrize("group", [1, 5, 16, 17, 40])
def test_attend_head_sizes_and_groups(dtype, dim, group):
    rng = np.random.default_rng([2, dim, group])
    lengths = [70, 3, 300]
    c = make_cache(rng, lengths, 2, dim, 32, dtype)
    q = dev(rng.standard_normal((3, 2 * group, dim)), dtype)
    check_attend(c, q, lengths, accumulate=True, softcap=3.0 if group == 5 else 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,heads,group,page", [([20000], 1, 8, 128), ([9000, 1, 0, 4000], 2, 2, 1024), ([1] * 70, 1, 1, 16),
                                                      ([2500] * 5 + [0] * 5, 4, 1, 16)])
def test_attend_split_over_the_length(dtype, lengths, heads, group, page):
    rng = np.random.default_rng([3, len(lengths), heads])
    c = make_cache(rng, lengths, heads, 64, page, dtype)
    q = dev(rng.standard_normal((len(lengths), heads * group, 64)) * 3, dtype)
    first = check_attend(c, q, lengths, accumulate=True, decay=0.9)
    for _ in range(2):                                    # the sums' order does not depend on who comes first
        assert torch.equal(first, c.attend(q)[0])
    assert int(c.scratch[:4 * (64 + 1024)].view(torch.int32).abs().sum()) == 0


def test_attend_many_sequences_and_short_capacity():
    rng = np.random.default_rng(4)
    lengths = [int(x) for x in rng.integers(0, 40, 700)]
    c = make_cache(rng, lengths, 1, 16, 16, F32)
    check_attend(c, dev(rng.standard_normal((700, 2, 16)), F32), lengths, accumulate=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_scores_far_apart(dtype):
    """Weights of exactly one token, of the lowest scores, and a maximum that keeps growing."""
    rng = np.random.default_rng(6)
    lengths = [200, 200, 200]
    c = make_cache(rng, lengths, 1, 64, 16, dtype)
    k = c.k_pages.float()
    tab = c.table.cpu().numpy()
    for j in range(200):
        k[tab[1, j // 16], 0, j % 16] = 0.0
        k[tab[1, j // 16], 0, j % 16, 0] = j                   # growing
        k[tab[2, j // 16], 0, j % 16] = 0.0
        k[tab[2, j // 16], 0, j % 16, 0] = -3e38 if dtype == F32 else -2e38
    c.k_pages.copy_(k.to(dtype))
    q = torch.zeros((3, 4, 64), device="cuda", dtype=dtype)
    q[0] = 20.0
    q[1:, :, 0] = 1.0
    check_attend(c, q, lengths, scale=1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_infinite_scores(dtype):
    """Keys whose score is minus infinity count for nothing; a sequence of such keys alone gives zeros."""
    rng = np.random.default_rng(7)
    lengths = [40, 40]
    c = make_cache(rng, lengths, 2, 32, 16, dtype)
    tab = c.table.cpu().numpy()
    for j in range(40):
        for s in (0, 1):
            if s == 1 or j % 3:
                c.k_pages[int(tab[s, j // 16]), :, j % 16, 5] = -math.inf
    q = dev(np.abs(rng.standard_normal((2, 4, 32))) + 0.1, dtype)
    out, lse = c.attend(q)
    assert torch.equal(out[1], torch.zeros_like(out[1])) and bool((lse[1] == -math.inf).all())
    check_attend(c, q, lengths, accumulate=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_slots_without_a_page(dtype):
    rng = np.random.default_rng(9)
    lengths = [100, 33, 16]
    c = make_cache(rng, lengths, 2, 64, 16, dtype)
    want_dead = [(0, 2), (0, 6), (1, 0), (2, 0)]
    q = dev(rng.standard_normal((3, 2, 64)), dtype)
    good = c.table.clone()
    for value in (-1, c.k_pages.shape[0], -2**31, 2**31 - 1):
        c.table.copy_(good)
        alive = c.table.cpu().numpy().copy()
        before = attend64(c, q, lengths, 0.125, 0.0, 1.0, set(want_dead))
        for s, p in want_dead:
            c.table[s, p] = value
        weight = c.weight.clone()
        out, lse = c.attend(q, accumulate=True)
        within(f64(out), before[0], before[3], "out")
        assert bool((lse[2] == -math.inf).all()) and not bool(out[2].any())
        within(f64(c.weight), before[2], before[5], "weight")
        c.weight.copy_(weight)
        assert alive.shape == tuple(c.table.shape)


@pytest.mark.parametrize("value", [-1, -2**31, 1000, 2**31 - 1])
def test_attend_lengths_out_of_range(value):
    """Taken as 0 or the capacity."""
    rng = np.random.default_rng(10)
    c = make_cache(rng, [48, 48], 1, 32, 16, F32)
    q = dev(rng.standard_normal((2, 2, 32)), F32)
    want = c.attend(q)[0].clone()
    c.lengths[1] = value
    got = c.attend(q)[0]
    assert torch.equal(got[0], want[0])
    assert torch.equal(got[1], want[1] if value > 0 else torch.zeros_like(want[1]))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_strides_and_given_outputs(dtype):
    rng = np.random.default_rng(11)
    lengths = [50, 150]
    c = make_cache(rng, lengths, 2, 40, 32, dtype)
    wide = dev(rng.standard_normal((2, 41 * 9 + 3)), dtype)
    q = wide.as_strided((2, 4, 40), (41 * 9 + 3, 41, 1), 1)              # unaligned heads
    out = torch.zeros((4, 2, 47), dtype=dtype, device="cuda")
    view = out.permute(1, 0, 2)[:, :, 3:43]
    lse = torch.zeros((2, 4), device="cuda")
    got = check_attend(c, q, lengths, out=view, lse=lse)
    assert got is view and bool((lse != 0).all())
    assert not bool(out[:, :, :3].any()) and not bool(out[:, :, 43:].any())
    # heads in the opposite order
    assert torch.equal(c.attend(q.flip(1).contiguous().flip(1))[0], c.attend(q.contiguous())[0])


def test_attend_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(12)
    lengths = [3000, 40]
    c = make_cache(rng, lengths, 2, 64, 64, BF16)
    q = dev(rng.standard_normal((2, 8, 64)), BF16)
    want, want_lse = c.attend(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, got_lse = c.attend(q)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)

    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    graph = torch.cuda.CUDAGraph()
    c.weight.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.attend(q, out=out, lse=lse, accumulate=True)
    for i in range(4):
        q.copy_(dev(rng.standard_normal((2, 8, 64)), BF16))
        c.lengths.copy_(dev(np.array([3000 - 700 * i, 1 + i], np.int32)))       # what a graph does not know
        c.weight.zero_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        weight = c.weight.clone()
        c.weight.zero_()
        eager, eager_lse = c.attend(q, accumulate=True)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse) and torch.equal(weight, c.weight)


# ---------------------------------------------------------------- append
def append64(c, start, offsets, n, k, v, pos):
    """(pages' cells that change: {(page, head, row): (k row, v row)}, slots: {(s, slot): row}, lengths)."""
    page = c.k_pages.shape[2]
    table = c.table.cpu().numpy()
    slots, lengths = {}, []
    for s in range(c.n_seq):
        a, b = (s, s + 1) if offsets is None else (min(offsets[s], n), min(offsets[s + 1], n))
        at = min(max(int(start[s]), 0), c.capacity)
        for i in range(a, b):
            if at + i - a < c.capacity:
                slots[(s, at + i - a)] = i
        lengths.append(min(at + b - a, c.capacity))
    cells = {}
    for (s, j), i in slots.items():
        p = table[s, j // page]
        if 0 <= p < c.k_pages.shape[0]:
            cells[(int(p), j % page)] = i
    return cells, slots, lengths


def check_append(c, k, v, pos, rot, q=None, offsets=None, start=None, pairs=None, layout=0, ladder=0):
    n, dtype = k.shape[0], c.k_pages.dtype
    s0 = c.lengths.cpu().numpy() if start is None else start
    cells, slots, lengths = append64(c, s0, offsets, n, k, v, pos)
    kp, vp = f64(c.k_pages), f64(c.v_pages)
    weight, time = c.weight.cpu().numpy().copy(), c.time.cpu().numpy().copy()
    tol = np.zeros(kp.shape)
    k64 = f64(k)
    want_k = k64 if rot is None else turned64(k64, pos, pairs, 10000.0, layout, ladder)
    ktol = np.zeros(k64.shape) if rot is None else rotary_tolerance(want_k, k64, pairs, layout, dtype)
    if rot is not None:
        rest = 2 * sum(pairs)
        ktol[..., rest:] = 0.0                          # copies
    for (p, r), i in cells.items():
        kp[p, :, r], vp[p, :, r], tol[p, :, r] = want_k[i], f64(v[i]), ktol[i]
    for (s, j), i in slots.items():
        weight[s, :, j] = 0.0
        time[s, :, j] = j if pos is None else pos[i, 0]
    got = c.append(k, v, None if pos is None else dev(pos), rotary=rot, q=q, offsets=None if offsets is None else dev(np.array(offsets, np.int32)),
                   start=None if start is None else dev(np.array(start, np.int32)))
    torch.cuda.synchronize()
    a = f64(c.k_pages)
    same = np.isnan(kp)
    assert np.array_equal(np.isnan(a), same)
    within(np.where(same, 0, a), np.where(same, 0, kp), tol, "k pages")
    assert np.array_equal(f64(c.v_pages), vp, equal_nan=True)
    assert np.array_equal(c.weight.cpu().numpy(), weight) and np.array_equal(c.time.cpu().numpy(), time)
    assert c.lengths.cpu().tolist() == lengths
    if q is not None:
        last = n if offsets is None else min(offsets[-1], n)
        q64 = f64(q)
        want = turned64(q64, pos, pairs, 10000.0, layout, ladder)
        within(f64(got)[:last], want[:last], rotary_tolerance(want, q64, pairs, layout, dtype)[:last], "q")
    assert int(c.scratch[:4].view(torch.int32)) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [[1, 1, 1], [0, 5, 0], [3, 0, 90], [0, 0, 0], [200, 17, 300]])
@pytest.mark.parametrize("given", [False, True])
def test_append_ragged(dtype, new, given):
    rng = np.random.default_rng([20] + new)
    dim, pairs = 64, (8, 12, 12)
    c = make_cache(rng, [10, 0, 30], 2, dim, 16, dtype, capacity=400)
    n = sum(new)
    offsets = np.concatenate([[0], np.cumsum(new)]).tolist()
    kv = dev(rng.standard_normal((n, 4, dim)), dtype)
    q = dev(rng.standard_normal((n, 6, dim)), dtype)
    pos = rng.integers(0, 1000, (n, 3)).astype(np.int32)
    check_append(c, kv[:, :2], kv[:, 2:], pos, cb.Rotary(dim, pairs), q=q, offsets=offsets, start=[7, 33, 0] if given else None, pairs=pairs)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dim,pairs", [(8, (1, 1, 1)), (80, (8, 12, 10)), (40, (5, 5, 5)), (256, (32, 48, 48))])
def test_append_one_token_each(dtype, layout, dim, pairs):
    rng = np.random.default_rng([21, dim])
    c = make_cache(rng, [0, 15, 16, 31, 100], 3, dim, 16, dtype, capacity=112)
    k, v, q = (dev(rng.standard_normal((5, h, dim)), dtype) for h in (3, 3, 9))
    pos = rng.integers(0, 1000, (5, 3)).astype(np.int32)
    check_append(c, k, v, pos, cb.Rotary(dim, pairs, layout=layout, ladder=1), q=q, pairs=pairs, layout=layout, ladder=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_as_they_are(dtype):
    """No rotary; times are slots without positions; a token's first row behind an unaligned address."""
    rng = np.random.default_rng(22)
    c = make_cache(rng, [3, 20], 2, 24, 16, dtype, capacity=64)
    wide = dev(rng.standard_normal((9, 2 * 25 + 1)), dtype)
    k = wide.as_strided((9, 2, 24), (51, 25, 1), 1)
    v = wide.flip(0).as_strided((9, 2, 24), (51, 25, 1), 2)
    check_append(c, k, v, None, None, offsets=[0, 4, 9])
    pos = rng.integers(0, 9, (9, 1)).astype(np.int32)
    check_append(c, k, v, pos, None, offsets=[0, 9, 9])


def test_append_beyond_the_capacity_without_a_page_and_rows_of_nobody():
    rng = np.random.default_rng(23)
    dim, pairs = 32, (4, 6, 6)
    c = make_cache(rng, [30, 0, 48], 2, dim, 16, F32, capacity=48)
    c.table[1, 1] = -1
    c.table[1, 2] = c.k_pages.shape[0]
    n = 120
    k, v, q = (dev(rng.standard_normal((n, h, dim)), F32) for h in (2, 2, 2))
    pos = rng.integers(0, 1000, (n, 3)).astype(np.int32)
    rot = cb.Rotary(dim, pairs)
    # 25 rows for 18 places, 48 with a page for 16 of them, none for a full sequence; rows 75 .. 119 are nobody's
    q_out = torch.full((n, 2, dim), 7.0, device="cuda")
    cells, _, lengths = append64(c, [30, 0, 48], [0, 25, 73, 75], n, k, v, pos)
    assert lengths == [48, 48, 48] and len(cells) == 18 + 16
    c.append(k, v, dev(pos), rotary=rot, q=q, q_out=q_out, offsets=dev(np.array([0, 25, 73, 75], np.int32)), start=dev(np.array([30, 0, 48], np.int32)))
    assert bool((q_out[75:] == 7.0).all()) and not bool((q_out[:75] == 7.0).all(-1).any())
    c2 = make_cache(np.random.default_rng(23), [30, 0, 48], 2, dim, 16, F32, capacity=48)
    c2.table[1, 1] = -1
    c2.table[1, 2] = c2.k_pages.shape[0]
    check_append(c2, k, v, pos, rot, q=None, offsets=[0, 25, 73, 75], pairs=pairs)


@pytest.mark.parametrize("n", [300, 20000])
def test_append_in_a_graph(n):
    """The cache grows replay by replay; few and many workgroups."""
    rng = np.random.default_rng([24, n])
    dim, pairs = 32, (4, 6, 6)
    c, e, warm = (cb.TokenCache.create(2, 1, dim, 4 * n, F32, 16) for _ in range(3))
    k, v = (dev(rng.standard_normal((n, 1, dim)), F32) for _ in range(2))
    pos = dev(rng.integers(0, 1000, (n, 3)).astype(np.int32))
    offsets = dev(np.array([0, n // 3, n], np.int32))
    rot = cb.Rotary(dim, pairs)
    warm.append(k, v, pos, rot, offsets=offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.append(k, v, pos, rot, offsets=offsets)
    for i in range(4):
        k.copy_(torch.randn(k.shape, device="cuda"))
        offsets[1] = (i * n) // 5
        graph.replay()
        torch.cuda.synchronize()
        e.append(k, v, pos, rot, offsets=offsets)
        torch.cuda.synchronize()
        for name in ("k_pages", "v_pages", "lengths", "weight", "time"):
            assert torch.equal(getattr(c, name), getattr(e, name)), (i, name)


# ---------------------------------------------------------------- evict
def kept64(weight, time, n, budget, window):
    """Slots that stay, in ascending order."""
    if n <= budget:
        return list(range(n))
    newest = max(int(t) for t in time[:n])
    recent = [j for j in range(n) if int(time[j]) > newest - window]
    key = lambda j: -math.inf if math.isnan(weight[j]) else float(weight[j])  # noqa: E731
    if len(recent) >= budget:
        return sorted(sorted(range(n), key=lambda j: (-int(time[j]), j))[:budget])
    rest = [j for j in range(n) if j not in set(recent)]
    # a weight that is not a number ranks below minus infinity
    rest.sort(key=lambda j: (math.isnan(weight[j]), -key(j) if not math.isnan(weight[j]) else 0, j))
    return sorted(recent + rest[:budget - len(recent)])


def check_evict(c, budget, window, weight=None, time=None, lengths=None):
    page = c.k_pages.shape[2]
    table = c.table.cpu().numpy()
    w0, t0 = (c.weight if weight is None else weight).cpu().numpy(), (c.time if time is None else time).cpu().numpy()
    n0 = (c.lengths if lengths is None else lengths).cpu().numpy()
    k, v = c.k_pages.clone(), c.v_pages.clone()
    w, t, n = c.weight.cpu().numpy().copy(), c.time.cpu().numpy().copy(), []
    for s in range(c.n_seq):
        m = min(max(int(n0[s]), 0), c.capacity)
        n.append(min(m, budget))
        for h in range(c.n_kv_heads):
            keep = kept64(w0[s, h], t0[s, h], m, budget, window)
            stay, move = [j for j in keep if j < budget], [j for j in keep if j >= budget]
            free = sorted(set(range(min(m, budget))) - set(stay))
            assert len(free) == len(move)
            for j in stay:
                w[s, h, j], t[s, h, j] = w0[s, h, j], t0[s, h, j]
            for a, b in zip(move, free):
                w[s, h, b], t[s, h, b] = w0[s, h, a], t0[s, h, a]
                pa, pb = int(table[s, a // page]), int(table[s, b // page])
                if 0 <= pa < k.shape[0] and 0 <= pb < k.shape[0]:
                    k[pb, h, b % page], v[pb, h, b % page] = c.k_pages[pa, h, a % page], c.v_pages[pa, h, a % page]
    c.evict(budget, window, weight=weight, time=time, lengths=lengths)
    torch.cuda.synchronize()
    bits = torch.int16 if k.dtype == BF16 else torch.int32
    assert c.lengths.cpu().tolist() == n
    assert np.array_equal(c.weight.cpu().numpy(), w, equal_nan=True) and np.array_equal(c.time.cpu().numpy(), t)
    assert torch.equal(c.k_pages.view(bits), k.view(bits)) and torch.equal(c.v_pages.view(bits), v.view(bits))


@pytest.mark.parametrize("dtype,dim", [(F32, 8), (BF16, 8), (BF16, 128), (F32, 80)])
@pytest.mark.parametrize("budget", [1, 16, 100, 511, 512])
@pytest.mark.parametrize("window", [0, 1, 7, 60])
def test_evict(dtype, dim, budget, window):
    rng = np.random.default_rng([30, dim, budget, window])
    c = make_cache(rng, [512, 0, 99, 100, 101, 1], 2, dim, 16, dtype)
    check_evict(c, budget, window)
    before = c.k_pages.clone()
    check_evict(c, budget, window)              # within the budget: nothing moves
    assert torch.equal(before.nan_to_num(), c.k_pages.nan_to_num())


@pytest.mark.parametrize("budget", [5, 40, 64])
def test_evict_ties_and_odd_weights(budget):
    rng = np.random.default_rng([31, budget])
    c = make_cache(rng, [90, 90, 90, 90], 1, 16, 16, F32)
    w = rng.integers(0, 3, (4, 1, c.capacity)).astype(np.float32)
    w[1] = 0.0
    w[1, 0, ::2] = -0.0                                     # zeros are equal
    w[2, 0, ::3], w[2, 0, 1::7], w[2, 0, 2::7], w[2, 0, 3::7] = math.nan, math.inf, -math.inf, -5.0
    w[3] = math.nan
    c.weight.copy_(dev(w))
    c.time.zero_()
    check_evict(c, budget, 0)


@pytest.mark.parametrize("budget", [3, 30])
def test_evict_times_at_the_ends_of_the_range(budget):
    rng = np.random.default_rng(32)
    c = make_cache(rng, [60, 60], 2, 16, 16, F32)
    c.time.copy_(dev(rng.choice([-2**31, -2**31 + 1, -1, 0, 2**31 - 2, 2**31 - 1], c.time.shape).astype(np.int32)))
    check_evict(c, budget, 2)
    c = make_cache(rng, [60, 60], 2, 16, 16, F32)
    c.time.fill_(-2**31)
    check_evict(c, budget, 2**31 - 1)


@pytest.mark.parametrize("n,budget,page", [(9000, 4096, 64), (70000, 65000, 1024), (40000, 100, 256), (5000, 4999, 16)])
def test_evict_long(n, budget, page):
    rng = np.random.default_rng([33, n])
    cap = -(-n // page)
    k = torch.randn((cap + 1, 1, page, 8), device="cuda")
    v, table = torch.randn_like(k), torch.arange(cap, 0, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    c = cb.TokenCache(k, v, table, dev(np.array([n], np.int32)), dev(rng.random((1, 1, cap * page)).astype(np.float32)),
                      dev(rng.integers(0, 1000, (1, 1, cap * page)).astype(np.int32)))
    check_evict(c, budget, 5)


def test_evict_by_other_arrays():
    """The cache's own arrays receive what is left, the given ones stay as they are."""
    rng = np.random.default_rng(34)
    c = make_cache(rng, [90, 20, 50], 2, 32, 16, BF16)
    w, t = torch.rand_like(c.weight), torch.randint(0, 30, c.time.shape, dtype=torch.int32, device="cuda")
    held = c.lengths.clone()
    given = [x.clone() for x in (w, t, held)]
    for kw in (dict(weight=w, time=t, lengths=held), dict(weight=w), dict(time=t, lengths=held)):
        c.lengths.copy_(held)
        check_evict(c, 40, 3, **kw)
        assert all(torch.equal(a, b) for a, b in zip(given, (w, t, held)))


def test_evict_without_a_page():
    rng = np.random.default_rng(35)
    c = make_cache(rng, [90], 2, 32, 16, F32)
    c.table[0, 1] = -1
    c.table[0, 4] = c.k_pages.shape[0]
    check_evict(c, 40, 3)


def test_evict_in_a_graph():
    rng = np.random.default_rng(36)
    c = make_cache(rng, [300, 300], 2, 16, 16, F32)
    e = cb.TokenCache(c.k_pages.clone(), c.v_pages.clone(), c.table, c.lengths.clone(), c.weight.clone(), c.time.clone())
    held = c.lengths.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.evict(100, 4)
    for i in range(3):
        w = torch.rand_like(c.weight)
        for x in (c, e):
            x.weight.copy_(w)
            x.lengths.copy_(held - 70 * i)
        graph.replay()
        torch.cuda.synchronize()
        e.evict(100, 4)
        for name in ("k_pages", "v_pages", "lengths", "weight", "time"):
            a, b = getattr(c, name), getattr(e, name)
            assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b), name


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pages_beyond_4_gb(dtype):
    """Append, attend and evict where offsets into the pages pass 2^32 bytes (and 2^31 values in bfloat16)."""
    rng = np.random.default_rng(40)
    heads, dim, page, pairs = 8, 128, 128, (16, 24, 24)
    size = heads * dim * page * (4 if dtype == F32 else 2)
    n_pages = (6 << 30) // size
    kp, vp = (torch.empty((n_pages, heads, page, dim), dtype=dtype, device="cuda") for _ in range(2))
    table = dev(np.array([[n_pages - 1, 0, n_pages - 2, n_pages // 2]], np.int32))
    small = cb.TokenCache.create(1, heads, dim, 4 * page, dtype, page)
    zeros = lambda t: torch.zeros((1, heads, 4 * page), dtype=t, device="cuda")  # noqa: E731
    big = cb.TokenCache(kp, vp, table, torch.zeros(1, dtype=torch.int32, device="cuda"), zeros(F32), zeros(torch.int32))
    n = 500
    k, v, q = (dev(rng.standard_normal((n, heads, dim)), dtype) for _ in range(3))
    pos = dev(rng.integers(0, 400, (n, 3)).astype(np.int32))
    for c in (big, small):
        c.append(k, v, pos, cb.Rotary(dim, pairs), offsets=dev(np.array([0, n], np.int32)))
        c.attend(q[:1], accumulate=True)
        c.evict(300, 2)
    for x, y in ((kp, small.k_pages), (vp, small.v_pages)):
        assert torch.equal(x[table[0].long()].transpose(0, 1).flatten(1, 2)[:, :300], y.transpose(0, 1).flatten(1, 2)[:, :300])
    assert torch.equal(big.weight, small.weight)
    assert torch.equal(big.attend(q[:1])[0], small.attend(q[:1])[0])


def test_caches_that_share_a_scratch_buffer():
    rng = np.random.default_rng(41)
    lengths = [700, 20, 3000]
    a, b = make_cache(rng, lengths, 2, 128, 64, BF16), make_cache(rng, [90], 1, 32, 16, F32)
    qa, qb = dev(rng.standard_normal((3, 36, 128)), BF16), dev(rng.standard_normal((1, 3, 32)), F32)
    shared = torch.zeros(max(a.scratch_bytes(36), b.scratch_bytes(3)) + 256, dtype=torch.uint8, device="cuda")
    shared = shared[(-shared.data_ptr()) % 256:]
    want = a.attend(qa)[0].clone(), b.attend(qb)[0].clone()
    a2 = cb.TokenCache(a.k_pages, a.v_pages, a.table, a.lengths, a.weight.clone(), a.time.clone(), scratch=shared)
    b2 = cb.TokenCache(b.k_pages, b.v_pages, b.table, b.lengths, b.weight.clone(), b.time.clone(), scratch=shared)
    for _ in range(3):
        assert torch.equal(a2.attend(qa, accumulate=True)[0], want[0])
        assert torch.equal(b2.attend(qb, accumulate=True)[0], want[1])
    assert a2.scratch.data_ptr() == shared.data_ptr() == b2.scratch.data_ptr()


def test_what_python_refuses():
    c = cb.TokenCache.create(2, 2, 32, 64, F32, 16)
    q = torch.zeros((2, 4, 32), device="cuda")
    for bad in (q.double(), q[:1], q[..., :16], q.cpu(), torch.zeros((2, 4, 64), device="cuda")[..., ::2]):
        with pytest.raises((AssertionError, KeyError)):
            c.attend(bad)
    with pytest.raises(cb.CBError):
        c.attend(q[:, :3])
    k = torch.zeros((5, 2, 32), device="cuda")
    with pytest.raises(AssertionError):
        c.append(k, k[:4])
    with pytest.raises(AssertionError):
        c.append(k, k, torch.zeros((5, 3), dtype=torch.int64, device="cuda"))
    with pytest.raises(AssertionError):
        c.append(k, k, offsets=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(cb.CBError):
        c.append(k, k)                              # five rows, two sequences
    with pytest.raises(cb.CBError):
        c.evict(0)
    with pytest.raises(AssertionError):
        cb.TokenCache(c.k_pages, c.v_pages, c.table.long(), c.lengths)
    with pytest.raises(cb.CBError):
        cb.TokenCache(c.k_pages.view(8, 2, 16, 32)[:, :, :8].contiguous(), c.v_pages[:, :, :8].contiguous(), c.table, c.lengths)


def test_a_graph_keeps_the_scratch_buffer_that_it_was_recorded_with():
    rng = np.random.default_rng(42)
    c = make_cache(rng, [5000, 40], 2, 64, 64, BF16)
    q, more = (dev(rng.standard_normal((2, heads, 64)), BF16) for heads in (4, 32))
    want, want_lse = c.attend(q)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(q, out=out, lse=lse)
    nbytes = c.scratch.numel()
    wider = c.attend(more)[0]
    assert c.scratch.numel() > nbytes
    others = [torch.full((nbytes + 256,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]      # would take a buffer that is free
    for _ in range(3):
        out.zero_()
        lse.zero_()
        graph.replay()
        assert torch.equal(c.attend(more)[0], wider)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert all(bool((x == 0x5A).all()) for x in others)


def test_no_scratch_buffer_is_made_while_a_graph_is_recorded():
    rng = np.random.default_rng(43)
    c = make_cache(rng, [300, 40], 2, 64, 64, BF16)
    q = dev(rng.standard_normal((2, 32, 64)), BF16)
    x = torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        with pytest.raises(AssertionError, match="attend once before"):
            c.attend(q)
    want = c.attend(q)[0]
    graph.replay()
    assert torch.equal(c.attend(q)[0], want) and bool((x == 1).all())


def test_append_refuses_more_rows_than_its_count_holds():
    c = cb.TokenCache.create(2, 2, 32, 64, F32, 16)
    rows = torch.zeros((1, 2, 32), device="cuda").expand(2 ** 32 + 2, 2, 32)       # 2 rows, were the count cut to 32 bits
    with pytest.raises(cb.CBError):
        c.append(rows, rows)
    assert not bool(c.lengths.any())


def small_cache(k, v, page=16, weight=False):
    """A cache of one head whose sequences hold k and v (sequences x tokens x dim)."""
    n_seq, n, dim = k.shape
    c = cb.TokenCache.create(n_seq, 1, dim, n, k.dtype, page, evictable=weight)
    c.append(k.reshape(-1, 1, dim), v.reshape(-1, 1, dim), offsets=torch.arange(0, n_seq * n + 1, n, dtype=torch.int32, device="cuda"))
    return c


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_weights_keep_the_bits_of_float32(dim):
    """Two tokens whose values nearly cancel, each in its own way: what is left shows the weights' own rounding."""
    b, heads = 8, 16
    k = torch.zeros((b, 2, dim), dtype=BF16, device="cuda")
    k[:, 1, 0] = -1.0
    v = torch.ones((b, 2, dim), dtype=BF16, device="cuda")
    v[:, 1] = -(1 + (torch.arange(dim, device="cuda") % 64) / 64).to(BF16)
    c = small_cache(k, v)
    q = torch.zeros((b, heads, dim), dtype=BF16, device="cuda")
    q[..., 0] = (1 + torch.arange(b * heads, device="cuda").view(b, heads) / 128).to(BF16)          # 128 numbers of 8 bits
    out, _ = c.attend(q, scale=0.25)
    p = np.exp(-0.25 * f64(q)[..., 0])[..., None]       # (of exact scores)
    want = (1 + p * f64(v)[0, 1]) / (1 + p)
    # of sums of up to 2: a weight to 1.5 units in its last place (3 EPS of values up to 2), three sums (2 EPS each), over 1.6; and the result's rounding
    within(f64(out), want, 8 * EPS + ROUND[BF16] * np.abs(want), "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,dim", [(1, 64), (7, 80), (40, 256), (200, 128), (20000, 64)])
def test_attend_infinite_values(dtype, n, dim):
    """A weight that is not zero times infinity is infinity, wherever the token is; infinities of both signs, or a value that is not a number,
    give what is not a number; all else is as it was."""
    rng = np.random.default_rng([50, n, dim])
    c = make_cache(rng, [n, n], 1, dim, 16, dtype)
    q = dev(rng.standard_normal((2, 3, dim)), dtype)
    finite = attend64(c, q, [n, n], dim ** -0.5, 0.0)
    want = finite[0].copy()
    tab = c.table.cpu().numpy()
    for d in range(40):                                 # (values 40 and above stay finite, and so does sequence 1)
        kind, j = d % 5, int(rng.integers(n))
        x = [math.inf, -math.inf, math.nan, math.inf, math.inf][kind]
        c.v_pages[int(tab[0, j // 16]), 0, j % 16, d] = x
        want[0, :, d] = x
        if kind >= 3 and n > 1:                         # a second one: of the other sign, or the same
            i = (j + 1 + int(rng.integers(n - 1))) % n
            c.v_pages[int(tab[0, i // 16]), 0, i % 16, d] = -math.inf if kind == 3 else math.inf
            want[0, :, d] = math.nan if kind == 3 else math.inf
    out = f64(c.attend(q)[0])
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isposinf(out), np.isposinf(want))
    assert np.array_equal(np.isneginf(out), np.isneginf(want))
    fine = np.isfinite(want)
    within(out[fine], want[fine], finite[3][fine], "finite values")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 2, 31, 64, 257, 30000])
def test_attend_values_near_the_largest(dtype, n):
    """A weighted mean is no larger than the largest value, however many tokens it is of."""
    dim = 64
    k = torch.zeros((1, n, dim), dtype=dtype, device="cuda")
    k[0, :, 1] = torch.arange(n, device="cuda") % 2
    v = torch.full((1, n, dim), 3e38, dtype=dtype, device="cuda")
    v[..., dim // 2:] *= -1
    q = torch.zeros((1, 4, dim), dtype=dtype, device="cuda")
    q[0, 2:, 1] = 1.5                                   # heads with equal scores, and with two sizes of them
    c = small_cache(k, v)
    out, lse = c.attend(q, scale=1.0)
    want = np.broadcast_to(f64(v)[0, 0], (1, 4, dim))
    # weights of one size and their sum, in pieces: as in attend64, without an error of the scores
    within(f64(out) / 1e38, want / 1e38, ((16 + 2 * math.sqrt(n)) * EPS + ROUND[dtype]) * np.abs(want) / 1e38, "out")
    z = math.log(sum(math.exp(1.5 * (j % 2)) for j in range(n)))
    within(f64(lse)[0, 2:], [z, z], (16 + abs(z)) * 4 * EPS, "lse")


def test_attend_exponentials_are_exact_to_float32():
    """One token of weight 1 and value 0, one of weight e^x and value 1: what comes out is e^x / (1 + e^x)."""
    dim, heads = 64, 512
    k = torch.zeros((1, 2, dim), device="cuda")
    k[0, 1, 0] = 1.0
    v = torch.zeros((1, 2, dim), device="cuda")
    v[0, 1] = 1.0
    c = small_cache(k, v, weight=True)
    q = torch.zeros((1, heads, dim), device="cuda")
    q[0, :, 0] = -torch.from_numpy(np.random.default_rng(51).uniform(0.0, 80.0, heads).astype(np.float32)).cuda()
    out, lse = c.attend(q, scale=1.0, accumulate=True)
    x = f64(q)[0, :, 0]
    want = np.exp(x) / (1 + np.exp(x))
    # e^x to 1 unit in the last place (2 EPS) and its second term, the sum, the division and its factor
    within(f64(out)[0, :, 0], want, 8 * EPS * want, "out")
    within(f64(lse)[0], np.log1p(np.exp(x)), 4 * EPS, "lse")
    # both tokens' weights over all heads: the same, and 512 sums
    total = np.array([heads - want.sum(), want.sum()])
    within(f64(c.weight)[0, 0, :2], total, (8 + 512) * EPS * total, "weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [3, 200, 5000])
@pytest.mark.parametrize("score", [0.0, 1e3, -1e4, 1e5, 1e6, -1e8, 3e38, -3e38])
def test_weights_that_are_added_up_are_those_of_the_softmax(dtype, n, score):
    """Every head's weights add up to one, however large the scores are that they come from."""
    dim, group = 32, 3
    k = torch.zeros((1, n, dim), dtype=dtype, device="cuda")
    k[..., 3] = score
    v = torch.randn((1, n, dim), device="cuda").to(dtype)
    c = small_cache(k, v, weight=True)
    q = torch.zeros((1, group, dim), dtype=dtype, device="cuda")
    q[..., 3] = 1.0
    c.attend(q, scale=1.0, accumulate=True)
    got = f64(c.weight)[0, 0]
    # equal scores: e^0 over a sum of n ones (exact below 2^24), a division, a product, a sum over the heads
    within(got[:n], np.full(n, group / n), 8 * EPS * group / n, "weights")
    assert not got[n:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_of_scores_far_apart(dtype):
    """Growing scores, scores of the lowest values, and small steps between large scores."""
    n, dim = 200, 64
    k = torch.zeros((3, n, dim), dtype=dtype, device="cuda")
    k[0, :, 0] = torch.arange(n, device="cuda")
    k[1, :, 0] = -3e38 if dtype == F32 else -2e38
    k[2, :, 0] = torch.arange(n, device="cuda") % 2
    k[2, :, 1] = 100000.0 if dtype == F32 else 99840.0
    v = torch.randn((3, n, dim), device="cuda").to(dtype)
    c = small_cache(k, v, weight=True)
    q = torch.zeros((3, 4, dim), dtype=dtype, device="cuda")
    q[:2, :, 0] = 1.0
    q[2, :, :2] = 1.0
    check_attend(c, q, [n] * 3, scale=1.0)
    c.weight.zero_()
    c.attend(q, scale=1.0, accumulate=True)
    scores = f64(k)[:, :, :2] @ np.ones(2)
    scores[:2] = f64(k)[:2, :, 0]
    p = np.exp(scores - scores.max(1, keepdims=True))
    want = 4 * p / p.sum(1, keepdims=True)
    # exact scores and differences: e^x of up to -100 in two terms, a sum, a division, products
    within(f64(c.weight)[:, 0, :n], want, (16 + 2 * math.sqrt(n)) * EPS * want + 1e-37, "weights")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_of_slots_without_a_page_do_not_fade(dtype):
    """They hold no token: their weight is left alone, whatever the page number is that is none."""
    rng = np.random.default_rng(52)
    lengths = [100, 33, 16]
    c = make_cache(rng, lengths, 2, 64, 16, dtype)
    dead = [(0, 2), (0, 6), (1, 0), (2, 0)]
    q = dev(rng.standard_normal((3, 2, 64)), dtype)
    want = attend64(c, q, lengths, 0.125, 0.0, 0.5, set(dead))
    for (s, p), value in zip(dead, (-1, c.k_pages.shape[0], -2**31, 2**31 - 1)):
        c.table[s, p] = value
        want[2][s, :, p * 16:p * 16 + 16] = f64(c.weight)[s, :, p * 16:p * 16 + 16]
    before = c.weight.clone()
    c.attend(q, accumulate=True, decay=0.5)
    within(f64(c.weight), want[2], want[5], "weight")
    for s, p in dead:
        assert torch.equal(c.weight[s, :, p * 16:p * 16 + 16], before[s, :, p * 16:p * 16 + 16])


def test_copies_of_a_rotary():
    """A copy goes by its own frequencies, whatever becomes of the first one."""
    rng = np.random.default_rng(53)
    q, pos = dev(rng.standard_normal((9, 2, 64)), F32), dev(rng.integers(0, 500, (9, 3)).astype(np.int32))
    first = cb.Rotary(64, (8, 12, 12))
    want = first.rotate(q, pos)
    others = [copy.deepcopy(first), pickle.loads(pickle.dumps(first))]
    for r in others:
        assert torch.equal(r.rotate(q, pos), want)
    first.plan.desc.pairs[0] = 99                       # is refused from here on
    with pytest.raises(cb.CBError):
        first.rotate(q, pos)
    c = cb.TokenCache.create(9, 2, 64, 16, F32, 16)
    for r in others:
        assert torch.equal(r.rotate(q, pos), want)
        c.append(q, q, pos, rotary=r, start=torch.zeros(9, dtype=torch.int32, device="cuda"))
        assert torch.equal(c.k_pages[:, :, 0], want)


def test_a_cache_is_not_copied():
    """Neither object could know of a scratch buffer that the other one makes or lets go."""
    c = cb.TokenCache.create(2, 2, 32, 64, F32, 16)
    for made in (copy.copy, copy.deepcopy, pickle.dumps):
        with pytest.raises(TypeError, match="not copied"):
            made(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradients_go_through_the_rotation(dtype, layout, inverse):
    rng = np.random.default_rng([54, layout])
    n, dim, pairs = 21, 40, (5, 6, 6)
    pos = dev(rng.integers(0, 300, (n, 3)).astype(np.int32))
    rot = cb.Rotary(dim, pairs, layout=layout)
    qkv = dev(rng.standard_normal((n, 7, dim)), dtype)
    gq, gk = dev(rng.standard_normal((n, 4, dim)), dtype), dev(rng.standard_normal((n, 2, dim)), dtype)
    want = rot.rotate(qkv[:, :4], pos, k=qkv[:, 4:6], inverse=inverse)
    back = rot.rotate(gq, pos, k=gk, inverse=not inverse)
    x = qkv.clone().requires_grad_()
    out = rot.rotate(x[:, :4], pos, k=x[:, 4:6], inverse=inverse)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    torch.autograd.backward(out, (gq, gk))
    assert torch.equal(x.grad[:, :4], back[0]) and torch.equal(x.grad[:, 4:6], back[1]) and not bool(x.grad[:, 6:].any())
    # q alone, and k alone of both; gradients of any strides (a sum's are one value, repeated)
    x.grad = None
    rot.rotate(x[:, :4], pos, inverse=inverse).sum().backward()
    ones = torch.ones_like(gq)
    assert torch.equal(x.grad[:, :4], rot.rotate(ones, pos, inverse=not inverse)) and not bool(x.grad[:, 4:].any())
    x.grad = None
    q, k = rot.rotate(qkv[:, :4], pos, k=x[:, 4:6], inverse=inverse)
    assert not q.requires_grad
    k.backward(gk.transpose(1, 2).contiguous().transpose(1, 2))
    assert torch.equal(x.grad[:, 4:6], back[1]) and not bool(x.grad[:, :4].any())
    # one of two results is used
    x.grad = None
    rot.rotate(x[:, :4], pos, k=x[:, 4:6], inverse=inverse)[0].backward(gq)
    assert torch.equal(x.grad[:, :4], back[0]) and not bool(x.grad[:, 4:].any())
    # outputs that are given are written outside of autograd's sight
    for kw in (dict(q_out=torch.empty_like(gq)), dict(k=gk, k_out=torch.empty_like(gk))):
        with pytest.raises(AssertionError, match="gradient"):
            rot.rotate(x[:, :4], pos, **kw)
    with torch.no_grad():
        got = torch.empty_like(gq)
        assert torch.equal(rot.rotate(x[:, :4], pos, inverse=inverse, q_out=got), want[0]) and not got.requires_grad


def test_gradient_of_the_gradient_of_the_rotation():
    """Linear in q: what a loss of the gradient gives back is the rotation itself."""
    rng = np.random.default_rng(55)
    pos = dev(rng.integers(0, 300, (5, 2)).astype(np.int32))
    rot = cb.Rotary(16, (3, 4))
    x, g, u = (dev(rng.standard_normal((5, 2, 16)), F32) for _ in range(3))
    x.requires_grad_()
    g.requires_grad_()
    grad, = torch.autograd.grad(rot.rotate(x, pos), x, g, create_graph=True)
    again, = torch.autograd.grad(grad, g, u)
    assert torch.equal(again, rot.rotate(u, pos))


def test_the_cache_refuses_what_wants_a_gradient():
    """What is cached, and what is read from it, carries none: a graph that would end there without a word is refused."""
    c = cb.TokenCache.create(2, 2, 32, 64, F32, 16)
    k, v, q = torch.randn((2, 2, 32), device="cuda"), torch.randn((2, 2, 32), device="cuda"), torch.randn((2, 4, 32), device="cuda")
    pos, rot = torch.zeros((2, 1), dtype=torch.int32, device="cuda"), cb.Rotary(32, (16,))
    wants = lambda x: x.clone().requires_grad_()  # noqa: E731
    for args, kw in (((wants(k), v), {}), ((k, wants(v)), {}), ((k, v, pos, rot), dict(q=wants(q)))):
        with pytest.raises(AssertionError, match="gradient"):
            c.append(*args, **kw)
    assert not bool(c.lengths.any())
    with pytest.raises(AssertionError, match="gradient"):
        c.attend(wants(q))
    with torch.no_grad():
        c.append(wants(k), wants(v), pos, rot, q=wants(q))
        c.attend(wants(q))
    assert c.lengths.tolist() == [1, 1]
    c.append(wants(k).detach(), v)
    assert c.lengths.tolist() == [2, 2]


@pytest.mark.parametrize("network", [True, False])
def test_lists_of_layers_that_take_them_over(network):
    """A propagated 1 x 1 layer's list is its producer's, which may have taken it over itself; behind a pooling stage it is the layer's own."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    h, w = 20, 28
    layers = [cb.Layer(rand(8, 3, 3, 3), None, 1, 1, h, w, True)]
    layers += [cb.Layer(rand(8, 8, 1, 1), None, 1, 0, h, w, True, mode=cb.CB_PROPAGATE) for _ in range(2)]
    pools = [None, None, cb.Pool(layers[-1], 2)]
    layers.append(cb.Layer(rand(4, 8, 1, 1), None, 1, 0, h // 2, w // 2, True, mode=cb.CB_PROPAGATE))
    pools.append(None)
    net = cb.Network(layers, pools)
    image = rand(3, h, w)
    for frame in range(3):
        if frame:
            image = image.clone()
            image[:, 3 + frame:6, 4:9] += 1.0
        if network:
            net.forward(image, [0.01] * 4)
        else:
            x = layers[0].process_frame(image, 0.01)
            for i in (1, 2):
                x = layers[i].process_frame_propagated(x, layers[i - 1])
            layers[3].process_frame_propagated(pools[2].process(), pools[2])
        for layer in layers:
            want = layer.changes_host()
            pixel, count = layer.listed()
            assert pixel.shape == (layer.Ho * layer.Wo,) and int(count) == want[3] > 0
            assert np.array_equal(pixel[:int(count)].cpu().numpy(), want[2])
        assert layers[2].listed()[0].data_ptr() == layers[0].listed()[0].data_ptr() or frame == 0


def test_outputs_of_nothing_are_refused():
    """An output without its input would come back unwritten."""
    c = cb.TokenCache.create(2, 2, 32, 64, F32, 16)
    k, out = torch.zeros((2, 2, 32), device="cuda"), torch.zeros((2, 4, 32), device="cuda")
    pos, rot = torch.zeros((2, 1), dtype=torch.int32, device="cuda"), cb.Rotary(32, (16,))
    with pytest.raises(AssertionError, match="q_out"):
        c.append(k, k, pos, rot, q_out=out)
    assert not bool(c.lengths.any())
    with pytest.raises(AssertionError, match="k_out"):
        rot.rotate(out, pos, k_out=k)


def class_cache(rng, lengths, heads, dim, page, dtype):
    """Long sequences over 64 pages that are only read: the tables name them in no order, again and again.  A page is of one of 16 classes (another
    one for each key head): query head i of 16 scores 0 at pages of class i and so little at others that their weight is zero; values
    i, i + 16, ... of those pages are zero, and large on all others."""
    cls = (np.arange(64)[:, None] + 5 * np.arange(heads)) % 16
    k = np.where(np.arange(16) == cls[..., None], 0.0, -30000.0)
    v = np.where(np.arange(dim) % 16 == cls[..., None], 0.0, 2.0 ** 20)
    k = np.concatenate([k, np.zeros((64, heads, dim - 16))], 2)
    pages = [dev(x.astype(np.float32)).to(dtype)[:, :, None].expand(-1, -1, page, -1).contiguous() for x in (k, v)]
    table = rng.integers(0, 64, (len(lengths), -(-max(lengths) // page))).astype(np.int32)
    c = cb.TokenCache(*pages, dev(table), dev(np.array(lengths, np.int32)))
    q = torch.zeros((len(lengths), heads, 16, dim), dtype=dtype, device="cuda")
    q[:, :, range(16), range(16)] = 1.0
    counts = np.zeros((len(lengths), heads, 16))        # tokens of a class
    for s, n in enumerate(lengths):
        held = np.bincount(table[s], np.clip(n - page * np.arange(table.shape[1]), 0, page), 64)
        for h in range(heads):
            counts[s, h] = np.bincount(cls[:, h], held, 16)
    return c, q.flatten(1, 2), counts


@pytest.mark.parametrize("dtype,dim,page,lengths,heads", [
    # a run within one pair (dealt to the wavefronts in turn): up to 137 tiles a wavefront on 256 compute units, page numbers come for 32 or 64 at a time
    (BF16, 64, 32, [9_000_000], 1), (F32, 64, 32, [9_000_001], 1), (BF16, 256, 16, [1_400_000], 1), (F32, 128, 64, [2_500_017], 1),
    (BF16, 64, 16, [1_500_000, 3, 0, 1_700_000, 40_000], 2), (F32, 256, 32, [70_000] * 16 + [1, 17], 1),
    # more pairs than workgroups: runs over ends of heads and sequences
    (BF16, 64, 64, [40_000, 1, 0, 37_001, 16, 45_000, 39_999] + [20_000] * 6, 96), (F32, 64, 16, [40_000, 1, 0, 37_001, 16] + [20_000] * 8, 48),
    (BF16, 128, 32, [40_000, 1, 0, 37_001, 16] + [20_000] * 8, 48), (F32, 256, 64, [40_000, 1, 0, 37_001, 16] + [20_000] * 8, 24)])
def test_attend_wavefronts_with_more_tiles_than_page_numbers(dtype, dim, page, lengths, heads):
    rng = np.random.default_rng([56, dim, len(lengths)])
    c, q, counts = class_cache(rng, lengths, heads, dim, page, dtype)
    out, lse = c.attend(q, scale=1.0)
    out = f64(out).reshape(counts.shape + (dim,))
    own = np.arange(dim) % 16 == np.arange(16)[:, None]
    some = counts > 0
    # a wrong page among the values: 2^20 / n at least
    assert not out[np.broadcast_to(own, out.shape) & some[..., None]].any()
    # a wrong page among the keys: a whole page's tokens less or more; counts below 2^24 are exact, and so is the maximum, zero
    n = np.array(lengths)[:, None, None] + np.zeros_like(counts)
    least = float(c.k_pages.float().min())              # (-30000 as the type holds it)
    with np.errstate(divide="ignore"):
        want = np.where(some, np.log(counts), least + np.log(n))
    got = f64(lse).reshape(counts.shape)
    assert np.array_equal(np.isneginf(got), n == 0)
    fine = n > 0
    within(got[fine], want[fine], (4 * EPS * (1 + np.abs(want)))[fine], "lse")


@pytest.mark.parametrize("budget,window", [(600, 0), (30_000, 3), (30_720, 0), (39_000, 8)])
def test_evict_sequences_that_fit_beside_some_that_do_not(budget, window):
    """Room for more slots than ranks fit on chip; sequences around that number, and short ones, in one call."""
    rng = np.random.default_rng([58, budget])
    lengths, page, dim = [40_000, 30_720, 30_721, 500, 0, 700], 64, 8
    pages = -(-max(lengths) // page)
    k = torch.randn((len(lengths) * pages, 1, page, dim), device="cuda")
    table = dev(rng.permutation(len(lengths) * pages).astype(np.int32).reshape(len(lengths), pages))
    slots = (len(lengths), 1, pages * page)
    c = cb.TokenCache(k, torch.randn_like(k), table, dev(np.array(lengths, np.int32)),
                      dev(rng.integers(0, 3000, slots).astype(np.float32)), dev(rng.integers(0, 1000, slots).astype(np.int32)))
    check_evict(c, budget, window)


def backwards(t, step_tokens=True, step_heads=True):
    """cb_heads of t's memory read from its last token and head on."""
    n, heads, dim = t.shape
    a, b = t.stride()[:2]
    at = (n - 1) * a * step_tokens + (heads - 1) * b * step_heads
    return cb.binding.cb_heads(t.data_ptr() + at * t.element_size(), -a if step_tokens else a, -b if step_heads else b, heads, 0)


def forwards(t):
    return cb.binding.cb_heads(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1], 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens,heads", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("pad", [0, 1, 2])
def test_tensors_in_the_opposite_order(dtype, tokens, heads, pad):
    """Strides of any sign, in inputs and in outputs (torch has none below zero: through the C ABI)."""
    rng = np.random.default_rng([59, pad])
    L, code = cb.lib(), cb.CB_F32 if dtype == F32 else cb.CB_BF16
    dims, dim, pairs = [d for d, on in ((0, tokens), (1, heads)) if on], 32, (4, 6, 6)
    stream = torch.cuda.current_stream().cuda_stream
    wide = lambda n, h: dev(rng.standard_normal((n, h, dim + pad)), dtype)[:, :, :dim]  # noqa: E731
    n = 37
    pos, rot = dev(rng.integers(0, 500, (n, 3)).astype(np.int32)), cb.Rotary(dim, pairs)
    q, k, q_out, k_out = wide(n, 6), wide(n, 2), wide(n, 6), wide(n, 2)
    assert L.cb_rotate(C.byref(rot.plan), code, n, pos.data_ptr(), C.byref(backwards(q, tokens, heads)), C.byref(forwards(q_out)),
                       C.byref(forwards(k)), C.byref(backwards(k_out, tokens, heads)), 0, stream) == cb.CB_OK
    assert torch.equal(q_out, rot.rotate(q.flip(dims), pos))
    assert torch.equal(k_out, rot.rotate(k, pos).flip(dims))

    a, b = cb.TokenCache.create(1, 2, dim, 64, dtype, 16), cb.TokenCache.create(1, 2, dim, 64, dtype, 16)
    v, offsets = wide(n, 2), dev(np.array([0, n], np.int32))
    want = a.append(k.flip(dims), v.flip(dims), pos, rot, q=q, offsets=offsets).flip(dims)
    assert L.cb_cache_append(C.byref(b.desc), C.byref(rot.plan), n, pos.data_ptr(), offsets.data_ptr(), None, C.byref(backwards(k, tokens, heads)),
                             C.byref(backwards(v, tokens, heads)), C.byref(forwards(q)), C.byref(backwards(q_out, tokens, heads)), stream) == cb.CB_OK
    assert torch.equal(q_out, want) and torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)

    c = make_cache(rng, [50, 150, 7], 2, dim, 32, dtype)
    q, out = wide(3, 4), wide(3, 4)
    c.attend(q)                                         # (its scratch buffer)
    prm = cb.binding.cb_attend_params(0.25, 0.0, 1.0, 0, 0)
    want = c.attend(q.flip(dims), scale=0.25)[0].flip(dims)
    assert L.cb_cache_attend(C.byref(c.desc), C.byref(prm), C.byref(backwards(q, tokens, heads)), C.byref(backwards(out, tokens, heads)), None,
                             stream) == cb.CB_OK
    assert torch.equal(out, want)
