"""Norms of heads with their rotation and gradients, caches in 8 bits, bounds of pages and attention over those that are chosen, on the GPU against plain
implementations in 64 bits on the host; a run of them together; streams, graphs and what Python refuses."""
import ctypes as C
import gc
import math
import types

import numpy as np
import pytest
import torch

import paper_1808_05488_amd as cb
from test_gpu_tokens import BF16, EPS, F32, ROUND, attend64, dev, f64, make_cache, pair_size, rows, turned64, within

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
ANGLE = 2 * math.pi * 2.0 ** -25           # an angle rounded to 2^-25 of a turn


# ---------------------------------------------------------------- norms with rotation
def norm64(x, w, pos, pairs, layout, ladder, eps):
    """(out, n, r) in 64 bits: x tokens x heads x dim."""
    eps = float(np.float32(eps))
    r = 1.0 / np.sqrt((x * x).mean(2, keepdims=True) + eps)
    return turned64(x * r * w, pos, pairs, 10000.0, layout, ladder), x * r, r


def norm_back64(x, w, g_out, pos, pairs, layout, ladder, eps):
    _, n, r = norm64(x, w, pos, pairs, layout, ladder, eps)
    g = turned64(g_out, pos, pairs, 10000.0, layout, ladder, -1.0)
    gx = r * (w * g - n * (w * g * n).mean(2, keepdims=True))
    return gx, (g * n).sum((0, 1)), n, r


def turned_size(x, pairs, layout):
    """What bounds a turned value: |x| + |y| of its pair, itself behind the pairs."""
    return np.maximum(pair_size(x, pairs, layout), np.abs(x))


def norm_tolerance(y, want, pairs, layout, dtype):
    # r: a sum of squares of up to 16 values a lane and 6 steps across lanes, scaled, eps added (25), its root (half of that), root and inverse (2): 15;
    # two products more, then the turn: two products, a sum, sine and cosine within 2 units each
    return (17 * EPS + 8 * EPS + ANGLE) * turned_size(y, pairs, layout) + ROUND[dtype] * np.abs(want)


def check_norm(rot, q, w, pos, pairs, layout, ladder, eps, got, what):
    x, w = f64(q), f64(w)
    want, n, _ = norm64(x, w, pos, pairs, layout, ladder, eps)
    within(f64(got), want, norm_tolerance(n * w, want, pairs, layout, q.dtype), what)


SHAPES = [(8, (1,), 1, 1, 1), (8, (1, 1, 2), 3, 2, 150), (16, (1, 0, 2), 3, 1, 5), (64, (8, 12, 12), 4, 2, 77), (80, (8, 12, 10), 5, 1, 33), (128, (16, 24, 24), 32, 8, 19),
          (72, (7, 9, 9, 2), 2, 2, 65), (256, (32, 48, 48), 2, 1, 19), (192, (24, 36, 36), 1, 3, 300), (40, (20,), 3, 3, 2100), (248, (31, 31, 31, 31), 2, 2, 21)]


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("layout,ladder", [(cb.CB_PAIRS_HALVES, cb.CB_LADDER_SHARED), (cb.CB_PAIRS_ADJACENT, cb.CB_LADDER_PER_AXIS)])
@pytest.mark.parametrize("dim,pairs,hq,hk,n", SHAPES)
def test_norm_rotate_and_its_gradients(dtype, wdtype, layout, ladder, dim, pairs, hq, hk, n):
    rng = np.random.default_rng([dim, hq, n, layout])
    q, k = dev(3 * rng.standard_normal((n, hq, dim)), dtype), dev(0.2 * rng.standard_normal((n, hk, dim)), dtype)
    wq, wk = (dev(1 + 0.3 * rng.standard_normal(dim), wdtype) for _ in range(2))
    gq, gk = dev(rng.standard_normal(q.shape), dtype), dev(rng.standard_normal(k.shape), dtype)
    pos = rng.integers(-5, 2000, (n, len(pairs))).astype(np.int32)
    rot, eps = cb.Rotary(dim, pairs, layout=layout, ladder=ladder), 1e-3
    a, b = rot.norm_rotate(q, dev(pos), wq, k=k, k_weight=wk, eps=eps)
    check_norm(rot, q, wq, pos, pairs, layout, ladder, eps, a, "q")
    check_norm(rot, k, wk, pos, pairs, layout, ladder, eps, b, "k")
    assert torch.equal(a, rot.norm_rotate(q, dev(pos), wq, eps=eps))
    # gradients: the same outputs, and those of the four leaves
    leaves = [t.clone().requires_grad_() for t in (q, wq, k, wk)]
    out = rot.norm_rotate(leaves[0], dev(pos), leaves[1], k=leaves[2], k_weight=leaves[3], eps=eps)
    assert torch.equal(out[0], a) and torch.equal(out[1], b)
    got = torch.autograd.grad(out, leaves, (gq, gk))
    for x, w, g, gx, gw in ((q, wq, gq, got[0], got[1]), (k, wk, gk, got[2], got[3])):
        check_back(x, w, g, pos, pairs, layout, ladder, eps, gx, gw)


def check_back(x, w, g, pos, pairs, layout, ladder, eps, gx, gw):
    heads, tokens = x.shape[1], x.shape[0]
    want_x, want_w, n, r = norm_back64(f64(x), f64(w), f64(g), pos, pairs, layout, ladder, eps)
    size = turned_size(f64(g), pairs, layout)                     # bounds every value of the gradient turned back
    wabs = np.abs(f64(w))
    if gx is not None:
        # r is within 15 units and comes in three times at most, the sum over a head within 24, products, differences and the turn 16
        spread = r * (wabs * size + np.abs(n) * (wabs * size * np.abs(n)).mean(2, keepdims=True))
        within(f64(gx), want_x, (96 * EPS + ANGLE) * spread + ROUND[gx.dtype] * np.abs(want_x), "gradient of x")
    if gw is not None:
        # a lane adds up the heads / 4 + 3 rows that it has of a stretch, of tokens / 1024 stretches; up to 256 lanes' sums follow one by one
        terms = (2 * heads // 4 + 3) * -(-tokens // 1024) + 256 + 32
        within(f64(gw), want_w, (terms * EPS + ANGLE) * (size * np.abs(n)).sum((0, 1)) + ROUND[gw.dtype] * np.abs(want_w), "gradient of the weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1, 2, 3])
def test_norm_rotate_strided_unaligned_and_in_place(dtype, off):
    rng = np.random.default_rng([15, off])
    n, dim, pairs, eps = 37, 32, (4, 6, 4), 1e-6
    flat = dev(rng.standard_normal(n * 7 * (dim + off) + 8), dtype)
    q = flat.as_strided((n, 3, dim), (7 * (dim + off), dim + off, 1), off)
    k = flat.as_strided((n, 2, dim), (7 * (dim + off), 2 * (dim + off), 1), off + 3 * (dim + off))
    w = dev(rng.standard_normal(dim + off), F32)[off:] if off else dev(rng.standard_normal(dim), F32)
    pos = rng.integers(0, 500, (n, 3)).astype(np.int32)
    rot, before = cb.Rotary(dim, pairs), flat.clone()
    out = torch.zeros((3, n, dim), dtype=dtype, device="cuda").transpose(0, 1)
    a, b = rot.norm_rotate(q, dev(pos), w, k=k, k_weight=w, q_out=out)
    assert a is out
    check_norm(rot, q, w, pos, pairs, 0, 0, eps, a, "q")
    check_norm(rot, k, w, pos, pairs, 0, 0, eps, b, "k")
    assert torch.equal(flat, before)
    # gradients of parts of one tensor, the gradient that comes a broadcast one
    x, v = flat.clone().requires_grad_(), w.clone().requires_grad_()
    y = rot.norm_rotate(x.as_strided(q.shape, q.stride(), q.storage_offset()), dev(pos), v)
    gx, gw = torch.autograd.grad(y.sum(), (x, v))
    ones = torch.ones_like(q, memory_format=torch.contiguous_format)
    check_back(q, w, ones, pos, pairs, 0, 0, eps, gx.as_strided(q.shape, q.stride(), q.storage_offset()), gw)
    assert rot.norm_rotate(q, dev(pos), w, q_out=q) is q
    assert torch.equal(q, a)
    inside = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
    inside.as_strided(q.shape, q.stride(), q.storage_offset()).fill_(True)
    assert torch.equal(flat[~inside], before[~inside])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e-12, 1e12, 1e18, 1e30, 1e37])
def test_norm_of_very_small_and_very_large_heads(dtype, size):
    """Squares that leave float32's range."""
    rng = np.random.default_rng(5)
    n, dim, pairs = 9, 64, (8, 12, 12)
    q, g = dev(size * rng.standard_normal((n, 3, dim)), dtype), dev(rng.standard_normal((n, 3, dim)), dtype)
    w, pos, rot = dev(rng.standard_normal(dim), F32), rng.integers(0, 99, (n, 3)).astype(np.int32), cb.Rotary(dim, pairs)
    for eps in (0.0, 1e-6) if size > 1e-6 else (0.0, 1e-45):
        check_norm(rot, q, w, pos, pairs, 0, 0, eps, rot.norm_rotate(q, dev(pos), w, eps=eps), f"eps = {eps}")
    if 1e-19 < size < 1e19:                      # (the gradient of x is about 1 / size: within float32's normal range, and bfloat16's)
        x, v = q.clone().requires_grad_(), w.clone().requires_grad_()
        gx, gw = torch.autograd.grad(rot.norm_rotate(x, dev(pos), v, eps=0.0), (x, v), g)
        check_back(q, w, g, pos, pairs, 0, 0, 0.0, gx, gw)


def test_norm_of_zeros_infinities_and_nan_keeps_to_its_head():
    rng = np.random.default_rng(6)
    n, dim, pairs = 5, 64, (8, 12, 12)
    q, w, pos = rng.standard_normal((n, 4, dim)), dev(np.ones(dim), F32), dev(rng.integers(0, 99, (n, 3)).astype(np.int32))
    q[1, 2] = 0.0
    q[2, 1, 7], q[3, 3, 60], q[4, 0, 11] = np.nan, np.inf, -np.inf
    rot = cb.Rotary(dim, pairs)
    clean = dev(np.where(np.isfinite(q), q, 0.5), F32)
    got, want = rot.norm_rotate(dev(q, F32), pos, w), rot.norm_rotate(clean, pos, w)
    touched = torch.zeros((n, 4), dtype=torch.bool)
    touched[2, 1] = touched[3, 3] = touched[4, 0] = True
    assert torch.equal(got.cpu()[~touched], want.cpu()[~touched])
    assert (got[1, 2] == 0).all() and torch.isnan(got[2, 1]).all()
    for at, d in (((3, 3), 60), ((4, 0), 11)):                   # 1 / infinity is zero: zeros, and what is not a number where the infinity was
        h = got[at].cpu()
        assert torch.isnan(h[d]) and (torch.isnan(h) | (h == 0)).all()
    # a head of zeros without eps is not a number, and no other head is touched
    zero = rot.norm_rotate(dev(np.where(np.isfinite(q), q, 0.5), F32), pos, w, eps=0.0)
    assert torch.isnan(zero[1, 2]).all() and torch.isnan(zero).sum() == dim


def test_gradients_of_the_norm_against_differences():
    rng = np.random.default_rng(8)
    n, heads, dim, pairs, eps = 7, 2, 24, (3, 4, 3), 1e-2
    pos = rng.integers(0, 300, (n, 3)).astype(np.int32)
    x, g, u = (rng.standard_normal((n, heads, dim)).astype(np.float32) for _ in range(3))
    w, t = (rng.standard_normal(dim).astype(np.float32) for _ in range(2))
    for layout in (0, 1):
        rot = cb.Rotary(dim, pairs, layout=layout)
        a, b = dev(x).requires_grad_(), dev(w).requires_grad_()
        gx, gw = torch.autograd.grad(rot.norm_rotate(a, dev(pos), b, eps=eps), (a, b), dev(g))
        along = float((f64(gx) * u).sum() + (f64(gw) * t).sum())
        f = lambda h: norm64(x + h * u.astype(np.float64), w + h * t.astype(np.float64), pos, pairs, layout, 0, eps)[0]  # noqa: E731
        h = 1e-5
        diff = float(((f(h) - f(-h)) / (2 * h) * g).sum())
        # what the gradients are off by, and a difference quotient by about h^2 and 2^-53 / h times third derivatives of order 1 and values
        sizes = norm_back64(x.astype(np.float64), w, g, pos, pairs, layout, 0, eps)
        size = turned_size(g, pairs, layout)
        spread = sizes[3] * (np.abs(w) * size + np.abs(sizes[2]) * (np.abs(w) * size * np.abs(sizes[2])).mean(2, keepdims=True))
        tol = (97 * EPS + ANGLE) * (spread * np.abs(u)).sum() + (400 * EPS + ANGLE) * ((size * np.abs(sizes[2])).sum((0, 1)) * np.abs(t)).sum() + 1e-6
        assert abs(along - diff) <= tol
        # and quotients of the kernel itself, at a step that float32 resolves, against the definition's at the same step
        h = 2.0 ** -6
        kernel = lambda s: f64(rot.norm_rotate(dev((x + s * h * u).astype(np.float32)), dev(pos), dev((w + s * h * t).astype(np.float32)), eps=eps))  # noqa: E731
        mine, want = ((kernel(1) - kernel(-1)) / (2 * h) * g).sum(), ((f(h) - f(-h)) / (2 * h) * g).sum()
        largest = np.abs(f(0)) + np.abs(f(h)) + np.abs(f(-h)) + 1
        # (inputs are rounded too: a few units more)
        assert abs(mine - want) <= ((64 * EPS + ANGLE) * (turned_size(largest, pairs, layout) * np.abs(g)).sum()) / h


@pytest.mark.parametrize("which", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 0, 0, 1), (0, 1, 1, 0), (1, 1, 1, 1)])
@pytest.mark.parametrize("used", ["q", "k", "both"])
def test_gradients_that_are_asked_for(which, used):
    rng = np.random.default_rng(12)
    n, dim, pairs = 70, 48, (6, 8, 8)
    make = [dev(rng.standard_normal(s), F32) for s in ((n, 3, dim), (dim,), (n, 2, dim), (dim,))]
    pos, rot = dev(rng.integers(0, 99, (n, 3)).astype(np.int32)), cb.Rotary(dim, pairs)
    gq, gk = dev(rng.standard_normal((n, 3, dim)), F32), dev(rng.standard_normal((n, 2, dim)), F32)

    def grads(flags):
        leaves = [t.clone().requires_grad_(bool(f)) for t, f in zip(make, flags)]
        q, k = rot.norm_rotate(leaves[0], pos, leaves[1], k=leaves[2], k_weight=leaves[3])
        loss = (q * gq).sum() * (used != "k") + (k * gk).sum() * (used != "q") if used == "both" else ((q * gq).sum() if used == "q" else (k * gk).sum())
        wanted = [t for t in leaves if t.requires_grad]
        if not loss.requires_grad:
            return None
        return dict(zip([i for i, f in enumerate(flags) if f], torch.autograd.grad(loss, wanted, allow_unused=True)))

    got, want = grads(which), grads((1, 1, 1, 1))
    if got is None:
        assert (used == "q" and not (which[0] or which[1])) or (used == "k" and not (which[2] or which[3]))
        return
    for i, g in got.items():
        if g is None:
            assert want[i] is None and ((used == "q" and i >= 2) or (used == "k" and i < 2))
        elif i % 2 == 0:
            assert torch.equal(g, want[i])
        else:
            # sums over 140 - 210 heads, dealt to lanes by how many heads take part, queries' and keys': two orders of the same terms, each of which is off by
            # no more than a unit for every term from the exact sum
            x, out_grad = make[i - 1], gq if i == 1 else gk
            _, _, norms, _ = norm_back64(f64(x), f64(make[i]), f64(out_grad), pos.cpu().numpy(), pairs, 0, 0, 1e-6)
            size = (turned_size(f64(out_grad), pairs, 0) * np.abs(norms)).sum((0, 1))
            within(f64(g), f64(want[i]), 2 * 210 * EPS * size, "gradient of a weight")


def test_gradients_of_gradients_of_the_norm_are_refused():
    rot, pos = cb.Rotary(16, (8,)), torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    x, w = torch.randn((2, 1, 16), device="cuda", requires_grad=True), torch.ones(16, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(rot.norm_rotate(x, pos, w).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)


def test_gradients_of_shared_and_broadcast_inputs():
    """One weight for queries and keys, queries that are one token's repeated, the same tensor as queries and keys."""
    rng = np.random.default_rng(14)
    n, heads, dim, pairs = 40, 3, 32, (4, 6, 6)
    pos, rot = rng.integers(0, 99, (n, 3)).astype(np.int32), cb.Rotary(32, (4, 6, 6))
    one, w = dev(rng.standard_normal((1, heads, dim)), F32).requires_grad_(), dev(rng.standard_normal(dim), F32).requires_grad_()
    gq, gk = (dev(rng.standard_normal((n, heads, dim)), F32) for _ in range(2))
    x = one.expand(n, heads, dim)
    q, k = rot.norm_rotate(x, dev(pos), w, k=x, k_weight=w)
    g_one, g_w = torch.autograd.grad((q, k), (one, w), (gq, gk))
    want_x, want_w, spread_x, spread_w = 0.0, 0.0, 0.0, 0.0
    for g in (gq, gk):
        a, b, norms, r = norm_back64(f64(x), f64(w), f64(g), pos, pairs, 0, 0, 1e-6)
        size, wabs = turned_size(f64(g), pairs, 0), np.abs(f64(w))
        want_x, want_w = want_x + a, want_w + b
        spread_x = spread_x + r * (wabs * size + np.abs(norms) * (wabs * size * np.abs(norms)).mean(2, keepdims=True))
        spread_w = spread_w + (size * np.abs(norms)).sum((0, 1))
    # (every term as in check_back, and sums of 80 of them: 80 units more at most)
    within(f64(g_one), want_x.sum(0, keepdims=True), (176 * EPS + ANGLE) * spread_x.sum(0, keepdims=True), "gradient of one token's")
    within(f64(g_w), want_w, (400 * EPS + ANGLE) * spread_w, "gradient of the weight")


def test_norm_of_nothing():
    rot, pos = cb.Rotary(16, (8,)), torch.empty((0, 1), dtype=torch.int32, device="cuda")
    q, w = torch.empty((0, 3, 16), device="cuda", requires_grad=True), torch.ones(16, device="cuda", requires_grad=True)
    y = rot.norm_rotate(q, pos, w)
    gx, gw = torch.autograd.grad(y.sum(), (q, w))
    assert y.shape == gx.shape == (0, 3, 16) and (gw == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_and_gradients_do_not_vary(dtype):
    rng = np.random.default_rng(9)
    n, dim, pairs = 4100, 128, (16, 24, 24)
    q, w, g = dev(rng.standard_normal((n, 5, dim)), dtype).requires_grad_(), dev(rng.standard_normal(dim), F32).requires_grad_(), dev(rng.standard_normal((n, 5, dim)), dtype)
    pos, rot = dev(rng.integers(0, 99, (n, 3)).astype(np.int32)), cb.Rotary(dim, pairs)
    first = None
    for _ in range(4):
        y = rot.norm_rotate(q, pos, w)
        now = (y.detach(),) + torch.autograd.grad(y, (q, w), g)
        first = now if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_norm_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(10)
    n, dim, pairs = 300, 64, (8, 12, 12)
    q, w, g = dev(rng.standard_normal((n, 4, dim)), BF16).requires_grad_(), dev(rng.standard_normal(dim), F32).requires_grad_(), dev(rng.standard_normal((n, 4, dim)), BF16)
    pos, rot = dev(rng.integers(0, 99, (n, 3)).astype(np.int32)), cb.Rotary(dim, pairs)

    def step():
        y = rot.norm_rotate(q, pos, w)
        return (y.detach(),) + torch.autograd.grad(y, (q, w), g)

    want = [step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
        side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[0], got))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        with torch.no_grad():
            q.copy_(dev(rng.standard_normal(q.shape), BF16))
            w.copy_(dev(rng.standard_normal(dim), F32))
        graph.replay()
        again = [t.clone() for t in held]
        torch.cuda.synchronize()
        for a, b in zip(again, step()):
            assert torch.equal(a, b), i


def test_a_training_step_of_norms_in_a_graph():
    """forward, backward() and a step of the weights in one graph, with eager work on leaves of its own between the replays."""
    rng = np.random.default_rng(11)
    n, dim, pairs = 130, 48, (8, 4, 12)
    x, g = dev(rng.standard_normal((n, 3, dim)), BF16), dev(rng.standard_normal((n, 3, dim)), BF16)
    w = dev(1 + 0.1 * rng.standard_normal(dim), F32)
    pos, rot = dev(rng.integers(0, 99, (n, 3)).astype(np.int32)), cb.Rotary(dim, pairs)

    def step(q, w):
        q.grad = w.grad = None
        rot.norm_rotate(q, pos, w).backward(g)
        with torch.no_grad():
            w -= 0.01 * w.grad
        return q.grad, w.grad

    held, eager = ([t.clone().requires_grad_() for t in (x, w)] for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    with torch.no_grad():
        held[1].copy_(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = step(*held)
    for i in range(4):
        with torch.no_grad():
            x.copy_(dev(rng.standard_normal(x.shape), BF16))
            held[0].copy_(x)
            eager[0].copy_(x)
        graph.replay()
        again = [t.clone() for t in grads] + [held[1].detach().clone()]
        torch.cuda.synchronize()
        for a, b in zip(again, step(*eager) + (eager[1],)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("leaf", ["q", "weight", "k"])
def test_a_recorded_backward_pass_is_refused_while_another_graph_of_the_leaves_lives(leaf):
    rng = np.random.default_rng(13)
    x, w = dev(rng.standard_normal((20, 2, 16)), BF16), dev(rng.standard_normal(16), F32)
    t = (w if leaf == "weight" else x).clone().requires_grad_()
    pos, rot, g = torch.zeros((20, 1), dtype=torch.int32, device="cuda"), cb.Rotary(16, (8,)), torch.ones_like(x)

    def step():
        if leaf == "k":
            return rot.norm_rotate(x, pos, w, k=t, k_weight=w)[1]
        return rot.norm_rotate(x, pos, t) if leaf == "weight" else rot.norm_rotate(t, pos, w)

    alive = step()
    want = torch.autograd.grad(alive, t, g, retain_graph=True)[0]
    torch.cuda.synchronize()
    with pytest.raises(AssertionError, match="same leaves"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            torch.autograd.grad(step(), t, g)
    del alive
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(step(), t, g)[0]
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,pairs", [(64, (8, 12, 12)), (72, (7, 9, 9)), (256, (31,))])
def test_gradients_in_the_place_of_what_they_come_from(dtype, dim, pairs):
    """cb_norm_rotate_back where x_grad is out_grad."""
    rng = np.random.default_rng([dim, 12])
    n, heads = 90, 5
    q, w, g = dev(rng.standard_normal((n, heads, dim)), dtype).requires_grad_(), dev(rng.standard_normal(dim), F32).requires_grad_(), dev(rng.standard_normal((n, heads, dim)), dtype)
    pos, rot = dev(rng.integers(0, 99, (n, len(pairs))).astype(np.int32)), cb.Rotary(dim, pairs)
    want = torch.autograd.grad(rot.norm_rotate(q, pos, w, eps=1e-5), (q, w), g)
    L = cb.binding.lib()
    at = lambda t: cb.binding.cb_heads(t.data_ptr(), heads * dim, dim, heads, 0)      # noqa: E731
    gw, size = torch.empty_like(w), C.c_size_t()
    assert L.cb_norm_rotate_back_scratch_bytes(C.byref(rot.plan), C.byref(size)) == 0
    scratch = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    back = cb.binding.cb_norm_back(at(q), at(g), at(g), w.data_ptr(), gw.data_ptr())
    assert L.cb_norm_rotate_back(C.byref(rot.plan), 1 if dtype == BF16 else 0, n, pos.data_ptr(), 1e-5, 0, C.byref(back), None, scratch.data_ptr(), size.value,
                                 torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(g, want[0]) and torch.equal(gw, want[1])


def test_what_norm_rotate_refuses():
    rot = cb.Rotary(16, (8,))
    x, w = torch.zeros((2, 3, 16), device="cuda"), torch.ones(16, device="cuda")
    pos = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    for call in (lambda: rot.norm_rotate(x.half(), pos, w), lambda: rot.norm_rotate(x, pos, w.half()), lambda: rot.norm_rotate(x, pos, w[:8]),
                 lambda: rot.norm_rotate(x, pos, torch.ones(32, device="cuda")[::2]), lambda: rot.norm_rotate(x, pos.long(), w),
                 lambda: rot.norm_rotate(x, pos[:1], w), lambda: rot.norm_rotate(x[..., :8], pos, w), lambda: rot.norm_rotate(x, pos, w, k=x),
                 lambda: rot.norm_rotate(x, pos, w, k_weight=w), lambda: rot.norm_rotate(x, pos, w, k=x.bfloat16(), k_weight=w),
                 lambda: rot.norm_rotate(x, pos, w, k=x, k_weight=w.bfloat16()), lambda: rot.norm_rotate(x, pos, w, k_out=x),
                 lambda: rot.norm_rotate(x, pos, w, k=x[:1], k_weight=w), lambda: rot.norm_rotate(x, pos, w.cpu()),
                 lambda: rot.norm_rotate(x.clone().requires_grad_(), pos, w, q_out=x)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(cb.binding.CBError if hasattr(cb, "binding") else RuntimeError):
        rot.norm_rotate(x, pos, w, eps=-1.0)


# ---------------------------------------------------------------- caches in 8 bits
def codes64(pages):
    return pages.cpu().view(torch.uint8).view(E4M3).double().numpy()


def held64(c, which):
    """Keys or values of all pages, float64."""
    pages, scale = getattr(c, which + "_pages"), getattr(c, which + "_scale")
    return f64(pages) if scale is None else codes64(pages) * np.repeat(f64(scale), 16, 2)[..., None]


def make_bytes(rng, lengths, heads, dim, page, capacity=None, spare=3, powers=True, bounded=False, weight=False):
    """A cache in 8 bits whose pages lie in no order; slots that hold no token, and scales of blocks without one, are not numbers."""
    pages = [-(-x // page) for x in lengths]
    width = max(1, max(pages)) if capacity is None else -(-capacity // page)
    own = [width if capacity is not None else p for p in pages]
    n_pages = sum(own) + spare
    order = rng.permutation(n_pages).tolist()
    table = np.full((len(lengths), width), -1, np.int32)
    code = {x: np.full((n_pages, heads, page, dim), 0x7F, np.uint8) for x in "kv"}
    scale = {x: np.full((n_pages, heads, page // 16), np.nan, np.float32) for x in "kv"}
    for s, n in enumerate(lengths):
        table[s, :own[s]], order = order[:own[s]], order[own[s]:]
        for x in "kv":
            for p in range(-(-n // page)):
                m = min(page, n - p * page)
                some = rng.integers(0, 0x78, (heads, m, dim)).astype(np.uint8) | (rng.integers(0, 2, (heads, m, dim)) << 7).astype(np.uint8)
                code[x][table[s, p], :, :m] = some                       # (up to 240: all that 8 bits hold but the largest, subnormal ones among them)
                b = -(-m // 16)
                scale[x][table[s, p], :, :b] = 2.0 ** rng.integers(-9, -5, (heads, b)) if powers else 0.01 * (0.3 + rng.random((heads, b)))
    cap = width * page
    tensors = {x: dev(code[x]).view(E4M3) for x in "kv"}
    bounds = torch.zeros((n_pages, heads, 2, dim), dtype=BF16, device="cuda") if bounded else None
    return cb.TokenCache(tensors["k"], tensors["v"], dev(table), dev(np.array(lengths, np.int32)),
                         dev(rng.random((len(lengths), heads, cap)).astype(np.float32)) if weight else None,
                         k_scale=dev(scale["k"]), v_scale=dev(scale["v"]), bounds=bounds)


def wide(c):
    """The cache as one that holds its values in 64 bits, for attend64 (which leaves out the slots without a page by itself)."""
    table = torch.where((c.table >= 0) & (c.table < c.k_pages.shape[0]), c.table, 0)
    return types.SimpleNamespace(k_pages=torch.from_numpy(held64(c, "k")), v_pages=torch.from_numpy(held64(c, "v")), table=table, weight=c.weight,
                                 n_kv_heads=c.n_kv_heads, head_dim=c.head_dim)


def check_attend_bytes(c, q, lengths, softcap=0.0, scale=None, accumulate=False, decay=1.0, dead=(), **kw):
    want = attend64(wide(c), q, lengths, c.head_dim ** -0.5 if scale is None else scale, softcap, decay if accumulate else None, dead)
    out, lse = c.attend(q, softcap=softcap, scale=scale, accumulate=accumulate, decay=decay, **kw)
    within(f64(out), want[0], want[3], "out")
    got = f64(lse)
    assert np.array_equal(np.isneginf(got), np.isneginf(want[1]))
    fine = np.isfinite(want[1])
    within(got[fine], want[1][fine], want[4][fine], "lse")
    if accumulate:
        within(f64(c.weight), want[2], want[5], "weight")
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page,heads,group,dim", [(16, 2, 1, 64), (32, 1, 4, 128), (64, 3, 3, 80), (128, 1, 17, 32), (16, 4, 16, 256), (1024, 1, 2, 16)])
@pytest.mark.parametrize("powers", [True, False])
def test_attend_in_8_bits_at_the_edges_of_tiles_and_pages(dtype, page, heads, group, dim, powers):
    lengths = [0, 1, 15, 16, 17, 31, 32, 33, 63, 65, 127, 129, page, page + 1, 2 * page - 1, 300]
    rng = np.random.default_rng([page, heads, dim])
    c = make_bytes(rng, lengths, heads, dim, page, powers=powers)
    check_attend_bytes(c, dev(2 * rng.standard_normal((len(lengths), heads * group, dim)), dtype), lengths)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [16, 48, 64, 96, 112, 128, 144, 192, 240, 256])
def test_attend_in_8_bits_head_sizes(dtype, dim):
    rng = np.random.default_rng(dim)
    lengths = [700, 3, 65]
    c = make_bytes(rng, lengths, 2, dim, 32, weight=True)
    check_attend_bytes(c, dev(2 * rng.standard_normal((3, 10, dim)), dtype), lengths, softcap=5.0, accumulate=True, decay=0.9)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,heads,group,page,dim", [([20011], 1, 4, 128, 128), ([9001, 1, 0, 5000], 4, 3, 32, 80), ([4097] * 3, 8, 1, 16, 64)])
def test_attend_in_8_bits_split_over_the_length(dtype, lengths, heads, group, page, dim):
    rng = np.random.default_rng([heads, page])
    c = make_bytes(rng, lengths, heads, dim, page)
    q = dev(2 * rng.standard_normal((len(lengths), heads * group, dim)), dtype)
    out = check_attend_bytes(c, q, lengths)
    assert torch.equal(out, c.attend(q)[0])                      # and does not vary


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attend_in_8_bits_without_pages_and_with_nan(dtype):
    rng = np.random.default_rng(21)
    lengths = [200, 150, 40]
    c = make_bytes(rng, lengths, 2, 64, 32)
    q = dev(rng.standard_normal((3, 4, 64)), dtype)
    c.table[0, 2], c.table[1, 0], c.table[1, 4] = -1, 1 << 30, c.k_pages.shape[0]
    dead = {(0, 2), (1, 0), (1, 4)}
    check_attend_bytes(c, q, lengths, dead=dead)
    # a value that is not a number is one of its place alone
    page, row = int(c.table[2, 1]), 3
    raw = c.v_pages.view(torch.uint8)
    raw[page, 1, row, 5] = 0x7F
    out, _ = c.attend(q)
    bad = torch.isnan(out)
    assert bad[2, 2:, 5].all() and bad.sum() == 2


@pytest.mark.parametrize("size", [1e30, 3e38, 1e-30])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_8_bits_hold_very_large_and_very_small_values(dtype, size):
    rng = np.random.default_rng(31)
    c = cb.TokenCache.create(1, 1, 32, 64, dtype=E4M3, page_tokens=16)
    v = dev(np.clip(size * rng.standard_normal((1, 1, 32)), -3e38, 3e38), dtype)
    k = torch.zeros_like(v)
    c.append(k, v)
    out, lse = c.attend(torch.ones((1, 1, 32), dtype=dtype, device="cuda"))
    want = held64(c, "v")[int(c.table[0, 0]), 0, 0]
    assert float(lse) == 0.0
    within(f64(out)[0, 0], want, (16 * EPS + ROUND[dtype]) * np.abs(want) + 1e-38, "one token")
    if size > 1:
        within(want, f64(v)[0, 0], 2.0 ** -4 * np.abs(f64(v)[0, 0]) + 2.0 ** -10 * float(c.v_scale[int(c.table[0, 0]), 0, 0]), "held")


def scale64(top):
    """The smallest power of two, 2^-64 .. 2^120, of which 448 times reaches top."""
    e = -64
    while e < 120 and 448.0 * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def bytes_append64(c, k, v, starts, ends):
    """What an append leaves: codes and scales, k and v as they are rounded (float64)."""
    out = {x + "_pages": c_clone(getattr(c, x + "_pages")) for x in "kv"}
    out.update({x + "_scale": f64(getattr(c, x + "_scale")) for x in "kv"})
    table, page = c.table.cpu().numpy(), c.k_pages.shape[2]
    for s, start in enumerate(starts):
        n = ends[s + 1] - ends[s]
        for b in range(start // 16, -(-(start + n) // 16) if n > 0 else start // 16):
            if b * 16 >= c.capacity or not 0 <= table[s, b * 16 // page] < c.k_pages.shape[0]:
                continue
            p, r0 = table[s, b * 16 // page], b * 16 % page
            new = [j for j in range(16) if start <= 16 * b + j < start + n]
            old = [j for j in range(16) if 16 * b + j < start]
            for name, x in (("k", k), ("v", v)):
                rows_ = x[[ends[s] + 16 * b + j - start for j in new]]
                for h in range(c.n_kv_heads):
                    y = rows_[:, h]
                    top = np.abs(np.where(np.isfinite(y), y, 0)).max()
                    was = out[name + "_scale"][p, h, r0 // 16]
                    now = max(scale64(top), was) if old else scale64(top)
                    out[name + "_scale"][p, h, r0 // 16] = now
                    pages = out[name + "_pages"]
                    if old and now != was:
                        held = pages[p, h, [r0 + j for j in old]].double() * was
                        pages[p, h, [r0 + j for j in old]] = rounded(held.numpy() / now)
                    pages[p, h, [r0 + j for j in new]] = rounded(y / now)
    return out


def c_clone(pages):
    return pages.cpu().view(torch.uint8).clone().view(E4M3)


def rounded(x):
    """The nearest that 8 bits hold (x is exact in float32)."""
    t = torch.from_numpy(np.ascontiguousarray(x)).float()
    return torch.where(torch.isnan(t), t, t.clamp(-448, 448)).to(E4M3)


def same_codes(got, want, what):
    a, b = got.cpu().view(torch.uint8).numpy(), want.view(torch.uint8).numpy()
    nan = (a & 0x7F) == 0x7F
    assert np.array_equal(nan, (b & 0x7F) == 0x7F), what
    assert np.array_equal(a[~nan], b[~nan]), (what, np.argwhere((a != b) & ~nan)[:3])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,heads,page", [(64, 2, 16), (128, 8, 64), (80, 3, 32), (16, 1, 128), (256, 2, 16), (208, 1, 64)])
@pytest.mark.parametrize("given", [False, True])
def test_append_in_8_bits(dtype, dim, heads, page, given):
    rng = np.random.default_rng([dim, page, given])
    held, new = [0, 1, 15, 16, 33, 200, 47, 0, 5], [40, 16, 1, 3, 0, 31, 33, 1, 100]
    c = make_bytes(rng, held, heads, dim, page, capacity=320)
    ends = np.concatenate([[0], np.cumsum(new)])
    n = int(ends[-1]) + 5                                          # rows of nobody behind the last sequence's
    size = np.exp(2 * rng.standard_normal((n, 2 * heads, 1)))
    kv = dev(rng.standard_normal((n, 2 * heads, dim)) * size, dtype)
    kv[3, 0, 2], kv[50, heads, 5], kv[60, 1 if heads > 1 else 0, 1], kv[70] = math.inf, -math.inf, math.nan, 0.0
    k, v = kv[:, :heads], kv[:, heads:]
    want = bytes_append64(c, f64(k), f64(v), held, ends)
    start = dev(np.array(held, np.int32)) if given else None
    if given:
        c.lengths.fill_(7)
    c.append(k, v, offsets=dev(ends.astype(np.int32)), start=start)
    for x in "kv":
        same_codes(getattr(c, x + "_pages"), want[x + "_pages"], x)
        assert np.array_equal(f64(getattr(c, x + "_scale")), want[x + "_scale"], equal_nan=True), x
    assert c.lengths.tolist() == [a + b for a, b in zip(held, new)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [0, 1, 2])
def test_append_in_8_bits_one_token_at_a_time(dtype, off):
    """Forty steps of one row a sequence, each louder or quieter than the one before: what was there is rounded again where the scale grows."""
    rng = np.random.default_rng(41)
    seqs, heads, dim = 3, 2, 48
    c = make_bytes(rng, [0, 9, 30], heads, dim, 32, capacity=96)
    at = [0, 9, 30]
    for i in range(40):
        flat = dev(rng.standard_normal(seqs * 2 * heads * (dim + off) + 2) * 2.0 ** rng.integers(-6, 7), dtype)
        k = flat.as_strided((seqs, heads, dim), (2 * heads * (dim + off), dim + off, 1), off)
        v = flat.as_strided((seqs, heads, dim), (2 * heads * (dim + off), dim + off, 1), off + heads * (dim + off))
        want = bytes_append64(c, f64(k), f64(v), at, [0, 1, 2, 3])
        c.append(k, v)
        for x in "kv":
            same_codes(getattr(c, x + "_pages"), want[x + "_pages"], (i, x))
            assert np.array_equal(f64(getattr(c, x + "_scale")), want[x + "_scale"], equal_nan=True)
        at = [x + 1 for x in at]
    assert c.lengths.tolist() == at


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [cb.CB_PAIRS_HALVES, cb.CB_PAIRS_ADJACENT])
@pytest.mark.parametrize("dim,pairs", [(64, (8, 12, 12)), (128, (16, 24, 24)), (80, (8, 12, 10)), (256, (10, 3, 7))])
def test_append_in_8_bits_with_rotation(dtype, layout, dim, pairs):
    rng = np.random.default_rng([dim, layout])
    heads, hq, held, new = 2, 4, [5, 0, 100], [50, 17, 1]
    ends = np.concatenate([[0], np.cumsum(new)])
    n = int(ends[-1]) + 3
    c = make_bytes(rng, held, heads, dim, 32, capacity=128, weight=True)
    time = torch.full((3, heads, c.capacity), -9, dtype=torch.int32, device="cuda")
    c = cb.TokenCache(c.k_pages, c.v_pages, c.table, c.lengths, c.weight, time, k_scale=c.k_scale, v_scale=c.v_scale)
    k, v, q = (dev(rng.standard_normal((n, h, dim)), dtype) for h in (heads, heads, hq))
    pos = rng.integers(0, 900, (n, len(pairs))).astype(np.int32)
    rot = cb.Rotary(dim, pairs, layout=layout)
    q_out = torch.full_like(q, 77.0)
    weight = f64(c.weight)
    before = c_clone(c.k_pages)
    c.append(k, v, dev(pos), rotary=rot, q=q, offsets=dev(ends.astype(np.int32)), q_out=q_out)
    assert (q_out[int(ends[-1]):] == 77.0).all()
    assert torch.equal(q_out[:int(ends[-1])], rot.rotate(q, dev(pos))[:int(ends[-1])])
    turned = turned64(f64(k), pos, pairs, 10000.0, layout, 0)
    off = (8 * EPS + ANGLE) * turned_size(f64(k), pairs, layout)
    got, table = held64(c, "k"), c.table.cpu().numpy()
    scale = f64(c.k_scale)
    touched = np.zeros(got.shape[:3], bool)
    for s in range(3):
        for j in range(new[s]):
            slot, row = held[s] + j, int(ends[s]) + j
            p, r = table[s, slot // 32], slot % 32
            touched[p, :, r] = True
            for h in range(heads):
                step = scale[p, h, r // 16]
                want = turned[row, h]
                tol = off[row, h] + np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step)
                within(got[p, h, r], want, tol, (s, j, h))
                assert step == 2.0 ** round(math.log2(step)) and 448 * step >= np.abs(want).max() - off[row, h].max()
    # scales are no larger than they have to be, where a block holds new tokens alone
    p = table[1, 0]
    for h in range(heads):
        top, most = np.abs(turned[ends[1]:ends[1] + 16, h]).max(), off[ends[1]:ends[1] + 16, h].max()
        assert scale64(top - most) <= scale[p, h, 0] <= scale64(top + most)
    for s in range(3):
        for j in range(new[s]):
            assert (time[s, :, held[s] + j] == int(pos[ends[s] + j, 0])).all()
            weight[s, :, held[s] + j] = 0.0
    assert np.array_equal(f64(c.weight), weight)
    untouched = ~torch.from_numpy(touched)
    slots = torch.zeros(touched.shape, dtype=torch.bool)                 # blocks of the tokens that were there may be rounded again
    for s in range(3):
        for j in range(held[s] // 16 * 16, held[s]):
            slots[table[s, j // 32], :, j % 32] = True
    stays = untouched & ~slots
    assert torch.equal(c.k_pages.cpu().view(torch.uint8)[stays], before.view(torch.uint8)[stays])


def test_append_in_8_bits_over_tokens_that_are_there():
    """From slots in front of the last token on: those behind the new ones stay as they are held, the lengths end with the new ones."""
    rng = np.random.default_rng(55)
    heads, dim, held, start, new = 2, 64, [100, 40, 33], [37, 0, 32], [20, 16, 1]
    ends = np.concatenate([[0], np.cumsum(new)])
    c = make_bytes(rng, held, heads, dim, 32, capacity=128)
    kv = dev(3 * rng.standard_normal((int(ends[-1]), 2 * heads, dim)), BF16)
    want = bytes_append64(c, f64(kv[:, :heads]), f64(kv[:, heads:]), start, ends)
    c.append(kv[:, :heads], kv[:, heads:], offsets=dev(ends.astype(np.int32)), start=dev(np.array(start, np.int32)))
    for x in "kv":
        same_codes(getattr(c, x + "_pages"), want[x + "_pages"], x)
        assert np.array_equal(f64(getattr(c, x + "_scale")), want[x + "_scale"], equal_nan=True)
    lengths = [a + b for a, b in zip(start, new)]
    assert c.lengths.tolist() == lengths
    check_attend_bytes(c, dev(rng.standard_normal((3, 4, dim)), BF16), lengths)


def test_append_in_8_bits_beyond_the_capacity_and_without_a_page():
    rng = np.random.default_rng(51)
    heads, dim = 2, 32
    held, new = [60, 10, 20], [30, 40, 5]
    ends = np.concatenate([[0], np.cumsum(new)])
    c = make_bytes(rng, held, heads, dim, 16, capacity=64)
    c.table[1, 1], c.table[2, 1] = -1, 1 << 28
    kv = dev(rng.standard_normal((int(ends[-1]), 2 * heads, dim)), F32)
    want = bytes_append64(c, f64(kv[:, :heads]), f64(kv[:, heads:]), held, ends)
    c.append(kv[:, :heads], kv[:, heads:], offsets=dev(ends.astype(np.int32)))
    for x in "kv":
        same_codes(getattr(c, x + "_pages"), want[x + "_pages"], x)
        assert np.array_equal(f64(getattr(c, x + "_scale")), want[x + "_scale"], equal_nan=True)
    assert c.lengths.tolist() == [64, 50, 25]


@pytest.mark.parametrize("n_seq", [1, 70, 300])
def test_append_in_8_bits_in_a_graph(n_seq):
    """Behind the tokens that are there, replayed: lengths grow on the device alone (by the last workgroup, or by a launch of its own)."""
    rng = np.random.default_rng(n_seq)
    heads, dim = 2, 64
    make = lambda: cb.TokenCache.create(n_seq, heads, dim, 64, dtype=E4M3, page_tokens=16)  # noqa: E731
    a, b = make(), make()
    k, v = (torch.zeros((n_seq, heads, dim), dtype=BF16, device="cuda") for _ in range(2))
    a.append(k, v)
    a.lengths.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.append(k, v)
    for i in range(5):
        k.copy_(dev(rng.standard_normal(k.shape), BF16))
        v.copy_(dev(rng.standard_normal(k.shape) * 4.0 ** i, BF16))
        graph.replay()
        torch.cuda.synchronize()
        b.append(k, v)
        assert torch.equal(a.lengths, b.lengths) and int(a.lengths[-1]) == i + 1
        for name in ("k_pages", "v_pages"):
            assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8))
        assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)


def test_what_caches_in_8_bits_refuse():
    c = cb.TokenCache.create(2, 2, 32, 64, dtype=E4M3, page_tokens=16)
    x = torch.zeros((2, 2, 32), device="cuda")
    p, s = c.k_pages, c.k_scale
    for call in (lambda: c.append(x, x.bfloat16()), lambda: c.append(x.half(), x.half()), lambda: c.attend(x.half()), lambda: c.append(x.to(E4M3), x.to(E4M3)),
                 lambda: cb.TokenCache(p, p, c.table, c.lengths), lambda: cb.TokenCache(p, p, c.table, c.lengths, k_scale=s),
                 lambda: cb.TokenCache(p, p, c.table, c.lengths, k_scale=s[:1], v_scale=s), lambda: cb.TokenCache(p, p, c.table, c.lengths, k_scale=s.double(), v_scale=s),
                 lambda: cb.TokenCache(p.float(), p.float(), c.table, c.lengths, k_scale=s, v_scale=s),
                 lambda: cb.TokenCache(p, p, c.table, c.lengths, k_scale=s, v_scale=s, bounds=torch.zeros(p.shape[:2] + (2, 32), device="cuda")),
                 lambda: c.attend(x.clone().requires_grad_()), lambda: c.append(x.clone().requires_grad_(), x)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: c.evict(4), lambda: c.bound(), lambda: c.choose(x, 4), lambda: cb.TokenCache.create(1, 1, 24, 64, dtype=E4M3)):
        with pytest.raises(RuntimeError):
            call()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pages_in_8_bits_beyond_4_gb(dtype):
    """Pages whose values lie behind 2^32 bytes: append, bounds, choice and attention find them."""
    heads, dim, page = 4, 128, 1024
    n_pages = (1 << 32) // (heads * dim * page) + 40
    pages = [torch.zeros((n_pages, heads, page, dim), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scale = [torch.ones((n_pages, heads, page // 16), device="cuda") for _ in range(2)]
    bounds = torch.zeros((n_pages, heads, 2, dim), dtype=BF16, device="cuda")
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7]], dtype=torch.int32, device="cuda")
    c = cb.TokenCache(*pages, table, torch.zeros(1, dtype=torch.int32, device="cuda"), k_scale=scale[0], v_scale=scale[1], bounds=bounds)
    rng = np.random.default_rng(61)
    n = 2 * page + 100
    k, v = (dev(rng.standard_normal((n, heads, dim)), dtype) for _ in range(2))
    c.append(k, v, offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    c.bound()
    q = dev(rng.standard_normal((1, 2 * heads, dim)), dtype)
    small = c.table[0].long()
    near = cb.TokenCache(*(p.view(torch.uint8)[small].view(E4M3) for p in pages), torch.arange(3, dtype=torch.int32, device="cuda")[None], c.lengths,
                         k_scale=scale[0][small], v_scale=scale[1][small], bounds=torch.zeros((3, heads, 2, dim), dtype=BF16, device="cuda"))
    near.bound()
    assert torch.equal(near.bounds, bounds[small])
    assert float((near.k_pages.float() != 0).float().mean()) > 0.6
    for a, b in zip(c.attend(q), near.attend(q)):
        assert torch.equal(a, b)
    picks = c.choose(q, 2, recent=1), near.choose(q, 2, recent=1)
    assert torch.equal(picks[0][0], picks[1][0])
    for a, b in zip(c.attend(q, chosen=picks[0]), near.attend(q, chosen=picks[1])):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- bounds and choice
def bounds64(c, lengths, since):
    """The bounds of the pages from since on, as float64 of what the array holds; None where they stay."""
    keys, table, page = held64(c, "k"), c.table.cpu().numpy(), c.k_pages.shape[2]
    out = {}
    for s, n in enumerate(lengths):
        for p in range(min(max(since[s], 0), c.capacity) // page, -(-n // page)):
            if 0 <= table[s, p] < keys.shape[0]:
                x = keys[table[s, p], :, :n - p * page]
                out[int(table[s, p])] = np.stack([x.min(1), x.max(1)], 1)
    return out


def with_bounds(rng, kind, lengths, heads, dim, page, **kw):
    """A cache of that kind ("f32", "bf16", "e4m3" or "odd": e4m3 with scales that are no powers of two), its bounds not numbers."""
    if kind in ("e4m3", "odd"):
        c = make_bytes(rng, lengths, heads, dim, page, powers=kind == "e4m3", **kw)
        return cb.TokenCache(c.k_pages, c.v_pages, c.table, c.lengths, k_scale=c.k_scale, v_scale=c.v_scale,
                             bounds=torch.full((c.k_pages.shape[0], heads, 2, dim), math.nan, dtype=BF16, device="cuda"))
    dtype = F32 if kind == "f32" else BF16
    c = make_cache(rng, lengths, heads, dim, page, dtype, evictable=False, **kw)
    return cb.TokenCache(c.k_pages, c.v_pages, c.table, c.lengths, bounds=torch.full((c.k_pages.shape[0], heads, 2, dim), math.nan, dtype=dtype, device="cuda"))


KINDS = ["f32", "bf16", "e4m3", "odd"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,dim,page", [(2, 64, 16), (3, 80, 32), (1, 256, 64), (8, 128, 128), (2, 16, 1024), (2, 8, 16), (1, 248, 32), (3, 72, 16),
                                            (2, 136, 32), (1, 144, 64), (2, 152, 16), (1, 160, 16), (1, 120, 32)])
def test_bounds(kind, heads, dim, page):
    if dim % 16 and kind in ("e4m3", "odd"):
        pytest.skip("heads of 8 bits are multiples of 16")
    rng = np.random.default_rng([dim, page])
    lengths = [0, 1, 15, 16, 17, page, page + 1, 3 * page - 1, 500]
    c = with_bounds(rng, kind, lengths, heads, dim, page)
    c.table[8, 0] = -1
    for since in (None, [0, 0, 20, 3, 16, page - 1, page, 2 * page, -5], [9] * 8 + [1 << 30]):
        c.bounds.fill_(math.nan)
        c.bound(None if since is None else dev(np.array(since, np.int32)))
        want, got = bounds64(c, lengths, [0] * 9 if since is None else since), f64(c.bounds)
        for p in range(got.shape[0]):
            if p not in want:
                assert np.isnan(got[p]).all()
            elif kind != "odd":
                assert np.array_equal(got[p], want[p]), p
            else:                                                        # outwards, by less than a step of bfloat16 (and a rounding of the product)
                lo, hi = want[p][:, 0], want[p][:, 1]
                slack = EPS * np.abs(want[p])
                assert (got[p][:, 0] <= lo + slack[:, 0]).all() and (got[p][:, 1] >= hi - slack[:, 1]).all()
                assert (np.abs(got[p] - want[p]) <= (2.0 ** -7 + 2 * EPS) * np.abs(want[p])).all()


def test_bounds_of_keys_that_are_not_numbers():
    c = cb.TokenCache.create(1, 1, 16, 64, dtype=BF16, page_tokens=16, bounded=True, evictable=False)
    k = torch.randn((40, 1, 16), device="cuda").to(BF16)
    k[5, 0, 3], k[20, 0, 1], k[21, 0, 2] = math.nan, math.inf, -math.inf
    c.append(k, k, offsets=torch.tensor([0, 40], dtype=torch.int32, device="cuda"))
    c.bound()
    b = c.bounds.float().cpu()
    assert torch.isnan(b[0, 0, :, 3]).all() and torch.isnan(b).sum() == 2
    assert b[1, 0, 1, 1] == math.inf and b[1, 0, 0, 2] == -math.inf
    # such a page is not ruled out by anything
    chosen, count = c.choose(torch.ones((1, 1, 16), dtype=BF16, device="cuda"), 1)
    assert chosen.tolist() == [[[0]]] and count.tolist() == [[1]]


def choose64(c, q, lengths, budget, first, recent):
    page, group = c.k_pages.shape[2], q.shape[1] // c.n_kv_heads
    bounds, table, q = f64(c.bounds), c.table.cpu().numpy(), f64(q)
    out = []
    for s, n in enumerate(lengths):
        total = -(-n // page)
        for h in range(c.n_kv_heads):
            score = np.full(total, -np.inf)
            for p in range(total):
                if 0 <= table[s, p] < bounds.shape[0]:
                    lo, hi = bounds[table[s, p], h]
                    score[p] = np.float32(max((np.where(x >= 0, hi, lo) * x).sum() for x in q[s, h * group:(h + 1) * group]))
            rank = np.where((np.arange(total) < first) | (np.arange(total) >= total - recent), np.inf, score)
            out.append(np.sort(np.argsort(-rank, kind="stable")[:budget]))
    return out


def check_choose(c, q, lengths, budget, first, recent):
    chosen, count = c.choose(q, budget, first=first, recent=recent)
    got, n = chosen.cpu().numpy(), count.cpu().numpy()
    for i, want in enumerate(choose64(c, q, lengths, budget, first, recent)):
        s, h = divmod(i, c.n_kv_heads)
        assert n[s, h] == len(want) and np.array_equal(got[s, h, :len(want)], want), (s, h)
        assert (got[s, h, len(want):] == -1).all()
    return chosen, count


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,group,dim,page,budget,first,recent", [(2, 1, 64, 16, 8, 1, 2), (1, 4, 128, 64, 3, 0, 0), (3, 5, 80, 16, 33, 2, 4), (2, 17, 16, 32, 4, 2, 2),
                                                                      (1, 2, 256, 16, 1, 0, 0), (4, 3, 48, 16, 1000, 1, 1), (2, 2, 8, 16, 5, 0, 1),
                                                                      (1, 6, 248, 32, 7, 1, 0), (2, 9, 72, 16, 12, 0, 3), (2, 2, 136, 16, 5, 0, 1),
                                                                      (1, 3, 152, 32, 4, 1, 1)])
def test_choose(kind, heads, group, dim, page, budget, first, recent):
    if dim % 16 and kind in ("e4m3", "odd"):
        pytest.skip("heads of 8 bits are multiples of 16")
    rng = np.random.default_rng([dim, budget])
    lengths = [0, 1, 16 * budget if budget < 100 else 64, 700, 2000, 1311, page, 5 * page + 1]
    c = with_bounds(rng, kind, lengths, heads, dim, page)
    c.bound()
    q = dev(rng.standard_normal((len(lengths), heads * group, dim)), F32 if kind in ("f32", "odd") else BF16)
    check_choose(c, q, lengths, budget, first, recent)


@pytest.mark.parametrize("n,budget", [(40000, 1), (40000, 777), (300000, 5), (300000, 18000)])
def test_choose_of_many_pages(n, budget):
    """More pages than the ranks' LDS has room for, in one sequence (300 000 tokens in pages of 16: 18 750)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + budget)
    pages, dim = n // 16, 16
    k = torch.zeros((pages, 1, 16, dim), dtype=BF16, device="cuda")
    bounds = torch.randn((pages, 1, 2, dim), generator=g, device="cuda").sort(2).values.to(BF16)
    c = cb.TokenCache(k, k, torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None], torch.tensor([n], dtype=torch.int32, device="cuda"), bounds=bounds)
    check_choose(c, torch.randn((1, 2, dim), generator=g, device="cuda").to(BF16), [n], budget, 1 if budget > 1 else 0, 2 if budget > 3 else 0)


@pytest.mark.parametrize("values", [1, 2, 3])
def test_choose_ties_go_to_the_lowest(values):
    rng = np.random.default_rng(values)
    n, page, dim = 5000, 16, 16
    pages = -(-n // page)
    k = torch.zeros((pages, 2, page, dim), device="cuda")
    bounds = dev(rng.integers(0, values, (pages, 2, 1, 1)).astype(np.float32)).expand(-1, -1, 2, dim).contiguous()
    c = cb.TokenCache(k, k, torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"), bounds=bounds)
    for budget, first, recent in ((7, 0, 0), (100, 3, 4), (300, 10, 0), (5, 2, 3), (pages, 0, 0), (pages - 1, 0, 0)):
        for sign in (1.0, -1.0, 0.0):
            check_choose(c, torch.full((1, 2, dim), sign, device="cuda"), [n], budget, first, recent)


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("seqs,heads", [(70, 3), (700, 8)])
def test_choose_of_many_sequences(kind, seqs, heads):
    """More sequences than a wavefront has lanes, more (sequence, key head) pairs than there are counters; sequences read the same pages."""
    rng = np.random.default_rng([seqs, heads])
    pages, page, dim = 300, 16, 16
    lengths = rng.integers(0, pages * page + 1, seqs)
    lengths[:5] = [0, 1, 16 * 20, 16 * 20 + 1, pages * page]
    one = make_bytes(rng, [pages * page], heads, dim, page) if kind == "e4m3" else make_cache(rng, [pages * page], heads, dim, page, F32 if kind == "f32" else BF16, evictable=False)
    dtype = one.bounds.dtype if one.bounds is not None else (BF16 if kind == "e4m3" else one.dtype)
    bounds = torch.sort(dev(rng.standard_normal((one.k_pages.shape[0], heads, 2, dim)), dtype), 2).values
    tables = np.stack([one.table.cpu().numpy()[0][rng.permutation(pages)] for _ in range(seqs)])
    c = cb.TokenCache(one.k_pages, one.v_pages, dev(tables), dev(lengths.astype(np.int32)), k_scale=one.k_scale, v_scale=one.v_scale, bounds=bounds)
    q = dev(rng.standard_normal((seqs, 2 * heads, dim)), F32 if kind == "f32" else BF16)
    pick = check_choose(c, q, lengths.tolist(), 20, 1, 2)
    if seqs < 100:
        check_chosen(c, q, lengths.tolist(), pick)
        want = [c.attend(q)[0][s] for s in (3, 4, 69)]
        small = cb.TokenCache(one.k_pages, one.v_pages, dev(tables[[3, 4, 69]]), dev(lengths[[3, 4, 69]].astype(np.int32)), k_scale=one.k_scale, v_scale=one.v_scale)
        got = small.attend(q[[3, 4, 69]].contiguous())[0]
        within(f64(got), f64(torch.stack(want)), 64 * EPS + 2 * ROUND[q.dtype] * np.abs(f64(got)), "the same sequences among others")
        since = dev(np.maximum(lengths - 30, 0).astype(np.int32))
        alone = cb.TokenCache(one.k_pages, one.v_pages, dev(one.table.cpu().numpy()), dev(np.array([pages * page], np.int32)), k_scale=one.k_scale, v_scale=one.v_scale, bounds=torch.zeros_like(bounds))
        alone.bound()
        full = dev(np.full(seqs, pages * page, np.int32))
        c.lengths.copy_(full)                                    # (whole pages: whichever sequence writes a page's bounds writes the same)
        c.bound(torch.minimum(since, full))
        touched = torch.zeros(bounds.shape[0], dtype=torch.bool)
        for s in range(seqs):
            touched[tables[s, int(since[s]) // page:]] = True
        assert torch.equal(c.bounds.cpu()[touched], alone.bounds.cpu()[touched])


def test_choose_scores_far_apart_and_without_pages():
    rng = np.random.default_rng(71)
    n, page, dim = 3000, 16, 32
    pages = -(-n // page)
    k = torch.zeros((pages, 1, page, dim), device="cuda")
    size = 10.0 ** rng.integers(-30, 31, (pages, 1, 1, 1))
    bounds = dev((np.sort(rng.standard_normal((pages, 1, 2, dim)), 2) * size).astype(np.float32))
    c = cb.TokenCache(k, k, torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"), bounds=bounds)
    q = dev(rng.standard_normal((1, 3, dim)), F32)
    check_choose(c, q, [n], 20, 0, 1)
    c.table[0, 10:180] = -1
    check_choose(c, q, [n], 20, 0, 1)
    check_choose(c, q, [n], 40, 0, 1)                              # more than there are pages with a number
    for bad in (-4, 0, n + 1, 1 << 30):
        c.lengths.fill_(bad)
        check_choose(c, q, [min(max(bad, 0), c.capacity)], 20, 0, 1)


# ---------------------------------------------------------------- attention over chosen pages
def attend_chosen64(c, q, lengths, chosen, count, scale, softcap):
    """out, lse and the tolerances of both, as attend64 has them, over the tokens that the lists name."""
    b, hq, dim = q.shape
    group, page = hq // c.n_kv_heads, c.k_pages.shape[2]
    keys, values, table, q64 = held64(c, "k"), held64(c, "v"), c.table.cpu().numpy(), f64(q)
    out, lse, tol, ltol = np.zeros(q64.shape), np.full((b, hq), -np.inf), np.zeros(q64.shape), np.zeros((b, hq))
    for s, n in enumerate(lengths):
        for h in range(c.n_kv_heads):
            at = []
            for p in chosen[s, h][:max(0, min(count[s, h], -(-n // page)))]:
                if 0 <= p < table.shape[1] and 0 <= table[s, p] < keys.shape[0]:
                    at += [(table[s, p], r) for r in range(max(0, min(page, n - p * page)))]
            if not at:
                continue
            i, r = np.array(at).T
            k, v = keys[i, h, r], values[i, h, r]
            for g in range(h * group, (h + 1) * group):
                x = (k * q64[s, g]).sum(1) * scale
                es = (2 * math.sqrt(dim) + 8) * EPS * np.abs(k * q64[s, g]).sum(1).max() * abs(scale)
                if softcap:
                    x = softcap * np.tanh(x / softcap)
                    es += 8 * EPS * softcap
                z = np.logaddexp.reduce(x)
                p = np.exp(x - z)
                out[s, g], lse[s, g] = p @ v, z
                rel = 2 * es + (16 + 2 * math.sqrt(len(at))) * EPS
                tol[s, g] = rel * (p @ np.abs(v)) + ROUND[q.dtype] * np.abs(out[s, g])
                ltol[s, g] = es + (16 + abs(z)) * 4 * EPS
    return out, lse, tol, ltol


def check_chosen(c, q, lengths, pick, softcap=0.0, scale=None):
    want = attend_chosen64(c, q, lengths, pick[0].cpu().numpy(), pick[1].cpu().numpy(), c.head_dim ** -0.5 if scale is None else scale, softcap)
    out, lse = c.attend(q, chosen=pick, softcap=softcap, scale=scale)
    within(f64(out), want[0], want[2], "out")
    got, fine = f64(lse), np.isfinite(want[1])
    assert np.array_equal(np.isneginf(got), np.isneginf(want[1]))
    within(got[fine], want[1][fine], want[3][fine], "lse")
    return out, lse


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,group,dim,page,budget,first,recent", [(2, 1, 64, 16, 8, 1, 2), (1, 4, 128, 64, 3, 0, 0), (3, 5, 80, 16, 33, 2, 4), (2, 17, 16, 32, 4, 2, 2),
                                                                      (1, 2, 256, 16, 1, 0, 0), (2, 3, 48, 16, 1000, 1, 1)])
def test_attend_over_chosen_pages(kind, heads, group, dim, page, budget, first, recent):
    rng = np.random.default_rng([dim, budget, 1])
    lengths = [0, 1, 16 * budget if budget < 100 else 64, 700, 2000, 1311, page, 5 * page + 1]
    c = with_bounds(rng, kind, lengths, heads, dim, page)
    c.bound()
    q = dev(2 * rng.standard_normal((len(lengths), heads * group, dim)), F32 if kind in ("f32", "odd") else BF16)
    pick = check_choose(c, q, lengths, budget, first, recent)
    a = check_chosen(c, q, lengths, pick)
    b = c.attend(q, chosen=pick)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_chosen(c, q, lengths, pick, softcap=4.0, scale=0.3)


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
def test_attend_over_all_pages_is_attention(kind):
    rng = np.random.default_rng(81)
    lengths = [5000, 3, 0, 777]
    c = with_bounds(rng, kind, lengths, 2, 64, 32)
    c.bound()
    q = dev(rng.standard_normal((4, 6, 64)), F32 if kind == "f32" else BF16)
    chosen, count = c.choose(q, c.capacity // 32)
    out, lse = check_chosen(c, q, lengths, (chosen, count))
    want = c.attend(q)
    within(f64(lse), f64(want[1]), 64 * EPS * (1 + np.abs(np.where(np.isfinite(f64(want[1])), f64(want[1]), 0))), "lse") if not np.isneginf(f64(lse)).any() else None
    assert torch.equal(torch.isinf(lse), torch.isinf(want[1]))


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
def test_attend_over_lists_of_any_kind(kind):
    """Places in no order, named twice, out of range, behind the last token, without a page; counts that lie."""
    rng = np.random.default_rng(82)
    lengths, heads, page = [400, 90, 16, 0, 333], 2, 16
    c = with_bounds(rng, kind, lengths, heads, 48, page)
    c.table[0, 7] = 1 << 29
    q = dev(rng.standard_normal((5, 4, 48)), F32 if kind == "f32" else BF16)
    chosen = rng.integers(-2, 30, (5, heads, 9)).astype(np.int32)
    chosen[0, 0, :4], chosen[0, 1, 3], chosen[4, 0] = [24, 7, 24, 3], 2**31 - 1, -2**31
    for count in (rng.integers(-3, 14, (5, heads)).astype(np.int32), np.full((5, heads), 9, np.int32), np.full((5, heads), 2**31 - 1, np.int32)):
        check_chosen(c, q, lengths, (dev(chosen), dev(count)))


def test_what_choosing_refuses():
    c = cb.TokenCache.create(2, 2, 32, 64, dtype=BF16, page_tokens=16, bounded=True, evictable=False)
    q = torch.zeros((2, 4, 32), dtype=BF16, device="cuda")
    chosen, count = c.choose(q, 3)
    since = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call in (lambda: c.bound(since.long()), lambda: c.bound(since[:1]), lambda: c.choose(q.float(), 3), lambda: c.choose(q[:1], 3), lambda: c.choose(q, 0),
                 lambda: c.choose(q, 1 << 31), lambda: c.choose(q.clone().requires_grad_(), 3), lambda: c.attend(q, chosen=(chosen.long(), count)),
                 lambda: c.attend(q, chosen=(chosen, count[:1])), lambda: c.attend(q, chosen=(chosen[:, :1], count)), lambda: c.attend(q, chosen=(chosen[0], count)),
                 lambda: c.attend(q, chosen=(chosen.transpose(0, 1), count)), lambda: c.attend(q, chosen=(chosen.cpu(), count))):
        with pytest.raises(AssertionError):
            call()
    w = cb.TokenCache.create(2, 2, 32, 64, dtype=BF16, page_tokens=16, bounded=True)
    for call in (lambda: c.choose(q, 3, first=2, recent=2), lambda: c.choose(q, 3, first=-1), lambda: w.attend(q, chosen=(chosen, count), accumulate=True),
                 lambda: c.choose(q[:, :3].contiguous(), 3)):
        with pytest.raises(RuntimeError):
            call()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("seqs", [64, 65, 300])
def test_attend_over_pages_of_many_sequences(kind, seqs):
    rng = np.random.default_rng([seqs, 83])
    lengths = [int(x) for x in rng.integers(0, 200, seqs)]
    lengths[seqs // 2], lengths[-1] = 1500, 0
    c = with_bounds(rng, kind, lengths, 2, 32, 16)
    c.bound()
    q = dev(rng.standard_normal((seqs, 6, 32)), F32 if kind in ("f32", "odd") else BF16)
    check_chosen(c, q, lengths, check_choose(c, q, lengths, 6, 1, 1))
    if kind in ("e4m3", "odd"):
        check_attend_bytes(c, q, lengths)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("off", [0, 1, 3])
def test_queries_and_answers_of_any_strides(kind, off):
    """Rows of a wider tensor, heads apart, from addresses that divide into no vector; what lies between stays as it was."""
    rng = np.random.default_rng([off, 84])
    lengths, heads, hq, dim = [700, 0, 33, 2000], 2, 6, 80
    dtype = F32 if kind in ("f32", "odd") else BF16
    c = with_bounds(rng, kind, lengths, heads, dim, 16)
    c.bound()
    pitch, step = (hq + 1) * (dim + off) + off, dim + off
    flat, room = dev(rng.standard_normal(4 * pitch + 8), dtype), torch.full((4 * pitch + 8,), 7.0, dtype=dtype, device="cuda")
    view = lambda t: t.as_strided((4, hq, dim), (pitch, step, 1), off + step)      # noqa: E731
    q, out = view(flat), view(room)
    plain = q.contiguous()
    pick, same = c.choose(q, 5, first=1, recent=1), c.choose(plain, 5, first=1, recent=1)
    assert torch.equal(pick[0], same[0]) and torch.equal(pick[1], same[1])
    for kw in ({}, {"chosen": pick}):
        want = c.attend(plain, **kw)
        room.fill_(7.0)
        got = c.attend(q, out=out, **kw)
        assert got[0].data_ptr() == out.data_ptr() and torch.equal(out, want[0]) and torch.equal(got[1], want[1])
        kept = room.clone()
        view(kept).fill_(7.0)
        assert (kept == 7.0).all()
        # one query head's tensor, the same for all sequences
        shared = plain[:1, :1].expand(4, 2, dim)
        a, b = c.attend(shared, **kw), c.attend(shared.contiguous(), **kw)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---------------------------------------------------------------- all head sizes
@pytest.mark.parametrize("dim", range(8, 257, 8))
def test_norm_of_every_head_size(dim):
    for i, pairs in enumerate([(dim // 2,), (dim // 2 - 1,), (dim // 4, 1), (dim // 8, 0, dim // 8)]):
        for dtype, layout in ((F32, cb.CB_PAIRS_ADJACENT), (BF16, cb.CB_PAIRS_HALVES)):
            test_norm_rotate_and_its_gradients(dtype, (F32, BF16)[i % 2], layout, cb.CB_LADDER_SHARED, dim, pairs, 1 + i, 3, 9)


@pytest.mark.parametrize("dim", range(16, 257, 16))
def test_append_in_8_bits_of_every_head_size(dim):
    for pairs in ((dim // 2,), (dim // 2 - 1,), (dim // 4, 1, 1)):
        for dtype, layout in ((F32, cb.CB_PAIRS_ADJACENT), (BF16, cb.CB_PAIRS_HALVES)):
            test_append_in_8_bits_with_rotation(dtype, layout, dim, pairs)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", range(8, 257, 8))
def test_pages_of_every_head_size(kind, dim):
    if dim % 16 and kind in ("e4m3", "odd"):
        pytest.skip("heads of 8 bits are multiples of 16")
    test_bounds(kind, 2, dim, 32)
    test_attend_over_chosen_pages(kind, 2, 3, dim, 16, 5, 1, 1)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
def test_steps_of_streams(kind):
    """Norm and rotate, append, bound, choose, attend: eagerly and as a graph that is replayed, every step against 64 bits from what the cache holds."""
    rng = np.random.default_rng(91)
    dtype, seqs, heads, hq, dim, pairs, page, budget = (F32 if kind == "f32" else BF16), 3, 2, 6, 64, (8, 12, 12), 16, 4
    make = lambda: cb.TokenCache.create(seqs, heads, dim, 512, dtype=E4M3 if kind == "e4m3" else dtype, page_tokens=page, evictable=False, bounded=True)  # noqa: E731
    rot, eager, held = cb.Rotary(dim, pairs), make(), make()
    n = 64                                                           # rows at most; offsets say how many there are
    x = torch.zeros((n, 2 * heads, dim), dtype=dtype, device="cuda")
    query, wq, wk = torch.zeros((seqs, hq, dim), dtype=dtype, device="cuda"), dev(1 + 0.2 * rng.standard_normal(dim), F32), dev(1 + 0.2 * rng.standard_normal(dim), F32)
    pos, now, offsets = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((n, 3), (seqs, 3), (seqs + 1,)))

    def step(c, since):
        since.copy_(c.lengths)
        k = rot.norm_rotate(x[:, :heads], pos, wk)
        c.append(k, x[:, heads:], pos[:, :1].contiguous(), offsets=offsets)
        c.bound(since=since)
        q = rot.norm_rotate(query, now, wq)
        pick = c.choose(q, budget, first=1, recent=1)
        return (k, q) + pick + c.attend(q, chosen=pick)

    sinces = [torch.zeros(seqs, dtype=torch.int32, device="cuda") for _ in range(2)]
    step(held, sinces[1])                                            # (a scratch buffer for these query heads is made once, before the graph)
    held.lengths.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step(held, sinces[1])
    lengths = [0] * seqs
    for i in range(6):
        new = rng.multinomial(int(rng.integers(0, n + 1)), [0.6, 0.1, 0.3])
        x.copy_(dev(rng.standard_normal(x.shape), dtype))
        query.copy_(dev(rng.standard_normal(query.shape), dtype))
        pos.copy_(dev(rng.integers(0, 90, (n, 3)).astype(np.int32)))
        now.fill_(i)
        offsets.copy_(dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        graph.replay()
        again = [t.clone() for t in recorded]
        torch.cuda.synchronize()
        got = step(eager, sinces[0])
        assert all(torch.equal(a, b) for a, b in zip(got, again)), i
        lengths = [a + int(b) for a, b in zip(lengths, new)]
        assert eager.lengths.tolist() == lengths == held.lengths.tolist()
        # the cache holds the normed keys, to a rounding more
        ends = np.concatenate([[0], np.cumsum(new)])
        keys, table = held64(eager, "k"), eager.table.cpu().numpy()
        for s in range(seqs):
            for j in range(int(new[s])):
                slot = lengths[s] - int(new[s]) + j
                want = f64(got[0])[ends[s] + j]
                p, r = table[s, slot // page], slot % page
                tol = 0.0 if kind != "e4m3" else np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * f64(eager.k_scale)[p, :, r // 16][:, None])
                within(keys[p, :, r], want, tol, "keys")
        check_norm(rot, query, wq, now.cpu().numpy(), pairs, 0, 0, 1e-6, got[1], "query")
        check_choose(eager, got[1], lengths, budget, 1, 1)
        check_chosen(eager, got[1], lengths, got[2:4])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_bounds_after_an_eviction(kind):
    rng = np.random.default_rng(92)
    dtype, lengths = (F32 if kind == "f32" else BF16), [200, 90]
    c = make_cache(rng, lengths, 2, 32, 16, dtype)
    c = cb.TokenCache(c.k_pages, c.v_pages, c.table, c.lengths, c.weight, c.time, bounds=torch.zeros((c.k_pages.shape[0], 2, 2, 32), dtype=dtype, device="cuda"))
    c.bound()
    c.evict(64, window=3)
    c.bound()
    lengths = c.lengths.tolist()
    assert lengths == [64, 64]
    q = dev(rng.standard_normal((2, 4, 32)), dtype)
    check_chosen(c, q, lengths, check_choose(c, q, lengths, 2, 0, 1))


def test_calls_on_another_device_than_the_current_one(monkeypatch):
    """Such calls make the tensors' device current for themselves.  (Which one is current is made up here: there may be one alone.)"""
    rng = np.random.default_rng(94)
    made, at = [], [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            made.append(self.index)
            at.append(self.index)

        def __exit__(self, *_):
            at.pop()

    dim, rot = 16, cb.Rotary(16, (8,))
    x, w, pos, g = dev(rng.standard_normal((2, 2, dim)), BF16), dev(rng.standard_normal(dim), F32), dev(np.array([[3], [4]], np.int32)), torch.ones((2, 2, dim), dtype=BF16, device="cuda")
    leaf = x.clone().requires_grad_()

    def work():
        c = cb.TokenCache.create(2, 2, dim, 64, dtype=BF16, page_tokens=16, bounded=True)
        y = rot.norm_rotate(x, pos, w)
        grad, = torch.autograd.grad(rot.norm_rotate(leaf, pos, w), leaf, g)
        q = c.append(rot.rotate(x, pos), x, pos, rot, q=y)
        c.bound()
        pick = c.choose(q, 1)
        out = c.attend(q, chosen=pick) + c.attend(q, accumulate=True)
        c.evict(1)
        return (y, grad, q, c.k_pages, c.bounds, c.weight) + pick + out

    want = work()
    assert not made
    monkeypatch.setattr(cb.binding, "_current_device", lambda: at[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    at[0] = 1
    got = work()
    assert made == [0] * 9 and at == [1]
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Caches and plans of their own on streams of their own: results are those of one after the other."""
    rng = np.random.default_rng(93)
    lengths = [3000, 17, 900]
    sides = [torch.cuda.Stream() for _ in range(2)]
    caches = [with_bounds(np.random.default_rng(i), kind, lengths, 2, 64, 32) for i, kind in enumerate(("e4m3", "bf16"))]
    q = dev(rng.standard_normal((3, 8, 64)), BF16)

    def work(c):
        c.bound()
        pick = c.choose(q, 9, recent=1)
        return pick + c.attend(q, chosen=pick) + c.attend(q)

    want = [work(c) for c in caches]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (c, side) in enumerate(zip(caches, sides)):
            with torch.cuda.stream(side):
                got[i].append(work(c))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [cb.CB_PAIRS_HALVES, cb.CB_PAIRS_ADJACENT])
@pytest.mark.parametrize("dim,pairs", [(64, (24,)), (128, (16, 8, 8)), (72, (20,)), (24, (10,)), (40, (15,)), (256, (31,)), (128, (32,))])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite_behind_the_pairs_stays_in_its_place(dtype, layout, dim, pairs, bad):
    """Values behind the pairs are not turned: what one of them is shows nowhere else, but through the mean of its head."""
    rng = np.random.default_rng([dim, 71])
    n, heads = 5, 3
    x, w, g = rng.standard_normal((n, heads, dim)), rng.standard_normal(dim), rng.standard_normal((n, heads, dim))
    pos, rot = dev(rng.integers(1, 99, (n, len(pairs))).astype(np.int32)), cb.Rotary(dim, pairs, layout=layout)

    def step(x, w, g):
        a, b = dev(x, dtype).requires_grad_(), dev(w, F32).requires_grad_()
        y = rot.norm_rotate(a, pos, b)
        return [t.detach().cpu() for t in (y, *torch.autograd.grad(y, (a, b), dev(g, dtype)))]

    def but(t, *at):
        t = t.copy()
        t[at] = bad
        return t

    clean = step(x, w, g)
    first = 2 * sum(pairs)
    for d in sorted({first, first + 1, (first + dim) // 2, dim - 1}):
        other = torch.arange(dim) != d
        # of x: 1 / infinity is zero, and so is all of the head but that value; what is not a number is in the whole head
        y = step(but(x, 1, 2, d), w, g)[0]
        assert torch.isnan(y[1, 2, d])
        assert torch.isnan(y[1, 2]).all() if math.isnan(bad) else (y[1, 2, other] == 0).all()
        kept = torch.ones((n, heads), dtype=torch.bool)
        kept[1, 2] = False
        assert torch.equal(y[kept], clean[0][kept])
        # of the weight: that value of all heads; its own gradient does not hang on it, the others' do by the mean alone
        y, _, gw = step(x, but(w, d), g)
        assert not torch.isfinite(y[..., d]).any() and torch.equal(y[..., other], clean[0][..., other]) and torch.equal(gw, clean[2])
        # of the output's gradient: that weight's gradient, and the head's
        y, gx, gw = step(x, w, but(g, 1, 2, d))
        assert torch.equal(y, clean[0]) and torch.equal(gx[kept], clean[1][kept])
        assert not torch.isfinite(gw[d]) and torch.equal(gw[other], clean[2][other])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,grad", [(1e13, 1e26), (1e-13, 1e-26), (1e-14, 1e-29), (1e8, 1e31), (1e-9, 1e-30), (1e14, 1e-12), (1e-14, 1e10), (1e13, 1e30)])
def test_gradients_of_the_norm_far_from_one(dtype, size, grad):
    """Values and gradients whose products leave float32's range, where neither they nor the results do."""
    rng = np.random.default_rng(72)
    n, dim, pairs = 9, 64, (8, 12, 12)
    q, g = dev(size * rng.standard_normal((n, 3, dim)), dtype).requires_grad_(), dev(grad * rng.standard_normal((n, 3, dim)), dtype)
    w, pos, rot = dev(rng.standard_normal(dim), F32).requires_grad_(), rng.integers(0, 99, (n, 3)).astype(np.int32), cb.Rotary(dim, pairs)
    gx, gw = torch.autograd.grad(rot.norm_rotate(q, dev(pos), w, eps=0.0), (q, w), g)
    check_back(q, w, g, pos, pairs, 0, 0, 0.0, gx, gw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,group,dim", [(2, 3, 64), (1, 17, 128), (3, 1, 80), (2, 2, 256)])
def test_attend_in_8_bits_of_large_queries_over_small_keys(dtype, heads, group, dim):
    """A query times a key's codes, before their scale, may be more than float32 holds; heads of ordinary size beside it are what they were."""
    rng = np.random.default_rng([heads, dim, 73])
    lengths = [300, 40, 1]
    c = make_bytes(rng, lengths, heads, dim, 32)
    q = dev(2 * rng.standard_normal((3, heads * group, dim)), dtype)
    all_pages = (torch.arange(c.table.shape[1], dtype=torch.int32, device="cuda").expand(3, heads, -1).contiguous(),
                 torch.full((3, heads), c.table.shape[1], dtype=torch.int32, device="cuda"))
    ordinary = c.attend(q)[0]
    large = (q * 2.0 ** 118).to(dtype)
    c.k_scale.mul_(2.0 ** -52)
    scale = float(np.float32(2.0 ** -66 * dim ** -0.5))
    for t in (large, torch.where(torch.arange(heads * group, device="cuda")[None, :, None] % 2 == 0, large, q)):
        assert torch.isfinite(t).all()
        check_attend_bytes(c, t, lengths, scale=scale)
        again, lse = c.attend(t, scale=scale, chosen=all_pages)
        want = attend64(wide(c), t, lengths, scale, 0.0)
        within(f64(again), want[0], want[3], "out over chosen pages")
    c.k_scale.mul_(2.0 ** 52)
    assert torch.equal(c.attend(q)[0], ordinary)


# ---------------------------------------------------------------- calls with more work than there are wavefronts
def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


def dealt(dim, pairs, hq, hk, vector):
    """How a wavefront of the norms is dealt (cb_norm.hip, launch): tokens of a stretch, steps of the queries, of the keys."""
    pieces = -(-dim // (2 * vector))
    lanes = 1
    while lanes < pieces and lanes < 64:
        lanes *= 2
    # heads at a time: the fewest lanes without one, the most heads of those that leave as few
    cost, at_once = min((-(-hq // h) * h + -(-hk // h) * h, -h) for h in (1 << i for i in range(7)) if lanes * h <= 64)
    return 64 // lanes // -at_once, -(-hq // -at_once), -(-hk // -at_once)


@pytest.mark.parametrize("dtype,layout,dim,pairs,hq,hk,vector,n", [(BF16, cb.CB_PAIRS_HALVES, 128, (16, 24, 24), 8, 8, 8, 7001), (F32, cb.CB_PAIRS_ADJACENT, 16, (4, 4), 3, 1, 4, 250003),
                                                                   (BF16, cb.CB_PAIRS_ADJACENT, 80, (8, 12, 10), 6, 2, 2, 9001), (F32, cb.CB_PAIRS_HALVES, 40, (15,), 5, 2, 1, 13001)])
def test_gradients_of_more_stretches_than_wavefronts(dtype, layout, dim, pairs, hq, hk, vector, n):
    """Every wavefront of the backward pass goes through several stretches of tokens, some through one less than others."""
    rng = np.random.default_rng([dim, n])
    tokens, q_steps, k_steps = dealt(dim, pairs, hq, hk, vector)
    waves = 3 * units() * 4
    stretches = -(-n // tokens)
    assert stretches > 2 * waves and stretches % waves
    q, k = dev(rng.standard_normal((n, hq, dim), dtype=np.float32), dtype).requires_grad_(), dev(rng.standard_normal((n, hk, dim), dtype=np.float32), dtype).requires_grad_()
    gq, gk = dev(rng.standard_normal((n, hq, dim), dtype=np.float32), dtype), dev(rng.standard_normal((n, hk, dim), dtype=np.float32), dtype)
    wq, wk = (dev(1 + 0.3 * rng.standard_normal(dim), F32).requires_grad_() for _ in range(2))
    pos, rot, eps = rng.integers(-5, 2000, (n, len(pairs))).astype(np.int32), cb.Rotary(dim, pairs, layout=layout), 1e-3
    out = rot.norm_rotate(q, dev(pos), wq, k=k, k_weight=wk, eps=eps)
    got = torch.autograd.grad(out, (q, wq, k, wk), (gq, gk))
    for x, w, g, y, gx, gw, steps in ((q, wq, gq, out[0], got[0], got[1], q_steps), (k, wk, gk, out[1], got[2], got[3], k_steps)):
        total, size = np.zeros(dim), np.zeros(dim)
        for a in range(0, n, 20000):
            part = slice(a, min(a + 20000, n))
            check_norm(rot, x[part], w, pos[part], pairs, layout, 0, eps, y[part], "output")
            check_back(x[part], w, g[part], pos[part], pairs, layout, 0, eps, gx[part], None)
            _, some, norms, _ = norm_back64(f64(x[part]), f64(w), f64(g[part]), pos[part], pairs, layout, 0, eps)
            total += some
            size += (turned_size(f64(g[part]), pairs, layout) * np.abs(norms)).sum((0, 1))
        # a term is off by 32 units; a lane adds up `steps` of each of its wavefront's stretches, six additions join a wavefront's lanes and four a workgroup's
        # wavefronts, in float32; rows of workgroups are added in float64 and rounded once
        terms = steps * -(-stretches // waves) + 6 + 4 + 32
        within(f64(gw), total, (terms * EPS + ANGLE) * size + ROUND[gw.dtype] * np.abs(total), "gradient of the weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,dim,page", [(8, 32, 64), (16, 16, 16), (8, 80, 128)])
def test_append_in_8_bits_of_more_blocks_than_wavefronts(dtype, heads, dim, page):
    """A wavefront takes two heads of a block, where there are so many blocks."""
    rng = np.random.default_rng([heads, dim, 74])
    held, new = [0, 17, 5, 0, 48], [3001, 16, 5000, 0, 1300]
    assert 2 * (sum(new) // 16 + 2 * len(new)) >= 4 * units()
    c = make_bytes(rng, held, heads, dim, page, capacity=5120)
    ends = np.concatenate([[0], np.cumsum(new)])
    n = int(ends[-1])
    kv = dev(rng.standard_normal((n, 2 * heads, dim)) * np.exp(2 * rng.standard_normal((n, 2 * heads, 1))), dtype)
    k, v = kv[:, :heads], kv[:, heads:]
    want = bytes_append64(c, f64(k), f64(v), held, ends)
    c.append(k, v, offsets=dev(ends.astype(np.int32)))
    for x in "kv":
        same_codes(getattr(c, x + "_pages"), want[x + "_pages"], x)
        assert np.array_equal(f64(getattr(c, x + "_scale")), want[x + "_scale"], equal_nan=True), x
    assert c.lengths.tolist() == [a + b for a, b in zip(held, new)]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_in_8_bits_at_once_and_by_blocks(dtype):
    """With rotation: one call of many blocks leaves what many calls of few leave."""
    rng = np.random.default_rng(75)
    heads, dim, n, step = 8, 64, 9008, 16 * 113
    rot = cb.Rotary(dim, (8, 12, 12))
    k, v = (dev(rng.standard_normal((n, heads, dim)) * np.exp(rng.standard_normal((n, 1, 1))), dtype) for _ in range(2))
    q, pos = dev(rng.standard_normal((n, heads, dim)), dtype), dev(rng.integers(0, 500, (n, 3)).astype(np.int32))
    a, b = (cb.TokenCache.create(1, heads, dim, n, dtype=E4M3) for _ in range(2))
    turned = a.append(k, v, pos, rot, q, offsets=dev(np.array([0, n], np.int32)))
    for i in range(0, n, step):
        j = min(i + step, n)
        assert torch.equal(b.append(k[i:j], v[i:j], pos[i:j], rot, q[i:j], offsets=dev(np.array([0, j - i], np.int32))), turned[i:j])
    for x in ("k_pages", "v_pages"):
        assert torch.equal(getattr(a, x).view(torch.uint8), getattr(b, x).view(torch.uint8))
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale) and a.lengths.tolist() == b.lengths.tolist() == [n]


@pytest.mark.parametrize("seed", range(4))
def test_choose_of_scores_whose_terms_cancel(seed):
    """Terms of 2^-40 .. 2^40 and of both signs: a score is the exact one but for a rounding a term in float64 and one to float32, and where that leaves two pages
    in either order either may be chosen."""
    rng = np.random.default_rng([seed, 76])
    pages, dim, group, budget = 300, 32, 3, 40
    k = torch.zeros((pages, 1, 16, dim), device="cuda")
    lo = rng.standard_normal((pages, dim)) * 2.0 ** rng.integers(-20, 21, (pages, dim))
    lo[:, 1::2] = -lo[:, ::2] * (1 + 2.0 ** -20 * rng.integers(-1, 2, (pages, dim // 2)))       # (pairs of terms that all but cancel, or do)
    bounds = dev(np.stack([lo, lo], 1)[:, None].astype(np.float32))
    q = rng.standard_normal((1, group, dim)) * 2.0 ** rng.integers(-20, 21, (1, group, 1))
    q[..., 1::2] = q[..., ::2]
    q = dev(q, F32)
    c = cb.TokenCache(k, k, torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([16 * pages], dtype=torch.int32, device="cuda"), bounds=bounds)
    chosen, count = c.choose(q, budget)
    got = chosen[0, 0].tolist()
    assert count.item() == budget and got == sorted(set(got)) and 0 <= got[0] and got[-1] < pages
    x, q64 = f64(bounds)[:, 0, 0], f64(q)[0]
    least, most = np.empty(pages, np.float32), np.empty(pages, np.float32)
    for p in range(pages):
        exact = [math.fsum(x[p] * q64[g]) for g in range(group)]                          # (products are exact in float64)
        off = [(dim + 1) * 2.0 ** -53 * np.abs(x[p] * q64[g]).sum() for g in range(group)]
        least[p], most[p] = max(a - b for a, b in zip(exact, off)), max(a + b for a, b in zip(exact, off))
    out = np.setdiff1d(np.arange(pages), got)
    assert (most[got][:, None] >= least[out][None]).all()
    sure = [p for p in got if (least[p] > most[out]).all()]
    assert len(sure) >= budget // 2                                                        # (most of them are no near thing)
