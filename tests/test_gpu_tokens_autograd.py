"""How the token operators stand to torch's autograd: outputs that are given, modes that carry derivatives."""
import gc

import pytest
import torch

import paper_1808_05488_amd as cb

pytestmark = pytest.mark.gpu

N, DIM = 3, 16


def values(heads=2, **kw):
    return torch.randn((N, heads, DIM), device="cuda", **kw)


def operands():
    rot, pos, w = cb.Rotary(DIM, (8,)), torch.zeros((N, 1), dtype=torch.int32, device="cuda"), torch.ones(DIM, device="cuda")
    return rot, pos, w, cb.TokenCache.create(N, 2, DIM, 64, dtype=torch.float32, bounded=True)


# what is written, of which shape; x: what a call takes
GIVEN = {
    "norm_rotate q_out": lambda x, t: operands()[0].norm_rotate(x, *operands()[1:3], q_out=t),
    "norm_rotate k_out": lambda x, t: operands()[0].norm_rotate(x, *operands()[1:3], k=x, k_weight=operands()[2], k_out=t),
    "rotate q_out": lambda x, t: operands()[0].rotate(x, operands()[1], q_out=t),
    "rotate k_out": lambda x, t: operands()[0].rotate(x, operands()[1], k=x, k_out=t),
    "append q_out": lambda x, t: operands()[3].append(x, x, operands()[1], operands()[0], q=x, q_out=t),
    "attend out": lambda x, t: operands()[3].attend(x, out=t),
    "attend lse": lambda x, t: operands()[3].attend(x, lse=t),
}


def output(which, **kw):
    return torch.randn((N, 2), device="cuda", **kw) if which == "attend lse" else values(**kw)


@pytest.mark.parametrize("which", GIVEN)
def test_a_graph_notices_that_what_it_has_saved_was_written(which):
    t, leaf = output(which), torch.ones((), device="cuda", requires_grad=True)
    y = leaf * t                                                   # (its backward pass needs t)
    before = t._version
    GIVEN[which](values(), t)
    assert t._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("which", GIVEN)
def test_outputs_that_want_a_gradient(which):
    t = output(which, requires_grad=True)
    before = t.detach().clone()
    with pytest.raises(AssertionError, match="carries no gradient"):
        GIVEN[which](values(), t)
    assert torch.equal(t, before)
    with torch.no_grad():
        GIVEN[which](values(), t)
    assert not torch.equal(t, before)


@pytest.mark.parametrize("which", GIVEN)
def test_outputs_in_inference_mode(which):
    t = output(which)
    before = t.clone()
    with torch.inference_mode():
        made = output(which)
        then = made.clone()
        GIVEN[which](values(), t)
        GIVEN[which](values(), made)
    assert not torch.equal(t, before) and not torch.equal(made, then)


@pytest.mark.parametrize("again", ["norm_rotate", "rotate"])
def test_a_norm_in_place_of_what_a_recorded_one_has_saved(again):
    rot, pos, w, _ = operands()
    q, w = values(), w.clone().requires_grad_()
    y = rot.norm_rotate(q, pos, w)
    with torch.no_grad():
        if again == "norm_rotate":
            rot.norm_rotate(q, pos, w, q_out=q)
        else:
            rot.rotate(q, pos, q_out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_inputs_and_new_outputs_keep_their_version():
    rot, pos, w, cache = operands()
    x = values()
    tensors = [x, pos, w]
    before = [t._version for t in tensors]
    a, b = rot.norm_rotate(x, pos, w, k=x, k_weight=w)
    cache.append(x, x)
    out, lse = cache.attend(x)
    assert [t._version for t in tensors] == before and a._version == b._version == out._version == lse._version == 0


def test_forward_mode_and_batched_gradients_are_refused():
    rot, pos, w, cache = operands()
    x = values()
    with torch.autograd.forward_ad.dual_level():
        d = torch.autograd.forward_ad.make_dual(x, x)
        for call in (lambda: rot.norm_rotate(d, pos, w), lambda: rot.rotate(d, pos), lambda: cache.append(d, x), lambda: cache.attend(d), lambda: cache.choose(d, 1)):
            with pytest.raises(AssertionError, match="forward-mode"):
                call()
        assert torch.equal(rot.rotate(x, pos), x)
    with pytest.raises(AssertionError, match="forward-mode"):
        torch.func.jvp(lambda t: rot.norm_rotate(t, pos, w), (x,), (x,))
    q = x.clone().requires_grad_()
    for f in (lambda t: rot.norm_rotate(t, pos, w), lambda t: rot.rotate(t, pos)):
        with pytest.raises(RuntimeError):
            torch.autograd.grad(f(q), q, torch.stack([x, x]), is_grads_batched=True)


@pytest.mark.parametrize("first", ["rotate", "norm_rotate"])
@pytest.mark.parametrize("recorded", ["rotate", "norm_rotate"])
@pytest.mark.parametrize("as_k", [False, True])
def test_a_recorded_backward_pass_of_a_leaf_that_another_stream_has_in_a_graph(first, recorded, as_k):
    rot, pos, w, _ = operands()
    x, t, g = values(), values().requires_grad_(), values()

    def step(which):
        if which == "rotate":
            return rot.rotate(x, pos, k=t)[1] if as_k else rot.rotate(t, pos)
        return rot.norm_rotate(x, pos, w, k=t, k_weight=w)[1] if as_k else rot.norm_rotate(t, pos, w)

    alive = step(first)
    want, = torch.autograd.grad(step(recorded), t, g)
    torch.cuda.synchronize()
    with pytest.raises(AssertionError, match="same leaves"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            torch.autograd.grad(step(recorded), t, g)
    del alive
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, = torch.autograd.grad(step(recorded), t, g)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
