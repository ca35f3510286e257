"""The host side of norms with rotation, caches in 8 bits and chosen pages: every refusal.  Nothing here launches anything: addresses are made up, and a call
that would not refuse them is not made."""
import ctypes as C
import math

import pytest

import paper_1808_05488_amd as cb
from paper_1808_05488_amd import binding
from test_tokens_abi import FAKE, cache, heads, rotary, without_asserts

OK, EINVAL, ENOMEM = cb.CB_OK, cb.CB_EINVAL, cb.CB_ENOMEM


def ref(x):
    return None if x is None else C.byref(x)


def bytes_cache(**kw):
    v = dict(dtype=cb.CB_E4M3, values_dtype=cb.CB_BF16, k_scale_dev=9 * FAKE, v_scale_dev=10 * FAKE, bounds_dev=11 * FAKE)
    v.update(kw)
    return cache(**v)


def test_norm_rotate_refusals():
    L, r, p, w = binding.lib(), rotary(), 8 * FAKE, 9 * FAKE

    def call(rot=r, dtype=cb.CB_F32, n=5, pos=p, eps=1e-6, wdtype=cb.CB_F32, q=heads(), qw=w, qo=heads(), k=heads(2), kw=w, ko=heads(2)):
        return L.cb_norm_rotate(ref(rot), dtype, n, pos, eps, wdtype, ref(q), qw, ref(qo), ref(k), kw, ref(ko), None)

    bad = rotary()
    bad.desc.pairs[0] = 99
    for kw in (dict(rot=None), dict(rot=bad), dict(dtype=2), dict(dtype=cb.CB_E4M3), dict(n=-1), dict(n=1 << 31), dict(pos=None), dict(eps=-1e-6),
               dict(eps=math.inf), dict(eps=math.nan), dict(wdtype=2), dict(wdtype=cb.CB_E4M3), dict(q=None), dict(qw=None), dict(qo=None),
               dict(k=None), dict(kw=None), dict(ko=None), dict(qw=w + 2), dict(kw=w + 1), dict(wdtype=cb.CB_BF16, qw=w + 1), dict(q=heads(3)),
               dict(k=heads(3)), dict(q=heads(0)), dict(q=heads(data=None)), dict(qo=heads(data=FAKE + 2)), dict(k=heads(2, reserved=1))):
        assert call(**kw) == EINVAL, kw
    nothing = heads(data=None)
    assert call(n=0, pos=None, q=nothing, qo=nothing, k=None, kw=None, ko=None) == OK


def test_norm_rotate_back_refusals():
    L, r, p, w, n = binding.lib(), rotary(), 8 * FAKE, 9 * FAKE, C.c_size_t()
    assert L.cb_norm_rotate_back_scratch_bytes(C.byref(r), C.byref(n)) == OK and n.value >= 2 * 64 * 4
    assert L.cb_norm_rotate_back_scratch_bytes(None, C.byref(n)) == EINVAL and L.cb_norm_rotate_back_scratch_bytes(C.byref(r), None) == EINVAL

    def side(x=heads(), g=heads(), xg=heads(), weight=w, wg=w):
        return binding.cb_norm_back(x, g, xg, weight, wg)

    def call(rot=r, dtype=cb.CB_F32, tokens=5, pos=p, eps=1e-6, wdtype=cb.CB_F32, q=side(), k=side(), scratch=10 * FAKE, size=n.value):
        return L.cb_norm_rotate_back(ref(rot), dtype, tokens, pos, eps, wdtype, ref(q), ref(k), scratch, size, None)

    for kw in (dict(rot=None), dict(dtype=2), dict(tokens=-1), dict(tokens=1 << 31), dict(pos=None), dict(eps=-1.0), dict(wdtype=3), dict(q=None, k=None),
               dict(q=side(g=heads(3))), dict(k=side(xg=heads(5))), dict(q=side(weight=None)), dict(q=side(weight=w + 2)), dict(k=side(wg=w + 1)),
               dict(q=side(x=heads(data=None))), dict(q=side(g=heads(data=FAKE + 1))), dict(k=side(xg=heads(data=FAKE + 2))), dict(scratch=None),
               dict(scratch=10 * FAKE + 8)):
        assert call(**kw) == EINVAL, kw
    assert call(size=n.value - 1) == ENOMEM


@pytest.mark.parametrize("kw", [dict(head_dim=24), dict(head_dim=8), dict(values_dtype=2), dict(values_dtype=cb.CB_E4M3), dict(values_dtype=-1), dict(reserved2=1),
                                dict(k_scale_dev=None), dict(v_scale_dev=None), dict(k_scale_dev=FAKE + 2), dict(v_scale_dev=FAKE + 1), dict(bounds_dev=FAKE + 8),
                                dict(dtype=2), dict(dtype=3)])
def test_caches_in_8_bits_that_are_refused(kw):
    L, c = binding.lib(), bytes_cache(**kw)
    prm, ch = binding.cb_attend_params(1.0, 0.0, 1.0, 0, 0), binding.cb_choose_params(4, 0, 0, 0)
    a, b = C.byref(heads()), C.byref(heads(8))
    assert L.cb_cache_append(C.byref(c), None, 2, None, None, None, a, a, None, None, None) == EINVAL
    assert L.cb_cache_attend(C.byref(c), C.byref(prm), b, b, None, None) == EINVAL
    assert L.cb_cache_attend_chosen(C.byref(c), C.byref(prm), b, b, None, FAKE, FAKE, 4, None) == EINVAL
    assert L.cb_cache_bound(C.byref(c), None, None) == EINVAL
    assert L.cb_cache_choose(C.byref(c), C.byref(ch), b, FAKE, FAKE, None) == EINVAL


def test_a_cache_in_8_bits_is_not_cut_back():
    p = binding.cb_evict_params(8, 0, None, None, None)
    assert binding.lib().cb_cache_evict(C.byref(bytes_cache()), C.byref(p), None) == EINVAL


def test_bound_and_choose_refusals():
    L = binding.lib()
    assert L.cb_cache_bound(None, None, None) == EINVAL
    assert L.cb_cache_bound(C.byref(cache()), None, None) == EINVAL                 # no bounds
    assert L.cb_cache_bound(C.byref(bytes_cache(scratch_bytes=100)), None, None) == ENOMEM

    def call(c=bytes_cache(), budget=4, first=1, recent=2, reserved=0, q=heads(8), chosen=FAKE, count=FAKE):
        return L.cb_cache_choose(ref(c), C.byref(binding.cb_choose_params(budget, first, recent, reserved)), ref(q), chosen, count, None)

    for kw in (dict(c=None), dict(c=cache()), dict(budget=0), dict(budget=-4), dict(budget=2 ** 30 + 1), dict(budget=2 ** 31 - 1), dict(first=-1), dict(recent=-1), dict(first=2, recent=3),
               dict(first=2 ** 31 - 1, recent=2 ** 31 - 1, budget=2 ** 31 - 1), dict(reserved=1), dict(q=None), dict(q=heads(6)), dict(q=heads(8, data=None)),
               dict(q=heads(8, data=FAKE + 1)), dict(chosen=None), dict(count=None)):
        assert call(**kw) == EINVAL, kw
    assert L.cb_cache_choose(C.byref(bytes_cache()), None, C.byref(heads(8)), FAKE, FAKE, None) == EINVAL
    # pages' scores need room, where there are bounds
    sizes = []
    for bounds in (None, 11 * FAKE):
        n, c = C.c_size_t(), cache(weight_dev=None, max_pages=1 << 12, bounds_dev=bounds)
        assert L.cb_cache_scratch_bytes(C.byref(c), 0, C.byref(n)) == OK
        sizes.append(n.value)
    assert sizes[1] >= 2 * 4 * (1 << 12) * 4 > sizes[0]
    # pages of all sequences and heads are counted in 32 bits
    for f in (lambda c: L.cb_cache_bound(C.byref(c), None, None), lambda c: call(c=c)):
        assert f(bytes_cache(n_seq=1024, n_kv_heads=64, max_pages=1 << 14, weight_dev=None, scratch_bytes=1 << 62)) == EINVAL
    assert call(c=cache(weight_dev=None, max_pages=1 << 12, bounds_dev=11 * FAKE, scratch_bytes=sizes[0])) == ENOMEM


def test_attend_chosen_refusals():
    L = binding.lib()

    def call(c=bytes_cache(), q=heads(8), out=heads(8), scale=1.0, cap=0.0, decay=1.0, accumulate=0, chosen=FAKE, count=FAKE, budget=4):
        p = binding.cb_attend_params(scale, cap, decay, accumulate, 0)
        return L.cb_cache_attend_chosen(ref(c), C.byref(p), ref(q), ref(out), None, chosen, count, budget, None)

    for kw in (dict(c=None), dict(q=None), dict(out=None), dict(q=heads(6), out=heads(6)), dict(out=heads(4)), dict(scale=math.inf), dict(cap=-1.0),
               dict(decay=2.0), dict(accumulate=1), dict(chosen=None), dict(count=None), dict(budget=0), dict(budget=-1), dict(budget=2 ** 30 + 1), dict(q=heads(8, data=None))):
        assert call(**kw) == EINVAL, kw
    assert call(c=bytes_cache(scratch_bytes=100)) == ENOMEM


def test_tensors_of_the_host_are_refused_without_asserts():
    got = without_asserts("""
        cb.Rotary(32, (16,)).norm_rotate(torch.zeros(1, 2, 32), torch.zeros((1, 1), dtype=torch.int32), torch.ones(32))""")
    assert got.startswith("AssertionError") and "on a GPU" in got
    got = without_asserts("""
        cb.Rotary(32, (16,)).norm_rotate(torch.zeros(1, 2, 32), torch.zeros((1, 1), dtype=torch.int32), torch.ones(32), k=torch.zeros(1, 2, 32))""")
    assert got.startswith("AssertionError") and "together" in got
    got = without_asserts("""
        x = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
        p = x(4, 2, 16, 32, dtype=torch.float8_e4m3fn)
        cb.TokenCache(p, p, x(2, 2, dtype=torch.int32), x(2, dtype=torch.int32))""")
    assert got.startswith("AssertionError") and "on a GPU" in got
    got = without_asserts("cb.TokenCache.create(1, 2, 32, 64, dtype=torch.float8_e4m3fn, device='cpu', evictable=True)")
    assert got.startswith("AssertionError") and "cut back" in got
