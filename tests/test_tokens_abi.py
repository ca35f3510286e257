"""The token operators' host side: frequencies, scratch sizes, and every refusal.  Nothing here launches anything: addresses are made
up, and a call that would not refuse them is not made."""
import ctypes as C
import math
import os
import subprocess
import sys
import textwrap

import pytest

import paper_1808_05488_amd as cb
from paper_1808_05488_amd import binding

FAKE = 1 << 20                      # an aligned address that is never read


def rotary_desc(head_dim=64, pairs=(8, 12, 12), layout=0, ladder=0, base=10000.0):
    d = binding.cb_rotary_desc()
    d.head_dim, d.n_axes, d.layout, d.ladder, d.base = head_dim, len(pairs), layout, ladder, base
    for a, n in enumerate(pairs):
        d.pairs[a] = n
    return d


def rotary(**kw):
    r = binding.cb_rotary()
    assert binding.lib().cb_rotary_init(C.byref(rotary_desc(**kw)), C.byref(r)) == cb.CB_OK
    return r


def cache(**kw):
    d = binding.cb_cache()
    v = dict(n_seq=2, n_kv_heads=4, head_dim=64, page_tokens=16, max_pages=8, n_pages=16, dtype=cb.CB_F32, k_pages_dev=FAKE,
             v_pages_dev=2 * FAKE, table_dev=3 * FAKE, lengths_dev=4 * FAKE, weight_dev=5 * FAKE, time_dev=6 * FAKE,
             scratch_dev=7 * FAKE, scratch_bytes=1 << 40)
    v.update(kw)
    for name, x in v.items():
        setattr(d, name, x)
    return d


def heads(n=4, data=FAKE, reserved=0):
    return binding.cb_heads(data, n * 64, 64, n, reserved)


@pytest.mark.parametrize("ladder", [cb.CB_LADDER_SHARED, cb.CB_LADDER_PER_AXIS])
def test_frequencies(ladder):
    pairs, base = (3, 0, 8, 5), 500.0
    r = rotary(head_dim=40, pairs=pairs, ladder=ladder, base=base)
    want, total = [], sum(pairs)
    for n in pairs:
        for i in range(n):
            e = len(want) / total if ladder == cb.CB_LADDER_SHARED else i / n
            want.append(base ** -e / (2 * math.pi))
    got = list(r.turns)
    assert got[total:] == [0.0] * (cb.CB_ROTARY_MAX_PAIRS - total)
    assert all(abs(g - w) <= 4e-16 * w for g, w in zip(got, want))


@pytest.mark.parametrize("kw", [dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(pairs=()), dict(pairs=(0, 0)),
                                dict(pairs=(16, 17)), dict(pairs=(-1, 8)), dict(layout=2), dict(layout=-1), dict(ladder=2),
                                dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan)])
def test_rotary_descriptions_that_are_refused(kw):
    r = binding.cb_rotary()
    assert binding.lib().cb_rotary_init(C.byref(rotary_desc(**kw)), C.byref(r)) == cb.CB_EINVAL


def test_rotary_descriptions_that_are_refused_by_field():
    L, r = binding.lib(), binding.cb_rotary()
    d = rotary_desc()
    d.n_axes = 5
    assert L.cb_rotary_init(C.byref(d), C.byref(r)) == cb.CB_EINVAL
    d = rotary_desc(pairs=(8, 8))
    d.pairs[2] = 1                  # behind the axes
    assert L.cb_rotary_init(C.byref(d), C.byref(r)) == cb.CB_EINVAL
    d = rotary_desc()
    d.reserved = 1
    assert L.cb_rotary_init(C.byref(d), C.byref(r)) == cb.CB_EINVAL
    assert L.cb_rotary_init(None, C.byref(r)) == cb.CB_EINVAL
    assert L.cb_rotary_init(C.byref(rotary_desc()), None) == cb.CB_EINVAL


def test_rotate_refusals():
    L, r, p = binding.lib(), rotary(), 8 * FAKE

    def call(rot=r, dtype=cb.CB_F32, n=5, pos=p, q=heads(), qo=heads(), k=heads(2), ko=heads(2), inverse=0):
        ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
        return L.cb_rotate(ref(rot), dtype, n, pos, ref(q), ref(qo), ref(k), ref(ko), inverse, None)

    bad = rotary()
    bad.desc.pairs[0] = 99
    for kw in (dict(rot=None), dict(rot=bad), dict(dtype=2), dict(n=-1), dict(n=1 << 31), dict(pos=None), dict(q=None), dict(qo=None),
               dict(k=None), dict(ko=None), dict(inverse=2), dict(q=heads(3)), dict(k=heads(3)), dict(q=heads(0)),
               dict(q=heads(4, data=None)), dict(q=heads(4, data=FAKE + 2)), dict(q=heads(reserved=1)),
               dict(q=heads(65537), qo=heads(65537))):
        assert call(**kw) == cb.CB_EINVAL, kw
    assert call(n=0, pos=None, q=heads(data=None), qo=heads(data=None), k=None, ko=None) == cb.CB_OK      # nothing to do


BAD_CACHES = [dict(n_seq=0), dict(n_seq=65536), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=4), dict(head_dim=36),
              dict(head_dim=264), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(max_pages=0),
              dict(max_pages=1 << 27), dict(n_pages=0), dict(dtype=2), dict(reserved=1)]
BAD_BUFFERS = [dict(k_pages_dev=None), dict(v_pages_dev=None), dict(k_pages_dev=FAKE + 8), dict(v_pages_dev=FAKE + 4),
               dict(table_dev=None), dict(lengths_dev=None), dict(scratch_dev=None), dict(scratch_dev=FAKE + 128),
               dict(weight_dev=FAKE + 4), dict(time_dev=FAKE + 8)]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_caches_that_are_refused(kw):
    L, c, n = binding.lib(), cache(**kw), C.c_size_t()
    prm, ev = binding.cb_attend_params(1.0, 0.0, 1.0, 0, 0), binding.cb_evict_params(8, 0, None, None, None)
    assert L.cb_cache_scratch_bytes(C.byref(c), 0, C.byref(n)) == cb.CB_EINVAL
    assert L.cb_cache_append(C.byref(c), None, 2, None, None, None, C.byref(heads()), C.byref(heads()), None, None, None) == cb.CB_EINVAL
    assert L.cb_cache_attend(C.byref(c), C.byref(prm), C.byref(heads()), C.byref(heads()), None, None) == cb.CB_EINVAL
    assert L.cb_cache_evict(C.byref(c), C.byref(ev), None) == cb.CB_EINVAL


@pytest.mark.parametrize("kw", BAD_BUFFERS + [dict(scratch_bytes=100)])
def test_buffers_that_are_refused(kw):
    L, c = binding.lib(), cache(**kw)
    want = cb.CB_ENOMEM if "scratch_bytes" in kw else cb.CB_EINVAL
    prm, ev = binding.cb_attend_params(1.0, 0.0, 1.0, 0, 0), binding.cb_evict_params(8, 0, None, None, None)
    assert L.cb_cache_append(C.byref(c), None, 2, None, None, None, C.byref(heads()), C.byref(heads()), None, None, None) == want
    assert L.cb_cache_attend(C.byref(c), C.byref(prm), C.byref(heads()), C.byref(heads()), None, None) == want
    assert L.cb_cache_evict(C.byref(c), C.byref(ev), None) == want


def test_append_refusals():
    L, c, r = binding.lib(), cache(), rotary()

    def call(c=c, rot=r, n=2, pos=FAKE, off=None, k=heads(), v=heads(), q=heads(8), qo=heads(8)):
        ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
        return L.cb_cache_append(ref(c), ref(rot), n, pos, off, None, ref(k), ref(v), ref(q), ref(qo), None)

    bad = rotary()
    bad.desc.base = 0.0
    for kw in (dict(c=None), dict(rot=bad), dict(rot=rotary(head_dim=80)), dict(n=-1, off=FAKE), dict(n=1 << 24, off=FAKE), dict(n=3), dict(pos=None), dict(k=None),
               dict(v=None), dict(k=heads(2)), dict(v=heads(5)), dict(qo=None), dict(q=None), dict(qo=heads(4)), dict(rot=None),
               dict(k=heads(data=None)), dict(v=heads(data=FAKE + 1)), dict(q=heads(8, reserved=3))):
        assert call(**kw) == cb.CB_EINVAL, kw


def test_attend_refusals():
    L = binding.lib()

    def call(c=cache(), q=heads(8), out=heads(8), scale=1.0, cap=0.0, decay=1.0, accumulate=0, reserved=0):
        ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
        p = binding.cb_attend_params(scale, cap, decay, accumulate, reserved)
        return L.cb_cache_attend(ref(c), C.byref(p), ref(q), ref(out), None, None)

    for kw in (dict(c=None), dict(q=None), dict(out=None), dict(q=heads(6), out=heads(6)), dict(out=heads(4)), dict(scale=math.inf),
               dict(scale=math.nan), dict(cap=-1.0), dict(cap=math.nan), dict(decay=-0.1), dict(decay=1.5), dict(decay=math.nan),
               dict(accumulate=2), dict(reserved=1), dict(accumulate=1, c=cache(weight_dev=None)), dict(q=heads(8, data=None)),
               dict(out=heads(8, data=FAKE + 2))):
        assert call(**kw) == cb.CB_EINVAL, kw
    assert L.cb_cache_attend(C.byref(cache()), None, C.byref(heads()), C.byref(heads()), None, None) == cb.CB_EINVAL
    # room for appending and eviction is not room for query heads
    n = C.c_size_t()
    assert L.cb_cache_scratch_bytes(C.byref(cache()), 0, C.byref(n)) == cb.CB_OK
    assert call(c=cache(scratch_bytes=n.value)) == cb.CB_ENOMEM


def test_evict_refusals():
    L = binding.lib()
    for c, budget, window in ((cache(weight_dev=None), 8, 0), (cache(time_dev=None), 8, 0), (cache(), 0, 0), (cache(), 129, 0),
                              (cache(), 8, -1), (None, 8, 0)):
        p = binding.cb_evict_params(budget, window, None, None, None)
        assert L.cb_cache_evict(None if c is None else C.byref(c), C.byref(p), None) == cb.CB_EINVAL
    assert L.cb_cache_evict(C.byref(cache()), None, None) == cb.CB_EINVAL
    for bad in (binding.cb_evict_params(8, 0, FAKE + 4, None, None), binding.cb_evict_params(8, 0, None, FAKE + 8, None)):
        assert L.cb_cache_evict(C.byref(cache()), C.byref(bad), None) == cb.CB_EINVAL


def test_attention_whose_work_is_not_counted_in_32_bits_is_refused():
    L, p = binding.lib(), binding.cb_attend_params(1.0, 0.0, 1.0, 0, 0)
    for kw in (dict(n_seq=65535, n_kv_heads=4, max_pages=1 << 13, page_tokens=1024), dict(n_seq=4, max_pages=1 << 20, page_tokens=1024)):
        c = cache(weight_dev=None, scratch_bytes=1 << 62, **kw)
        assert L.cb_cache_attend(C.byref(c), C.byref(p), C.byref(heads(512)), C.byref(heads(512)), None, None) == cb.CB_EINVAL


def test_scratch_sizes():
    L, n = binding.lib(), C.c_size_t()

    def size(heads, **kw):
        assert L.cb_cache_scratch_bytes(C.byref(cache(**kw)), heads, C.byref(n)) == cb.CB_OK
        return n.value

    assert size(0) < size(4) <= size(16)
    assert size(8, weight_dev=None) <= size(8)
    assert size(0, weight_dev=None) < 1 << 16                 # counters alone
    assert size(8, max_pages=1 << 14) > 2 * 8 * (1 << 18) * 4       # a score a query head and slot
    for bad in (-1, 3, 65540):
        assert L.cb_cache_scratch_bytes(C.byref(cache()), bad, C.byref(n)) == cb.CB_EINVAL
    assert L.cb_cache_scratch_bytes(C.byref(cache()), 4, None) == cb.CB_EINVAL
    assert L.cb_cache_scratch_bytes(None, 4, C.byref(n)) == cb.CB_EINVAL


def without_asserts(code):
    """What python -O prints of the code (assert statements are gone there), with the error's type in place of one that is raised."""
    text = "import torch\nimport paper_1808_05488_amd as cb\ntry:\n" + textwrap.indent(textwrap.dedent(code), "    ") + \
           "\nexcept Exception as e:\n    print(type(e).__name__, e)\nelse:\n    print('done')\n"
    r = subprocess.run([sys.executable, "-O", "-c", text], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr
    return r.stdout.strip()


def test_addresses_of_the_host_are_refused_without_asserts():
    got = without_asserts("""
        x = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
        cb.TokenCache(x(4, 2, 16, 32), x(4, 2, 16, 32), x(2, 2, dtype=torch.int32), x(2, dtype=torch.int32))""")
    assert got.startswith("AssertionError") and "on a GPU" in got
    got = without_asserts("""
        cb.Rotary(32, (16,)).rotate(torch.zeros(0, 2, 32), torch.zeros((0, 1), dtype=torch.int32))""")
    assert got.startswith("AssertionError") and "on a GPU" in got


def test_what_a_scratch_buffer_has_to_be_is_checked_without_asserts():
    # (a stand-in for a cache: nothing here has a GPU)
    code = """
        import types
        from unittest import mock
        me = types.SimpleNamespace(scratch_bytes=lambda n: 512, _room=-1, device=torch.device("cpu"), desc=types.SimpleNamespace())
        with mock.patch.object(torch.cuda, "is_current_stream_capturing", return_value=%s):
            cb.TokenCache._scratch(me, 4, %s)"""
    got = without_asserts(code % (True, None))
    assert got.startswith("AssertionError") and "attend once before" in got
    for given in ("torch.zeros(512, dtype=torch.int32)", "torch.zeros(1024, dtype=torch.uint8)[::2]", "torch.zeros(512, dtype=torch.uint8, device='meta')"):
        got = without_asserts(code % (False, given))
        assert got.startswith("AssertionError") and "scratch" in got
    assert without_asserts(code % (False, "torch.zeros(512, dtype=torch.uint8)")) == "done"
