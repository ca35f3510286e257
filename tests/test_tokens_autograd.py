"""How the token operators stand to torch's modes, as far as it shows without a GPU."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code):
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    return r.stdout.strip()


def test_the_package_is_imported_in_inference_mode():
    assert run("import torch\nwith torch.inference_mode():\n    import paper_1808_05488_amd as cb\nprint(cb.Rotary(32, (16,)).head_dim)") == "32"


def test_an_import_makes_no_tensors():
    # (where there is no GPU one on it would raise, where there is one it would initialise it)
    assert run("import torch\ntorch.set_default_device('cuda')\nimport paper_1808_05488_amd\nprint(torch.cuda.is_initialized())") == "False"


def test_tensors_with_a_tangent_are_refused_before_anything_is_read():
    got = run("""
import types
import torch
import torch.autograd.forward_ad as fw
import paper_1808_05488_amd as cb
rot, one, pos = cb.Rotary(16, (8,)), torch.ones(16), torch.zeros((2, 1), dtype=torch.int32)
me = types.SimpleNamespace()                     # (a stand-in for a cache: nothing here has a GPU)
x = torch.ones(2, 3, 16)
calls = lambda d, w: (lambda: rot.rotate(d, pos), lambda: rot.rotate(x, pos, k=d), lambda: rot.rotate(x, pos, q_out=d), lambda: rot.norm_rotate(d, pos, one),
                      lambda: rot.norm_rotate(x, pos, w), lambda: rot.norm_rotate(x, pos, one, k=d, k_weight=one), lambda: rot.norm_rotate(x, pos, one, k=x, k_weight=w),
                      lambda: rot.norm_rotate(x, pos, one, q_out=d), lambda: cb.TokenCache.append(me, d, x), lambda: cb.TokenCache.append(me, x, d),
                      lambda: cb.TokenCache.append(me, x, x, q=d), lambda: cb.TokenCache.append(me, x, x, q=x, q_out=d), lambda: cb.TokenCache.attend(me, d),
                      lambda: cb.TokenCache.attend(me, x, out=d), lambda: cb.TokenCache.attend(me, x, lse=d), lambda: cb.TokenCache.choose(me, d, 1))
n = 0
with fw.dual_level():
    for call in calls(fw.make_dual(x, x), fw.make_dual(one, one)):
        try:
            call()
        except AssertionError as e:
            n += 'forward-mode' in str(e)
        except Exception as e:
            print(type(e), e)
    # a graph of such tensors is refused by torch
    try:
        rot.norm_rotate(fw.make_dual(x.clone().requires_grad_(), x), pos, one)
    except (AssertionError, NotImplementedError):
        n += 1
    # and one without a tangent gets as far as to what it needs
    try:
        rot.rotate(x, pos)
    except AssertionError as e:
        n += 'on a GPU' in str(e)
print(n)""")
    assert got == "18"
