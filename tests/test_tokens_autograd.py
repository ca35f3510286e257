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
