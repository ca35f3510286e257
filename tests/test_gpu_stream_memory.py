"""The example's stream memory: every frame's answer against the same steps in float64 on the host, from the tokens that the
trunk's list names; the cache stays within its budget, its lists and weights are the ones that the definition keeps."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def example():
    spec = importlib.util.spec_from_file_location("stream_memory", os.path.join(ROOT, "examples", "stream_memory.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_frames_of_a_stream(dtype):
    ex = example()
    budget, window = 300, 2
    mem = ex.StreamMemory(96, 128, budget, window=window, dtype=dtype)
    c, plan = mem.cache, mem.rotary.plan
    pairs = [plan.desc.pairs[a] for a in range(3)]
    n = sum(pairs)
    axis = np.repeat(np.arange(3), pairs)
    freq = 10000.0 ** (-np.arange(n) / n)

    def turned(x, pos):
        angle = pos[:, axis] * freq
        y, cos, sin = x.copy(), np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[..., :n], y[..., n:2 * n] = x[..., :n] * cos - x[..., n:2 * n] * sin, x[..., :n] * sin + x[..., n:2 * n] * cos
        return y

    def held(pages, length):
        p, table = pages.float().cpu().double().numpy(), c.table.cpu().numpy()[0]
        return np.stack([p[table[j // 64], :, j % 64] for j in range(length)], 1) if length else np.zeros((mem.heads, 0, mem.head_dim))

    u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    for t, image in enumerate(ex.video(96, 128, 7, dtype)):
        before = int(c.lengths[0])
        k0, v0 = held(c.k_pages, before), held(c.v_pages, before)
        w0, t0 = c.weight.cpu().numpy()[0].astype(np.float64), c.time.cpu().numpy()[0].copy()
        answer, lse = mem.step(image)
        torch.cuda.synchronize()
        count = int(mem.count)
        pixel = mem.listed[:count].long().cpu().numpy()
        assert (np.diff(pixel) > 0).all()
        length = before + count
        assert int(c.lengths[0]) == min(length, budget)
        # what was attended over: the tokens that were there, and the new ones, read back where they were put or moved to
        pos = np.stack([np.full(count, t), pixel // mem.w, pixel % mem.w], 1)
        q = turned(mem.query.float().cpu().double().numpy(), np.array([[t, mem.h // 2, mem.w // 2]]))[0]
        q = torch.from_numpy(q).to(dtype).double().numpy()
        new = new_tokens(mem, pixel)
        kn = torch.from_numpy(turned(new[0], pos)).to(dtype).double().numpy()
        k = np.concatenate([k0, kn.transpose(1, 0, 2)], 1)
        v = np.concatenate([v0, new[1].transpose(1, 0, 2)], 1)
        group = q.shape[0] // mem.heads
        for h in range(mem.heads):
            x = q[h * group:(h + 1) * group] @ k[h].T / math.sqrt(mem.head_dim)
            z = np.logaddexp.reduce(x, 1)
            p = np.exp(x - z[:, None])
            want = p @ v[h]
            # a rounding of the query, of the new keys, and of the answer, each of a score's size or the value's
            es = 4 * u * (np.abs(q[h * group:(h + 1) * group]) @ np.abs(k[h]).T).max() / math.sqrt(mem.head_dim)
            tol = (2 * es + 64 * 2.0 ** -24) * (p @ np.abs(v[h])) + 2 * u * np.abs(want)
            got = answer[0, h * group:(h + 1) * group].float().cpu().double().numpy()
            assert (np.abs(got - want) <= tol).all(), (t, h)
            assert np.allclose(lse[0, h * group:(h + 1) * group].cpu().numpy(), z, atol=es + 1e-5)
            # and what is kept: the weights and times of the tokens that the definition keeps, up to ties within rounding
            weight = np.concatenate([w0[h, :before], np.zeros(count)]) * 0.95 + p.sum(0)
            time = np.concatenate([t0[h, :before], np.full(count, t)])
            kept = np.sort(c.time.cpu().numpy()[0, h, :min(length, budget)])
            recent = time > t - window
            if length > budget:
                if recent.sum() >= budget:
                    assert (kept == np.sort(np.sort(time)[-budget:])).all()
                else:
                    assert (kept > t - window).sum() == recent.sum()
                    rest = np.sort(c.weight.cpu().numpy()[0, h, :budget][c.time.cpu().numpy()[0, h, :budget] <= t - window])
                    best = np.sort(weight[~recent])[len(weight[~recent]) - len(rest):]
                    assert np.allclose(rest, best, rtol=4 * es + 1e-5, atol=1e-6)


def new_tokens(mem, pixel):
    """(keys, values) of the listed pixels before rotation, as the example projects them."""
    out = mem.net.layers[-1]
    features = torch.empty((out.O, out.Ho, out.Wo), dtype=mem.dtype, device="cuda")
    state = torch.empty((out.C, out.H, out.W), dtype=mem.dtype, device="cuda")
    from paper_1808_05488_amd import binding
    binding.cb_layer_export_state(out.handle, state, features)
    torch.cuda.synchronize()
    every = mem.listed.long().clamp(0, mem.h * mem.w - 1)
    tokens = features.reshape(out.O, -1)[:, every].t() @ mem.to_kv
    kv = tokens[:len(pixel)].view(-1, 2, mem.heads, mem.head_dim).double().cpu().numpy()
    return kv[:, 0], kv[:, 1]
