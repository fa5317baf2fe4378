"""The example decoder: its caches hold what they should after prompt and steps, and a layer's attention on the evicted cache
matches the float64 oracle."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from tests import attn_utils as au

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import importlib.util
    spec = importlib.util.spec_from_file_location("decode_with_cache", os.path.join(ROOT, "examples", "decode_with_cache.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("budget,prompt,window", [(64, 300, 0), (64, 40, 0), (80, 200, 50)])
def test_caches_and_attention_of_the_example(example, budget, prompt, window):
    m = example.Decoder(layers=2, budget=budget, n_sink=4, n_recent=16, window=window, observe=20)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = m.prompt(torch.randn(prompt, m.d, generator=g, device="cuda").to(m.dtype))
    for step in range(5):
        x = m.step(x)
    torch.cuda.synchronize()
    assert m.status.item() == 0 and torch.isfinite(x.float()).all()
    entries, seen = min(prompt + 5, budget), prompt + 5
    assert m.length.item() == entries and m.position.item() == seen
    for c in m.caches:
        for h in range(m.hkv):
            pos = c.pos[0, h, :entries].tolist()
            assert len(set(pos)) == entries and set(range(4)) <= set(pos) and set(range(seen - 16, seen)) <= set(pos) and max(pos) == seen - 1
    # one more token through layer 0's attention: the stored entry is the projection's, the result the oracle's
    c = m.caches[0]
    q, k, v = m.split(torch.matmul(example.norm(x), m.w_qkv[0].T))
    kk, vv, pos = c.k.clone(), c.v.clone(), c.pos.clone()
    kk[:, :, entries], vv[:, :, entries], pos[:, :, entries] = k, v, seen
    out = m.attend(0, x)
    torch.cuda.synchronize()
    ref = au.reference(q[:, None], kk, vv, [entries + 1], window, 4, m.scale, pos.cpu().numpy(), [seen])
    au.check_out(out[:, None], ref, "bf16", m.hd)
    if entries == budget:       # at the budget something had to go, and it was neither a sink nor recent
        gone = [set(pos[0, h, :entries + 1].tolist()) - set(c.pos[0, h, :budget].tolist()) for h in range(m.hkv)]
        assert all(len(s) == 1 and 4 <= min(s) < seen - 15 for s in gone)
    assert np.isfinite(c.weight[0, :, :min(entries + 1, budget)].cpu().numpy()).all()


def test_example_runs_as_a_command():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_with_cache.py"), "--prompt", "300", "--steps", "8", "--budget", "128",
                          "--layers", "2"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "cache 128 of 309 positions" in out.stdout, out.stdout + out.stderr[-1500:]
