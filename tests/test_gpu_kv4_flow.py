"""The calls on the cache in 4 bits together, as they are used: a prompt in chunks, decoding with eviction, captured and replayed,
on other streams, strided and shared memory; and the example decoder on such caches."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as ko
from tests import attn_utils as au
from tests import kv4_utils as k4
from tests.test_gpu_cache_example import example  # noqa: F401  (the module of the example, as a fixture)

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def _i(*v):
    return torch.tensor(v, **I32)


def test_a_prompt_in_chunks_and_then_tokens(api):
    """Chunks are attended to over what was stored so far, read back, and their own keys and values as they are; every chunk and
    every token against the oracle over exactly that."""
    H, Hq, D, group, chunks, steps = 2, 6, 128, 32, [45, 100, 1], 3
    cap, scale = 192, 1.0 / math.sqrt(D)
    g = torch.Generator().manual_seed(0)
    length, status = _i(0), _i(0)
    cache = api.KV4Cache.empty(1, H, cap, D, group, torch.bfloat16, length)
    cache.data.fill_(0xFF)
    k_all, v_all = (torch.zeros(1, H, cap, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))       # as they were computed
    stored = [np.zeros((1, H, cap, D)) for _ in range(2)]                                                   # what the cache stands for
    n = 0
    for T in chunks:
        wide = torch.randn(1, T, (Hq + 2 * H), D, generator=g).to(torch.bfloat16).cuda()
        q, k, v = wide[:, :, :Hq], wide[:, :, Hq:Hq + H].transpose(1, 2), wide[:, :, Hq + H:].transpose(1, 2)
        scratch = api.KVCache(*(torch.zeros(1, H, n + T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)), _i(n + T))
        if n:
            api.si_kv4_load(cache, scratch, None, n, None, status)
        scratch.k[:, :, n:], scratch.v[:, :, n:] = k, v
        out, lse = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, T, Hq, device="cuda")
        api.si_attn_prefill(scratch, q, 0, 0, scale, out, lse, scratch.workspace(Hq, T), status)
        for x, s in ((scratch.k, stored[0]), (scratch.v, stored[1])):
            assert np.array_equal(au.f64(x[:, :, :n]), ko.round16(s[:, :, :n], "bf16"))
        ref = au.reference(q, scratch.k, scratch.v, [n + T], 0, 0, scale)
        au.check_out(out, ref, "bf16", D)
        api.si_kv4_store(api.KVCache(k, v, _i(T)), cache, None, status)
        k_all[:, :, n:n + T], v_all[:, :, n:n + T] = k, v
        for s, x in zip(stored, (k, v)):
            m, st, c = ko.quantise(au.f64(x), group, "bf16")
            s[:, :, n:n + T] = m + st * c
        n += T
        length.fill_(n)
    ws = cache.workspace(Hq)
    for _ in range(steps):
        wide = torch.randn(1, Hq + 2 * H, D, generator=g).to(torch.bfloat16).cuda()
        out, lse = torch.empty(1, Hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(1, Hq, device="cuda")
        api.si_kv4_attn_decode(cache, wide[:, :Hq], None, wide[:, Hq:Hq + H], wide[:, Hq + H:], 0, 0, scale, out, lse, 0, ws, status)
        k_all[:, :, n], v_all[:, :, n] = wide[:, Hq:Hq + H], wide[:, Hq + H:]
        n += 1
        length.fill_(n)
        made = k4.Made.__new__(k4.Made)
        made.k, made.v = k_all, v_all
        made.kq, made.vq = (list(ko.quantise(au.f64(x), group, "bf16")) for x in (k_all, v_all))
        k4.check(out, lse, k4.reference(made, wide[:, :Hq], [n], 0, 0, scale), "bf16", D)
    assert status.item() == 0


@pytest.mark.parametrize("D,group,Hq,H", [(128, 32, 8, 2), (64, 64, 4, 4), (128, 64, 20, 1)])
def test_steps_at_a_budget_captured_and_replayed(api, D, group, Hq, H):
    """A step -- token, weights, eviction, lengths -- captured once and replayed gives the bits of the same steps made one by one."""
    B, budget, cap, steps = 3, 100, 128, 6

    def fresh():
        pos = torch.arange(cap, **I32).expand(B, H, cap).contiguous()
        weight = torch.rand(B, H, cap, generator=torch.Generator().manual_seed(1)).cuda()
        made = k4.Made(api, B, H, D, cap, group, "bf16", [100, 97, 3], seed=D, pos=pos, weight=weight)
        made.position = _i(100, 97, 3)
        return made

    g = torch.Generator().manual_seed(3)
    tokens = torch.randn(steps, B, Hq + 2 * H, D, generator=g).to(torch.bfloat16).cuda()

    def step(made, x, out, ws, status):
        c = made.cache
        api.si_kv4_attn_decode(c, x[:, :Hq], made.position, x[:, Hq:Hq + H], x[:, Hq + H:], 0, 0, 0.09, out, None, api.SI_FLAG_ACC_WEIGHT, ws, status)
        api.si_kv4_evict(c, c, made.position, 1, budget, 2, 8, None, c.length, ws, status)
        made.position.add_(1)

    one, status = fresh(), _i(0)
    ws = one.cache.workspace(Hq)
    outs = []
    for t in range(steps):
        outs.append(torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda"))
        step(one, tokens[t], outs[-1], ws, status)
    torch.cuda.synchronize()
    assert status.item() == 0 and one.cache.length.tolist() == [100, 100, 9]
    for b in range(B):
        for h in range(H):
            p = one.cache.pos[b, h, :one.cache.length[b]].tolist()
            assert len(set(p)) == len(p) and max(p) == one.position[b].item() - 1 and {0, 1} <= set(p)
    # two captured steps (on two models) that share one workspace, replayed in turn
    models, graphs, x = [fresh(), fresh()], [], torch.empty_like(tokens[0])
    out = torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for m in models:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(m, x, out, ws, status)
        graphs.append(graph)
    for t in range(steps):
        x.copy_(tokens[t])
        for graph in graphs:
            ws.fill_(0xA5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), outs[t].view(torch.int16))
    for m in models:
        n = one.cache.length.tolist()
        assert m.cache.length.tolist() == n and status.item() == 0
        for x1, x2 in zip(m.read(m.cache.length), one.read(one.cache.length)):
            assert torch.equal(x1.view(torch.int16), x2.view(torch.int16))
        for b in range(B):
            assert torch.equal(m.cache.pos[b, :, :n[b]], one.cache.pos[b, :, :n[b]]) and torch.equal(m.cache.weight[b, :, :n[b]], one.cache.weight[b, :, :n[b]])


def test_calls_on_a_stream_of_their_own(api):
    """Work queued on a stream that is not the current one, behind a long kernel there."""
    made = k4.Made(api, 2, 2, 128, 2048, 32, "f16", [2000, 1500], seed=5)
    q = torch.randn(2, 8, 128, device="cuda").half()
    ws, outs = made.cache.workspace(8), []
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        out = torch.empty_like(q)
        back = api.KVCache(*(torch.zeros(2, 2, 2048, 128, dtype=torch.float16, device="cuda") for _ in range(2)), made.length)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                (big @ big).sum()
        api.si_kv4_attn_decode(made.cache, q, None, None, None, 0, 0, 0.09, out, None, 0, ws, None, stream)
        api.si_kv4_load(made.cache, back, None, 2000, None, None, stream)
        torch.cuda.synchronize()
        outs.append((out, back.k, back.v))
    for other in outs[1:]:
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("D,group", [(128, 32), (64, 32)])
def test_strided_and_shared_rows(api, D, group):
    """Rows apart by more than their length, heads in front of sequences, two sequences on the same rows (read only)."""
    B, H, tiles, Hq = 2, 3, 5, 6
    tb = api.si_kv4_tile_bytes(D, group)
    big = torch.full((H, B, tiles + 2, tb), 0xFF, dtype=torch.uint8, device="cuda")
    data = big.permute(1, 0, 2, 3)[:, :, 1:1 + tiles]
    length = _i(150, 77)
    k, v = (torch.randn(B, H, 160, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = api.KV4Cache(data, D, group, torch.bfloat16, length)
    api.si_kv4_store(api.KVCache(k, v, length), api.KV4Cache(data, D, group, torch.bfloat16, _i(0, 0)))
    plain = api.KV4Cache.empty(B, H, 160, D, group, torch.bfloat16, length)
    api.si_kv4_store(api.KVCache(k, v, length), api.KV4Cache(plain.data, D, group, torch.bfloat16, _i(0, 0)))
    assert (big[:, :, 0] == 0xFF).all() and (big[:, :, -1] == 0xFF).all()
    q = torch.randn(B, Hq, D, device="cuda").to(torch.bfloat16)
    outs = []
    for c in (cache, plain):
        out = torch.empty_like(q)
        api.si_kv4_attn_decode(c, q, None, None, None, 0, 0, 0.1, out, None, 0, c.workspace(Hq))
        outs.append(out)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    # sequence 1 on the rows of sequence 0
    shared = api.KV4Cache(plain.data[:1].expand(B, -1, -1, -1), D, group, torch.bfloat16, _i(150, 150))
    out = torch.empty_like(q)
    api.si_kv4_attn_decode(shared, q, None, None, None, 0, 0, 0.1, out, None, 0, shared.workspace(Hq))
    assert torch.equal(out[0].view(torch.int16), outs[1][0].view(torch.int16))
    one = api.KV4Cache(plain.data[:1], D, group, torch.bfloat16, _i(150))
    alone = torch.empty_like(q[:1])
    api.si_kv4_attn_decode(one, q[1:], None, None, None, 0, 0, 0.1, alone, None, 0, one.workspace(Hq))
    err = (alone[0].float() - out[1].float()).abs().max().item()
    assert err <= 2 * 2.0 ** -8 * out[1].float().abs().max().item()        # other runs: one rounding of the result apart
    with pytest.raises(api.SelectInferError):
        api.si_kv4_attn_decode(shared, q, None, k[:, :, 0].contiguous(), v[:, :, 0].contiguous(), 0, 0, 0.1, out, None, 0, shared.workspace(Hq))


def test_rows_beyond_four_gigabytes(api):
    """Tiles whose offsets need more than 32 bits: the last entries of a long cache are stored, read back and attended to."""
    D, H, n = 128, 1, 27_000_000 // 32 * 32
    length = _i(n - 5)
    cache = api.KV4Cache.empty(1, H, n, D, 32, torch.bfloat16, length)
    assert cache.data.numel() > 1 << 32
    k, v = (torch.randn(1, H, 3, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    status = _i(0)
    api.si_kv4_store(api.KVCache(k, v, _i(3)), cache, None, status)
    length.fill_(n - 2)
    back = api.KVCache(torch.zeros_like(k), torch.zeros_like(v), _i(0))
    api.si_kv4_load(cache, back, _i(n - 5), 3, back.length, status)
    assert back.length.item() == 3
    for x, y in ((k, back.k), (v, back.v)):
        assert np.array_equal(au.f64(y), ko.read_back(*ko.quantise(au.f64(x), 32, "bf16"), "bf16"))
    q = torch.randn(1, 4, D, device="cuda").to(torch.bfloat16)
    new = torch.randn(2, 1, H, D, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(1, 4, device="cuda")
    api.si_kv4_attn_decode(cache, q, None, new[0], new[1], 4, 0, 0.1, out, lse, 0, cache.workspace(4), status)       # the window: the stored ones and the new one
    assert status.item() == 0
    made = k4.Made.__new__(k4.Made)
    made.k, made.v = torch.cat([k, new[0][:, :, None]], 2), torch.cat([v, new[1][:, :, None]], 2)
    made.kq, made.vq = (list(ko.quantise(au.f64(x), 32, "bf16")) for x in (made.k, made.v))
    k4.check(out, lse, k4.reference(made, q, [4], 0, 0, 0.1), "bf16", D)


@pytest.mark.parametrize("budget,prompt,window", [(64, 300, 0), (64, 40, 0), (80, 200, 50)])
def test_the_example_on_caches_in_4_bits(example, budget, prompt, window):  # noqa: F811
    m = example.Decoder(layers=2, budget=budget, n_sink=4, n_recent=16, window=window, observe=20, bits=4)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = m.prompt(torch.randn(prompt, m.d, generator=g, device="cuda").to(m.dtype))
    for _ in range(5):
        x = m.step(x)
    torch.cuda.synchronize()
    assert m.status.item() == 0 and torch.isfinite(x.float()).all()
    entries, seen = min(prompt + 5, budget), prompt + 5
    assert m.length.item() == entries and m.position.item() == seen
    for c in m.caches:
        for h in range(m.hkv):
            pos = c.pos[0, h, :entries].tolist()
            assert len(set(pos)) == entries and set(range(4)) <= set(pos) and set(range(seen - 16, seen)) <= set(pos) and max(pos) == seen - 1
    # one more token through layer 0's attention, against the oracle over what the cache held and the token's own entry in 4 bits
    from paper_2607_18081_b200 import api
    c = m.caches[0]
    q, k, v = m.split(torch.matmul(example.norm(x), m.w_qkv[0].T))
    held = api.KVCache(*(torch.zeros(1, m.hkv, c.capacity, m.hd, dtype=m.dtype, device="cuda") for _ in range(2)), m.length)
    api.si_kv4_load(c, held, None, entries, None)
    pos = c.pos.clone()
    pos[:, :, entries] = seen
    new = [ko.quantise(au.f64(t), 32, "bf16") for t in (k, v)]
    out = m.attend(0, x)
    torch.cuda.synchronize()
    kk, vv = au.f64(held.k), au.f64(held.v)
    for a, (lo, s, code) in zip((kk, vv), new):
        a[:, :, entries] = lo + s * code
    for hq in range(m.hq):
        h = hq // (m.hq // m.hkv)
        from oracle import attention_oracle as ao
        want, _, w, reach, size = ao.attend(au.f64(q[:, hq]), kk[0, h, :entries + 1], vv[0, h, :entries + 1], pos[0, h, :entries + 1].cpu().numpy(), np.array([seen]), window, 4, m.scale)
        # the values that were read back are rounded to bf16, half a step each: 2^-8 of keys (in the scores) and of values
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 * (2 * size[0] + 1) + 2.0 ** -10) * reach + 1e-6
        assert np.all(np.abs(au.f64(out[:, hq]) - want) <= bound)


def test_the_example_runs_as_a_command_in_4_bits():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode_with_cache.py"), "--prompt", "300", "--steps", "8", "--budget", "128",
                          "--layers", "2", "--bits", "4"], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "cache 128 of 309 positions" in out.stdout, out.stdout + out.stderr[-1500:]
