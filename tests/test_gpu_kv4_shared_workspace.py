"""The calls on a cache in 4 bits between multi-token FFN calls that share a workspace with them: the same bits as with
workspaces of their own, and the FFN's union stage never starts ahead of them."""
import pytest
import torch

from tests.test_gpu_shared_workspace import ROUNDS, _call, _shared, api, c1, ffn  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def _cache(api, B, H, cap, D, pos):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(B, H, cap, D, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16) for _ in range(2))
    length = torch.full((B,), cap, dtype=torch.int32, device="cuda")
    weight = torch.rand(B, H, cap, generator=g, device="cuda")
    p = torch.arange(cap, dtype=torch.int32, device="cuda").expand(B, H, cap).contiguous() if pos else None
    cache = api.KV4Cache.empty(B, H, cap, D, 32, torch.bfloat16, length, p, weight)
    wide = api.KVCache(k, v, length, p, weight.clone())
    return cache, wide, g


def test_every_call_and_a_multi_token_call(api, c1, ffn):  # noqa: F811
    B, H, Hq, cap, D, budget = 36, 8, 32, 16384, 64, 6000
    cache, wide, g = _cache(api, B, H, cap, D, True)
    start = api.KV4Cache(cache.data, D, 32, torch.bfloat16, torch.zeros_like(cache.length), cache.pos, cache.weight)
    q = torch.randn(B, Hq, D, generator=g, device="cuda").to(torch.bfloat16)
    q_pos = cache.length - 1
    ws = _shared(c1, ffn, api.si_kv4_workspace_bytes(cache, Hq))
    outs = []
    for own in (True, False):
        out, y = torch.empty_like(q), torch.empty_like(ffn[4])
        dst = api.KV4Cache.empty(B, H, 6016, D, 32, torch.bfloat16, torch.zeros_like(cache.length), torch.zeros(B, H, 6016, dtype=torch.int32, device="cuda"),
                                 torch.zeros(B, H, 6016, device="cuda"))
        dst.data.zero_()
        back = api.KVCache(*(torch.zeros(B, H, budget, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)), torch.zeros_like(cache.length))
        mine, theirs = (cache.workspace(Hq), c1.store.workspace(ffn[3], ffn[2], 1)) if own else (ws, ws)
        torch.cuda.synchronize()
        for _ in range(ROUNDS // 3):
            for call in (lambda: api.si_kv4_store(wide, start),
                         lambda: api.si_kv4_attn_decode(cache, q, q_pos, None, None, 0, 0, 0.125, out, None, api.SI_FLAG_ACC_WEIGHT, mine),
                         lambda: api.si_kv4_evict(cache, dst, q_pos, 0, budget, 4, 64, None, dst.length, mine),
                         lambda: api.si_kv4_load(dst, back, None, budget, None)):
                _call(api, c1, ffn, theirs, y)
                call()
                assert not api.si_debug_union_ahead(c1.store.handle, ffn[3], ffn[2], theirs)
        _call(api, c1, ffn, theirs, y)
        torch.cuda.synchronize()
        outs.append((out, cache.weight.clone(), dst.pos, dst.weight, dst.length, dst.data, back.k, back.v, y))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert torch.equal(outs[0][-1], ffn[4])
