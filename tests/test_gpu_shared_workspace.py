"""Calls of different kinds that share one workspace in stream order, with nothing between them: the same bits as with
workspaces of their own.  Multi-token FFN calls may start their union stage while the kernel ahead still runs; behind
anything that still uses the workspace (or writes a list) they must not."""
import numpy as np
import pytest
import torch

from paper_2607_18081_b200 import workloads as wl
from tests.gpu_utils import LoadedModel, assert_close, from_dev, to_dev

pytestmark = pytest.mark.gpu
ROUNDS = 12


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


@pytest.fixture(scope="module")
def c1(api):
    return LoadedModel(wl.CONFIGS["c1"])


@pytest.fixture(scope="module")
def ffn(api, c1):
    """Arguments of a 16-token call with lists of its own, and its result in a workspace of its own."""
    cfg, T = c1.cfg, 16
    k = cfg.k_active
    lists = wl.zipf_lists(cfg, 0, T, slot_of_rank=c1.slot_of_rank[0])
    x, idx = to_dev(wl.x_tokens(cfg, 0, T), cfg.dtype), torch.from_numpy(np.ascontiguousarray(lists, np.int32)).cuda()
    y = torch.empty(T, cfg.d_model, dtype=torch.float32, device="cuda")
    api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, y, 0, c1.store.workspace(T, k, 1))
    torch.cuda.synchronize()
    return x, idx, k, T, y


def _call(api, c1, ffn, ws, y):
    x, idx, k, T, _ = ffn
    api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, y, 0, ws)


def _cache(api, B, H, cap, D, pos):
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(B, H, cap, D, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16) for _ in range(2))
    length = torch.full((B,), cap, dtype=torch.int32, device="cuda")
    weight = torch.rand(B, H, cap, generator=g, device="cuda")
    p = torch.arange(cap, dtype=torch.int32, device="cuda").expand(B, H, cap).contiguous() if pos else None
    return api.KVCache(k, v, length, p, weight), g


def _shared(c1, ffn, need):
    """One buffer for both: the FFN's union stage lies behind 64 MB of it, so the cache's scratch has to reach there."""
    assert need > 66 << 20
    size = max(need, c1.store.workspace(ffn[3], ffn[2], 1).numel())
    return torch.zeros(size, dtype=torch.uint8, device="cuda")


def test_decode_then_a_multi_token_call(api, c1, ffn):
    B, H, Hq, cap, D = 36, 8, 32, 16384, 64
    cache, g = _cache(api, B, H, cap, D, False)
    q = torch.randn(B, Hq, D, generator=g, device="cuda").to(torch.bfloat16)
    ws = _shared(c1, ffn, api.si_kv_workspace_bytes(cache, Hq, 1))
    start = cache.weight.clone()
    outs = []
    for own in (True, False):
        cache.weight.copy_(start)
        out, y = torch.empty_like(q), torch.empty_like(ffn[4])
        mine, theirs = (cache.workspace(Hq, 1), c1.store.workspace(ffn[3], ffn[2], 1)) if own else (ws, ws)
        torch.cuda.synchronize()
        for _ in range(ROUNDS):
            _call(api, c1, ffn, theirs, y)
            api.si_attn_decode(cache, q, None, None, None, 0, 0, 0.125, out, None, api.SI_FLAG_ACC_WEIGHT, mine)
            assert not api.si_debug_union_ahead(c1.store.handle, ffn[3], ffn[2], theirs)
        _call(api, c1, ffn, theirs, y)
        torch.cuda.synchronize()
        outs.append((out, cache.weight.clone(), y))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert torch.equal(outs[0][2], ffn[4])


def test_eviction_then_a_multi_token_call(api, c1, ffn):
    B, H, cap, D, budget = 72, 8, 16384, 64, 6000
    cache, _ = _cache(api, B, H, cap, D, True)
    ws = _shared(c1, ffn, api.si_kv_workspace_bytes(cache, 0, 0))
    q_pos = cache.length - 1
    keep = [t.clone() for t in (cache.k, cache.v, cache.pos, cache.weight)]
    outs = []
    for own in (True, False):
        dk, dv = (torch.zeros(B, H, budget, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dst = api.KVCache(dk, dv, torch.zeros_like(cache.length), torch.zeros(B, H, budget, dtype=torch.int32, device="cuda"),
                          torch.zeros(B, H, budget, device="cuda"))
        y = torch.empty_like(ffn[4])
        mine, theirs = (cache.workspace(0, 0), c1.store.workspace(ffn[3], ffn[2], 1)) if own else (ws, ws)
        torch.cuda.synchronize()
        for r in range(ROUNDS):                            # by turns into another cache (two kernels) and, few over the budget, in place (one)
            _call(api, c1, ffn, theirs, y)
            api.si_kv_evict(cache, dst, q_pos, 0, budget, 4, 64, None, dst.length, mine)
            assert not api.si_debug_union_ahead(c1.store.handle, ffn[3], ffn[2], theirs)
            _call(api, c1, ffn, theirs, y)
            api.si_kv_evict(cache, cache, q_pos, 0, cap - 200 + 10 * r, 4, 64, None, None, mine)
        _call(api, c1, ffn, theirs, y)
        torch.cuda.synchronize()
        outs.append((dk, dv, dst.pos, dst.weight, dst.length, cache.k.clone(), cache.v.clone(), cache.pos.clone(), cache.weight.clone(), y))
        for t, s in zip((cache.k, cache.v, cache.pos, cache.weight), keep):
            t.copy_(s)
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert torch.equal(outs[0][-1], ffn[4])


def test_prefill_and_weights_then_a_multi_token_call(api, c1, ffn):
    cache, g = _cache(api, 1, 2, 9000, 128, False)
    q = torch.randn(1, 20, 8, 128, generator=g, device="cuda").to(torch.bfloat16)
    ws = torch.zeros(max(api.si_kv_workspace_bytes(cache, 8, 20), c1.store.workspace(ffn[3], ffn[2], 1).numel()), dtype=torch.uint8, device="cuda")
    start, outs = cache.weight.clone(), []
    for own in (True, False):
        cache.weight.copy_(start)
        out, lse, y = torch.empty_like(q), torch.empty(1, 20, 8, device="cuda"), torch.empty_like(ffn[4])
        mine, theirs = (cache.workspace(8, 20), c1.store.workspace(ffn[3], ffn[2], 1)) if own else (ws, ws)
        torch.cuda.synchronize()
        for _ in range(ROUNDS):
            api.si_attn_prefill(cache, q, 0, 0, 0.09, out, lse, mine)
            assert not api.si_debug_union_ahead(c1.store.handle, ffn[3], ffn[2], theirs)
            _call(api, c1, ffn, theirs, y)
            api.si_attn_weights(cache, q, 0, 0, 0.09, lse, mine)
            assert not api.si_debug_union_ahead(c1.store.handle, ffn[3], ffn[2], theirs)
            _call(api, c1, ffn, theirs, y)
        torch.cuda.synchronize()
        outs.append((out, lse, cache.weight.clone(), y))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_multi_token_calls_of_different_sizes_in_one_workspace(api, c1):
    """Another token count is another layout of the workspace: the next call's union stage may not run beside the call before."""
    cfg = c1.cfg
    k, sizes = cfg.k_active, [17, 16, 100, 3, 200, 33, 2, 130, 16, 16, 15]
    ws = c1.store.workspace(max(sizes), k, 1)
    args = []
    for T in sizes:
        lists = np.ascontiguousarray(wl.zipf_lists(cfg, 0, T, slot_of_rank=c1.slot_of_rank[0]), np.int32)
        args.append((T, to_dev(wl.x_tokens(cfg, 0, T), cfg.dtype), torch.from_numpy(lists).cuda()))
    want = []
    for T, x, idx in args:
        y = torch.empty(T, cfg.d_model, dtype=torch.float32, device="cuda")
        api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, y, 0, c1.store.workspace(T, k, 1))
        torch.cuda.synchronize()
        want.append(y)
    got = [torch.empty_like(y) for y in want]
    torch.cuda.synchronize()
    before = None
    for _ in range(ROUNDS):
        for (T, x, idx), y in zip(args, got):
            assert api.si_debug_union_ahead(c1.store.handle, T, k, ws) == (T == before)
            api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, y, 0, ws)
            before = T
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_lists_selected_right_in_front_of_a_multi_token_call(api, c1):
    """si_select's kernel lets its dependents start before it has written the list: the call behind it has to wait for it."""
    cfg, T = c1.cfg, 16
    k = cfg.k_active
    sc = wl.scores(cfg, 0, 6 + T)
    x_bits = wl.x_tokens(cfg, 0, T)
    x, y = to_dev(x_bits, cfg.dtype), torch.empty(T, cfg.d_model, dtype=torch.float32, device="cuda")
    ws, sel_ws = c1.store.workspace(T, k, 1), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    idx = torch.zeros(k, dtype=torch.int32, device="cuda")
    n_out = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = [torch.from_numpy(sc[r].copy()).cuda() for r in range(6)]
    more = torch.from_numpy(sc[6:].copy()).cuda()
    ys = []
    torch.cuda.synchronize()
    for r in range(6):
        api.si_select(rows[r], api.SI_SELECT_TOPK, k, 0.0, 0, idx, n_out, sel_ws)
        assert not api.si_debug_union_ahead(c1.store.handle, T, k, ws)
        api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, y, api.SI_FLAG_SHARED_LIST, ws)
        ys.append(y.clone())
    for _ in range(3):
        api.si_layer_forward(c1.store.handle, 0, x, T, more, k, None, None, y, 0, ws)
    torch.cuda.synchronize()
    from oracle import selectinfer_oracle as so
    for r in range(6):
        sel = so.select_topk(sc[r], k)
        for t in (0, T - 1):
            assert_close(from_dev(ys[r][t]), c1.oracle_y(0, x_bits[t], sel), (r, t))
    for t in range(T):
        assert_close(from_dev(y[t]), c1.oracle_y(0, x_bits[t], so.select_topk(sc[6 + t], k)), t)


def test_calls_captured_into_a_graph_alternate_and_match(api, c1, ffn):
    ws = c1.store.workspace(ffn[3], ffn[2], 1)
    y = [torch.zeros_like(ffn[4]) for _ in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    x, idx, k, T, want = ffn
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for i, o in enumerate(y):
            assert api.si_debug_union_ahead(c1.store.handle, T, k, ws, stream=s) == (i > 0)
            api.si_ffn_forward(c1.store.handle, 0, x, T, idx, None, k, o, 0, ws, stream=s)
    assert not api.si_debug_union_ahead(c1.store.handle, T, k, ws, stream=s)      # the capture is over
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for o in y:
        assert torch.equal(o, want)
