"""GPU parity of attention over the key/value cache -- prefill, single token, accumulated weights -- against the float64
oracle, within the bounds of attn_utils."""
import math

import numpy as np
import pytest
import torch

from tests import attn_utils as au

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def _prefill(api, q, k, v, length, window, n_sink, scale, weight=None):
    cache = api.KVCache(k, v, length, None, weight)
    B, T, Hq, D = q.shape
    out = torch.full((B, T, Hq, D), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((B, T, Hq), 7.0, dtype=torch.float32, device="cuda")
    ws = cache.workspace(Hq, T)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.si_attn_prefill(cache, q, window, n_sink, scale, out, lse, ws, status)
    if weight is not None:
        api.si_attn_weights(cache, q, window, n_sink, scale, lse, ws, status)
    torch.cuda.synchronize()
    assert status.item() == 0
    return out, lse


PREFILL = [
    # B, T, lens, Hq, Hkv, D, window, n_sink
    (1, 1, [1], 1, 1, 64, 0, 0),
    (1, 1, [300], 4, 1, 128, 0, 0),
    (2, 5, [5, 3], 8, 2, 128, 0, 0),             # the second sequence is shorter than T: rows that see nothing
    (1, 33, [33], 3, 1, 64, 0, 0),               # three query heads to a key head
    (2, 130, [130, 257], 6, 2, 128, 0, 0),
    (1, 200, [333], 7, 1, 64, 17, 3),
    (1, 129, [129], 2, 2, 128, 1, 0),            # a window of one: every query sees itself only
    (2, 300, [300, 511], 4, 2, 64, 128, 130),    # more sinks than the window is long
    (3, 64, [0, 64, 1000], 4, 4, 128, 100, 4),   # an empty sequence
    (1, 515, [1027], 8, 1, 128, 256, 1),
    (1, 700, [700], 5, 1, 64, 0, 0),
    (1, 40, [2100], 32, 4, 128, 0, 0),           # few rows, a long axis
    (1, 3, [1500], 128, 1, 64, 0, 0),            # 128 query heads on one key head
    (1, 260, [900], 1, 1, 128, 300, 64),
    (2, 30, [0, 2500], 8, 2, 128, 0, 0),         # keys split over CTAs, an empty sequence beside a long one
    (1, 20, [3000], 8, 2, 64, 1500, 5),          # ... with a window and sinks
    (1, 1, [5000], 12, 4, 128, 0, 0),
]


@pytest.mark.parametrize("B,T,lens,Hq,Hkv,D,window,n_sink", PREFILL)
@pytest.mark.parametrize("dtype,order", [("bf16", "hnd"), ("f16", "nhd")])
def test_prefill_and_weights(api, B, T, lens, Hq, Hkv, D, window, n_sink, dtype, order):
    scale = 1.0 / math.sqrt(D)
    cap = max(lens) + 9
    q, k, v, length = au.make(B, Hq, Hkv, D, cap, dtype, order, T, 11 * T + D, lens)
    before = np.random.default_rng(T).random((B, Hkv, cap)).astype(np.float32)
    weight = torch.from_numpy(before).cuda()
    out, lse = _prefill(api, q, k, v, length, window, n_sink, scale, weight)
    ref = au.reference(q, k, v, lens, window, n_sink, scale)
    au.check_out(out, ref, dtype, D)
    au.check_lse(lse, ref, D)
    au.check_weight(weight, before.astype(np.float64), ref, D, T)


def test_prefill_with_scores_far_apart_and_negative_scale(api):
    """Scores of several hundred: the running maximum moves a lot, most weights vanish; a negative scale turns the order."""
    for scale in (2.0, -0.7):
        q, k, v, length = au.make(1, 4, 2, 64, 400, "bf16", "hnd", 150, 5, [390], spread=4.0)
        k[:, :, :390] *= torch.linspace(0.1, 3.0, 390, device="cuda", dtype=k.dtype)[None, None, :, None]   # the maximum keeps growing
        out, lse = _prefill(api, q, k, v, length, 0, 0, scale)
        ref = au.reference(q, k, v, [390], 0, 0, scale)
        au.check_out(out, ref, "bf16", 64)
        au.check_lse(lse, ref, 64)


def test_prefill_is_repeatable_and_leaves_the_cache_alone(api):
    q, k, v, length = au.make(2, 8, 2, 128, 700, "bf16", "nhd", 400, 3, [700, 555])
    k0, v0 = k.clone(), v.clone()
    a, la = _prefill(api, q, k, v, length, 200, 4, 0.09)
    for _ in range(3):
        b, lb = _prefill(api, q, k, v, length, 200, 4, 0.09)
        assert torch.equal(a, b) and torch.equal(la, lb)
    assert torch.equal(k.view(torch.int16), k0.view(torch.int16)) and torch.equal(v.view(torch.int16), v0.view(torch.int16))


DECODE = [
    # B, lens, Hq, Hkv, D, window, n_sink, positions given, new entry
    (1, [0], 4, 1, 128, 0, 0, False, True),        # the very first token
    (1, [1], 1, 1, 64, 0, 0, False, False),
    (2, [0, 5], 8, 2, 64, 0, 0, False, False),     # an empty cache: nothing to see
    (3, [6, 16, 17], 8, 2, 128, 0, 0, False, True),
    (4, [15, 127, 128, 129], 4, 4, 128, 0, 0, False, True),
    (2, [1000, 31], 24, 8, 128, 0, 0, False, True),
    (2, [777, 2500], 16, 2, 64, 100, 4, False, True),
    (1, [5000], 32, 8, 128, 0, 0, False, True),
    (2, [900, 901], 7, 1, 128, 64, 70, False, True),
    (1, [600], 20, 1, 64, 0, 0, False, True),      # more query heads to a key head than one matrix tile holds
    (2, [400, 333], 8, 2, 128, 0, 0, True, True),
    (2, [400, 2333], 4, 2, 64, 150, 8, True, True),
    (2, [300, 20], 8, 4, 128, 90, 2, True, False),
    (40, [3 + 37 * i for i in range(40)], 4, 2, 64, 0, 0, False, True),
    (1, [3000], 128, 1, 64, 0, 0, False, True),
]


@pytest.mark.parametrize("B,lens,Hq,Hkv,D,window,n_sink,given,new", DECODE)
@pytest.mark.parametrize("dtype,order,acc", [("bf16", "hnd", True), ("f16", "nhd", False), ("bf16", "nhd", True)])
def test_decode(api, B, lens, Hq, Hkv, D, window, n_sink, given, new, dtype, order, acc):
    scale = 1.0 / math.sqrt(D)
    cap = max(lens) + 5
    q, k, v, length = au.make(B, Hq, Hkv, D, cap, dtype, order, 1, 7 * Hq + D, lens)
    rng = np.random.default_rng(B + Hq)
    before = rng.random((B, Hkv, cap)).astype(np.float32)
    weight = torch.from_numpy(before).cuda()
    pos = q_pos = None
    if given:   # positions with gaps, in no order, other ones per head; the query's is the newest
        q_pos = torch.tensor([2 * n + 1 for n in lens], dtype=torch.int32, device="cuda")
        pos = torch.full((B, Hkv, cap), -5, dtype=torch.int32)
        for b, n in enumerate(lens):
            for h in range(Hkv):
                pos[b, h, :n] = torch.from_numpy(rng.permutation(2 * n + 1)[:n].astype(np.int32))
        pos = pos.cuda()
    wide = torch.randn(B, 3 * Hkv * D, device="cuda").to(q.dtype)
    kn, vn = wide[:, :Hkv * D].view(B, Hkv, D), wide[:, Hkv * D:2 * Hkv * D].view(B, Hkv, D)
    cache = api.KVCache(k, v, length, pos, weight)
    out = torch.full((B, Hq, D), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((B, Hq), 7.0, dtype=torch.float32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k0, v0 = k.clone(), v.clone()
    api.si_attn_decode(cache, q[:, 0], q_pos, kn if new else None, vn if new else None, window, n_sink, scale, out, lse,
                       api.SI_FLAG_ACC_WEIGHT if acc else 0, cache.workspace(Hq, 1), status)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert length.tolist() == list(lens)
    total = [n + 1 if new else n for n in lens]
    start = before.astype(np.float64)
    for b, n in enumerate(lens):
        if new:
            k0[b, :, n], v0[b, :, n] = kn[b], vn[b]
            if acc:
                start[b, :, n] = 0.0
            if given:
                assert pos[b, :, n].tolist() == [int(q_pos[b])] * Hkv
    assert torch.equal(k.view(torch.int16), k0.view(torch.int16)) and torch.equal(v.view(torch.int16), v0.view(torch.int16))
    ref = au.reference(q, k, v, total, window, n_sink, scale, None if pos is None else pos.cpu().numpy(), None if q_pos is None else q_pos.tolist())
    au.check_out(out[:, None], ref, dtype, D)
    au.check_lse(lse[:, None], ref, D)
    if acc:
        au.check_weight(weight, start, ref, D, 1)
    else:
        assert np.array_equal(weight.cpu().numpy(), before)


def test_decode_ignores_what_hidden_entries_hold(api):
    """NaN and infinities in entries outside the window or after the query, and beyond the length, never reach the result."""
    for D, Hq, Hkv in ((64, 8, 2), (128, 3, 1)):
        n, window, n_sink = 700, 50, 3
        q, k, v, length = au.make(1, Hq, Hkv, D, 720, "bf16", "hnd", 1, 1, [n])
        ref = au.reference(q, k, v, [n], window, n_sink, 0.1)
        k[:, :, n_sink:n - window], v[:, :, n_sink:n - window] = float("inf"), float("nan")
        cache = api.KVCache(k, v, length)
        out = torch.empty(1, Hq, D, dtype=q.dtype, device="cuda")
        lse = torch.empty(1, Hq, dtype=torch.float32, device="cuda")
        api.si_attn_decode(cache, q[:, 0], None, None, None, window, n_sink, 0.1, out, lse, 0, cache.workspace(Hq, 1))
        au.check_out(out[:, None], ref, "bf16", D)
        au.check_lse(lse[:, None], ref, D)
        # the same with positions: every third entry lies after the query
        pos = torch.arange(720, dtype=torch.int32, device="cuda").expand(1, Hkv, 720).contiguous()
        pos[..., ::3] += 5000
        q2, k2, v2, _ = au.make(1, Hq, Hkv, D, 720, "bf16", "hnd", 1, 2, [n])
        q_pos = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
        ref = au.reference(q2, k2, v2, [n], 0, 0, 0.1, pos.cpu().numpy(), [n - 1])
        k2[:, :, ::3], v2[:, :, ::3] = float("nan"), float("inf")
        cache = api.KVCache(k2, v2, length, pos)
        api.si_attn_decode(cache, q2[:, 0], q_pos, None, None, 0, 0, 0.1, out, lse, 0, cache.workspace(Hq, 1))
        au.check_out(out[:, None], ref, "bf16", D)
        au.check_lse(lse[:, None], ref, D)


def test_new_entries_that_their_query_does_not_see_are_stored_all_the_same(api):
    """Entries without positions and a query position of the caller's: before the entry, far behind it (a window between), at it."""
    lens, at, window, D = [100, 100, 100, 50], [40, 300, 100, 49], 64, 128
    q, k, v, length = au.make(4, 4, 2, D, 120, "bf16", "nhd", 1, 12, lens)
    kn, vn = (torch.randn(4, 2, D, device="cuda").to(q.dtype) for _ in range(2))
    q_pos = torch.tensor(at, dtype=torch.int32, device="cuda")
    cache = api.KVCache(k, v, length)
    out = torch.empty(4, 4, D, dtype=q.dtype, device="cuda")
    lse = torch.empty(4, 4, dtype=torch.float32, device="cuda")
    api.si_attn_decode(cache, q[:, 0], q_pos, kn, vn, window, 0, 0.1, out, lse, 0, cache.workspace(4, 1))
    for b, n in enumerate(lens):
        assert torch.equal(k[b, :, n], kn[b]) and torch.equal(v[b, :, n], vn[b])
    ref = au.reference(q, k, v, [n + 1 for n in lens], window, 0, 0.1, np.broadcast_to(np.arange(120), (4, 2, 120)), at)
    au.check_out(out[:, None], ref, "bf16", D)
    au.check_lse(lse[:, None], ref, D)


def test_decode_equals_prefill_of_one_token_and_is_repeatable(api):
    q, k, v, length = au.make(3, 16, 4, 128, 1300, "f16", "nhd", 1, 9, [1300, 64, 801])
    cache = api.KVCache(k, v, length)
    res = []
    for _ in range(3):
        out = torch.empty(3, 16, 128, dtype=q.dtype, device="cuda")
        api.si_attn_decode(cache, q[:, 0], None, None, None, 500, 2, 0.08, out, None, 0, cache.workspace(16, 1))
        res.append(out)
    assert torch.equal(res[0], res[1]) and torch.equal(res[0], res[2])
    ref = au.reference(q, k, v, [1300, 64, 801], 500, 2, 0.08)
    au.check_out(res[0][:, None], ref, "f16", 128)
    out, _ = _prefill(api, q, k, v, length, 500, 2, 0.08)
    au.check_out(out, ref, "f16", 128)


def test_caches_whose_offsets_pass_32_bits(api):
    """Entries more than 2^32 elements apart: a token-major cache of one sequence with a row stride of 2^22 elements."""
    D, rs, n = 64, 1 << 22, 1100
    mem = torch.zeros(2, (n - 1) * rs + 4 * D, dtype=torch.bfloat16, device="cuda") if torch.cuda.mem_get_info()[0] > 40 << 30 else None
    if mem is None:
        pytest.skip("needs 40 GB free")
    k, v = (m.as_strided((1, 2, n, D), (0, 2 * D, rs, 1)) for m in mem)
    g = torch.Generator(device="cuda").manual_seed(1)
    k.copy_(torch.randn(1, 2, n, D, generator=g, device="cuda")); v.copy_(torch.randn(1, 2, n, D, generator=g, device="cuda"))
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 70, 8, D, generator=g, device="cuda").to(torch.bfloat16)
    weight = torch.zeros(1, 2, n, device="cuda")
    ref = au.reference(q, k, v, [n], 0, 0, 0.125)
    out, lse = _prefill(api, q, k, v, length, 0, 0, 0.125, weight)
    au.check_out(out, ref, "bf16", D)
    au.check_weight(weight, np.zeros((1, 2, n)), ref, D, 70)
    cache = api.KVCache(k, v, length)
    o1 = torch.empty(1, 8, D, dtype=q.dtype, device="cuda")
    api.si_attn_decode(cache, q[:, -1], None, None, None, 0, 0, 0.125, o1, None, 0, cache.workspace(8, 1))
    last = {x: ref[x][:, -1:] for x in ("out", "reach", "lse", "size", "n")}
    au.check_out(o1[:, None], last, "bf16", D)


@pytest.mark.parametrize("D,order", [(128, "hnd"), (64, "nhd")])
def test_sequences_that_share_one_cache_through_a_zero_stride(api, D, order):
    """Every sequence of the batch reads the same keys and values (expand: a stride of zero), at lengths of its own."""
    lens, Hq, Hkv, T, cap = [400, 150, 399], 8, 2, 37, 410
    q, k, v, _ = au.make(1, Hq, Hkv, D, cap, "bf16", order, T, 8, [cap])
    k, v = k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1)
    q = torch.cat([q, q.flip(1), -q]).contiguous()
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    weight = torch.zeros(3, Hkv, cap, device="cuda")
    out, lse = _prefill(api, q, k, v, length, 0, 0, 0.1, weight)
    ref = au.reference(q, k, v, lens, 0, 0, 0.1)
    au.check_out(out, ref, "bf16", D)
    au.check_lse(lse, ref, D)
    au.check_weight(weight, np.zeros(weight.shape), ref, D, T)
    cache = api.KVCache(k, v, length)
    o1 = torch.empty(3, Hq, D, dtype=q.dtype, device="cuda")
    api.si_attn_decode(cache, q[:, -1], None, None, None, 0, 0, 0.1, o1, None, 0, cache.workspace(Hq, 1))
    au.check_out(o1[:, None], {x: ref[x][:, -1:] for x in ("out", "reach", "lse", "size", "n")}, "bf16", D)


def test_prefill_weights_and_eviction_in_one_graph(api):
    lens = [300, 170]
    q, k, v, length = au.make(2, 8, 2, 128, 320, "bf16", "nhd", 60, 6, lens)
    weight = torch.zeros(2, 2, 320, device="cuda")
    src = api.KVCache(k, v, length, None, weight)
    dk, dv = (torch.zeros(2, 2, 64, 128, dtype=q.dtype, device="cuda") for _ in range(2))
    dst = api.KVCache(dk, dv, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.int32, device="cuda"),
                      torch.zeros(2, 2, 64, device="cuda"))
    out, lse = torch.empty(2, 60, 8, 128, dtype=q.dtype, device="cuda"), torch.empty(2, 60, 8, device="cuda")
    ws = src.workspace(8, 60)

    def calls(stream=None):
        weight.zero_()
        api.si_attn_prefill(src, q, 0, 0, 0.09, out, lse, ws, stream=stream)
        api.si_attn_weights(src, q, 0, 0, 0.09, lse, ws, stream=stream)
        api.si_kv_evict(src, dst, None, 0, 64, 4, 8, None, dst.length, ws, stream=stream)

    calls()
    torch.cuda.synchronize()
    first = [t.clone() for t in (out, lse, weight, dk, dv, dst.pos, dst.weight)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls(s)
    for t in (out, lse, dk, dv, dst.pos, dst.weight):
        t.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert dst.length.tolist() == [64, 64]
    for a, b in zip(first, (out, lse, weight, dk, dv, dst.pos, dst.weight)):
        assert torch.equal(a, b)
    ref = au.reference(q, k, v, lens, 0, 0, 0.09)
    au.check_out(out, ref, "bf16", 128)
    au.check_weight(weight, np.zeros(weight.shape), ref, 128, 60)


def test_lengths_outside_the_capacity_and_a_full_cache_are_reported(api):
    q, k, v, _ = au.make(2, 4, 2, 64, 64, "bf16", "hnd", 1, 1, [64, 64])
    out = torch.empty(2, 4, 64, dtype=q.dtype, device="cuda")
    kn = torch.zeros(2, 2, 64, dtype=q.dtype, device="cuda")
    for lens, new in (([65, 3], None), ([-1, 3], None), ([64, 3], kn)):
        length = torch.tensor(lens, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache = api.KVCache(k, v, length)
        k0 = k.clone()
        api.si_attn_decode(cache, q[:, 0], None, new, new, 0, 0, 0.1, out, None, 0, cache.workspace(4, 1), status)
        torch.cuda.synchronize()
        assert status.item() == api.SI_ERR_OUT_OF_RANGE
        if new is not None:
            assert torch.equal(k[0].view(torch.int16), k0[0].view(torch.int16)) and torch.count_nonzero(k[1, :, 3]) == 0
        status.zero_()
        o4 = torch.empty(2, 1, 4, 64, dtype=q.dtype, device="cuda")
        api.si_attn_prefill(cache, q, 0, 0, 0.1, o4, None, cache.workspace(4, 1), status)
        torch.cuda.synchronize()
        assert status.item() == (api.SI_ERR_OUT_OF_RANGE if lens[0] != 64 else 0)


def test_calls_run_on_the_given_stream_and_in_a_graph(api):
    lens = [200, 90]
    q, k, v, length = au.make(2, 8, 2, 128, 256, "bf16", "hnd", 1, 4, lens)
    weight = torch.zeros(2, 2, 256, device="cuda")
    cache = api.KVCache(k, v, length, None, weight)
    ws = cache.workspace(8, 1)
    out, lse = torch.empty(2, 8, 128, dtype=q.dtype, device="cuda"), torch.empty(2, 8, dtype=torch.float32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        api.si_attn_decode(cache, q[:, 0], None, None, None, 0, 0, 0.09, out, lse, api.SI_FLAG_ACC_WEIGHT, ws, stream=s)
    for want in (lens, [17, 230]):               # the lengths live on the device: a captured call follows them
        kk, vv = au.make(2, 8, 2, 128, 256, "bf16", "hnd", 1, 4, [256, 256])[1:3]
        k.copy_(kk); v.copy_(vv)
        length.copy_(torch.tensor(want, dtype=torch.int32))
        weight.zero_()
        graph.replay()
        torch.cuda.synchronize()
        ref = au.reference(q, k, v, want, 0, 0, 0.09)
        au.check_out(out[:, None], ref, "bf16", 128)
        au.check_weight(weight, np.zeros((2, 2, 256)), ref, 128, 1)


def test_one_workspace_for_long_and_short_chunks_and_fewer_heads(api):
    """A program sizes its scratch once, for its longest chunk and all heads; its last chunk is short (and split over CTAs)."""
    n, D, Hkv = 3000, 128, 2
    _, k, v, length = au.make(1, 32, Hkv, D, n + 8, "bf16", "nhd", 1, 4, [n])
    cache = api.KVCache(k, v, length)
    ws = cache.workspace(32, 2048)
    for T, Hq in ((21, 32), (130, 8), (1, 2)):
        q = au.make(1, Hq, Hkv, D, 8, "bf16", "hnd", T, T, [8])[0]
        out, lse = torch.empty(1, T, Hq, D, dtype=q.dtype, device="cuda"), torch.empty(1, T, Hq, device="cuda")
        api.si_attn_prefill(cache, q, 0, 0, 0.09, out, lse, ws)
        ref = au.reference(q, k, v, [n], 0, 0, 0.09)
        au.check_out(out, ref, "bf16", D)
        au.check_lse(lse, ref, D)


def _whole_numbers(B, Hq, Hkv, D, n, T, dtype, seed, lift=0, step=False):
    """Queries and keys of small whole numbers: every score is exact in fp32.  lift: a common 2^20 in all scores of all queries;
    step: the scores also grow by one from key to key."""
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randint(-2, 3, (B, T, Hq, D), generator=g).float(), torch.randint(-2, 3, (B, Hkv, n, D), generator=g).float()
    if lift:
        q[..., :3], k[..., 0] = torch.tensor([1024.0, 16.0, 1.0]), 1024.0
        j = torch.arange(n) if step else torch.zeros(n)
        k[..., 1], k[..., 2] = j // 16, j % 16
    v = torch.randn(B, Hkv, n, D, generator=g)
    dt = au.TDT[dtype]
    return q.to(dt).cuda(), k.to(dt).cuda(), v.to(dt).cuda(), torch.full((B,), n, dtype=torch.int32, device="cuda")


def _check_exact_scores(out, lse, ref, dtype, reach_of=60.0):
    """Bounds where the scores carry no error: p is relative to the type (u) and to the exponent's difference (8 e * reach_of; what
    lies further below the maximum is nothing), sums n e, the result rounded once more; lse 4 e of itself."""
    u, E = au.U[dtype], au.E
    rel = 8 * E * reach_of + (ref["n"] + 8) * E
    bound = (u * np.abs(ref["out"]) + (u + rel[..., None]) * ref["reach"]) * 1.01
    if dtype == "f16":
        bound += (ref["n"][..., None] * 5.0 + 1.0) * 2.0 ** -25
    assert np.all(np.abs(au.f64(out) - ref["out"]) <= bound)
    assert np.all(np.abs(au.f64(lse) - ref["lse"]) <= 4 * E * np.abs(ref["lse"]) + (ref["n"] + 8) * E)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,n,T", [(128, 390, 150), (64, 3000, 20), (64, 300, 300)])     # the second: keys split over CTAs
@pytest.mark.parametrize("scale", [1e6, -1e6, 3e9, 1e30])
def test_scores_far_beyond_the_mantissa(api, D, n, T, scale, dtype):
    """Scaled scores above 2^24, where neighbouring fp32 numbers are more than one apart: the softmax picks the largest scores."""
    q, k, v, length = _whole_numbers(1, 4, 2, D, n, T, dtype, n)
    out, lse = _prefill(api, q, k, v, length, 0, 0, scale)
    ref = au.reference(q, k, v, [n], 0, 0, scale)
    _check_exact_scores(out, lse, ref, dtype)
    o1, l1 = torch.empty(1, 4, D, dtype=q.dtype, device="cuda"), torch.empty(1, 4, device="cuda")
    cache = api.KVCache(k, v, length)
    api.si_attn_decode(cache, q[:, -1].contiguous(), None, None, None, 0, 0, scale, o1, l1, 0, cache.workspace(4, 1))
    last = {x: ref[x][:, -1:] for x in ("out", "reach", "lse", "n")}
    _check_exact_scores(o1[:, None], l1[:, None], last, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,n,T", [(128, 700, 200), (64, 3000, 20)])
@pytest.mark.parametrize("scale", [0.04, 0.04332, 0.05, 0.5, -0.04333])
@pytest.mark.parametrize("step", [False, True])
def test_scores_with_a_large_common_part(api, D, n, T, scale, step, dtype):
    """All scores lie near 2^20 * scale; what they differ by decides.  With `step` the running maximum grows from tile to tile."""
    q, k, v, length = _whole_numbers(1, 4, 2, D, n, T, dtype, n + 1, lift=1, step=step)
    out, lse = _prefill(api, q, k, v, length, 0, 0, scale)
    _check_exact_scores(out, lse, au.reference(q, k, v, [n], 0, 0, scale), dtype)


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f16")])
def test_accumulated_weights_keep_nan(api, D, dtype):
    """A query that is not a number makes the weight of every entry it sees one too, in every tile and column alike, and of no other."""
    B, T, Hq, Hkv, n = 1, 300, 8, 2, 700
    q, k, v, length = au.make(B, Hq, Hkv, D, n + 3, dtype, "hnd", T, 21, [n])
    ref = au.reference(q, k, v, [n], 0, 0, 0.1)
    lse = torch.from_numpy(ref["lse"].astype(np.float32)).cuda()
    for i, hq in ((64, 0), (64, 1), (68, 4), (77, 2), (299, 7), (0, 5), (192, 0), (131, 3)):
        qb, lb = q.clone(), lse.clone()
        qb[0, i, hq, 5], lb[0, i, hq] = float("nan"), float("nan")
        weight = torch.zeros(B, Hkv, n + 3, device="cuda")
        cache = api.KVCache(k, v, length, None, weight)
        api.si_attn_weights(cache, qb, 0, 0, 0.1, lb, cache.workspace(Hq, T))
        got, seen = weight.cpu().numpy(), n - T + i + 1
        h = hq // (Hq // Hkv)
        assert np.isnan(got[0, h, :seen]).all(), (i, hq, np.nonzero(~np.isnan(got[0, h, :seen]))[0][:5])
        assert np.isfinite(got[0, h, seen:]).all() and np.isfinite(got[0, 1 - h]).all()


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 3, 1), (128, 20, 1)])
@pytest.mark.parametrize("n,bad", [(1, [0]), (17, [16]), (40, list(range(16, 40))), (5000, [4999]), (5000, list(range(2000, 2600)))])
def test_decode_keeps_nan(api, D, Hq, Hkv, n, bad):
    """Visible keys that are not numbers: the output, lse and every weight of their head are not either; other heads as ever."""
    q, k, v, length = au.make(2, Hq, Hkv, D, n + 2, "bf16", "hnd", 1, 31, [n, n])
    k[1, 0, bad] = float("nan")
    weight = torch.zeros(2, Hkv, n + 2, device="cuda")
    cache = api.KVCache(k, v, length, None, weight)
    out, lse = torch.empty(2, Hq, D, dtype=q.dtype, device="cuda"), torch.empty(2, Hq, device="cuda")
    api.si_attn_decode(cache, q[:, 0], None, None, None, 0, 0, 0.1, out, lse, api.SI_FLAG_ACC_WEIGHT, cache.workspace(Hq, 1))
    G = Hq // Hkv
    assert torch.isnan(out[1, :G]).all() and torch.isnan(weight[1, 0, :n]).all()
    assert torch.isnan(lse[1, :G]).all()
    for t in (out[0], out[1, G:], lse[0], lse[1, G:], weight[0], weight[1, 1:]):
        assert torch.isfinite(t).all()
    o, l = _prefill(api, q, k, v, length, 0, 0, 0.1)
    assert torch.isnan(o[1, 0, :G]).all() and torch.isnan(l[1, 0, :G]).all()
    assert torch.isfinite(o[0]).all() and torch.isfinite(l[0]).all() and torch.isfinite(l[1, 0, G:]).all()


def test_decode_with_nan_adds_nothing_to_hidden_entries(api):
    n, window, n_sink, D = 700, 50, 3, 64
    for positions in (False, True):
        q, k, v, length = au.make(1, 4, 1, D, n + 4, "f16", "hnd", 1, 41, [n])
        k[0, 0, n - 7] = float("nan")
        weight = torch.zeros(1, 1, n + 4, device="cuda")
        pos = torch.arange(n + 4, dtype=torch.int32, device="cuda").view(1, 1, -1).contiguous() if positions else None
        cache = api.KVCache(k, v, length, pos, weight)
        out = torch.empty(1, 4, D, dtype=q.dtype, device="cuda")
        api.si_attn_decode(cache, q[:, 0], length - 1, None, None, window, n_sink, 0.1, out, None, api.SI_FLAG_ACC_WEIGHT, cache.workspace(4, 1))
        got = weight[0, 0].cpu().numpy()
        assert np.isnan(got[:n_sink]).all() and np.isnan(got[n - window:n]).all()
        assert (got[n_sink:n - window] == 0).all() and (got[n:] == 0).all()


@pytest.mark.parametrize("T,n,Hq,Hkv,D,window,n_sink,dtype", [
    (1500, 4000, 4, 1, 128, 0, 0, "bf16"),          # many key tiles, blocks of queries of many lengths
    (2000, 2000, 3, 3, 64, 0, 0, "f16"),
    (1000, 9000, 2, 1, 128, 700, 130, "bf16"),
    (60, 12000, 8, 2, 64, 0, 0, "bf16"),            # long keys split over CTAs
    (5, 30000, 16, 2, 128, 0, 0, "f16"),
])
def test_prefill_of_long_sequences(api, T, n, Hq, Hkv, D, window, n_sink, dtype):
    q, k, v, length = au.make(1, Hq, Hkv, D, n + 1, dtype, "nhd", T, T + n, [n])
    weight = torch.zeros(1, Hkv, n + 1, device="cuda")
    out, lse = _prefill(api, q, k, v, length, window, n_sink, 0.1, weight)
    # rows of every part of the range against the oracle, and all of them through the sum of what they gave
    rows = sorted({0, 1, T // 3, T // 2, T - 2, T - 1} | set(range(0, T, max(1, T // 40))))
    rows = [r for r in rows if 0 <= r < T]
    G = Hq // Hkv
    from oracle import attention_oracle as ao
    kn, vn, qn = au.f64(k)[0, :, :n], au.f64(v)[0, :, :n], au.f64(q)[0]
    ref = {x: np.zeros((1, len(rows), Hq) + ((D,) if x in ("out", "reach") else ())) for x in ("out", "reach", "lse", "size", "n")}
    for h in range(Hq):
        o, l, w, r, z = ao.attend(qn[rows, h], kn[h // G], vn[h // G], np.arange(n), n - T + np.asarray(rows), window, n_sink, 0.1)
        for x, y in (("out", o), ("reach", r), ("lse", l), ("size", z), ("n", (w > 0).sum(-1))):
            ref[x][0, :, h] = y
    au.check_out(out[:, rows], ref, dtype, D)
    au.check_lse(lse[:, rows], ref, D)
    total = au.f64(weight)[0].sum(-1)                # every query gives each of its G heads' entries a weight of one in all
    assert np.all(np.abs(total - T * G) <= T * G * (4 * au.delta(ref, D).max() + 3e-5))
