"""GPU parity of the cache eviction: exact against the oracle, in place and into another cache."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def _weights(kind, shape, rng):
    w = rng.random(shape).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 4).astype(np.float32) / 4
    elif kind == "equal":
        w[:] = 0.5
    elif kind == "odd":          # signed zeros, infinities, NaN, denormals among ties
        w = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-45, 1.0, 2.0, -3.0], np.float32), size=shape)
    return w


CASES = [
    # lens, n_new, cap, budget, n_sink, n_recent
    ([1], 0, 8, 1, 0, 0),
    ([0, 7], 0, 8, 5, 0, 0),
    ([5, 8], 0, 8, 8, 2, 2),               # nothing to evict
    ([33, 2], 0, 40, 7, 2, 3),
    ([100, 64, 65], 0, 128, 64, 4, 16),
    ([64, 64], 1, 70, 64, 4, 8),           # a decode step at the budget
    ([66, 67], 1, 70, 64, 4, 8),           # three and four over it
    ([2050, 1026], 2, 2052, 2048, 2040, 8),  # half of the entries are protected
    ([1030, 2049], 0, 2050, 1024, 1, 1000),
    ([5000], 0, 5001, 4999, 0, 1),
    ([3000, 777], 0, 3001, 100, 100, 0),   # only protected entries fit
    ([20000], 0, 20000, 333, 4, 100),
    ([60000], 0, 60001, 30000, 16, 128),
    ([60000, 13], 0, 60004, 30001, 16, 128),   # an aligned row length
    ([16384, 9000], 0, 16384, 4096, 4, 256),
]


@pytest.mark.parametrize("lens,n_new,cap,budget,n_sink,n_recent", CASES)
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(api, lens, n_new, cap, budget, n_sink, n_recent, kind, in_place):
    B, H, D = len(lens), 3, 64 if kind != "ties" else 128
    rng = np.random.default_rng(cap + budget)
    w = _weights(kind, (B, H, cap), rng)
    pos = np.stack([np.stack([rng.permutation(2 * cap)[:cap] for _ in range(H)]) for _ in range(B)]).astype(np.int32)
    last = np.array([2 * cap - 1 - b for b in range(B)], np.int32)
    k, v = (torch.randint(-30000, 30000, (B, H, cap, D), dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(2))
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    tpos, tw = torch.from_numpy(pos).cuda(), torch.from_numpy(w).cuda()
    src = api.KVCache(k, v, length, tpos, tw)
    k0, v0 = k.view(torch.int16).cpu().numpy().copy(), v.view(torch.int16).cpu().numpy().copy()
    if in_place:
        dst, dk, dv, dpos, dw = src, k, v, tpos, tw
    else:                                  # a token-major destination with room to spare
        dk, dv = (torch.zeros(B, budget + 3, H, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
        dpos = torch.full((B, H, budget + 3), -9, dtype=torch.int32, device="cuda")
        dw = torch.full((B, H, budget + 3), -9.0, device="cuda")
        dst = api.KVCache(dk, dv, length, dpos, dw)
    kept = torch.full((B, H, budget), -7, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.si_kv_evict(src, dst, torch.from_numpy(last).cuda(), n_new, budget, n_sink, n_recent, kept, length, src.workspace(0, 0), status)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert length.tolist() == [min(n + n_new, budget) for n in lens]
    got_k, got_v = dk.view(torch.int16).cpu().numpy(), dv.view(torch.int16).cpu().numpy()
    got_p, got_w = dpos.cpu().numpy(), dw.cpu().numpy()
    for b, n in enumerate(lens):
        n += n_new
        for h in range(H):
            want = ao.evict(w[b, h, :n], pos[b, h, :n].astype(np.int64), int(last[b]), budget, n_sink, n_recent)
            assert np.array_equal(kept[b, h].cpu().numpy(), want), (b, h)
            to = np.nonzero(want >= 0)[0]
            assert np.array_equal(got_k[b, h, to], k0[b, h, want[to]]) and np.array_equal(got_v[b, h, to], v0[b, h, want[to]])
            assert np.array_equal(got_p[b, h, to], pos[b, h, want[to]])
            assert np.array_equal(got_w[b, h, to].view(np.int32), w[b, h, want[to]].view(np.int32))
            rest = np.setdiff1d(np.arange(got_p.shape[2]), to)     # everything else is as it was
            assert np.array_equal(got_p[b, h, rest], pos[b, h, rest] if in_place else np.full(len(rest), -9))


def test_evict_of_a_prefilled_cache_without_positions(api):
    B, H, D, cap, budget = 2, 2, 128, 500, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(B, H, cap, D, generator=g, device="cuda").to(torch.float16) for _ in range(2))
    w = torch.rand(B, H, cap, generator=g, device="cuda")
    length = torch.tensor([500, 300], dtype=torch.int32, device="cuda")
    src = api.KVCache(k, v, length, None, w)
    dk, dv = (torch.zeros(B, H, budget, D, dtype=torch.float16, device="cuda") for _ in range(2))
    dpos, dw = torch.zeros(B, H, budget, dtype=torch.int32, device="cuda"), torch.zeros(B, H, budget, device="cuda")
    len_out = torch.zeros(B, dtype=torch.int32, device="cuda")
    dst = api.KVCache(dk, dv, len_out, dpos, dw)
    api.si_kv_evict(src, dst, None, 0, budget, 4, 16, None, len_out, src.workspace(0, 0))
    torch.cuda.synchronize()
    assert len_out.tolist() == [budget, budget]
    for b, n in enumerate([500, 300]):
        for h in range(H):
            want = ao.evict(w[b, h, :n].cpu().numpy(), np.arange(n), n - 1, budget, 4, 16)
            assert np.array_equal(dpos[b, h].cpu().numpy(), want)
            assert torch.equal(dk[b, h], k[b, h, torch.from_numpy(want).cuda()]) and torch.equal(dv[b, h], v[b, h, torch.from_numpy(want).cuda()])


def test_evict_into_a_cache_with_a_budget_above_the_source(api):
    """Nothing is over the budget: every entry is copied, further slots of `kept` are -1 and of the cache untouched."""
    B, H, D, cap, budget, lens = 2, 2, 64, 40, 100, [40, 7]
    k, v = (torch.randn(B, H, cap, D, device="cuda").to(torch.float16) for _ in range(2))
    w = torch.rand(B, H, cap, device="cuda")
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for with_kept in (True, False):
        dk, dv = (torch.zeros(B, H, budget, D, dtype=torch.float16, device="cuda") for _ in range(2))
        dpos, dw = torch.full((B, H, budget), -9, dtype=torch.int32, device="cuda"), torch.zeros(B, H, budget, device="cuda")
        kept = torch.full((B, H, budget), -7, dtype=torch.int32, device="cuda") if with_kept else None
        len_out = torch.zeros(B, dtype=torch.int32, device="cuda")
        src, dst = api.KVCache(k, v, length, None, w), api.KVCache(dk, dv, len_out, dpos, dw)
        api.si_kv_evict(src, dst, None, 0, budget, 4, 16, kept, len_out, src.workspace(0, 0))
        torch.cuda.synchronize()
        assert len_out.tolist() == lens
        for b, n in enumerate(lens):
            assert torch.equal(dk[b, :, :n], k[b, :, :n]) and torch.equal(dv[b, :, :n], v[b, :, :n]) and torch.equal(dw[b, :, :n], w[b, :, :n])
            assert (dpos[b, :, n:] == -9).all() and torch.count_nonzero(dk[b, :, n:]) == 0
            if with_kept:
                assert (kept[b, :, n:] == -1).all() and (kept[b, :, :n] == torch.arange(n, device="cuda")).all()


@pytest.mark.parametrize("n,budget", [(400000, 150000), (393217, 393000), (700001, 300000)])
def test_evict_of_rows_longer_than_shared_memory_holds(api, n, budget):
    """More keys than eight CTAs keep in shared memory: the weights are read again instead, in rounds."""
    rng = np.random.default_rng(n)
    w = np.floor(rng.random(n) * 1000).astype(np.float32)
    k, v = (torch.randint(-30000, 30000, (1, 1, n, 64), dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(2))
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    src = api.KVCache(k, v, length, None, torch.from_numpy(w).cuda().view(1, 1, n))
    dk, dv = (torch.zeros(1, 1, budget, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dst = api.KVCache(dk, dv, length, torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, budget, device="cuda"))
    kept = torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda")
    api.si_kv_evict(src, dst, None, 0, budget, 16, 1000, kept, None, src.workspace(0, 0))
    torch.cuda.synchronize()
    want = ao.evict(w, np.arange(n), n - 1, budget, 16, 1000)
    assert np.array_equal(kept[0, 0].cpu().numpy(), want) and np.array_equal(dst.pos[0, 0].cpu().numpy(), want)
    at = torch.from_numpy(want).cuda()
    assert torch.equal(dk[0, 0].view(torch.int16), k[0, 0, at].view(torch.int16)) and torch.equal(dv[0, 0].view(torch.int16), v[0, 0, at].view(torch.int16))


def test_evict_reports_lengths_outside_the_capacity(api):
    k = torch.zeros(1, 1, 16, 64, dtype=torch.float16, device="cuda")
    pos, w = torch.zeros(1, 1, 16, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, 16, device="cuda")
    for n, n_new in ((17, 0), (-1, 0), (16, 1)):
        c = api.KVCache(k, k.clone(), torch.tensor([n], dtype=torch.int32, device="cuda"), pos, w)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        api.si_kv_evict(c, c, torch.zeros(1, dtype=torch.int32, device="cuda"), n_new, 4, 0, 0, None, None, c.workspace(0, 0), status)
        torch.cuda.synchronize()
        assert status.item() == api.SI_ERR_OUT_OF_RANGE


def _evict_fast(w, budget, n_sink, n_recent):
    """ao.evict for entry j at position j without NaN, in numpy (the oracle's own takes minutes at millions of entries)."""
    n = len(w)
    rank = w.astype(np.float64)
    rank[:n_sink] = rank[n - n_recent:] = np.inf
    kept = np.zeros(n, bool)
    kept[np.argsort(-rank, kind="stable")[:budget]] = True
    src = np.where(kept[:budget], np.arange(budget), -1)
    src[src < 0] = budget + np.nonzero(kept[budget:])[0]
    return src


@pytest.mark.parametrize("D,n,budget", [(128, 4_400_000, 4_300_001), (64, 8_500_000, 8_400_000), (128, 3000, 777)])
def test_evict_with_budgets_of_millions(api, D, n, budget):
    """More slots than 65535 blocks of the moving kernel hold."""
    rng = np.random.default_rng(budget)
    w = np.floor(rng.random(n) * 1e5).astype(np.float32)
    want = _evict_fast(w, budget, 16, 1000 if n > 5000 else 100)
    if n <= 5000:
        assert np.array_equal(want, ao.evict(w, np.arange(n), n - 1, budget, 16, 100))
    k = torch.arange(n, dtype=torch.int32, device="cuda").view(1, 1, n, 1).expand(1, 1, n, D // 2).contiguous().view(torch.bfloat16)
    v = (torch.arange(n, dtype=torch.int32, device="cuda") ^ 0x5A5A).view(1, 1, n, 1).expand(1, 1, n, D // 2).contiguous().view(torch.bfloat16)
    length, len_out = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    src = api.KVCache(k, v, length, None, torch.from_numpy(w).cuda().view(1, 1, n))
    dk, dv = (torch.zeros(1, 1, budget, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dst = api.KVCache(dk, dv, len_out, torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, budget, device="cuda"))
    api.si_kv_evict(src, dst, None, 0, budget, 16, 1000 if n > 5000 else 100, None, len_out, src.workspace(0, 0))
    torch.cuda.synchronize()
    at = torch.from_numpy(want).cuda()
    assert len_out.item() == budget and torch.equal(dst.pos[0, 0].long(), at)
    assert torch.equal(dst.weight[0, 0], src.weight[0, 0, at])
    for d, x in ((dk, 0), (dv, 0x5A5A)):
        got = d[0, 0].view(torch.int32)
        assert all(torch.equal(got[:, c].long(), at ^ x) for c in (0, 5, D // 2 - 1))


@pytest.mark.parametrize("lens,n_new,cap,budget", [
    ([16384], 0, 16384, 16200),             # four CTAs to a row that select and move
    ([8300, 8299], 1, 8301, 8192),
    ([16384, 16383], 1, 16385, 16384),      # a decode step at the budget, and one below it
    ([50000], 0, 50003, 49999),
    ([65536], 0, 65536, 65300),
    ([3, 60000], 0, 60000, 59800),
])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
@pytest.mark.parametrize("with_kept", [True, False])
def test_evict_in_place_on_rows_of_several_ctas(api, lens, n_new, cap, budget, kind, with_kept):
    B, H, D, n_sink, n_recent = len(lens), 3, 64, 4, 100
    rng = np.random.default_rng(cap)
    w = _weights(kind, (B, H, cap), rng)
    pos = np.stack([np.stack([rng.permutation(2 * cap)[:cap] for _ in range(H)]) for _ in range(B)]).astype(np.int32)
    last = np.array([2 * cap - 1 - b for b in range(B)], np.int32)
    k, v = (torch.randint(-30000, 30000, (B, H, cap, D), dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(2))
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = api.KVCache(k, v, length, torch.from_numpy(pos).cuda(), torch.from_numpy(w).cuda())
    k0, v0 = k.view(torch.int16).clone(), v.view(torch.int16).clone()
    kept = torch.full((B, H, budget), -7, dtype=torch.int32, device="cuda") if with_kept else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.si_kv_evict(cache, cache, torch.from_numpy(last).cuda(), n_new, budget, n_sink, n_recent, kept, length, cache.workspace(0, 0), status)
    torch.cuda.synchronize()
    assert status.item() == 0 and length.tolist() == [min(n + n_new, budget) for n in lens]
    got_p, got_w = cache.pos.cpu().numpy(), cache.weight.cpu().numpy()
    for b, n in enumerate(lens):
        n += n_new
        for h in range(H):
            want = ao.evict(w[b, h, :n], pos[b, h, :n].astype(np.int64), int(last[b]), budget, n_sink, n_recent)
            if with_kept:
                assert np.array_equal(kept[b, h].cpu().numpy(), want)
            to = np.nonzero(want >= 0)[0]
            d, s = torch.from_numpy(to).cuda(), torch.from_numpy(want[to]).cuda()
            assert torch.equal(k[b, h, d].view(torch.int16), k0[b, h, s]) and torch.equal(v[b, h, d].view(torch.int16), v0[b, h, s])
            assert np.array_equal(got_p[b, h, to], pos[b, h, want[to]])
            assert np.array_equal(got_w[b, h, to].view(np.int32), w[b, h, want[to]].view(np.int32))
            assert np.array_equal(got_p[b, h, len(to):], pos[b, h, len(to):])            # slots beyond are as they were


@pytest.mark.parametrize("n,budget", [(393208, 100000), (393216, 393000), (200001, 199990)])
def test_evict_of_rows_that_just_fit_shared_memory(api, n, budget):
    rng = np.random.default_rng(n)
    w = np.floor(rng.random(n) * 1000).astype(np.float32)
    k, v = (torch.randint(-30000, 30000, (1, 1, n, 64), dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(2))
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    src = api.KVCache(k, v, length, None, torch.from_numpy(w).cuda().view(1, 1, n))
    dk, dv = (torch.zeros(1, 1, budget, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dst = api.KVCache(dk, dv, length, torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, budget, device="cuda"))
    api.si_kv_evict(src, dst, None, 0, budget, 16, 1000, None, None, src.workspace(0, 0))
    at = torch.from_numpy(_evict_fast(w, budget, 16, 1000)).cuda()
    assert torch.equal(dst.pos[0, 0].long(), at)
    assert torch.equal(dk[0, 0].view(torch.int16), k[0, 0, at].view(torch.int16)) and torch.equal(dv[0, 0].view(torch.int16), v[0, 0, at].view(torch.int16))
