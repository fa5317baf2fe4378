"""GPU parity of the cache in 4 bits -- storing, reading back, single-token attention, eviction -- against the float64 oracle:
codes exactly, attention within the bounds of kv4_utils."""
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import kv4_oracle as ko
from tests import attn_utils as au
from tests import kv4_utils as k4

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def bits(t):
    return t.contiguous().view(torch.int16)


def same(t, want):
    """16-bit tensor against float64 values: equal, NaN to NaN."""
    return np.array_equal(au.f64(t), want, equal_nan=True)


SHAPES = [(128, 32), (128, 64), (64, 32), (64, 64)]

STORE = [
    # B, H, entries there before, entries stored
    (1, 1, [0], [1]), (1, 2, [31], [1]), (1, 2, [32], [1]), (2, 3, [5, 6], [2, 3]), (1, 1, [0], [32]), (2, 2, [30, 33], [35, 0]),
    (3, 2, [0, 17, 64], [200, 77, 1]), (1, 8, [1], [127]), (2, 1, [63, 127], [130, 66]), (1, 2, [3], [1000]),
]


@pytest.mark.parametrize("B,H,past,new", STORE)
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("dtype,order", [("bf16", "nhd"), ("f16", "hnd")])
def test_stored_entries_come_back_as_the_format_says(api, B, H, past, new, D, group, dtype, order):
    """Whole and partial tiles; what was there before and what lies behind stays as it was, byte for byte of what it stands for."""
    cap = (max(p + n for p, n in zip(past, new)) + 40) // 32 * 32 + 32
    made = k4.Made(api, B, H, D, cap, group, dtype, [cap] * B, seed=D + group)
    g = torch.Generator().manual_seed(5)
    T = max(new)
    wide = (torch.randn(B, T, 5 * H, D, generator=g) * torch.exp(torch.randn(B, T, 5 * H, 1, generator=g))).to(made.dt).cuda()
    k, v = wide[:, :, H:2 * H].transpose(1, 2), wide[:, :, 3 * H:4 * H].transpose(1, 2)
    if order == "hnd":
        k, v = k.contiguous(), v.contiguous()
    before_k, before_v = made.read()
    assert same(before_k, ko.read_back(*made.kq, dtype)) and same(before_v, ko.read_back(*made.vq, dtype))
    dst = api.KV4Cache(made.cache.data, D, group, made.dt, torch.tensor(past, **I32))
    status = torch.zeros(1, **I32)
    api.si_kv4_store(api.KVCache(k, v, torch.tensor(new, **I32)), dst, None, status)
    after_k, after_v = made.read()
    assert status.item() == 0
    for x, after, before in ((k, after_k, before_k), (v, after_v, before_v)):
        want = ko.read_back(*ko.quantise(au.f64(x), group, dtype), dtype)
        for b in range(B):
            assert same(after[b, :, past[b]:past[b] + new[b]], want[b, :, :new[b]])
            assert torch.equal(bits(after[b, :, :past[b]]), bits(before[b, :, :past[b]]))
            assert torch.equal(bits(after[b, :, past[b] + new[b]:]), bits(before[b, :, past[b] + new[b]:]))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group", SHAPES)
def test_values_at_the_ends_of_the_type(api, D, group, dtype):
    """NaN, infinities, zeros of both signs, constants, subnormal numbers, the largest ones, values halfway between two codes."""
    big = 65504.0 if dtype == "f16" else 2.0 ** 93
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    g = torch.Generator().manual_seed(3)
    rows = [torch.zeros(D), torch.full((D,), -0.0), torch.full((D,), 3.140625), torch.randn(D, generator=g) * 2.0 ** -20, torch.randn(D, generator=g) * big / 8,
            torch.arange(D) % 31 * 0.5, (torch.arange(D) % 31 * 0.5 - 7) * 1.0703125, torch.randint(0, 9, (D,), generator=g) * tiny, torch.randint(-7, 8, (D,), generator=g) * tiny * 16,
            torch.where(torch.arange(D) % 2 == 0, big, -big), 100 + torch.arange(D) % 3 * 0.5, torch.randn(D, generator=g) * 1e-3 + 7]
    for special in (float("nan"), float("inf"), float("-inf")):
        for at in (0, 33, D - 1):
            x = torch.randn(D, generator=g)
            x[at] = special
            rows.append(x)
    if dtype == "bf16":
        rows += [torch.where(torch.arange(D) == 40, 2.0 ** 95, 1.0), torch.where(torch.arange(D) == 40, 3.0e38, -3.0e38), torch.arange(D) % 16 * 2.0 ** -126, torch.arange(D) % 16 * 2.0 ** -128]
    x = torch.stack([r.float() for r in rows])
    n = len(rows)
    cap = (n + 31) // 32 * 32
    full = torch.zeros(1, 1, cap, D)
    full[0, 0, :n] = x
    for swap in (False, True):
        made = k4.Made(api, 1, 1, D, cap, group, dtype, [n], k=full.flip(2) if swap else full, v=full)
        k, v = made.read(made.length)
        assert same(k[:, :, :n], ko.read_back(*made.kq, dtype)[:, :, :n]) and same(v[:, :, :n], ko.read_back(*made.vq, dtype)[:, :, :n])
        assert torch.equal(bits(k[:, :, n:]), torch.zeros_like(bits(k[:, :, n:])))


def test_positions_and_weights_go_along(api):
    B, H, D, cap = 2, 2, 64, 96
    for with_pos, with_weight, with_first in ((1, 1, 0), (0, 0, 1), (0, 1, 0), (1, 0, 1)):
        pos, weight = torch.full((B, H, cap), -7, **I32), torch.full((B, H, cap), -7.0, device="cuda")
        past, new = [10, 0], [33, 40]
        k, v = (torch.randn(B, H, 50, D, device="cuda").to(torch.bfloat16) for _ in range(2))
        spos = torch.randint(0, 1000, (B, H, 50), **I32) if with_pos else None
        sweight = torch.rand(B, H, 50, device="cuda") if with_weight else None
        dst = api.KV4Cache.empty(B, H, cap, D, 32, torch.bfloat16, torch.tensor(past, **I32), pos, weight)
        api.si_kv4_store(api.KVCache(k, v, torch.tensor(new, **I32), spos, sweight), dst, torch.tensor([500, 600], **I32) if with_first else None)
        for b in range(B):
            span = slice(past[b], past[b] + new[b])
            want = spos[b, :, :new[b]] if with_pos else (torch.arange(new[b], **I32) + ([500, 600][b] if with_first else past[b])).expand(H, -1)
            assert torch.equal(pos[b, :, span], want)
            assert torch.equal(weight[b, :, span], sweight[b, :, :new[b]] if with_weight else torch.zeros(H, new[b], device="cuda"))
            rest = torch.ones(cap, dtype=torch.bool, device="cuda")
            rest[span] = False
            assert (pos[b, :, rest] == -7).all() and (weight[b, :, rest] == -7.0).all()
        # and back
        back = api.KVCache(torch.zeros_like(k), torch.zeros_like(v), torch.zeros(B, **I32), torch.full((B, H, 50), -9, **I32), torch.full((B, H, 50), -9.0, device="cuda"))
        full = api.KV4Cache(dst.data, D, 32, torch.bfloat16, torch.tensor([43, 40], **I32), pos, weight)
        api.si_kv4_load(full, back, dst.length, 35, back.length)
        assert back.length.tolist() == [33, 35]
        for b, m in enumerate([33, 35]):
            assert torch.equal(back.pos[b, :, :m], pos[b, :, past[b]:past[b] + m]) and torch.equal(back.weight[b, :, :m], weight[b, :, past[b]:past[b] + m])
            assert (back.pos[b, :, m:] == -9).all() and (back.weight[b, :, m:] == -9.0).all()


@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("order", ["hnd", "nhd"])
def test_parts_are_read_back(api, D, group, order):
    """From any first entry, any number; lengths that end before it; rows of dst behind stay as they were."""
    B, H, cap = 4, 3, 320
    lens = [300, 47, 0, 320]
    made = k4.Made(api, B, H, D, cap, group, "bf16", lens, seed=9)
    want = [ko.read_back(*x, "bf16") for x in (made.kq, made.vq)]
    for first, n in (([0, 0, 0, 0], 320), ([1, 46, 0, 31], 2), ([299, 47, 5, 319], 1), ([300, 2 ** 31 - 1, 7, 0], 90), ([33, 15, 0, 64], 150), ([0, 0, 0, 0], 0)):
        shape = (B, H, 330, D) if order == "hnd" else (B, 330, H, D)
        out = [torch.full(shape, 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        view = [x if order == "hnd" else x.transpose(1, 2) for x in out]
        got, status = torch.full((B,), -1, **I32), torch.zeros(1, **I32)
        api.si_kv4_load(made.cache, api.KVCache(*view, torch.zeros(B, **I32)), torch.tensor(first, **I32), n, got, status)
        assert status.item() == 0
        for b in range(B):
            m = min(n, max(0, lens[b] - first[b]))
            assert got[b].item() == m
            for x, y in zip(view, want):
                assert same(x[b, :, :m], y[b, :, first[b]:first[b] + m]) and (x[b, :, m:] == 5.0).all()


def test_what_the_device_reports(api):
    """Entries that do not fit, lengths outside the cache, a negative first entry: an error code, and nothing outside is touched."""
    D, cap = 128, 64
    made = k4.Made(api, 2, 2, D, cap, 32, "bf16", [cap, cap], seed=1)
    before, _ = made.read()
    k, v = (torch.randn(2, 2, 40, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    status = torch.zeros(1, **I32)
    api.si_kv4_store(api.KVCache(k, v, torch.tensor([40, 3], **I32)), api.KV4Cache(made.cache.data, D, 32, made.dt, torch.tensor([50, 64], **I32)), None, status)
    after, _ = made.read()
    assert status.item() == api.SI_ERR_OUT_OF_RANGE
    assert torch.equal(bits(after[0, :, :50]), bits(before[0, :, :50])) and torch.equal(bits(after[1]), bits(before[1]))
    assert same(after[0, :, 50:], ko.read_back(*ko.quantise(au.f64(k[0, :, :14]), 32, "bf16"), "bf16"))
    out = api.KVCache(torch.zeros_like(k), torch.zeros_like(v), torch.zeros(2, **I32))
    for lens, first, want in (([-3, 70], [0, 60], [0, 4]), ([64, 5], [-1, 0], [40, 5])):
        status.zero_()
        got = torch.zeros(2, **I32)
        api.si_kv4_load(api.KV4Cache(made.cache.data, D, 32, made.dt, torch.tensor(lens, **I32)), out, torch.tensor(first, **I32), 40, got, status)
        assert status.item() == api.SI_ERR_OUT_OF_RANGE and got.tolist() == want
    # a full cache takes no new entry, and attends to what it has
    full = k4.Made(api, 1, 1, D, cap, 32, "bf16", [cap], seed=2)
    q, kn, vn, out = (torch.randn(1, h, D, device="cuda").to(torch.bfloat16) for h in (4, 1, 1, 4))
    b0, _ = full.read()
    status.zero_()
    api.si_kv4_attn_decode(full.cache, q, None, kn, vn, 0, 0, 0.1, out, None, 0, full.cache.workspace(4), status)
    b1, _ = full.read()
    assert status.item() == api.SI_ERR_OUT_OF_RANGE and torch.equal(bits(b0), bits(b1))
    k4.check(out, None, k4.reference(full, q, [cap], 0, 0, 0.1), "bf16", D)


DECODE = [
    # B, lens, Hq, Hkv, window, n_sink, positions given, new entry
    (1, [0], 4, 1, 0, 0, False, True),         # the very first token
    (1, [1], 1, 1, 0, 0, False, False),
    (2, [0, 5], 8, 2, 0, 0, False, False),     # an empty cache: nothing to see
    (4, [6, 31, 32, 33], 8, 2, 0, 0, False, True),
    (5, [15, 16, 63, 64, 65], 4, 4, 0, 0, False, True),
    (2, [1000, 31], 24, 8, 0, 0, False, True),
    (2, [777, 2500], 16, 2, 100, 4, False, True),
    (1, [9000], 32, 8, 0, 0, False, True),
    (2, [900, 901], 7, 1, 64, 70, False, True),
    (1, [600], 20, 1, 0, 0, False, True),      # more query heads to a key head than one matrix tile holds
    (2, [400, 333], 8, 2, 0, 0, True, True),
    (2, [400, 2333], 4, 2, 150, 8, True, True),
    (2, [300, 20], 8, 4, 90, 2, True, False),
    (40, [3 + 37 * i for i in range(40)], 4, 2, 0, 0, False, True),
    (1, [3000], 128, 1, 0, 0, False, True),
    (3, [5000, 0, 64], 16, 1, 33, 1, False, True),
]


def _decode_case(api, made, B, lens, Hq, Hkv, window, n_sink, given, new, acc, scale, seed=0, spread=1.0):
    D, cap = made.D, made.cache.capacity
    rng = np.random.default_rng(B + Hq + seed)
    g = torch.Generator().manual_seed(seed + 77)
    wide = (torch.randn(B, Hq + 2 * Hkv, D, generator=g) * spread).to(made.dt).cuda()
    q, kn, vn = wide[:, :Hq], wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:]
    before = rng.random((B, Hkv, cap)).astype(np.float32)
    weight = torch.from_numpy(before).cuda()
    pos = q_pos = None
    if given:   # positions with gaps, in no order, other ones per head; the query's is the newest
        q_pos = torch.tensor([2 * n + 1 for n in lens], **I32)
        pos = torch.full((B, Hkv, cap), -5, dtype=torch.int32)
        for b, n in enumerate(lens):
            for h in range(Hkv):
                pos[b, h, :n] = torch.from_numpy(rng.permutation(2 * n + 1)[:n].astype(np.int32))
        pos = pos.cuda()
    cache = api.KV4Cache(made.cache.data, D, made.group, made.dt, made.length, pos, weight)
    out, lse = torch.full((B, Hq, D), 7.0, dtype=made.dt, device="cuda"), torch.full((B, Hq), 7.0, device="cuda")
    status = torch.zeros(1, **I32)
    ws = cache.workspace(Hq)
    ws.fill_(0xFF)
    api.si_kv4_attn_decode(cache, q, q_pos, kn if new else None, vn if new else None, window, n_sink, scale, out, lse,
                           api.SI_FLAG_ACC_WEIGHT if acc else 0, ws, status)
    torch.cuda.synchronize()
    assert status.item() == 0 and made.length.tolist() == list(lens)
    total, start = [n + 1 if new else n for n in lens], before.astype(np.float64)
    for b, n in enumerate(lens):
        if new:
            made.set(b, n, kn[b], vn[b])
            if acc:
                start[b, :, n] = 0.0
            if given:
                assert pos[b, :, n].tolist() == [int(q_pos[b])] * Hkv
    stored = [au.f64(x) for x in made.read(torch.tensor(total, **I32))]
    for x, y in zip(stored, (made.kq, made.vq)):         # the new entry, and nothing else changed
        want = ko.read_back(*y, made.dtype)
        for b, n in enumerate(total):
            assert np.array_equal(x[b, :, :n], want[b, :, :n], equal_nan=True)
    ref = k4.reference(made, q, total, window, n_sink, scale, None if pos is None else pos.cpu().numpy(), None if q_pos is None else q_pos.tolist())
    k4.check(out, lse, ref, made.dtype, D)
    if acc:
        k4.check_weight(weight, start, ref, D)
    else:
        assert np.array_equal(weight.cpu().numpy(), before)


@pytest.mark.parametrize("B,lens,Hq,Hkv,window,n_sink,given,new", DECODE)
@pytest.mark.parametrize("D,group,dtype,acc", [(128, 32, "bf16", True), (64, 32, "f16", True), (128, 64, "f16", False), (64, 64, "bf16", False)])
def test_decode(api, B, lens, Hq, Hkv, window, n_sink, given, new, D, group, dtype, acc):
    made = k4.Made(api, B, Hkv, D, (max(lens) + 33) // 32 * 32, group, dtype, lens, seed=7 * Hq + D)
    _decode_case(api, made, B, lens, Hq, Hkv, window, n_sink, given, new, acc, 1.0 / math.sqrt(D))


@pytest.mark.parametrize("B,Hq,Hkv,D,group,dtype,given", [(300, 4, 2, 64, 32, "bf16", False), (260, 12, 1, 128, 64, "f16", False), (140, 6, 1, 64, 64, "bf16", True)])
def test_decode_of_many_short_sequences(api, B, Hq, Hkv, D, group, dtype, given):
    """More sequences than a CTA has threads, empty ones among them; twelve and six query heads to a key head."""
    lens = [(37 * b) % 71 if b % 5 else 0 for b in range(B)]
    made = k4.Made(api, B, Hkv, D, 96, group, dtype, lens, seed=B)
    _decode_case(api, made, B, lens, Hq, Hkv, 0 if given else 20, 2, given, True, True, 0.1, seed=B)
    made = k4.Made(api, B, Hkv, D, 96, group, dtype, lens, seed=B + 1)
    _decode_case(api, made, B, lens, Hq, Hkv, 0, 0, False, False, True, 0.1, seed=B)


@pytest.mark.parametrize("Hq,Hkv,window,n_sink", [(16, 1, 1, 0), (12, 1, 500, 700), (3, 1, 33, 1), (2, 2, 64, 64)])
def test_decode_at_the_edges_of_windows(api, Hq, Hkv, window, n_sink):
    """A window of one entry, more first positions than entries, windows that end inside a tile and on its boundary."""
    for D, group, dtype in ((128, 32, "f16"), (64, 64, "bf16")):
        lens = [639, 640, 641, 33]
        made = k4.Made(api, 4, Hkv, D, 672, group, dtype, lens, seed=window)
        _decode_case(api, made, 4, lens, Hq, Hkv, window, n_sink, False, True, True, 0.1)


def test_a_query_before_every_entry_sees_nothing(api):
    made = k4.Made(api, 2, 2, 64, 64, 32, "bf16", [40, 3], seed=1)
    q, kn, vn = (torch.randn(2, h, 64, device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    out, lse = torch.full_like(q, 7.0), torch.full((2, 4), 7.0, device="cuda")
    weight = torch.full((2, 2, 64), 0.5, device="cuda")
    cache = api.KV4Cache(made.cache.data, 64, 32, made.dt, made.length, None, weight)
    api.si_kv4_attn_decode(cache, q, torch.tensor([-1, -5], **I32), kn, vn, 0, 0, 0.1, out, lse, api.SI_FLAG_ACC_WEIGHT, cache.workspace(4))
    assert (out == 0).all() and torch.isneginf(lse).all()
    for b, n in enumerate([40, 3]):
        made.set(b, n, kn[b], vn[b])
        assert (weight[b, :, n] == 0).all() and (weight[b, :, :n] == 0.5).all() and (weight[b, :, n + 1:] == 0.5).all()
    for x, y in zip(made.read(torch.tensor([41, 4], **I32)), (made.kq, made.vq)):
        for b, n in enumerate([41, 4]):
            assert same(x[b, :, :n], ko.read_back(*y, "bf16")[b, :, :n])


@pytest.mark.parametrize("dtype,scale,spread", [("bf16", 2.0, 4.0), ("f16", -0.7, 3.0), ("bf16", 1e-3, 2.0 ** -40), ("f16", 0.1, 2.0 ** -12), ("bf16", 2.0 ** -40, 2.0 ** 40), ("f16", 1.0, 0.0)])
def test_decode_with_scores_far_apart_and_queries_of_any_size(api, dtype, scale, spread):
    """Maxima that keep growing, a negative scale, queries far below and above one, all of them zero."""
    n, D = 700, 128
    g = torch.Generator().manual_seed(8)
    k = torch.randn(1, 2, 704, D, generator=g) * torch.linspace(0.1, 3.0, 704)[:, None]
    made = k4.Made(api, 1, 2, D, 704, 32, dtype, [n], k=k, v=torch.randn(1, 2, 704, D, generator=g))
    _decode_case(api, made, 1, [n], 8, 2, 0, 0, False, False, True, scale, spread=spread)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["growing", "shrinking", "tiny", "large", "constant", "mixed", "offset"])
def test_decode_with_steps_of_very_different_sizes(api, dtype, kind):
    """Values whose steps grow or shrink by orders of magnitude along the cache, or are all zero, or lie beside a large offset."""
    n, D = 1000, 64
    g = torch.Generator().manual_seed(4)
    v = torch.randn(1, 1, 1024, D, generator=g)
    lo, hi = (-12.0, 12.0) if dtype == "f16" else (-60.0, 60.0)
    along = torch.linspace(lo, hi, 1024)[:, None]
    v = {"growing": v * 2.0 ** along, "shrinking": v * 2.0 ** -along, "tiny": v * 2.0 ** (lo + 2), "large": v * 2.0 ** hi, "constant": torch.ones_like(v) * 3.25,
         "mixed": v * 2.0 ** (torch.rand(1, 1, 1024, 1, generator=g) * 20 - 10), "offset": v * 2.0 ** -4 + 1000}[kind]
    made = k4.Made(api, 1, 1, D, 1024, 32, dtype, [n], k=torch.randn(1, 1, 1024, D, generator=g) * 0.3, v=v)
    _decode_case(api, made, 1, [n], 4, 1, 0, 0, False, False, True, 0.1)


def test_decode_ignores_what_hidden_entries_hold(api):
    """Entries outside the window, after the query and beyond the length hold NaN steps: they never reach the result."""
    for D, Hq, Hkv in ((64, 8, 2), (128, 3, 1)):
        n, window, n_sink = 700, 50, 3
        g = torch.Generator().manual_seed(6)
        k, v = (torch.randn(1, Hkv, 736, D, generator=g) for _ in range(2))
        k[:, :, n_sink:n - window], v[:, :, n_sink:n - window] = float("nan"), float("inf")
        made = k4.Made(api, 1, Hkv, D, 736, 32, "bf16", [n], k=k, v=v)
        q = torch.randn(1, Hq, D, device="cuda").to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty(1, Hq, device="cuda")
        api.si_kv4_attn_decode(made.cache, q, None, None, None, window, n_sink, 0.1, out, lse, 0, made.cache.workspace(Hq))
        k4.check(out, lse, k4.reference(made, q, [n], window, n_sink, 0.1), "bf16", D)
        # with positions: every third entry lies after the query
        k, v = (torch.randn(1, Hkv, 736, D, generator=g) for _ in range(2))
        k[:, :, ::3], v[:, :, ::3] = float("inf"), float("nan")
        pos = torch.arange(736, **I32).expand(1, Hkv, 736).contiguous()
        pos[..., ::3] += 5000
        made = k4.Made(api, 1, Hkv, D, 736, 32, "bf16", [n], k=k, v=v)
        cache = api.KV4Cache(made.cache.data, D, 32, torch.bfloat16, made.length, pos)
        api.si_kv4_attn_decode(cache, q, torch.tensor([n - 1], **I32), None, None, 0, 0, 0.1, out, lse, 0, cache.workspace(Hq))
        k4.check(out, lse, k4.reference(made, q, [n], 0, 0, 0.1, pos.cpu().numpy(), [n - 1]), "bf16", D)


def test_nan_reaches_exactly_the_heads_that_see_it(api):
    D, n = 128, 300
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(1, 3, 320, D, generator=g) for _ in range(2))
    k[0, 0, 150, 5] = float("nan")
    v[0, 1, 20, 40] = float("inf")
    made = k4.Made(api, 1, 3, D, 320, 32, "bf16", [n], k=k, v=v)
    q = torch.randn(1, 6, D, device="cuda").to(torch.bfloat16)
    q[0, 5, 17] = float("nan")
    out, lse = torch.empty_like(q), torch.empty(1, 6, device="cuda")
    api.si_kv4_attn_decode(made.cache, q, None, None, None, 0, 0, 0.1, out, lse, 0, made.cache.workspace(6))
    assert out[0, 0:2].isnan().all() and lse[0, 0:2].isnan().all()             # a key: the whole row of the head's queries
    assert out[0, 2:4, 32:64].isnan().all() and not out[0, 2:4, :32].isnan().any() and not out[0, 2:4, 64:].isnan().any()     # a value: its group
    assert not lse[0, 2:4].isnan().any() and not out[0, 4].isnan().any()
    assert out[0, 5].isnan().all() and lse[0, 5].isnan()


def test_new_entries_that_their_query_does_not_see_are_stored_all_the_same(api):
    lens, at, window, D = [100, 100, 100, 50], [40, 300, 100, 49], 64, 128
    made = k4.Made(api, 4, 2, D, 128, 32, "bf16", lens, seed=12)
    kn, vn = (torch.randn(4, 2, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(4, 4, D, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(4, 4, device="cuda")
    weight = torch.full((4, 2, 128), 0.5, device="cuda")
    cache = api.KV4Cache(made.cache.data, D, 32, made.dt, made.length, None, weight)
    api.si_kv4_attn_decode(cache, q, torch.tensor(at, **I32), kn, vn, window, 0, 0.1, out, lse, api.SI_FLAG_ACC_WEIGHT, cache.workspace(4))
    total = [n + 1 for n in lens]
    for b, n in enumerate(lens):
        made.set(b, n, kn[b], vn[b])
    for x, y in zip(made.read(torch.tensor(total, **I32)), (made.kq, made.vq)):
        for b, n in enumerate(total):
            assert same(x[b, :, :n], ko.read_back(*y, "bf16")[b, :, :n])
    ref = k4.reference(made, q, total, window, 0, 0.1, np.broadcast_to(np.arange(128), (4, 2, 128)), at)
    k4.check(out, lse, ref, "bf16", D)
    start = np.full((4, 2, 128), 0.5)
    for b, n in enumerate(lens):
        start[b, :, n] = 0.0
    k4.check_weight(weight, start, ref, D)


def test_decode_repeats_its_bits(api):
    made = k4.Made(api, 3, 2, 128, 4096, 32, "f16", [4000, 77, 1500], seed=3)
    q = torch.randn(3, 8, 128, device="cuda").half()
    ws = made.cache.workspace(8)
    got = []
    for _ in range(3):
        ws.random_(0, 255)
        out, lse = torch.empty_like(q), torch.empty(3, 8, device="cuda")
        api.si_kv4_attn_decode(made.cache, q, None, None, None, 0, 0, 0.09, out, lse, 0, ws)
        got.append((bits(out), lse))
    assert all(torch.equal(a, got[0][0]) and torch.equal(b, got[0][1]) for a, b in got)


EVICT = [
    # B, H, lens, capacity, budget, n_sink, n_recent, n_new, in place
    (1, 1, [40], 64, 20, 0, 0, 0, False), (2, 3, [500, 70], 512, 100, 4, 30, 0, False), (1, 2, [5000], 5024, 333, 4, 64, 0, False),
    (2, 2, [90, 33], 96, 64, 1, 5, 0, True), (3, 2, [256, 256, 200], 288, 256, 4, 20, 1, True), (1, 4, [2000], 2016, 500, 0, 100, 0, True),
    (2, 1, [31, 32], 64, 31, 0, 1, 1, True), (1, 1, [64], 64, 64, 0, 0, 0, True), (2, 2, [10, 0], 64, 32, 4, 4, 0, False),
]


@pytest.mark.parametrize("B,H,lens,cap,budget,n_sink,n_recent,n_new,in_place", EVICT)
@pytest.mark.parametrize("D,group", SHAPES)
def test_eviction(api, B, H, lens, cap, budget, n_sink, n_recent, n_new, in_place, D, group):
    total = [n + n_new for n in lens]
    made = k4.Made(api, B, H, D, cap, group, "bf16", total, seed=budget)
    rng = np.random.default_rng(cap + budget)
    weight = rng.random((B, H, cap)).astype(np.float32)
    weight[..., ::7] = 0.25                                             # ties
    weight[..., 3] = np.nan
    pos = np.stack([[rng.permutation(2 * cap)[:cap] for _ in range(H)] for _ in range(B)]).astype(np.int32) if in_place else np.broadcast_to(np.arange(cap, dtype=np.int32), (B, H, cap))
    last = [2 * cap] * B if in_place else [n - 1 for n in total]
    wt, pt = torch.from_numpy(weight).cuda(), torch.from_numpy(pos.copy()).cuda()
    length = torch.tensor(lens, **I32)
    src = api.KV4Cache(made.cache.data, D, group, made.dt, length, pt if in_place else None, wt)
    kept, len_out, status = torch.full((B, H, budget), -9, **I32), torch.zeros(B, **I32), torch.zeros(1, **I32)
    before = made.read()
    if in_place:
        dst = src
    else:
        other = k4.Made(api, B, H, D, (budget + 40) // 32 * 32, group, "bf16", [(budget + 40) // 32 * 32] * B, seed=1)
        dc = other.cache
        dst = api.KV4Cache(dc.data, D, group, made.dt, len_out, torch.full((B, H, dc.capacity), -3, **I32), torch.full((B, H, dc.capacity), -3.0, device="cuda"))
        held = other.read()
    api.si_kv4_evict(src, dst, torch.tensor(last, **I32) if in_place else None, n_new, budget, n_sink, n_recent, kept, len_out, src.workspace(0), status)
    after = made.read() if in_place else other.read()
    assert status.item() == 0 and len_out.tolist() == [min(n, budget) for n in total]
    stay = before if in_place else held
    for b in range(B):
        for h in range(H):
            n = total[b]
            want = ao.evict(weight[b, h, :n].astype(np.float64), pos[b, h, :n], last[b], budget, n_sink, n_recent)
            assert np.array_equal(kept[b, h].cpu().numpy(), want)
            m = int((want >= 0).sum())
            at = torch.from_numpy(want[:m]).cuda()
            for x, y, z in zip(after, before, stay):
                assert torch.equal(bits(x[b, h, :m]), bits(y[b, h, at])) and torch.equal(bits(x[b, h, m:]), bits(z[b, h, m:]))
            assert np.array_equal(dst.pos[b, h, :m].cpu().numpy(), pos[b, h, want[:m]])
            assert np.array_equal(dst.weight[b, h, :m].cpu().numpy(), weight[b, h, want[:m]], equal_nan=True)
