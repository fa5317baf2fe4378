"""Refusals of the cache calls that the host can see: no GPU, no launch (pointers below are never followed)."""
import ctypes

import numpy as np
import pytest

from oracle import attention_oracle as ao

P = ctypes.c_void_p
FAKE, NULL = 0x10000, None


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def _kv(api, **change):
    f = dict(k=FAKE, v=FAKE * 2, weight=FAKE * 3, pos=None, len=FAKE * 4, seq_stride=8 * 100 * 128, head_stride=100 * 128, row_stride=128,
             n_seqs=2, n_kv_heads=8, head_dim=128, capacity=100, dtype=api.SI_BF16)
    f.update(change)
    return api._KvDesc(**f)


def _prefill(api, kv, q=FAKE, ss=4096, ts=4096, T=4, hq=32, window=0, n_sink=0, scale=0.1, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 40):
    return api.lib().si_attn_prefill(ctypes.byref(kv), q, ss, ts, T, hq, window, n_sink, scale, out, lse, ws, ws_bytes, None, None)


def _weights(api, kv, q=FAKE, ss=4096, ts=4096, T=4, hq=32, window=0, n_sink=0, scale=0.1, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return api.lib().si_attn_weights(ctypes.byref(kv), q, ss, ts, T, hq, window, n_sink, scale, lse, ws, ws_bytes, None, None)


def _decode(api, kv, q=FAKE, ss=4096, hq=32, q_pos=None, kn=None, vn=None, ns=1024, window=0, n_sink=0, scale=0.1, out=FAKE, lse=None, flags=0,
            ws=FAKE, ws_bytes=1 << 40):
    return api.lib().si_attn_decode(ctypes.byref(kv), q, ss, hq, q_pos, kn, vn, ns, window, n_sink, scale, out, lse, flags, ws, ws_bytes, None, None)


def _evict(api, src, dst, q_pos=FAKE, n_new=0, budget=50, n_sink=4, n_recent=4, ws=FAKE, ws_bytes=1 << 40):
    return api.lib().si_kv_evict(ctypes.byref(src), ctypes.byref(dst), q_pos, n_new, budget, n_sink, n_recent, None, None, ws, ws_bytes, None, None)


BAD_CACHES = [
    (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(len=None), "INVALID_ARG"), (dict(n_seqs=-1), "INVALID_ARG"),
    (dict(n_kv_heads=0), "INVALID_ARG"), (dict(capacity=0), "INVALID_ARG"), (dict(dtype=3), "INVALID_ARG"), (dict(dtype=0), "INVALID_ARG"),
    (dict(head_dim=96), "UNSUPPORTED"), (dict(head_dim=256), "UNSUPPORTED"), (dict(row_stride=64), "INVALID_ARG"),
    (dict(head_stride=-8), "INVALID_ARG"), (dict(row_stride=132), "ALIGNMENT"), (dict(head_stride=4), "ALIGNMENT"), (dict(seq_stride=1), "ALIGNMENT"),
    (dict(k=FAKE + 2), "ALIGNMENT"), (dict(v=FAKE + 8), "ALIGNMENT"),
]


@pytest.mark.parametrize("change,err", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(api, change, err):
    want = getattr(api, "SI_ERR_" + err)
    kv, good = _kv(api, **change), _kv(api, pos=FAKE)
    assert _prefill(api, kv) == want and _weights(api, kv) == want and _decode(api, kv) == want
    assert _evict(api, kv, good) == want and _evict(api, good, kv) == want
    out = ctypes.c_size_t(0)
    assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), 32, 1, ctypes.byref(out)) == want


def test_bad_arguments_are_refused(api):
    I, U, A, N = api.SI_ERR_INVALID_ARG, api.SI_ERR_UNSUPPORTED, api.SI_ERR_ALIGNMENT, api.SI_ERR_NOMEM
    kv, pos = _kv(api), _kv(api, pos=FAKE)
    for call in (_prefill, _weights, _decode):
        assert call(api, kv, hq=0) == I and call(api, kv, hq=12) == I and call(api, kv, window=-1) == I and call(api, kv, n_sink=-1) == I
        assert call(api, kv, scale=float("nan")) == I and call(api, kv, scale=float("inf")) == I
        assert call(api, kv, hq=8 * 129) == U and call(api, kv, q=None) == I and call(api, kv, q=FAKE + 2) == A and call(api, kv, ss=4100) == A
        assert call(api, kv, ss=-8) == I
    for call in (_prefill, _weights):
        assert call(api, kv, T=-1) == I and call(api, kv, ts=12) == A and call(api, pos) == U and call(api, kv, ts=0) == U
        assert call(api, kv, T=0, q=None) == api.SI_OK and call(api, _kv(api, n_seqs=0, k=None, v=None, len=None)) == api.SI_OK
    assert _prefill(api, kv, out=None) == I and _prefill(api, kv, out=FAKE + 4) == A
    assert _weights(api, kv, lse=None) == I and _weights(api, _kv(api, weight=None)) == I
    assert _decode(api, kv, out=None) == I and _decode(api, pos) == I                       # positions without the query's
    assert _decode(api, kv, kn=FAKE) == I and _decode(api, kv, vn=FAKE) == I                # one of the two only
    assert _decode(api, kv, kn=FAKE + 2, vn=FAKE) == A and _decode(api, kv, kn=FAKE, vn=FAKE, ns=1022) == A
    assert _decode(api, kv, flags=1) == I and _decode(api, _kv(api, weight=None), flags=api.SI_FLAG_ACC_WEIGHT) == I
    need = ctypes.c_size_t(0)
    assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), 32, 1, ctypes.byref(need)) == api.SI_OK
    assert need.value > 0 and _decode(api, kv, ws_bytes=0) == N and _evict(api, pos, pos, ws_bytes=0) == N
    assert _decode(api, kv, ws=None) == I and _evict(api, pos, pos, ws=None) == I and _evict(api, pos, pos, ws=FAKE + 16) == A
    assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), 12, 1, ctypes.byref(need)) == I
    assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), 32, -1, ctypes.byref(need)) == I
    assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), 32, 1, None) == I


def test_bad_evictions_are_refused(api):
    I = api.SI_ERR_INVALID_ARG
    src, dst = _kv(api), _kv(api, k=FAKE * 8, v=FAKE * 9, pos=FAKE, weight=FAKE)
    pos = _kv(api, pos=FAKE)
    for bad in (dict(budget=0), dict(budget=101), dict(n_new=-1), dict(n_new=101), dict(n_sink=-1), dict(n_recent=-1), dict(n_sink=30, n_recent=21)):
        assert _evict(api, src, dst, **bad) == I
    for change in (dict(n_seqs=1), dict(n_kv_heads=4), dict(head_dim=64), dict(dtype=api.SI_F16), dict(pos=None), dict(weight=None)):
        f = {n: getattr(dst, n) for n, _ in dst._fields_}
        f.update(change)
        assert _evict(api, src, api._KvDesc(**f)) == I
    assert _evict(api, _kv(api, weight=None), dst) == I
    assert _evict(api, src, src) == I                                # in place without positions
    assert _evict(api, pos, dst, q_pos=None) == I                    # positions without the newest one
    assert _evict(api, pos, _kv(api, pos=FAKE, v=FAKE * 5)) == I     # half in place


def test_writes_to_shared_memory_are_refused(api):
    I, N = api.SI_ERR_INVALID_ARG, api.SI_ERR_NOMEM
    for change in (dict(seq_stride=0), dict(head_stride=0)):
        kv = _kv(api, **change)
        assert _decode(api, kv, kn=FAKE, vn=FAKE) == I and _decode(api, kv, ws_bytes=0) == N          # reading is fine
        assert _evict(api, _kv(api), _kv(api, k=FAKE * 8, v=FAKE * 9, pos=FAKE, weight=FAKE, **change)) == I
        assert _evict(api, _kv(api, pos=FAKE, **change), _kv(api, pos=FAKE, **change)) == I
        assert _evict(api, kv, _kv(api, k=FAKE * 8, v=FAKE * 9, pos=FAKE, weight=FAKE), ws_bytes=0) == N
        alone = _kv(api, n_seqs=1, n_kv_heads=1, **change)
        assert _decode(api, alone, kn=FAKE, vn=FAKE, ws_bytes=0) == N
    src = _kv(api, pos=FAKE * 7)
    apart = dict(k=FAKE * 8, v=FAKE * 9, pos=FAKE, weight=FAKE)
    assert _evict(api, src, _kv(api, **apart), ws_bytes=0) == N
    for same in (dict(v=src.v), dict(pos=src.pos), dict(weight=src.weight)):
        assert _evict(api, src, _kv(api, **{**apart, **same})) == I


def test_scales_beyond_the_type_are_refused(api):
    for scale in (2.5e38, -2.5e38):
        for call in (_prefill, _weights, _decode):
            assert call(api, _kv(api), scale=scale) == api.SI_ERR_INVALID_ARG


def test_oracle_eviction_by_hand():
    w = np.array([5.0, 1.0, 4.0, np.nan, 4.0, 0.5, 9.0])
    # budget 4, position 5 recent (protected): kept are slots 5, 6, 0 and the lower of the tied 2 and 4
    assert ao.evict(w, np.array([0, 1, 2, 3, 4, 7, 6]), 7, 4, 0, 1).tolist() == [0, 5, 2, 6]
    assert ao.evict(w, np.arange(7), 6, 9, 0, 0).tolist() == [0, 1, 2, 3, 4, 5, 6, -1, -1]
    assert ao.evict(np.array([np.nan, -np.inf, 1.0]), np.arange(3), 2, 2, 0, 0).tolist() == [2, 1]


def test_oracle_attention_against_the_definition():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    out, lse, w, _, _ = ao.attend(q, k, v, np.arange(6), np.array([1, 5, -1]), 2, 1, 0.5)
    # query at position 1 sees entries 0, 1; at 5: 4, 5 (window) and 0 (first position); at -1: nothing
    for i, see in ((0, [0, 1]), (1, [0, 4, 5])):
        e = np.exp(0.5 * k[see] @ q[i])
        assert np.allclose(out[i], e @ v[see] / e.sum()) and np.isclose(lse[i], np.log(e.sum())) and np.isclose(w[i].sum(), 1.0)
        assert np.array_equal(np.nonzero(w[i])[0], see)
    assert np.all(out[2] == 0) and np.isneginf(lse[2]) and np.all(w[2] == 0)


@pytest.mark.parametrize("shape", [dict(), dict(n_seqs=3), dict(head_dim=64, row_stride=64), dict(n_kv_heads=1), dict(n_seqs=20), dict(weight=None)])
@pytest.mark.parametrize("capacity", [100, 1200, 8192, 12288, 300001])
def test_a_workspace_covers_fewer_queries_and_heads(api, shape, capacity):
    """Fewer rows are split over more CTAs, so the need of one size says nothing about that of a smaller one: the size is for all."""
    f = dict(n_seqs=1, capacity=capacity)
    f.update(shape)
    kv = _kv(api, **f)
    need = ctypes.c_size_t(0)

    def size(hq, T):
        assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), hq, T, ctypes.byref(need)) == api.SI_OK
        return need.value

    heads, tokens = [kv.n_kv_heads * g for g in (1, 2, 3, 4, 7, 8, 20, 64, 128)], [1, 2, 13, 45, 64, 129, 512, 600, 2048, 8192]
    table = [[size(hq, T) for T in tokens] for hq in heads]
    for row in table:
        assert row == sorted(row)
    for col in zip(*table):
        assert list(col) == sorted(col)


def test_a_short_chunk_passes_with_the_workspace_of_a_long_one(api):
    """Splits of the keys need room (a workspace of NULL is refused behind the size check): never more than the larger size gave."""
    need = ctypes.c_size_t(0)
    for capacity, T_max, hq_max in ((8192, 2048, 32), (12288, 8192, 32), (8192, 1024, 64)):
        kv = _kv(api, n_seqs=1, capacity=capacity)
        assert api.lib().si_kv_workspace_bytes(ctypes.byref(kv), hq_max, T_max, ctypes.byref(need)) == api.SI_OK
        for T, hq in ((1, 32), (45, 32), (200, 8), (512, 32)):
            assert _prefill(api, kv, T=T, hq=hq, ws_bytes=0) == api.SI_ERR_NOMEM           # split: it does need room
            assert _prefill(api, kv, T=T, hq=hq, ws=None, ws_bytes=need.value) == api.SI_ERR_INVALID_ARG


class _On:
    """A tensor of host memory that says it lies on a CUDA device (its address is never followed: the calls below end before a launch)."""

    def __init__(self, t, device):
        self.t, self.n, self.is_cuda, self.device = t, device, device >= 0, f"cuda:{device}"

    def get_device(self):
        return self.n

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_the_binding_refuses_tensors_of_another_device(api, monkeypatch):
    import torch
    B, H, cap, D, Hq = 2, 2, 16, 64, 4
    bf16, i32, f32 = torch.bfloat16, torch.int32, torch.float32

    def on(device, *shape, dtype=bf16):
        return _On(torch.zeros(*shape, dtype=dtype), device)

    def cache(device=1, **other):
        t = dict(k=on(device, B, H, cap, D), v=on(device, B, H, cap, D), length=on(device, B, dtype=i32), pos=None, weight=on(device, B, H, cap, dtype=f32))
        t.update(other)
        return api.KVCache(t["k"], t["v"], t["length"], t["pos"], t["weight"])

    for name, shape, dtype in (("v", (B, H, cap, D), bf16), ("length", (B,), i32), ("pos", (B, H, cap), i32), ("weight", (B, H, cap), f32)):
        for device in (0, -1):
            with pytest.raises(ValueError):
                cache(**{name: on(device, *shape, dtype=dtype)})
    with pytest.raises(ValueError):
        cache(-1)
    here = 1
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    c, elsewhere = cache(), cache(0)

    class stream:
        device_index, cuda_stream = 0, 0

    def calls(c, at, T=0, **kw):          # T = 0: nothing to launch
        q, out, lse = on(at.get("q", 1), B, T, Hq, D), on(at.get("out", 1), B, T, Hq, D), on(at.get("lse", 1), B, T, Hq, dtype=f32)
        ws, status = on(at.get("ws", 1), 1 << 20, dtype=torch.uint8), on(at.get("status", 1), 1, dtype=i32)
        yield lambda: api.si_attn_prefill(c, q, 0, 0, 0.1, out, lse, ws, status, **kw)
        if "out" not in at:
            yield lambda: api.si_attn_weights(c, q, 0, 0, 0.1, lse, ws, status, **kw)

    for f in calls(c, {}):
        f()
    for at in (dict(q=0), dict(out=0), dict(lse=0), dict(ws=0), dict(status=0), dict(q=-1)):
        for f in calls(c, at):
            with pytest.raises(ValueError):
                f()
    for f in calls(c, {}, stream=stream):
        with pytest.raises(ValueError):
            f()
    new = [on(d, B, H, D) for d in (1, 0)]
    q1, out1, ws = on(1, B, Hq, D), on(1, B, Hq, D), on(1, 1 << 20, dtype=torch.uint8)
    for args in ((on(0, B, Hq, D), None, None, None), (q1, on(0, B, dtype=i32), None, None), (q1, None, new[1], new[1]), (q1, None, new[0], new[1])):
        with pytest.raises(ValueError):
            api.si_attn_decode(c, *args, 0, 0, 0.1, out1, None, 0, ws)
    with pytest.raises(ValueError):
        api.si_kv_evict(c, elsewhere, None, 0, 4, 0, 0, None, None, ws)
    with pytest.raises(ValueError):
        api.si_kv_evict(c, c, None, 0, 4, 0, 0, on(0, B, H, 4, dtype=i32), None, ws)
    here = 0                                # another device is current
    for f in calls(c, {}):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        api.si_attn_decode(c, q1, None, None, None, 0, 0, 0.1, out1, None, 0, ws)
    with pytest.raises(ValueError):
        api.si_kv_evict(c, c, None, 0, 4, 0, 0, None, None, ws)


def test_words_off_their_boundaries_are_refused(api):
    """Pointers that are not multiples of four would fault on the device.  (No workspace is given: without the check the calls end there.)"""
    A, N = api.SI_ERR_ALIGNMENT, api.SI_ERR_NOMEM
    kv, pos = _kv(api, n_seqs=1, capacity=8192), _kv(api, n_seqs=1, capacity=8192, pos=FAKE)
    calls = (_prefill, _weights, _decode)
    assert all(c(api, kv, ws_bytes=0) == N for c in calls) and _evict(api, pos, pos, ws_bytes=0) == N
    for change in (dict(weight=FAKE + 2), dict(len=FAKE + 1), dict(pos=FAKE + 3)):
        bad = _kv(api, n_seqs=1, capacity=8192, **{**dict(pos=None), **change})
        assert _decode(api, bad, q_pos=FAKE, ws_bytes=0) == A
        assert _evict(api, _kv(api, n_seqs=1, capacity=8192, **{**dict(pos=FAKE), **change}), pos, ws_bytes=0) == A
        if "pos" not in change:
            assert _prefill(api, bad, ws_bytes=0) == A and _weights(api, bad, ws_bytes=0) == A
    assert _prefill(api, kv, lse=FAKE + 2, ws_bytes=0) == A and _weights(api, kv, lse=FAKE + 2, ws_bytes=0) == A
    assert _decode(api, kv, lse=FAKE + 2, ws_bytes=0) == A and _decode(api, kv, q_pos=FAKE + 2, ws_bytes=0) == A
    assert _evict(api, pos, pos, q_pos=FAKE + 2, ws_bytes=0) == A
    lib, ref = api.lib(), ctypes.byref
    for kept, len_out, status in ((FAKE + 1, None, None), (None, FAKE + 2, None), (None, None, FAKE + 3)):
        assert lib.si_kv_evict(ref(pos), ref(pos), FAKE, 0, 50, 4, 4, kept, len_out, FAKE, 0, status, None) == A
    assert lib.si_attn_prefill(ref(kv), FAKE, 4096, 4096, 4, 32, 0, 0, 0.1, FAKE, None, FAKE, 0, FAKE + 2, None) == A
    assert lib.si_attn_weights(ref(kv), FAKE, 4096, 4096, 4, 32, 0, 0, 0.1, FAKE, FAKE, 0, FAKE + 2, None) == A
    assert lib.si_attn_decode(ref(kv), FAKE, 4096, 32, None, None, None, 0, 0, 0, 0.1, FAKE, None, 0, FAKE, 0, FAKE + 2, None) == A
