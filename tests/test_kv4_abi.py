"""The cache in 4 bits: refusals that the host can see (no GPU, no launch; pointers below are never followed), sizes, and the
oracle's statement of the format."""
import ctypes

import numpy as np
import pytest

from oracle import kv4_oracle as ko

FAKE = 0x10000
REF = ctypes.byref


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def _kv4(api, **change):
    f = dict(data=FAKE, weight=FAKE * 3, pos=None, len=FAKE * 4, seq_stride=8 * 4 * 5120, head_stride=4 * 5120, n_seqs=2, n_kv_heads=8,
             head_dim=128, capacity=128, group=32, dtype=api.SI_BF16)
    f.update(change)
    return api._Kv4Desc(**f)


def _kv(api, **change):
    f = dict(k=FAKE, v=FAKE * 2, weight=FAKE * 3, pos=None, len=FAKE * 4, seq_stride=8 * 100 * 128, head_stride=100 * 128, row_stride=128,
             n_seqs=2, n_kv_heads=8, head_dim=128, capacity=100, dtype=api.SI_BF16)
    f.update(change)
    return api._KvDesc(**f)


def _store(api, src, dst, first_pos=None, status=None):
    return api.lib().si_kv4_store(REF(src), REF(dst), first_pos, status, None)


def _load(api, src, dst, first=None, n=50, len_out=None, status=None):
    return api.lib().si_kv4_load(REF(src), REF(dst), first, n, len_out, status, None)


def _decode(api, kv, q=FAKE, ss=4096, hq=32, q_pos=None, kn=None, vn=None, ns=1024, window=0, n_sink=0, scale=0.1, out=FAKE, lse=None, flags=0,
            ws=FAKE, ws_bytes=1 << 40, status=None):
    return api.lib().si_kv4_attn_decode(REF(kv), q, ss, hq, q_pos, kn, vn, ns, window, n_sink, scale, out, lse, flags, ws, ws_bytes, status, None)


def _evict(api, src, dst, q_pos=FAKE, n_new=0, budget=50, n_sink=4, n_recent=4, kept=None, len_out=None, ws=FAKE, ws_bytes=1 << 40, status=None):
    return api.lib().si_kv4_evict(REF(src), REF(dst), q_pos, n_new, budget, n_sink, n_recent, kept, len_out, ws, ws_bytes, status, None)


BAD = [
    (dict(data=None), "INVALID_ARG"), (dict(len=None), "INVALID_ARG"), (dict(n_seqs=-1), "INVALID_ARG"), (dict(n_kv_heads=0), "INVALID_ARG"),
    (dict(capacity=0), "INVALID_ARG"), (dict(capacity=100), "INVALID_ARG"), (dict(capacity=16), "INVALID_ARG"), (dict(dtype=3), "INVALID_ARG"),
    (dict(head_dim=96), "UNSUPPORTED"), (dict(head_dim=256), "UNSUPPORTED"), (dict(group=16), "UNSUPPORTED"), (dict(group=128), "UNSUPPORTED"),
    (dict(head_stride=-16), "INVALID_ARG"), (dict(head_stride=8), "ALIGNMENT"), (dict(seq_stride=4), "ALIGNMENT"), (dict(data=FAKE + 8), "ALIGNMENT"),
    (dict(pos=FAKE + 4), "ALIGNMENT"), (dict(weight=FAKE + 8), "ALIGNMENT"), (dict(len=FAKE + 2), "ALIGNMENT"),
]


@pytest.mark.parametrize("change,err", BAD)
def test_bad_caches_are_refused_by_every_call(api, change, err):
    want, bad, good, kv = getattr(api, "SI_ERR_" + err), _kv4(api, **change), _kv4(api, data=FAKE * 8, pos=FAKE), _kv(api)
    assert _store(api, kv, bad) == want and _load(api, bad, kv) == want and _decode(api, bad, q_pos=FAKE, ws_bytes=0) == want
    assert _evict(api, bad, good) == want and _evict(api, good, bad) == want
    out = ctypes.c_size_t(0)
    assert api.lib().si_kv4_workspace_bytes(REF(bad), 32, REF(out)) == want


def test_bad_arguments_are_refused(api):
    I, U, A, N, OK = api.SI_ERR_INVALID_ARG, api.SI_ERR_UNSUPPORTED, api.SI_ERR_ALIGNMENT, api.SI_ERR_NOMEM, api.SI_OK
    kv4, kv, pos = _kv4(api), _kv(api), _kv4(api, pos=FAKE)
    # store and load: the 16-bit side's own checks, shapes that differ, writes to shared rows, words off their boundaries
    assert _store(api, _kv(api, k=None), kv4) == I and _load(api, kv4, _kv(api, v=FAKE + 2)) == A
    for change in (dict(n_seqs=1), dict(n_kv_heads=4), dict(head_dim=64), dict(dtype=api.SI_F16)):
        assert _store(api, _kv(api, **change), kv4) == I and _load(api, kv4, _kv(api, **change)) == I
    for change in (dict(seq_stride=0), dict(head_stride=0)):
        assert _store(api, kv, _kv4(api, **change)) == I and _load(api, kv4, _kv(api, **change)) == I
        assert _decode(api, _kv4(api, **change), kn=FAKE, vn=FAKE) == I and _decode(api, _kv4(api, **change), ws_bytes=0) == N
        assert _evict(api, kv4, _kv4(api, data=FAKE * 8, pos=FAKE, weight=FAKE, **change)) == I
    assert _load(api, kv4, kv, n=-1) == I and _load(api, kv4, kv, n=101) == I
    assert _store(api, kv, kv4, first_pos=FAKE + 2) == A and _store(api, kv, kv4, status=FAKE + 1) == A
    assert _load(api, kv4, kv, first=FAKE + 2) == A and _load(api, kv4, kv, len_out=FAKE + 2) == A and _load(api, kv4, kv, status=FAKE + 3) == A
    none4, none = _kv4(api, n_seqs=0, data=None, len=None), _kv(api, n_seqs=0, k=None, v=None, len=None)
    assert _store(api, none, none4) == OK and _load(api, none4, none) == OK and _decode(api, none4) == OK
    # attention: as si_attn_decode
    assert _decode(api, kv4, hq=0) == I and _decode(api, kv4, hq=12) == I and _decode(api, kv4, window=-1) == I and _decode(api, kv4, n_sink=-1) == I
    assert _decode(api, kv4, scale=float("nan")) == I and _decode(api, kv4, scale=2.5e38) == I and _decode(api, kv4, hq=8 * 129) == U
    assert _decode(api, kv4, q=None) == I and _decode(api, kv4, q=FAKE + 2) == A and _decode(api, kv4, ss=4100) == A and _decode(api, kv4, ss=-8) == I
    assert _decode(api, kv4, out=None) == I and _decode(api, kv4, out=FAKE + 4) == A and _decode(api, pos) == I
    assert _decode(api, kv4, kn=FAKE) == I and _decode(api, kv4, vn=FAKE) == I and _decode(api, kv4, kn=FAKE + 2, vn=FAKE) == A
    assert _decode(api, kv4, kn=FAKE, vn=FAKE, ns=1022) == A and _decode(api, kv4, flags=1) == I
    assert _decode(api, _kv4(api, weight=None), flags=api.SI_FLAG_ACC_WEIGHT) == I
    assert _decode(api, kv4, lse=FAKE + 2) == A and _decode(api, kv4, q_pos=FAKE + 2) == A and _decode(api, kv4, status=FAKE + 2) == A
    assert _decode(api, kv4, ws_bytes=0) == N and _decode(api, kv4, ws=None) == I and _decode(api, kv4, ws=FAKE + 16) == A
    assert _decode(api, _kv4(api, n_seqs=65535, n_kv_heads=65535, capacity=32, weight=None), hq=65535, ws_bytes=0) == api.SI_ERR_TOO_LARGE
    # eviction: as si_kv_evict
    dst = dict(data=FAKE * 8, pos=FAKE, weight=FAKE)
    for bad in (dict(budget=0), dict(budget=129), dict(n_new=-1), dict(n_new=129), dict(n_sink=-1), dict(n_recent=-1), dict(n_sink=30, n_recent=21)):
        assert _evict(api, kv4, _kv4(api, **dst), **bad) == I
    for change in (dict(n_seqs=1), dict(n_kv_heads=4), dict(head_dim=64), dict(dtype=api.SI_F16), dict(group=64), dict(pos=None), dict(weight=None)):
        assert _evict(api, kv4, _kv4(api, **{**dst, **change})) == I
    assert _evict(api, _kv4(api, weight=None), _kv4(api, **dst)) == I and _evict(api, kv4, kv4) == I
    assert _evict(api, pos, _kv4(api, **dst), q_pos=None) == I and _evict(api, pos, _kv4(api, pos=FAKE, weight=FAKE * 7)) == I
    src = _kv4(api, pos=FAKE * 7)
    for same in (dict(pos=src.pos), dict(weight=src.weight)):
        assert _evict(api, src, _kv4(api, **{**dst, **same})) == I
    assert _evict(api, pos, pos, ws_bytes=0) == N and _evict(api, pos, pos, ws=None) == I and _evict(api, pos, pos, ws=FAKE + 16) == A
    for word in (dict(q_pos=FAKE + 2), dict(kept=FAKE + 1), dict(len_out=FAKE + 2), dict(status=FAKE + 3)):
        assert _evict(api, pos, pos, **word) == A


def test_sizes(api):
    sizes = {(d, g): api.si_kv4_tile_bytes(d, g) for d in (64, 128) for g in (32, 64)}
    # 32 entries of two halves of D / 2 bytes, and 4 bytes per group of either
    assert sizes == {(64, 32): 2560, (64, 64): 2304, (128, 32): 5120, (128, 64): 4608}
    lib, out = api.lib(), ctypes.c_size_t(0)
    assert lib.si_kv4_tile_bytes(96, 32, REF(out)) == api.SI_ERR_UNSUPPORTED and lib.si_kv4_tile_bytes(64, 32, None) == api.SI_ERR_INVALID_ARG

    def ws(hq, **change):
        assert lib.si_kv4_workspace_bytes(REF(_kv4(api, **change)), hq, REF(out)) == api.SI_OK
        return out.value
    for change in (dict(), dict(capacity=8192), dict(weight=None), dict(n_seqs=40, head_dim=64)):
        assert ws(0, **change) <= ws(8, **change) <= ws(32, **change) <= ws(8 * 128, **change)
    kv4 = _kv4(api)
    assert lib.si_kv4_workspace_bytes(REF(kv4), 12, REF(out)) == api.SI_ERR_INVALID_ARG and lib.si_kv4_workspace_bytes(REF(kv4), 32, None) == api.SI_ERR_INVALID_ARG
    assert lib.si_kv4_workspace_bytes(REF(kv4), 8 * 129, REF(out)) == api.SI_ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_oracle_format(dtype):
    import torch
    dt = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    # by hand: 0 .. 15 are their own codes; a step of 1 + 1 / 15 is rounded up
    m, s, c = ko.quantise(np.arange(32) % 16, 32, dtype)
    assert np.all(m == 0) and np.all(s == 1) and np.array_equal(c, np.arange(32) % 16)
    m, s, c = ko.quantise(np.linspace(-8, 8, 32).round(), 32, dtype)
    up = 1.0703125 if dtype == "bf16" else 1.0673828125         # the next values above 16 / 15 = 1.0667
    assert np.all(m == -8) and np.all(s == up) and c[0] == 0 and c[-1] == 15
    # rounding agrees with torch's, and quantised values are within half a step
    x = torch.randn(40, 128, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * torch.exp(2 * torch.randn(40, 1, generator=torch.Generator().manual_seed(2), dtype=torch.float64))
    assert np.array_equal(ko.round16(x.float().double().numpy(), dtype), x.float().to(dt).double().numpy())
    x = x.to(dt).double().numpy()
    for group in (32, 64):
        m, s, c = ko.quantise(x, group, dtype)
        assert np.all(np.abs(m + s * c - x) <= s / 2 * (1 + 2.0 ** -20)) and np.array_equal(ko.round16(s, dtype), s) and np.array_equal(ko.round16(m, dtype), m)
        span = x.reshape(40, -1, group).max(-1) - x.reshape(40, -1, group).min(-1)
        step = s.reshape(40, -1, group)[..., 0]
        assert np.all(step * 15 >= span * (1 - 2.0 ** -23)) and np.all(step * 15 <= span * (1 + 2.0 ** -7))
    # a constant, a group with a NaN, one with an infinity, one with a range beyond the limit
    for v, want in ((np.full(32, 3.5), 3.5), (np.r_[np.nan, np.zeros(31)], np.nan), (np.r_[np.inf, np.zeros(31)], np.nan)):
        m, s, c = ko.quantise(v, 32, dtype)
        assert np.array_equal(ko.read_back(m, s, c, dtype), np.full(32, want), equal_nan=True)
    assert np.isnan(ko.quantise(np.r_[2.0 ** 95, np.zeros(31)], 32, "bf16")[1]).all()


class _On:
    """A tensor of host memory that says it lies on a CUDA device (its address is never followed)."""

    def __init__(self, t, device):
        self.t, self.n, self.is_cuda, self.device = t, device, device >= 0, f"cuda:{device}"

    def get_device(self):
        return self.n

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_the_binding_refuses_wrong_tensors(api, monkeypatch):
    import torch
    B, H, D, Hq = 2, 2, 64, 4
    u8, i32, f32, bf16 = torch.uint8, torch.int32, torch.float32, torch.bfloat16

    def on(device, *shape, dtype=bf16):
        return _On(torch.zeros(*shape, dtype=dtype), device)

    def cache(device=1, **other):
        t = dict(data=on(device, B, H, 3, 2560, dtype=u8), length=on(device, B, dtype=i32), pos=None, weight=None)
        t.update(other)
        return api.KV4Cache(t["data"], D, 32, bf16, t["length"], t["pos"], t["weight"])

    assert cache().capacity == 96
    for bad in (dict(data=on(1, B, H, 3, 2304, dtype=u8)), dict(data=on(1, B, H, 3, 2560, dtype=torch.int8)), dict(length=on(1, B + 1, dtype=i32)), dict(length=on(0, B, dtype=i32)),
                dict(pos=on(1, B, H, 95, dtype=i32)), dict(weight=on(1, B, H, 96, dtype=i32)), dict(weight=on(-1, B, H, 96, dtype=f32)),
                dict(data=_On(torch.zeros(B, H, 6, 2560, dtype=u8)[:, :, ::2], 1)), dict(pos=_On(torch.zeros(B, H, 192, dtype=i32)[..., ::2], 1))):
        with pytest.raises(ValueError):
            cache(**bad)
    with pytest.raises(ValueError):
        cache(-1)
    with pytest.raises(api.SelectInferError):
        api.KV4Cache(on(1, B, H, 3, 2560, dtype=u8), 96, 32, bf16, on(1, B, dtype=i32))
    with pytest.raises(ValueError):
        api.KV4Cache.empty(B, H, 40, D, 32, bf16, torch.zeros(B, dtype=i32))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    c, other = cache(), cache(0)
    wide = api.KVCache(on(0, B, H, 50, D), on(0, B, H, 50, D), on(0, B, dtype=i32))
    here = api.KVCache(on(1, B, H, 50, D), on(1, B, H, 50, D), on(1, B, dtype=i32))
    ws, q, out = on(1, 1 << 20, dtype=u8), on(1, B, Hq, D), on(1, B, Hq, D)
    for call in (lambda: api.si_kv4_store(wide, c), lambda: api.si_kv4_load(c, wide, None, 5, None), lambda: api.si_kv4_evict(c, other, None, 0, 4, 0, 0, None, None, ws),
                 lambda: api.si_kv4_store(here, c, on(0, B, dtype=i32)), lambda: api.si_kv4_load(c, here, on(1, B, dtype=f32), 5, None),
                 lambda: api.si_kv4_attn_decode(c, on(0, B, Hq, D), None, None, None, 0, 0, 0.1, out, None, 0, ws),
                 lambda: api.si_kv4_attn_decode(c, q, None, on(1, B, H, D), None, 0, 0, 0.1, out, None, 0, ws),
                 lambda: api.si_kv4_attn_decode(c, q, None, None, None, 0, 0, 0.1, out, None, 0, on(0, 1 << 20, dtype=u8))):
        with pytest.raises(ValueError):
            call()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (lambda: api.si_kv4_store(here, c), lambda: api.si_kv4_load(c, here, None, 5, None),
                 lambda: api.si_kv4_attn_decode(c, q, None, None, None, 0, 0, 0.1, out, None, 0, ws), lambda: api.si_kv4_evict(c, c, None, 0, 4, 0, 0, None, None, ws)):
        with pytest.raises(ValueError):
            call()
