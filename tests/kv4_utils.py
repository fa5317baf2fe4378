"""Helpers for the tests of the cache in 4 bits: packed caches and the float64 arrays they stand for, and the bounds that the
arithmetic allows.  No method arithmetic here.

Bounds (u, e as in attn_utils; y = m + s c the stored values):
  score    sum over groups of s (q . c) + m sum q in fp32, chopped additions allowed: |err| <= (2 D + 16) e * size with
           size = max_j sum_c |q_c| (s c + |m|) * |scale|; the argument of exp2 and back 4 e |score|, more e * 128 for a reference
           of exp2 that may lie up to 128 away from the maximum
  out      p s is rounded to 11 bits (2^-11 of sum_j p_j s_j c_j), below 2^-14 absolutely: at most 2^-25 where the largest p s is 2^5 or more, i.e.
           15 * 2^-30 of the largest of (s, |m| 2^-10) per entry; fp32 sums: relative 2 delta + (n + 8) e of sum_j p_j (s_j c_j + |m_j|); the result u.
"""
import numpy as np
import torch

from oracle import attention_oracle as ao
from oracle import kv4_oracle as ko
from tests import attn_utils as au

E = au.E


class Made:
    """A packed cache over random 16-bit entries, and what it stands for: m, s, c per key and value [B, H, cap, D] (float64)."""

    def __init__(self, api, B, H, D, cap, group, dtype, lens, seed=0, pos=None, weight=None, fill=0xFF, k=None, v=None):
        g = torch.Generator().manual_seed(seed)
        dt = au.TDT[dtype]
        size = torch.exp(0.7 * torch.randn(H, 1, D, generator=g))
        self.k = (torch.randn(B, H, cap, D, generator=g) * size if k is None else k).to(dt).cuda()
        self.v = (torch.randn(B, H, cap, D, generator=g) if v is None else v).to(dt).cuda()
        self.api, self.group, self.dtype, self.D, self.dt = api, group, dtype, D, dt
        self.lens = list(lens)
        self.length = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.cache = api.KV4Cache.empty(B, H, cap, D, group, dt, self.length, pos, weight)
        self.cache.data.fill_(fill)              # unused entries: steps and lowest values that are NaN
        start = torch.zeros_like(self.length)
        api.si_kv4_store(api.KVCache(self.k, self.v, self.length), api.KV4Cache(self.cache.data, D, group, dt, start))
        self.kq, self.vq = (list(ko.quantise(au.f64(x), group, dtype)) for x in (self.k, self.v))

    def values(self, which):
        m, s, c = self.kq if which == "k" else self.vq
        return m + s * c

    def set(self, b, j, k_new, v_new):
        """Entry j of sequence b becomes these 16-bit rows [H, D] in the oracle's arrays."""
        for q, x in ((self.kq, k_new), (self.vq, v_new)):
            for i, y in enumerate(ko.quantise(au.f64(x), self.group, self.dtype)):
                if not q[i].flags.writeable:
                    q[i] = q[i].copy()
                q[i][b, :, j] = y

    def read(self, length=None):
        """Everything in the cache, read back: k, v [B, H, cap, D]."""
        api, c = self.api, self.cache
        full = torch.full_like(self.length, c.capacity) if length is None else length
        k, v = (torch.zeros(c.n_seqs, c.n_kv_heads, c.capacity, self.D, dtype=self.dt, device="cuda") for _ in range(2))
        api.si_kv4_load(api.KV4Cache(c.data, self.D, self.group, self.dt, full), api.KVCache(k, v, full), None, c.capacity, None)
        return k, v


def reference(made, q, total, window, n_sink, scale, pos=None, q_pos=None):
    """Per (sequence, query head): attention over the first total[b] entries; q [B, Hq, D]."""
    B, Hq, D = q.shape
    H, cap = made.k.shape[1], made.k.shape[2]
    G = Hq // H
    qn, kn, vn = au.f64(q), made.values("k"), made.values("v")
    ka, sc = np.abs(made.kq[0]) + made.kq[1] * made.kq[2], made.vq[1] * made.vq[2]
    va = np.abs(made.vq[0]) + sc
    res = {"out": np.zeros((B, Hq, D)), "sc": np.zeros((B, Hq, D)), "reach": np.zeros((B, Hq, D)), "lse": np.zeros((B, Hq)), "size": np.zeros((B, Hq)),
           "weight": np.zeros((B, H, cap)), "n": np.zeros((B, Hq)), "peak": np.zeros((B, Hq))}
    for b in range(B):
        n = int(total[b])
        for hq in range(Hq):
            h = hq // G
            p = np.arange(n) if pos is None else np.asarray(pos[b][h][:n])
            s = [n - 1] if q_pos is None else [q_pos[b]]
            see = ao.visible(p, s, window, n_sink)[0]
            at = lambda a: np.where(see[:, None], a[b, h, :n], 0.0)  # noqa: E731
            o, l, w, _, _ = ao.attend(qn[b, hq][None], at(kn), at(vn), p, np.asarray(s), window, n_sink, scale)
            res["out"][b, hq], res["lse"][b, hq], res["sc"][b, hq], res["reach"][b, hq] = o[0], l[0], (w @ at(sc))[0], (w @ at(va))[0]
            if n:
                res["size"][b, hq] = (at(ka) @ np.abs(qn[b, hq])).max() * abs(scale)
                res["peak"][b, hq] = max(at(made.vq[1]).max(), np.abs(at(made.vq[0])).max() * 2.0 ** -10)
            res["n"][b, hq] = see.sum()
            res["weight"][b, h, :n] += w.sum(0)
    return res


def delta(ref, D):
    lse = np.where(np.isfinite(ref["lse"]), np.abs(ref["lse"]), 0.0)
    return (2 * D + 16) * E * ref["size"] + E * (4 * (lse + ref["size"]) + 128)


def check(out, lse, ref, dtype, D):
    d = delta(ref, D)
    rel = (2 * d + (ref["n"] + 8) * E)[..., None]
    bound = 1.01 * (au.U[dtype] * np.abs(ref["out"]) + 2.0 ** -11 * ref["sc"] + rel * ref["reach"] + (ref["n"] * ref["peak"])[..., None] * 15 * 2.0 ** -30)
    if dtype == "f16":
        bound += 2.0 ** -25
    err = np.abs(au.f64(out) - ref["out"])
    assert np.all(err <= bound), f"out: {np.max(err / np.maximum(bound, 1e-30)):.3f} of the bound"   # NaN fails too
    if lse is not None:
        got, empty = au.f64(lse), np.isinf(ref["lse"])
        assert np.array_equal(np.isneginf(got), empty)
        bound = (d + 4 * E * (np.abs(np.where(empty, 0, ref["lse"])) + 128) + ref["n"] * E)[~empty]
        err = np.abs(got[~empty] - ref["lse"][~empty])
        assert np.all(err <= bound), np.max(err / bound)


def check_weight(weight, before, ref, D):
    d = delta(ref, D).max()
    rel = 4 * d + (ref["n"].max() + ref["lse"].shape[-1] // weight.shape[1] + 16) * E
    want = before + ref["weight"]
    err = np.abs(au.f64(weight) - want)
    bound = rel * ref["weight"] + 2 * E * np.abs(want) + 1e-30
    assert np.all(err <= bound), np.max(err / bound)
