"""Helpers for the tests of attention over the key/value cache: caches in both memory orders with garbage beyond their
lengths, and the bounds that the arithmetic allows.  No method arithmetic here.

Bounds (u = unit roundoff of the 16-bit type: 2^-8 bf16, 2^-11 f16; e = 2^-24):
  score    a dot product of D exact products summed in fp32 in any order, chopped additions allowed: |err| <= 2 D e * size with
           size = max_j sum_c |q_c k_jc| * |scale|; turning it into the argument of exp2 and back costs 4 e * |score|.
           Both together: delta.
  lse      delta + 4 e (|lse| + log of the number of terms) + n e (the sum)
  p        relative 2 delta (score and lse) + n e
  out      p is rounded to the type (u, relative to the largest p of the row: an online softmax may hold p scaled, never above
           2^8 times its value, which keeps the relative error), out once more (u |out|); f16 also loses up to 2^-25 per p absolutely.
"""
import numpy as np
import torch

from oracle import attention_oracle as ao

E = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TDT = {"bf16": torch.bfloat16, "f16": torch.float16}


def make(B, Hq, Hkv, D, cap, dtype, order, T, seed, lens, spread=1.0):
    """Random cache and queries on the GPU; entries from lens[b] on hold NaN and infinities."""
    g = torch.Generator().manual_seed(seed)
    dt = TDT[dtype]
    shape = (B, Hkv, cap, D) if order == "hnd" else (B, cap, Hkv, D)
    k, v = (torch.randn(shape, generator=g).to(dt) for _ in range(2))
    if order == "nhd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
        v[b, :, n + 1:] = float("nan")
    wide = torch.randn(B, T, (Hq + 2 * Hkv) * D, generator=g).mul_(spread).to(dt).cuda()
    q = wide[..., :Hq * D].view(B, T, Hq, D)
    dev = lambda t: (t.cuda() if order == "hnd" else t.transpose(1, 2).contiguous().cuda().transpose(1, 2))  # noqa: E731
    return q, dev(k), dev(v), torch.tensor(lens, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def reference(q, k, v, lens, window, n_sink, scale, pos=None, q_pos=None):
    """Per (sequence, query head): attend() over the cache's entries.  q [B, T, Hq, D] -> dict of arrays."""
    B, T, Hq, D = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    G = Hq // Hkv
    qn, kn, vn = f64(q), f64(k), f64(v)
    res = {"out": np.zeros((B, T, Hq, D)), "reach": np.zeros((B, T, Hq, D)), "lse": np.zeros((B, T, Hq)),
           "size": np.zeros((B, T, Hq)), "weight": np.zeros((B, Hkv, cap)), "n": np.zeros((B, T, Hq))}
    for b in range(B):
        n = int(lens[b])
        for hq in range(Hq):
            h = hq // G
            p = np.arange(n) if pos is None else np.asarray(pos[b][h][:n])
            s = np.arange(n - T, n) if q_pos is None else np.asarray([q_pos[b]])
            o, l, w, r, z = ao.attend(qn[b, :, hq], kn[b, h, :n], vn[b, h, :n], p, s, window, n_sink, scale)
            res["out"][b, :, hq], res["lse"][b, :, hq], res["reach"][b, :, hq], res["size"][b, :, hq] = o, l, r, z
            res["n"][b, :, hq] = (w > 0).sum(-1)
            res["weight"][b, h, :n] += w.sum(0)
    return res


def delta(ref, D):
    lse = np.where(np.isfinite(ref["lse"]), np.abs(ref["lse"]), 0.0)
    return 2 * D * E * ref["size"] + 4 * E * (lse + ref["size"])


def check_out(out, ref, dtype, D):
    d = delta(ref, D)
    rel = 2 * d + (ref["n"] + 8) * E
    u = U[dtype]
    bound = (u * np.abs(ref["out"]) + (u + rel[..., None]) * ref["reach"]) * 1.01
    if dtype == "f16":
        bound += (ref["n"][..., None] * 5.0 + 1.0) * 2.0 ** -25
    err = np.abs(f64(out) - ref["out"])
    assert np.all(err <= bound), f"out: {np.max(err / np.maximum(bound, 1e-30)):.3f} of the bound"   # NaN fails too


def check_lse(lse, ref, D):
    got = f64(lse)
    empty = np.isinf(ref["lse"])
    assert np.array_equal(np.isneginf(got), empty)
    bound = (delta(ref, D) + 4 * E * (np.abs(np.where(empty, 0, ref["lse"])) + 20) + ref["n"] * E)[~empty]
    err = np.abs(got[~empty] - ref["lse"][~empty])
    assert np.all(err <= bound), np.max(err / bound)


def check_weight(weight, before, ref, D, T):
    d = delta(ref, D).max() if ref["size"].size else 0.0
    terms = T * (ref["lse"].shape[-1] // weight.shape[1])
    rel = 4 * d + (ref["n"].max() + terms + 16) * E if ref["n"].size else 0.0
    want = before + ref["weight"]
    err = np.abs(f64(weight) - want)
    bound = rel * ref["weight"] + 2 * E * np.abs(want) + 1e-30
    assert np.all(err <= bound), np.max(err / bound)
