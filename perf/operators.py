"""Timed cases of the cache operators: attention with a sliding window and always-visible first tokens (prefill and
single token), the attention weight every cache entry has received, and eviction by that weight.

A case is one call.  `run` makes it either through the package (`own`) or in a plain form of elementary torch
operations in 32 bits; `exact` states the same result in 64 bits, written on its own.

Common to all: a cache of one layer, k and v [n_seqs, n_kv_heads, capacity, head_dim] views (memory order head-major,
"hnd", or token-major, "nhd"), len[b] entries in use.  An entry at position p is visible to a query at position s if
p <= s and (window == 0 or p > s - window or p < n_sink).
"""
import math

import numpy as np
import torch

own = False

# n_q_heads, n_kv_heads, head_dim: grouped, one key head per query head, three and eight query heads per key head
HEADS = [(32, 8, 128), (32, 32, 128), (24, 8, 128), (16, 2, 128), (32, 8, 64)]


def listed():
    return [
        # a long prompt of one user, every earlier token visible: the largest matrix work of a model's attention
        dict(name="prefill_prompt", op="prefill", B=1, T=8192, past=0, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, n_sink=0, ragged=False, order="nhd"),
        # several prompts of different lengths behind one another's padding, sliding window with sinks, three heads to a group
        dict(name="prefill_window", op="prefill", B=3, T=4001, past=0, Hq=24, Hkv=8, D=128, dtype="f16", window=1024, n_sink=4, ragged=True, order="hnd"),
        # a short piece of a prompt against a long cache (chunked prefill): few rows, a long axis to split
        dict(name="prefill_chunk", op="prefill", B=1, T=45, past=12000, Hq=32, Hkv=8, D=64, dtype="bf16", window=0, n_sink=0, ragged=False, order="hnd"),
        # the first token after a prompt of a few words: nothing but latency
        dict(name="decode_first", op="decode", B=1, n=7, cap=4096, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, n_sink=0, ragged=False, pos=False, acc=True, order="hnd"),
        # a served batch at mixed lengths, weights accumulated for a later eviction
        dict(name="decode_batch", op="decode", B=32, n=8191, cap=8192, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, n_sink=0, ragged=True, pos=False, acc=True, order="hnd"),
        # one user's very long cache: a single sequence has to fill the GPU
        dict(name="decode_long", op="decode", B=1, n=130001, cap=131072, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, n_sink=0, ragged=False, pos=False, acc=False, order="nhd"),
        # a batch decoding with a window and sinks in long caches, one key head per query head
        dict(name="decode_window", op="decode", B=16, n=16000, cap=16384, Hq=32, Hkv=32, D=128, dtype="f16", window=2048, n_sink=4, ragged=False, pos=False, acc=False, order="hnd"),
        # decoding on caches that were cut to a budget: every entry carries its position, weights go on accumulating
        dict(name="decode_evicted", op="decode", B=24, n=2000, cap=2112, Hq=16, Hkv=2, D=128, dtype="bf16", window=0, n_sink=0, ragged=False, pos=True, acc=True, order="hnd"),
        # the weight every entry received from all queries of a prompt (what the eviction after a prefill ranks)
        dict(name="weights_prompt", op="weights", B=1, T=4096, past=0, Hq=32, Hkv=8, D=128, dtype="bf16", window=0, n_sink=0, ragged=False, order="nhd"),
        # the same from the last 32 queries only, of prompts of different lengths
        dict(name="weights_recent", op="weights", B=4, T=32, past=8150, Hq=32, Hkv=8, D=64, dtype="f16", window=0, n_sink=0, ragged=True, order="hnd"),
        # after a prefill: the prompt's keys and values cut to a budget, into the cache that decoding goes on with
        dict(name="evict_prompt", op="evict", B=8, n=16384, cap=16384, Hkv=32, D=128, dtype="bf16", budget=4096, n_sink=4, n_recent=256, ragged=False, step=False, order="nhd"),
        # every decode step of a batch at its budget: one entry has to go
        dict(name="evict_step", op="evict", B=16, n=2049, cap=2112, Hkv=8, D=128, dtype="bf16", budget=2048, n_sink=4, n_recent=128, ragged=False, step=True, order="hnd"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prefill", "decode", "weights", "evict"])
    Hq, Hkv, D = rng.choice(HEADS)
    c = dict(op=op, Hq=Hq, Hkv=Hkv, D=D, dtype=rng.choice(["bf16", "f16"]), order=rng.choice(["hnd", "nhd"]), ragged=rng.random() < 0.5)
    if op in ("prefill", "weights"):
        c.update(B=_log_int(rng, 1, 8), T=_log_int(rng, 1, 4096), past=rng.choice([0, _log_int(rng, 1, 12000)]))
        c.update(window=rng.choice([0, _log_int(rng, 16, 4096)]), n_sink=rng.choice([0, 1, 4, 64]))
        most = 1 << 30 if op == "prefill" else 1 << 28
        while c["B"] * Hq * c["T"] * (c["T"] + c["past"]) > most:
            c["T"], c["B"] = max(1, c["T"] * 2 // 3), max(1, c["B"] * 2 // 3)
    elif op == "decode":
        c.update(B=_log_int(rng, 1, 64), n=_log_int(rng, 1, 131000), pos=rng.random() < 0.4, acc=rng.random() < 0.5)
        c.update(window=rng.choice([0, _log_int(rng, 16, 8192)]), n_sink=rng.choice([0, 1, 4, 64]))
        while c["B"] * Hkv * D * 4 * c["n"] > 500_000_000:
            c["B"], c["n"] = max(1, c["B"] // 2), max(1, c["n"] * 2 // 3)
        c.update(cap=c["n"] + rng.randint(1, 200))
    else:
        del c["Hq"]
        c.update(B=_log_int(rng, 1, 16), n=_log_int(rng, 64, 65536), step=rng.random() < 0.4, n_sink=rng.choice([0, 4, 16]))
        while c["B"] * Hkv * D * 4 * c["n"] > 1_500_000_000:
            c["B"], c["n"] = max(1, c["B"] // 2), max(64, c["n"] * 2 // 3)
        c.update(budget=c["n"] - 1 if c["step"] else _log_int(rng, 32, max(32, c["n"] // 2)))
        c.update(n_recent=rng.randint(1, c["budget"] - c["n_sink"]) if c["budget"] > c["n_sink"] else 0, cap=c["n"] + rng.randint(0, 99))
        c["n_sink"] = min(c["n_sink"], c["budget"])
        c["ragged"] = c["ragged"] and not c["step"]
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _lens(case):
    """Entries of every sequence before the call (host ints): the same for every seed."""
    B, n = case["B"], case["n"] if "n" in case else case["T"] + case["past"]
    if not case["ragged"]:
        return [n] * B
    return [max(1, n - (n * ((b * 5) % B)) // (B + 1)) for b in range(B)]


def _cache(case, cap, g, dt):
    B, H, D = case["B"], case["Hkv"], case["D"]
    shape = (B, H, cap, D) if case["order"] == "hnd" else (B, cap, H, D)
    k, v = (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt) for _ in range(2))
    return (k, v) if case["order"] == "hnd" else (k.transpose(1, 2), v.transpose(1, 2))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    op, B, H, D = case["op"], case["B"], case["Hkv"], case["D"]
    i32 = dict(dtype=torch.int32, device="cuda")
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lens = _lens(case)
    st = {"case": case, "len": torch.tensor(lens, **i32), "scale": 1.0 / math.sqrt(D)}
    cap = case["cap"] if "cap" in case else max(lens)
    st["k"], st["v"] = _cache(case, cap, g, dt)
    if op in ("prefill", "weights", "decode"):
        # the first entries draw attention in every head, as a model's first tokens do
        mean = rand(B, H, 1, D)
        st["k"][:, :, :4] = (0.5 * mean + 0.5 * rand(B, H, min(4, cap), D)).to(dt)
        T = case["T"] if op != "decode" else 1
        G = case["Hq"] // H
        q = (rand(B, T, H, G, D) + mean[:, None]).to(dt)
        # the projection's output holds queries, keys and values side by side: the queries are a strided part of it
        wide = torch.empty(B, T, case["Hq"] * D + 2 * H * D, dtype=dt, device="cuda")
        wide[..., :case["Hq"] * D] = q.reshape(B, T, -1)
        st["q"] = wide[..., :case["Hq"] * D].view(B, T, case["Hq"], D)
        st["weight"] = torch.zeros(B, H, cap, dtype=torch.float32, device="cuda")
    if op == "weights":
        s, hidden = _scores(case, st, st["q"], st["len"].long())
        st["lse"] = _lse(s).permute(0, 2, 1, 3).reshape(B, case["T"], case["Hq"]).contiguous()
        del s, hidden
    if op == "decode":
        st["q"] = st["q"][:, 0]
        st["k_new"], st["v_new"] = rand(B, H, D).to(dt), rand(B, H, D).to(dt)
        if case["pos"]:   # a third of the positions seen so far are gone, other ones in every head
            seen = torch.tensor([n + n // 2 for n in lens], **i32)
            keep = torch.rand(B, H, max(int(seen.max()), cap), generator=g, device="cuda")
            keep.masked_fill_(torch.arange(keep.shape[2], device="cuda") >= seen[:, None, None], 2.0)
            st["pos"] = torch.argsort(keep, dim=-1)[..., :cap].to(torch.int32).contiguous()
            st["q_pos"] = seen
            st["weight"].copy_(torch.rand(B, H, cap, generator=g, device="cuda"))
    if op == "evict":
        st["weight"] = torch.exp(1.5 * rand(B, H, cap))   # a few heavy entries, many light ones
        st["pos"] = torch.arange(cap, **i32).expand(B, H, cap).contiguous()
        st["q_pos"] = st["len"] - 1
        st["kept"] = torch.zeros(B, H, case["budget"], **i32)
        st["len_out"] = torch.zeros(B, **i32)
        if case["step"]:
            st["len"] = st["len"] - 1
        else:
            st["dk"], st["dv"] = (torch.zeros(B, H, case["budget"], D, dtype=dt, device="cuda") for _ in range(2))
            st["dpos"] = torch.zeros(B, H, case["budget"], **i32)
            st["dweight"] = torch.zeros(B, H, case["budget"], dtype=torch.float32, device="cuda")
    if own:   # what a program keeps beside its tensors: the cache's description, output buffers, the workspace
        from paper_2607_18081_b200 import api
        st["cache"] = api.KVCache(st["k"], st["v"], st["len"], st.get("pos"), st.get("weight"))
        if op == "evict":
            st["dst"] = st["cache"] if case["step"] else api.KVCache(st["dk"], st["dv"], st["len_out"], st["dpos"], st["dweight"])
            st["ws"] = st["cache"].workspace(0, 0)
        else:
            st["ws"] = st["cache"].workspace(case["Hq"], case.get("T", 1))
            st["out"] = torch.empty(st["q"].shape, dtype=dt, device="cuda")
            if "lse" not in st:
                st["lse"] = torch.empty(st["q"].shape[:-1], dtype=torch.float32, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ plain form

def _scores(case, st, q, n):
    """Scaled scores [B, Hkv, T, G, capacity] with hidden entries at -inf, and the hidden mask; the queries are the last T of the n[b] positions."""
    B, T, Hq, D = q.shape
    H, cap = st["k"].shape[1], st["k"].shape[2]
    qf = q.float().view(B, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    s = torch.matmul(qf, st["k"].float().transpose(-1, -2)).view(B, H, T, Hq // H, cap)
    s.mul_(st["scale"])
    j = torch.arange(cap, device="cuda")
    at = st["q_pos"].long()[:, None] if "q_pos" in st else n[:, None] - T + torch.arange(T, device="cuda")[None]
    at = at[:, None, :, None]                                                     # [B, 1, T, 1]
    p = st["pos"].long()[:, :, None] if "pos" in st else j[None, None, None]      # [B | 1, H | 1, 1, cap]
    seen = (p <= at) & (j < n[:, None, None, None])
    if case["window"]:
        seen &= (p > at - case["window"]) | (p < case["n_sink"])
    hidden = ~seen
    return s.masked_fill_(hidden[:, :, :, None], -math.inf), hidden


def _lse(s):
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    return (torch.exp(s - m).sum(-1).log() + m[..., 0])


def _attend(case, st, q, n):
    s, _ = _scores(case, st, q, n)
    B, H, T, G, cap = s.shape
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)        # a row with nothing visible: all exp = 0
    e = s.sub_(m).exp_()
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, H, T * G, cap), st["v"].float()).view(B, H, T, G, -1) / l.clamp_min(torch.finfo(torch.float32).tiny)
    back = lambda x: x.permute(0, 2, 1, 3, 4).reshape(B, T, H * G, -1)  # noqa: E731
    return back(o).to(q.dtype), back(l.log() + m)[..., 0], e, l


def _evict(case, st):
    k, v, pos, weight = (st[x] for x in ("k", "v", "pos", "weight"))
    B, H, cap, D = k.shape
    n, budget = (st["len"] + (1 if case["step"] else 0)).long(), case["budget"]
    j = torch.arange(cap, device="cuda")
    used = (j < n[:, None])[:, None]                                              # [B, 1, cap]
    last = st["q_pos"].long()[:, None, None]
    safe = (pos < case["n_sink"]) | (pos > last - case["n_recent"])
    rank = torch.where(torch.isnan(weight), -math.inf, weight).masked_fill(safe, math.inf).masked_fill(~used, -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros(B, H, cap, dtype=torch.bool, device="cuda").scatter_(-1, best, True) & used
    # kept entries below the budget stay; the i-th kept entry beyond it goes to the i-th freed slot
    hole = ~kept[..., :budget]
    movers = torch.sort((kept & (j >= budget)).to(torch.int8), dim=-1, descending=True, stable=True).indices
    moves = (kept & (j >= budget)).sum(-1, keepdim=True)
    nth = (hole.long().cumsum(-1) - 1).clamp_min(0)
    source = torch.where(hole, movers.gather(-1, nth), j[:budget].expand(B, H, budget))
    filled = ~hole | (nth < moves)
    source = torch.where(filled, source, -1)
    st["kept"].copy_(source)
    st["len_out"].copy_(n.clamp_max(budget))
    dst = [k[:, :, :budget], v[:, :, :budget], pos[..., :budget], weight[..., :budget]] if case["step"] else [st[x] for x in ("dk", "dv", "dpos", "dweight")]
    at = source.clamp_min(0)
    wide = at[..., None].expand(B, H, budget, D)
    for d, x, i, ok in ((dst[0], k, wide, filled[..., None]), (dst[1], v, wide, filled[..., None]), (dst[2], pos, at, filled), (dst[3], weight, at, filled)):
        d.copy_(torch.where(ok, x.gather(2, i), d))


def run(st):
    case = st["case"]
    if own:
        from paper_2607_18081_b200 import api
    op = case["op"]
    if op == "prefill":
        if own:
            api.si_attn_prefill(st["cache"], st["q"], case["window"], case["n_sink"], st["scale"], st["out"], st["lse"], st["ws"])
            return {"out": st["out"], "lse": st["lse"]}
        out, lse, _, _ = _attend(case, st, st["q"], st["len"].long())
        return {"out": out, "lse": lse}
    if op == "weights":
        if own:
            api.si_attn_weights(st["cache"], st["q"], case["window"], case["n_sink"], st["scale"], st["lse"], st["ws"])
            return {"weight": st["weight"]}
        s, hidden = _scores(case, st, st["q"], st["len"].long())
        B, H, T, G, cap = s.shape
        s.sub_(st["lse"].view(B, T, H, G).permute(0, 2, 1, 3)[..., None]).exp_().masked_fill_(hidden[:, :, :, None], 0.0)
        st["weight"] += s.sum((2, 3))
        return {"weight": st["weight"]}
    if op == "decode":
        if own:
            api.si_attn_decode(st["cache"], st["q"], st.get("q_pos"), st["k_new"], st["v_new"], case["window"], case["n_sink"], st["scale"],
                               st["out"], st["lse"], api.SI_FLAG_ACC_WEIGHT if case["acc"] else 0, st["ws"])
            return {"out": st["out"], "lse": st["lse"], "weight": st["weight"]}
        n = st["len"].long()
        b = torch.arange(case["B"], device="cuda")
        st["k"][b, :, n], st["v"][b, :, n] = st["k_new"], st["v_new"]
        if "pos" in st:
            st["pos"][b, :, n] = st["q_pos"][:, None]
        out, lse, e, l = _attend(case, st, st["q"][:, None], n + 1)
        if case["acc"]:
            st["weight"][b, :, n] = 0.0
            st["weight"] += (e / l.clamp_min(torch.finfo(torch.float32).tiny)).sum((2, 3))
        return {"out": out[:, 0], "lse": lse[:, 0], "weight": st["weight"]}
    if own:
        api.si_kv_evict(st["cache"], st["dst"], st["q_pos"], 1 if case["step"] else 0, case["budget"], case["n_sink"], case["n_recent"],
                        st["kept"], st["len_out"], st["ws"])
    else:
        _evict(case, st)
    names = ("k", "v", "pos", "weight") if case["step"] else ("dk", "dv", "dpos", "dweight")
    return {x: st[y] for x, y in zip(("k", "v", "pos", "weight", "kept", "len"), names + ("kept", "len_out"))}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    # the inputs only; nothing of the plain form's arithmetic below (a weights case is given its lse as an input)
    st = prepare(case, seed)
    B, H, D = case["B"], case["Hkv"], case["D"]
    lens = st["len"].tolist()
    if case["op"] == "evict":
        return _exact_evict(case, st, lens)
    G = case["Hq"] // H
    T = case.get("T", 1)
    dev = dict(dtype=torch.float64, device="cuda")
    out, lse, weight = torch.zeros(B, T, case["Hq"], D, **dev), torch.zeros(B, T, case["Hq"], **dev), st["weight"].double()
    q = st["q"] if case["op"] != "decode" else st["q"][:, None]
    for b in range(B):
        for h in range(H):
            n = lens[b]
            k, v = st["k"][b, h, :n].double(), st["v"][b, h, :n].double()
            p = st["pos"][b, h, :n].double() if "pos" in st else torch.arange(n, **dev)
            if case["op"] == "decode":
                here = float(st["q_pos"][b]) if "pos" in st else float(n)
                k, v = torch.cat([k, st["k_new"][b, h].double()[None]]), torch.cat([v, st["v_new"][b, h].double()[None]])
                p = torch.cat([p, torch.full((1,), here, **dev)])
                if case["acc"]:
                    weight[b, h, n] = 0.0
                rows = torch.tensor([here], **dev)
            else:
                rows = torch.arange(n - T, n, **dev)
            for i0 in range(0, T, 1024):
                at = rows[i0:i0 + 1024, None]
                ok = p[None] <= at
                if case["window"]:
                    ok &= (at - p[None] < case["window"]) | (p[None] < case["n_sink"])
                for g in range(G):
                    hq = h * G + g
                    logit = (q[b, i0:i0 + 1024, hq].double() @ k.T * st["scale"]).masked_fill(~ok, -math.inf)
                    z = torch.logsumexp(logit, -1, keepdim=True)
                    if case["op"] == "weights":
                        z = st["lse"][b, i0:i0 + 1024, hq].double()[:, None]
                    w = torch.exp(logit - z).masked_fill(~ok, 0.0)
                    out[b, i0:i0 + 1024, hq], lse[b, i0:i0 + 1024, hq] = w @ v, z[:, 0]
                    if case["op"] == "weights" or (case["op"] == "decode" and case["acc"]):
                        weight[b, h, :len(p)] += w.sum(0)
    if case["op"] == "prefill":
        return {"out": out, "lse": lse}
    return {"weight": weight} if case["op"] == "weights" else {"out": out[:, 0], "lse": lse[:, 0], "weight": weight}


def _exact_evict(case, st, lens):
    budget, res = case["budget"], {}
    names = ("k", "v", "pos", "weight") if case["step"] else ("dk", "dv", "dpos", "dweight")
    for x, y in zip(("k", "v", "pos", "weight"), names):
        res[x] = st[y].clone() if x == "pos" else st[y].double()
    pos, weight = st["pos"].cpu().numpy(), st["weight"].double().cpu().numpy()
    kept = np.full((case["B"], case["Hkv"], budget), -1, np.int32)
    for b, n in enumerate(lens):
        n += 1 if case["step"] else 0
        for h in range(case["Hkv"]):
            p, w = pos[b, h, :n].astype(np.int64), weight[b, h, :n]
            held = (p < case["n_sink"]) | (int(st["q_pos"][b]) - p < case["n_recent"])
            order = sorted(range(n), key=lambda j: (not held[j], -w[j], j))[:budget] if n > budget else list(range(n))
            stay = [j for j in order if j < budget]
            free = sorted(set(range(min(budget, n))) - set(stay))
            kept[b, h, stay] = stay
            for slot, j in zip(free, sorted(j for j in order if j >= budget)):
                kept[b, h, slot] = j
    res["kept"] = torch.from_numpy(kept).cuda()
    to = (res["kept"] >= 0).nonzero(as_tuple=True)
    frm = (to[0], to[1], res["kept"][to].long())
    for x, y in zip(("k", "v", "pos", "weight"), ("k", "v", "pos", "weight")):
        res[x][to] = st[y][frm].to(res[x].dtype)
    res["len"] = torch.tensor([min(n + (1 if case["step"] else 0), budget) for n in lens], dtype=torch.int32)
    return res


# ------------------------------------------------------------------------------------------------ what a call cannot do without

def work(case):
    B, H, D = case["B"], case["Hkv"], case["D"]
    lens = _lens(case)
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in lens) * H
        moved = B * H if case["step"] else kept
        return {"bytes": sum(lens) * H * 8 + moved * (2 * 2 * D * 2 + 16) + kept * 4, "flops": 0}
    T = case.get("T", 1)
    pairs, read, w, s = 0, 0, case["window"], case["n_sink"]
    for n in lens:
        n += case["op"] == "decode"
        at = np.arange(max(0, n - T), n)
        if w and not case.get("pos"):
            pairs += int(np.sum(np.minimum(at + 1, w) + np.clip(np.minimum(at - w + 1, s), 0, None)))
            first = max(0, int(at[0]) - w + 1)
            read += n - first + min(s, first)
        elif w:   # positions thinned out by a third: two thirds of the window's positions are still there
            pairs += min(n, int(w * 2 / 3) + s)
            read += min(n, int(w * 2 / 3) + s)
        else:
            pairs += int(np.sum(at + 1)) if not case.get("pos") else n
            read += n
    qo = B * T * case["Hq"] * (2 * D + 4)
    if case["op"] == "weights":
        return {"bytes": qo + read * H * (2 * D + 8), "flops": 2 * D * pairs * case["Hq"]}
    more = (8 * read * H if case.get("acc") else 0) + (4 * sum(lens) * H if case.get("pos") else 0)
    return {"bytes": qo + B * T * case["Hq"] * 2 * D + read * H * 4 * D + more, "flops": 4 * D * pairs * case["Hq"]}
