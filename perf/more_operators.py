"""Timed cases of the cache held in 4 bits: quantising entries as they are stored and reading them back, attention of a
single token over such a cache, its eviction by accumulated weight, and the two as one decoding step.

`run` makes a case's calls either through the package (`own`) or in a plain form of elementary torch operations in 32 bits;
`exact` states the same result in 64 bits, written on its own.

The format: the head_dim values of a key (or value) are cut into groups of 32 or 64.  A group x holds its lowest value m, a
step s and 4-bit codes c, and stands for m + s c:
    s = (max x - min x) / 15, rounded up to the cache's 16-bit type,    m = min x,    c = nearest integer of (x - m) / s
(range, its fifteenth and x - m in fp32; the quotient is the exact product with the fp32 reciprocal of s).  An entry at position p is visible to a query
at position t if p <= t and (window == 0 or p > t - window or p < n_sink).
"""
import math

import numpy as np
import torch

own = False

# n_q_heads, n_kv_heads, head_dim: grouped, one key head per query head, three, eight and sixteen query heads per key head
HEADS = [(32, 8, 128), (32, 32, 128), (24, 8, 128), (16, 2, 128), (16, 1, 128), (32, 8, 64)]


def listed():
    return [
        # a prompt's keys and values, parts of the fused projection, go into the empty cache and come back for the next chunk's attention
        dict(name="store_prompt", op="store", B=1, T=8192, past=0, Hq=32, Hkv=8, D=128, dtype="bf16", group=32, ragged=False),
        # chunks of several prompts behind what their caches hold already, none of them on a tile's boundary
        dict(name="store_chunks", op="store", B=6, T=1001, past=1501, Hq=32, Hkv=8, D=64, dtype="f16", group=64, ragged=True),
        # one drafted token or two per sequence of a batch: nothing but latency
        dict(name="store_tokens", op="store", B=32, T=2, past=700, Hq=24, Hkv=8, D=128, dtype="bf16", group=32, ragged=False),
        # a long cache read back into the scratch cache that the next chunk of the prompt is prefilled on
        dict(name="load_long", op="load", B=1, n=65000, Hq=32, Hkv=8, D=128, dtype="bf16", group=32, ragged=False, order="nhd"),
        # several caches of different lengths
        dict(name="load_batch", op="load", B=7, n=3001, Hq=16, Hkv=2, D=128, dtype="f16", group=64, ragged=True, order="hnd"),
        # the first token after a prompt of a few words: nothing but latency
        dict(name="decode_first", op="decode", B=1, n=7, cap=4096, Hq=32, Hkv=8, D=128, dtype="bf16", group=32, window=0, n_sink=0, ragged=False, pos=False, acc=True),
        # a served batch at mixed lengths, weights accumulated for a later eviction
        dict(name="decode_batch", op="decode", B=32, n=8191, cap=8192, Hq=32, Hkv=8, D=128, dtype="bf16", group=32, window=0, n_sink=0, ragged=True, pos=False, acc=True),
        # one user's very long cache: a single sequence has to fill the GPU
        dict(name="decode_long", op="decode", B=1, n=260001, cap=260096, Hq=32, Hkv=8, D=128, dtype="bf16", group=64, window=0, n_sink=0, ragged=False, pos=False, acc=False),
        # a batch decoding with a window and sinks in long caches, one key head per query head
        dict(name="decode_window", op="decode", B=16, n=16000, cap=16384, Hq=32, Hkv=32, D=128, dtype="f16", group=32, window=2048, n_sink=4, ragged=False, pos=False, acc=False),
        # a prompt's cache in 4 bits cut to a budget, the kept part read back
        dict(name="evict_prompt", op="evict", B=4, n=16384, cap=16384, Hq=32, Hkv=32, D=128, dtype="bf16", group=32, budget=2048, n_sink=4, n_recent=256, ragged=False),
        # a decoding step of a batch at its budget: one token attends and adds its weights, one entry has to go
        dict(name="step_batch", op="step", B=24, n=2048, cap=2080, Hq=16, Hkv=2, D=128, dtype="bf16", group=32, window=0, n_sink=4, n_recent=128),
        # the same for one user, a small head size and a short budget
        dict(name="step_single", op="step", B=1, n=1000, cap=1024, Hq=32, Hkv=8, D=64, dtype="f16", group=32, window=0, n_sink=4, n_recent=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _tiles(n):
    """The least capacity that holds n entries: whole tiles of 32."""
    return (n + 31) // 32 * 32


def draw(rng):
    op = rng.choice(["store", "load", "decode", "decode", "evict", "step"])
    Hq, Hkv, D = rng.choice(HEADS)
    c = dict(op=op, Hq=Hq, Hkv=Hkv, D=D, dtype=rng.choice(["bf16", "f16"]), group=rng.choice([32, 64]))
    if op == "store":
        c.update(B=_log_int(rng, 1, 32), T=_log_int(rng, 1, 8192), past=rng.choice([0, _log_int(rng, 1, 4000)]), ragged=rng.random() < 0.5)
        while c["B"] * c["T"] * Hkv * D > 10_000_000:
            c["B"], c["T"] = max(1, c["B"] // 2), max(1, c["T"] * 2 // 3)
    elif op == "load":
        c.update(B=_log_int(rng, 1, 32), n=_log_int(rng, 1, 65000), ragged=rng.random() < 0.5, order=rng.choice(["hnd", "nhd"]))
        while c["B"] * c["n"] * Hkv * D > 66_000_000:
            c["B"], c["n"] = max(1, c["B"] // 2), max(1, c["n"] * 2 // 3)
    elif op == "decode":
        c.update(B=_log_int(rng, 1, 64), n=_log_int(rng, 1, 260000), pos=rng.random() < 0.4, acc=rng.random() < 0.5, ragged=rng.random() < 0.5)
        c.update(window=rng.choice([0, _log_int(rng, 16, 8192)]), n_sink=rng.choice([0, 1, 4, 64]))
        while c["B"] * Hkv * D * c["n"] > 130_000_000:
            c["B"], c["n"] = max(1, c["B"] // 2), max(1, c["n"] * 2 // 3)
        c.update(cap=_tiles(c["n"] + rng.randint(1, 200)))
    elif op == "evict":
        c.update(B=_log_int(rng, 1, 16), n=_log_int(rng, 64, 65536), n_sink=rng.choice([0, 4, 16]), ragged=rng.random() < 0.5)
        while c["B"] * Hkv * D * c["n"] > 260_000_000:
            c["B"], c["n"] = max(1, c["B"] // 2), max(64, c["n"] * 2 // 3)
        c.update(budget=_log_int(rng, 32, max(32, c["n"] // 4)), cap=_tiles(c["n"] + rng.randint(0, 99)))
        c.update(n_recent=rng.randint(0, c["budget"] - c["n_sink"]))
    else:
        c.update(B=_log_int(rng, 1, 32), n=_log_int(rng, 100, 4096), window=0, n_sink=rng.choice([0, 4, 16]))
        while c["B"] * Hkv * D * c["n"] > 130_000_000:
            c["B"] = max(1, c["B"] // 2)
        c.update(n_recent=rng.randint(1, c["n"] // 2), cap=_tiles(c["n"] + 1 + rng.randint(0, 50)))
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _lens(case, n):
    """Entries of every sequence (host ints): the same for every seed."""
    B = case["B"]
    if not case.get("ragged"):
        return [n] * B
    return [max(1, n - (n * ((b * 5) % B)) // (B + 1)) for b in range(B)]


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _raw(case, seed):
    """The 16-bit values everything starts from: keys whose channels differ in size, and the rest of a call's inputs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    dt, op, B, H, D, Hq = _dt(case), case["op"], case["B"], case["Hkv"], case["D"], case["Hq"]
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    st = {"case": case, "scale": 1.0 / math.sqrt(D)}
    channel = torch.exp(0.5 * rand(H, 1, D))
    if op == "store":
        T, past = case["T"], _lens(case, case["past"]) if case["past"] else [0] * B
        wide = rand(B, T, Hq + 2 * H, D)
        wide[:, :, Hq:Hq + H] *= channel[:, 0]
        wide = wide.to(dt)
        st["k"], st["v"] = wide[:, :, Hq:Hq + H].transpose(1, 2), wide[:, :, Hq + H:].transpose(1, 2)
        st["new"] = torch.tensor(_lens(case, T), **i32)
        st["past"] = torch.tensor(past, **i32)
        st["len"] = st["past"] + st["new"]
        st["cap"] = _tiles(T + max(past))
        st["out_k"], st["out_v"] = (torch.zeros(B, H, T, D, dtype=dt, device="cuda") for _ in range(2))
        return st
    n = case["n"]
    st["len"] = torch.tensor(_lens(case, n), **i32)
    cap = st["cap"] = case.get("cap", _tiles(n))
    k = torch.empty(B, H, cap, D, dtype=dt, device="cuda")
    v = torch.empty_like(k)
    mean = rand(B, H, 1, D)
    for b in range(B):
        k[b], v[b] = rand(H, cap, D).mul_(channel).to(dt), rand(H, cap, D).to(dt)
    # the first entries draw attention in every head, as a model's first tokens do
    k[:, :, :4] = (0.5 * mean + 0.5 * rand(B, H, 4, D)).to(dt)
    st["k"], st["v"] = k, v
    if op == "load":
        shape = (B, H, cap, D) if case["order"] == "hnd" else (B, cap, H, D)
        st["out_k"], st["out_v"] = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
        if case["order"] == "nhd":
            st["out_k"], st["out_v"] = st["out_k"].transpose(1, 2), st["out_v"].transpose(1, 2)
        return st
    if op in ("evict", "step") or case["acc"]:
        st["weight"] = torch.exp(1.5 * rand(B, H, cap))      # a few heavy entries, many light ones
    if op in ("decode", "step"):
        # the projection's output holds queries, keys and values side by side
        wide = rand(B, Hq + 2 * H, D)
        wide[:, :Hq] += mean.expand(B, H, Hq // H, D).reshape(B, Hq, D)
        wide[:, Hq:Hq + H] *= channel[:, 0]
        wide = wide.to(dt)
        st["q"], st["k_new"], st["v_new"] = wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:]
    if op == "step" or case.get("pos"):   # a third of the positions seen so far are gone, other ones in every head
        seen = st["len"] + st["len"] // 2
        keep = torch.rand(B, H, max(int(seen.max()), cap), generator=g, device="cuda")
        keep.masked_fill_(torch.arange(keep.shape[2], device="cuda") >= seen[:, None, None], 2.0)
        st["pos"], st["q_pos"] = torch.argsort(keep, dim=-1)[..., :cap].to(torch.int32).contiguous(), seen
    if op == "evict":
        st["dpos"] = torch.zeros(B, H, _tiles(case["budget"]), **i32)
        st["dweight"] = torch.zeros(B, H, _tiles(case["budget"]), dtype=torch.float32, device="cuda")
        st["out_k"], st["out_v"] = (torch.zeros(B, H, case["budget"], D, dtype=dt, device="cuda") for _ in range(2))
    if op in ("evict", "step"):
        st["kept"] = torch.zeros(B, H, case["budget"] if op == "evict" else n, **i32)
        st["len_out"] = torch.zeros(B, **i32)
    return st


def prepare(case, seed):
    st = _raw(case, seed)
    op, B, H, D = case["op"], case["B"], case["Hkv"], case["D"]
    if op in ("decode", "step"):
        st["out"] = torch.empty(B, case["Hq"], D, dtype=_dt(case), device="cuda")
        st["lse"] = torch.empty(B, case["Hq"], dtype=torch.float32, device="cuda")
    if own:   # the packed cache, its description, and what a program keeps beside it
        from paper_2607_18081_b200 import api
        new = lambda cap, length, pos=None, weight=None: api.KV4Cache.empty(B, H, cap, D, case["group"], _dt(case), length, pos, weight)  # noqa: E731
        if op == "store":
            st["src"] = api.KVCache(st["k"], st["v"], st["new"])
            st["cache"] = new(st["cap"], st["past"])
            st["after"] = api.KV4Cache(st["cache"].data, D, case["group"], _dt(case), st["len"])
            st["back"] = api.KVCache(st["out_k"], st["out_v"], st["new"])
            return st
        st["cache"] = new(st["cap"], st["len"], st.get("pos"), st.get("weight"))
        full = torch.full((B,), st["cap"], dtype=torch.int32, device="cuda")
        api.si_kv4_store(api.KVCache(st["k"], st["v"], full), api.KV4Cache(st["cache"].data, D, case["group"], _dt(case), torch.zeros_like(full)), None)
        if op == "load":
            st["back"] = api.KVCache(st["out_k"], st["out_v"], st["len"])
        if op == "evict":
            st["dst"] = new(_tiles(case["budget"]), st["len_out"], st["dpos"], st["dweight"])
            st["back"] = api.KVCache(st["out_k"], st["out_v"], st["len_out"])
        if op != "load":
            st["ws"] = st["cache"].workspace(case["Hq"])
    elif op != "store":
        st["kq"], st["vq"] = _quantise(st["k"], case["group"]), _quantise(st["v"], case["group"])
    if op != "store":
        del st["k"], st["v"]
    return st


# ------------------------------------------------------------------------------------------------ plain form

def _round_up(x, dt):
    """fp32 x >= 0 rounded up to dt."""
    y = x.to(dt)
    return torch.where(y.float() < x, (y.view(torch.int16) + 1).view(dt), y)


def _quantise(x, group):
    """[..., D] of a 16-bit type -> codes uint8 [..., D / group, group], steps and lowest values [..., D / group, 1]."""
    x = x.unflatten(-1, (-1, min(group, x.shape[-1])))
    m = x.amin(-1, keepdim=True)
    step = (x.amax(-1, keepdim=True).float() - m.float()) * torch.tensor(1.0 / 15.0, dtype=torch.float32, device=x.device)
    s = _round_up(step, x.dtype)
    r = torch.where(s > 0, 1.0 / s.float(), 0.0)
    c = torch.round((x.float() - m.float()).double() * r.double()).clamp_(0, 15)     # exact: quotients halfway between two codes are common
    return c.to(torch.uint8), s, m


def _values(c, s, m):
    return (c.float() * s.float() + m.float()).flatten(-2)


def _attend(case, st, n):
    """Attention of one query per sequence over the first n[b] entries: out, lse (32 bits) and the weights [B, Hkv, G, cap]."""
    B, H, D, Hq, cap = case["B"], case["Hkv"], case["D"], case["Hq"], st["cap"]
    s = torch.matmul(st["q"].float().view(B, H, Hq // H, D), _values(*st["kq"]).transpose(-1, -2)) * st["scale"]
    j = torch.arange(cap, device="cuda")
    at = (st["q_pos"].long() if "q_pos" in st else n - 1)[:, None, None]
    p = st["pos"].long() if "pos" in st else j[None, None]
    seen = (p <= at) & (j < n[:, None, None])
    if case["window"]:
        seen = seen & ((p > at - case["window"]) | (p < case["n_sink"]))
    s = s.masked_fill(~seen[:, :, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)        # a row with nothing visible: all exp = 0
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    w = e / total.clamp_min(torch.finfo(torch.float32).tiny)
    return torch.matmul(w, _values(*st["vq"])).view(B, Hq, D), (total.log() + top).view(B, Hq), w


def _decode(case, st):
    n = st["len"].long()
    b = torch.arange(case["B"], device="cuda")
    for to, x in ((st["kq"], st["k_new"]), (st["vq"], st["v_new"])):
        for a, y in zip(to, _quantise(x, case["group"])):
            a[b, :, n] = y
    if "pos" in st:
        st["pos"][b, :, n] = st["q_pos"][:, None]
    out, lse, w = _attend(case, st, n + 1)
    st["out"].copy_(out)
    st["lse"].copy_(lse)
    if "weight" in st:
        st["weight"][b, :, n] = 0.0
        st["weight"] += w.sum(2)


def _keep(case, st, n, budget, pos, last):
    """Source slot of every slot below the budget, -1 beyond the kept entries: protected positions first, then the largest weights."""
    B, H, cap = st["weight"].shape
    j = torch.arange(cap, device="cuda")
    used = (j < n[:, None])[:, None]
    safe = (pos < case["n_sink"]) | (pos > last[:, None, None] - case["n_recent"])
    rank = st["weight"].masked_fill(safe, math.inf).masked_fill(~used, -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros(B, H, cap, dtype=torch.bool, device="cuda").scatter_(-1, best, True) & used
    # kept entries below the budget stay; the i-th kept entry beyond it goes to the i-th freed slot
    hole = ~kept[..., :budget]
    movers = torch.sort((kept & (j >= budget)).to(torch.int8), dim=-1, descending=True, stable=True).indices
    moves = (kept & (j >= budget)).sum(-1, keepdim=True)
    nth = (hole.long().cumsum(-1) - 1).clamp_min(0)
    source = torch.where(hole, movers.gather(-1, nth), j[:budget].expand(B, H, budget))
    return torch.where(~hole | (nth < moves), source, -1)


def _pick(x, source):
    """Entries source[b, h, i] of x [B, H, cap, ...] (the first one where it is -1)."""
    i = source.clamp_min(0)
    return x.gather(2, i.view(*i.shape, *[1] * (x.dim() - 3)).expand(*i.shape, *x.shape[3:]))


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2607_18081_b200 import api
    if op == "store":
        if own:
            api.si_kv4_store(st["src"], st["cache"], None)
            api.si_kv4_load(st["after"], st["back"], st["past"], case["T"], None)
        else:
            here = (torch.arange(case["T"], device="cuda") < st["new"][:, None])[:, None, :, None]
            for out, x in ((st["out_k"], st["k"]), (st["out_v"], st["v"])):
                out.copy_(torch.where(here, _values(*_quantise(x, case["group"])).to(out.dtype), out))
        return {"k": st["out_k"], "v": st["out_v"]}
    if op == "load":
        if own:
            api.si_kv4_load(st["cache"], st["back"], None, st["cap"], None)
        else:
            here = (torch.arange(st["cap"], device="cuda") < st["len"][:, None])[:, None, :, None]
            for out, x in ((st["out_k"], st["kq"]), (st["out_v"], st["vq"])):
                out.copy_(torch.where(here, _values(*x).to(out.dtype), out))
        return {"k": st["out_k"], "v": st["out_v"]}
    if op == "evict":
        budget = case["budget"]
        if own:
            api.si_kv4_evict(st["cache"], st["dst"], None, 0, budget, case["n_sink"], case["n_recent"], st["kept"], st["len_out"], st["ws"])
            api.si_kv4_load(st["dst"], st["back"], None, budget, None)
        else:
            n = st["len"].long()
            source = _keep(case, st, n, budget, torch.arange(st["cap"], device="cuda").expand(st["weight"].shape), n - 1)
            ok = source >= 0
            st["kept"].copy_(source)
            st["len_out"].copy_(n.clamp_max(budget))
            for out, x in ((st["out_k"], st["kq"]), (st["out_v"], st["vq"])):
                out.copy_(torch.where(ok[..., None], _values(*(_pick(a, source) for a in x)).to(out.dtype), out))
            for out, x in ((st["dpos"], source), (st["dweight"], _pick(st["weight"], source))):
                out[..., :budget] = torch.where(ok, x.to(out.dtype), out[..., :budget])
        return {"k": st["out_k"], "v": st["out_v"], "pos": st["dpos"], "weight": st["dweight"], "kept": st["kept"], "len": st["len_out"]}
    if own:
        flags = api.SI_FLAG_ACC_WEIGHT if "weight" in st else 0
        api.si_kv4_attn_decode(st["cache"], st["q"], st.get("q_pos"), st["k_new"], st["v_new"], case["window"], case["n_sink"], st["scale"],
                               st["out"], st["lse"], flags, st["ws"])
    else:
        _decode(case, st)
    res = {"out": st["out"], "lse": st["lse"]}
    if op == "step":
        n = case["n"]
        if own:
            api.si_kv4_evict(st["cache"], st["cache"], st["q_pos"], 1, n, case["n_sink"], case["n_recent"], st["kept"], st["len_out"], st["ws"])
        else:
            source = _keep(case, st, st["len"].long() + 1, n, st["pos"], st["q_pos"].long())
            st["kept"].copy_(source)
            st["len_out"].copy_((st["len"] + 1).clamp_max(n))
            for x in (*st["kq"], *st["vq"], st["pos"], st["weight"]):
                x[:, :, :n] = _pick(x, source)
        res.update(pos=st["pos"], kept=st["kept"], len=st["len_out"])
    if "weight" in st:
        res["weight"] = st["weight"]
    return res


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_cache(x, group, dt):
    """What a 16-bit [..., D] stands for once held in 4 bits: the definition above, its fp32 roundings explicit ones of 64-bit results."""
    fl = lambda y: y.float().double()  # noqa: E731
    z = x.double().reshape(*x.shape[:-1], -1, min(group, x.shape[-1]))
    low, high = z.min(-1, keepdim=True).values, z.max(-1, keepdim=True).values
    fifteenth = fl(fl(high - low) * float(np.float32(1.0 / 15.0)))
    step = fifteenth.to(dt).double()
    bits = step.to(dt).view(torch.int16)
    step = torch.where(step < fifteenth, (bits + 1).view(dt).double(), step)
    inverse = torch.where(step > 0, fl(1.0 / step.clamp_min(1e-300)), 0.0)
    code = (fl(z - low) * inverse).round().clamp(0, 15)
    return (low + step * code).reshape(x.shape)


def exact(case, seed):
    st = _raw(case, seed)
    dt, group, op, B, H, D = _dt(case), case["group"], case["op"], case["B"], case["Hkv"], case["D"]
    if op in ("store", "load"):
        lens = (st["new"] if op == "store" else st["len"]).tolist()
        res = {"k": torch.zeros(st["out_k"].shape, dtype=torch.float64, device="cuda"), "v": torch.zeros(st["out_k"].shape, dtype=torch.float64, device="cuda")}
        for b, n in enumerate(lens):
            for x in ("k", "v"):
                for h in range(H):
                    res[x][b, h, :n] = _exact_cache(st[x][b, h, :n], group, dt)
        return res
    lens = st["len"].tolist()
    if op == "evict":
        return _exact_evict(case, st, lens, {})
    G = case["Hq"] // H
    out = torch.zeros(B, case["Hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, case["Hq"], dtype=torch.float64, device="cuda")
    weight = st["weight"].double() if "weight" in st else None
    for b, n in enumerate(lens):
        for h in range(H):
            k = _exact_cache(torch.cat([st["k"][b, h, :n], st["k_new"][b, h, None]]), group, dt)
            v = _exact_cache(torch.cat([st["v"][b, h, :n], st["v_new"][b, h, None]]), group, dt)
            p = torch.arange(n + 1, device="cuda") if "pos" not in st else torch.cat([st["pos"][b, h, :n], st["q_pos"][b, None]])
            here = int(st["q_pos"][b]) if "pos" in st else n
            ok = p <= here
            if case["window"]:
                ok &= (here - p < case["window"]) | (p < case["n_sink"])
            logit = (st["q"][b, h * G:(h + 1) * G].double() @ k.T * st["scale"]).masked_fill(~ok, -math.inf)
            z = torch.logsumexp(logit, -1, keepdim=True)
            w = torch.exp(logit - z).masked_fill(~ok, 0.0)
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = w @ v, z[:, 0]
            if weight is not None:
                weight[b, h, n] = 0.0
                weight[b, h, :n + 1] += w.sum(0)
            if "pos" in st:
                st["pos"][b, h, n] = here
    res = {"out": out, "lse": lse}
    if op == "step":
        st["weight"] = weight
        return _exact_evict(case, st, [n + 1 for n in lens], res)
    if weight is not None:
        res["weight"] = weight
    return res


def _exact_evict(case, st, lens, res):
    """The entries that stay, found by sorting row by row; in a step within the cache, otherwise into one of the budget's size."""
    step, H = case["op"] == "step", case["Hkv"]
    budget = case["n"] if step else case["budget"]
    weight = st["weight"].double().cpu().numpy()
    place = np.arange(weight.shape[2])
    kept = np.full((case["B"], H, budget), -1, np.int64)
    for b, n in enumerate(lens):
        last = int(st["q_pos"][b]) if step else n - 1
        for h in range(H):
            p, w = (st["pos"][b, h].cpu().numpy() if step else place)[:n].astype(np.int64), weight[b, h, :n]
            held = (p < case["n_sink"]) | (last - p < case["n_recent"])
            order = np.lexsort((np.arange(n), -w, ~held))[:budget]
            stay = np.sort(order[order < budget])
            free = np.setdiff1d(np.arange(min(budget, n)), stay)
            kept[b, h, stay] = stay
            come = np.sort(order[order >= budget])
            kept[b, h, free[:len(come)]] = come
    keep = torch.from_numpy(kept).cuda()
    got = keep >= 0
    res["kept"] = keep.int()
    res["len"] = torch.tensor([min(n, budget) for n in lens], dtype=torch.int32)
    if step:
        for x in ("pos", "weight"):
            res[x] = st[x].clone()
            res[x][:, :, :budget] = torch.where(got, st[x].gather(2, keep.clamp_min(0)), st[x][:, :, :budget])
        return res
    for x in ("dpos", "dweight"):
        y = keep if x == "dpos" else st["weight"].gather(2, keep.clamp_min(0)).double()
        res[x[1:]] = torch.zeros(st[x].shape, dtype=torch.int32 if x == "dpos" else torch.float64, device="cuda")
        res[x[1:]][..., :budget] = torch.where(got, y, 0).to(res[x[1:]].dtype)
    for x in ("k", "v"):
        res[x] = torch.zeros(st["out_k"].shape, dtype=torch.float64, device="cuda")
        b, h, i = got.nonzero(as_tuple=True)
        res[x][b, h, i] = _exact_cache(st[x][b, h, keep[b, h, i]], case["group"], _dt(case))
    return res


# ------------------------------------------------------------------------------------------------ what a call cannot do without

def work(case):
    op, B, H, D = case["op"], case["B"], case["Hkv"], case["D"]
    wide = 4 * D                                            # a key and a value in 16 bits
    entry = D + 8 * (D // min(case["group"], D))            # ... in 4 bits, with step and lowest value of every group
    if op == "store":                                       # and read back
        n = sum(_lens(case, case["T"])) * H
        return {"bytes": 2 * n * (wide + entry), "flops": 0}
    lens = _lens(case, case["n"])
    if op == "load":
        return {"bytes": sum(lens) * H * (wide + entry), "flops": 0}
    if op == "evict":                                       # weights in, entries moved, read back
        kept = sum(min(n, case["budget"]) for n in lens) * H
        return {"bytes": sum(lens) * H * 4 + kept * (3 * entry + wide + 16), "flops": 0}
    w, s = case["window"], case["n_sink"]
    seen = 0
    for n in lens:
        n += 1
        if w:
            n = min(n, (w if not case.get("pos") else int(w * 2 / 3)) + s)
        seen += n
    acc, pos = op == "step" or case["acc"], op == "step" or case.get("pos")
    bytes_ = seen * H * entry + B * case["Hq"] * (4 * D + 4) + B * H * (wide + entry) + (8 * seen * H if acc else 0) + (4 * sum(lens) * H if pos else 0)
    if op == "step":                                        # positions and weights for the choice, one entry moved
        bytes_ += sum(lens) * H * 12 + B * H * (2 * entry + 16)
    return {"bytes": bytes_, "flops": 4 * D * seen * case["Hq"]}
