"""Single-token attention over the cache in 4 bits where the values' steps differ by many orders of magnitude: between the groups of
an entry, between entries that matter and entries that do not, from one tile to the next, beside NaN.

Bounds (e = 2^-24, u the unit roundoff of the type; p softmax weights, s c the step and code of value j, m its lowest value), per
query head and channel, the channel's own group only:
  p s      rounded to 11 bits for the products with codes shifted to -8 .. 7: 8 * 2^-11 sum_j p_j s_j.  The scale that f16 is given follows the
           largest p s of the head and group and holds it above 2^7, so below 2^-14 a rounding is 2^-25 at most, 2^-32 of the largest: 8 n 2^-32 max_j p_j s_j
  sums     (2 delta + (n + 32) e) sum_j p_j (|m_j| + 16 s_j): partial sums hold the codes without the shift
  weights  below 2^-110 of the largest count as 0: 2^-108 sum_j (|m_j| + 16 s_j)
  result   u |out|, f16 2^-25
delta and the bounds of lse and of the weights as in kv4_utils."""
import numpy as np
import pytest
import torch

from tests import attn_utils as au
from tests import kv4_utils as k4

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
E = au.E

# head_dim, group, query heads per key head: every way of laying heads and groups out in the matrix products
FORMS = [(128, 32, 4), (128, 64, 3), (64, 32, 4), (64, 64, 4), (128, 32, 8), (128, 64, 6), (64, 32, 5), (128, 32, 16), (128, 64, 9), (64, 64, 12), (64, 32, 20)]


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def statement(made, q, n, scale):
    """float64: results of the first n entries of sequence 0 for queries q [Hq, D], and what the bounds need."""
    qn, H = au.f64(q), made.k.shape[1]
    G = len(qn) // H
    k = made.values("k")
    (km, ks, kc), (vm, vs, vc) = made.kq, made.vq
    r = {x: [] for x in ("out", "ps", "peak", "reach", "all", "lse", "size", "p")}
    with np.errstate(invalid="ignore", over="ignore"):
        for hq in range(len(qn)):
            h = hq // G
            x = k[0, h, :n] @ qn[hq] * scale
            p = np.exp(x - x.max())
            r["lse"].append(x.max() + np.log(p.sum()))
            r["size"].append(((np.abs(km[0, h, :n]) + ks[0, h, :n] * kc[0, h, :n]) @ np.abs(qn[hq])).max() * abs(scale))
            p /= p.sum()
            m, s, c = vm[0, h, :n], vs[0, h, :n], vc[0, h, :n]
            r["p"].append(p)
            r["out"].append(p @ (m + s * c))
            r["ps"].append(p @ s)
            r["peak"].append((p[:, None] * s).max(0))
            r["reach"].append(p @ (np.abs(m) + 16 * s))
            r["all"].append((np.abs(m) + 16 * s).sum(0))
    return {x: np.array(y) for x, y in r.items()} | {"n": n}


def attend(api, made, q, n, scale, rows):
    """q [Hq, D] over sequence 0, `rows` times as sequences that share its memory: out [rows, Hq, D], lse, weights [rows, H, cap]."""
    c, Hq = made.cache, len(q)
    cache = api.KV4Cache(c.data[:1].expand(rows, -1, -1, -1), made.D, made.group, made.dt, torch.full((rows,), n, **I32), None,
                         torch.zeros(rows, c.n_kv_heads, c.capacity, device="cuda"))
    out, lse = torch.full((rows, Hq, made.D), 7.0, dtype=made.dt, device="cuda"), torch.full((rows, Hq), 7.0, device="cuda")
    status, ws = torch.zeros(1, **I32), cache.workspace(Hq)
    ws.fill_(0xFF)
    api.si_kv4_attn_decode(cache, q.expand(rows, -1, -1).contiguous(), None, None, None, 0, 0, scale, out, lse, api.SI_FLAG_ACC_WEIGHT, ws, status)
    assert status.item() == 0
    return out, lse, cache.weight


def check(made, got, ref):
    """Every row against the statement; NaN exactly where the statement has it."""
    out, lse, weight = (au.f64(x) for x in got)
    n, H = ref["n"], weight.shape[1]
    d = (2 * made.D + 16) * E * ref["size"] + E * (4 * (np.abs(ref["lse"]) + ref["size"]) + 128)
    rel = (2 * d + (n + 32) * E)[:, None]
    bound = 1.01 * (au.U[made.dtype] * np.abs(ref["out"]) + 8 * 2.0 ** -11 * ref["ps"] + 8 * n * 2.0 ** -32 * ref["peak"] + rel * ref["reach"] + 2.0 ** -108 * ref["all"])
    bound = bound + (2.0 ** -25 if made.dtype == "f16" else 0.0)
    nan = np.isnan(ref["out"])
    assert np.array_equal(np.isnan(out), np.broadcast_to(nan, out.shape))
    err = np.where(nan, 0.0, np.abs(out - ref["out"]))
    bound = np.where(nan, 1.0, bound)
    assert np.all(err <= bound), f"out: {np.max(err / np.maximum(bound, 1e-300)):.3f} of the bound"
    bound = d + 4 * E * (np.abs(ref["lse"]) + 128) + n * E
    assert np.all(np.abs(lse - ref["lse"]) <= bound), np.max(np.abs(lse - ref["lse"]) / bound)
    want = ref["p"].reshape(H, -1, n).sum(1)
    bound = (4 * d.max() + (n + len(d) // H + 16) * E) * want + 2 * E * want + 1e-30
    assert np.all(np.abs(weight[:, :, :n] - want) <= bound) and (weight[:, :, n:] == 0).all()


def case(api, D, group, G, dtype, v, k=None, q=None, n=1000, scale=0.1, seed=0, H=2):
    g = torch.Generator().manual_seed(seed + G)
    cap = (n + 31) // 32 * 32
    k = torch.randn(1, H, cap, D, generator=g) * 0.3 if k is None else k
    made = k4.Made(api, 1, H, D, cap, group, dtype, [n], k=k, v=v)
    q = (torch.randn(G * H, D, generator=g) if q is None else q).to(made.dt).cuda()
    ref = statement(made, q, n, scale)
    for rows in (1, 400):                     # a run of tiles per warp: one or two tiles of one item, and many
        check(made, attend(api, made, q, n, scale, rows), ref)


def noise(D, n=1000, H=2, seed=1):
    return torch.randn(1, H, (n + 31) // 32 * 32, D, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,G", FORMS)
def test_nan_and_infinity_stay_in_their_group(api, D, group, G, dtype):
    """One group of one value, in the first tile or a later one: the other groups' results are what they are without it."""
    for at, special in ((3, float("inf")), (700, float("nan")), (999, float("-inf"))):
        v = noise(D)
        v[0, 1, at, D - 5] = special
        case(api, D, group, G, dtype, v)


FAR = ["apart", "zeros_large", "zeros_constant", "zeros_nan", "constant_small"]


@pytest.mark.parametrize("kind", FAR)
@pytest.mark.parametrize("D,group,G", FORMS)
def test_steps_that_jump_do_not_touch_the_softmax(api, D, group, G, kind):
    """bf16 values whose size changes at once by more than fp32 has exponents: with equal scores lse is log n and every weight 1 / n,
    whatever the values are."""
    v, n = noise(D), 1000
    first = torch.arange(v.shape[2])[:, None] < 500
    one = torch.ones_like(v)
    v = {"apart": torch.where(first, v * 2.0 ** -70, v * 2.0 ** 70), "zeros_large": torch.where(first, 0.0, v * 2.0 ** 60),
         "zeros_constant": torch.where(first, 0.0, one * 2.0 ** 100), "zeros_nan": torch.where(first, 0.0, v),
         "constant_small": torch.where(first, one * 2.0 ** 30, v * 2.0 ** -60)}[kind]
    if kind == "zeros_nan":
        v[0, 0, 600, 1], v[0, 1, 999, D - 1] = float("nan"), float("inf")
    case(api, D, group, G, "bf16", v, n=n)
    case(api, D, group, G, "bf16", v, k=torch.zeros_like(v), n=n)


def test_every_entry_of_a_constant_group_counts(api):
    """Groups without a step, zeros first: 2^30, and the largest number of bf16."""
    for top in (2.0 ** 30, 3.3e38):
        v = torch.zeros(1, 2, 320, 128)
        v[:, :, 200:] = top
        case(api, 128, 32, 4, "bf16", v, n=300)
        case(api, 64, 64, 12, "bf16", v[..., :64].contiguous(), n=300)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_largest_of_scores_beyond_2_to_24(api, dtype):
    """Scores that are exact and so far apart that one entry has all the weight: its value comes back."""
    n, D, H = 300, 64, 1
    g = torch.Generator().manual_seed(3)
    k = torch.ones(1, H, 320, D) * torch.randperm(320, generator=g).float()[:, None] / 64
    v = torch.randn(1, H, 320, D, generator=g) * (2.0 ** 40 if dtype == "bf16" else 64.0)
    for G, group in ((4, 32), (8, 64), (16, 32)):
        made = k4.Made(api, 1, H, D, 320, group, dtype, [n], k=k, v=v)
        q = torch.full((G, D), 8.0 if dtype == "f16" else 2.0 ** 24, dtype=made.dt, device="cuda")
        m, s, c = (x[0, 0, int(made.values("k")[0, 0, :n, 0].argmax())] for x in made.vq)
        for rows in (1, 400):
            out = au.f64(attend(api, made, q, n, 1.0 if dtype == "bf16" else 2.0 ** 20, rows)[0])
            want = m + s * c
            assert np.all(np.abs(out - want) <= 1.01 * (au.U[dtype] * np.abs(want) + 8 * 2.0 ** -11 * s) + (2.0 ** -25 if dtype == "f16" else 0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,G", FORMS)
def test_groups_of_very_different_sizes(api, D, group, G, dtype):
    """Channels of an entry 2^30 (f16: 2^22) apart, alone and with one entry that has most of the weight."""
    v, groups = noise(D), D // group
    reach = 30 if dtype == "bf16" else 22
    up = torch.arange(D) // group * (reach / max(groups - 1, 1)) - (15 if dtype == "bf16" else 12)
    case(api, D, group, G, dtype, v * 2.0 ** up)
    base = torch.randn(1, D, generator=torch.Generator().manual_seed(5))
    q = base + 0.1 * torch.randn(2 * G, D, generator=torch.Generator().manual_seed(6))
    k = noise(D, seed=7) * 0.1
    k[0, :, 450] = base * (4.2 / (0.1 * base.pow(2).sum()))
    case(api, D, group, G, dtype, v * 2.0 ** up.flip(0), k=k, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,G", FORMS)
@pytest.mark.parametrize("at", [0, 33, 620])
def test_one_large_entry_of_no_weight(api, D, group, G, dtype, at):
    """An entry whose steps are far above all others and whose weight is 0: the others keep their bits."""
    v, base = noise(D), torch.randn(1, D, generator=torch.Generator().manual_seed(5))
    q = base + 0.1 * torch.randn(2 * G, D, generator=torch.Generator().manual_seed(6))
    k = noise(D, seed=7) * 0.1
    k[0, :, at] = -base * (200.0 / (0.1 * base.pow(2).sum()))
    if dtype == "f16":
        v = v * 2.0 ** -10
    v[0, :, at] = v[0, :, at] * (2.0 ** 70 if dtype == "bf16" else 2.0 ** 23)
    case(api, D, group, G, dtype, v, k=k, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,G", FORMS)
def test_scores_grow_while_steps_shrink(api, D, group, G, dtype):
    """What is large comes first and loses its weight little by little, and at once; and the other way round."""
    base = torch.randn(1, D, generator=torch.Generator().manual_seed(5))
    q = base + 0.05 * torch.randn(2 * G, D, generator=torch.Generator().manual_seed(6))
    along = torch.linspace(0.0, 1.0, 1024)[:, None]
    unit = base / (0.1 * base.pow(2).sum())
    range2 = 40.0 if dtype == "bf16" else 20.0
    for shape in (along, torch.floor(along * 4) / 4):
        size = 2.0 ** (range2 * (0.5 - shape))
        for steps in (size, 1 / size):
            k = unit * shape * 25.0 + noise(D, seed=7) * 0.05
            case(api, D, group, G, dtype, noise(D) * steps, k=k, q=q)


@pytest.mark.parametrize("D,group,G", FORMS)
def test_queries_near_the_largest_number(api, D, group, G):
    """Finite bf16 queries of up to 2^127 with a scale that brings the scores back; a query and a scale of zero."""
    q = torch.randn(2 * G, D, generator=torch.Generator().manual_seed(4))
    q[0] = 0.0
    case(api, D, group, G, "bf16", noise(D), q=q.clamp(-1.9, 1.9) * 2.0 ** 126, scale=0.1 * 2.0 ** -126)
    one = torch.where(torch.arange(D) % 7 == 2, 1.9, 0.0) * 2.0 ** 126 * torch.ones(2 * G, 1)
    case(api, D, group, G, "bf16", noise(D), q=one, scale=0.1 * 2.0 ** -126)
    case(api, D, group, G, "bf16", noise(D), q=q, k=torch.sign(noise(D, seed=2)[..., :1]).expand(-1, -1, -1, D) * 3.0e38, scale=0.0)
    case(api, D, group, G, "bf16", noise(D), q=torch.zeros(2 * G, D), scale=1.9e38)


def test_scores_beyond_the_largest_number_are_nan(api):
    """Never finite and wrong: |scale q| of 2^130 is refused by NaN, and the other heads keep their results."""
    for D, group, G in FORMS:
        q = torch.randn(2 * G, D, generator=torch.Generator().manual_seed(4)) * 2.0 ** -20
        k = noise(D, seed=7)
        made = k4.Made(api, 1, 2, D, 1024, group, "bf16", [1000], k=k * 2.0 ** -100, v=noise(D))
        q[G - 1] = 2.0 ** 105
        q = q.to(made.dt).cuda()
        out, lse, _ = attend(api, made, q, 1000, 2.0 ** 25, 1)
        assert out[0, G - 1].isnan().all() and lse[0, G - 1].isnan()
        assert not out[0, :G - 1].isnan().any() and not out[0, G:].isnan().any()


@pytest.mark.parametrize("D,group,G", FORMS)
def test_results_end_where_f16_ends(api, D, group, G):
    """-65504 and 65504 in one group: the step is rounded up and m + 15 s is 65536.  The largest number comes back, from attention as from
    reading back; one entry (a result of one run of tiles) and many (parts that are joined)."""
    for n in (1, 900):
        v = torch.where(torch.arange(D) % 2 == 0, 65504.0, -65504.0) * torch.ones(1, 2, (n + 31) // 32 * 32, 1)
        made = k4.Made(api, 1, 2, D, v.shape[2], group, "f16", [n], k=torch.zeros_like(v), v=v)
        q = torch.randn(2 * G, D, device="cuda").half()
        back = made.read()[1][0, 0, 0]
        assert back.tolist() == [65504.0, -65504.0] * (D // 2)
        for rows in (1, 400):
            out, _, _ = attend(api, made, q, n, 0.1, rows)
            assert torch.equal(out, back.expand_as(out))


@pytest.mark.parametrize("D,group,G", FORMS)
def test_roundings_beyond_the_ends_of_f16(api, D, group, G):
    """The same values, one entry ahead of the others by 2 / (1 + 1.05 * 2^-11): p s of the others lies just above the middle of two f16 numbers and is
    rounded up, by 30 in what the lowest number comes out as.  Still a finite result."""
    v = torch.where(torch.arange(D) % 2 == 0, 65504.0, -65504.0) * torch.ones(1, 2, 32, 1)
    k = torch.zeros_like(v)
    k[:, :, 0] = 1.0
    scale = -float(np.log(0.5 * (1.0 + 1.05 * 2.0 ** -11))) / D
    case(api, D, group, G, "f16", v, k=k, q=torch.ones(2 * G, D), n=32, scale=scale)
