"""si_kv4_load where the number of entries read back goes into the array that the lengths, or the first entries, come from."""
import pytest
import torch

from tests import kv4_utils as k4
from tests.test_kv4_abi import FAKE, _kv, _kv4, _load

I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def api():
    from paper_2607_18081_b200 import api as _api
    return _api


def test_len_out_may_be_an_input_but_not_overlap_one(api):
    """One array for len_out and src->len (or `first`) is written after all of it was read; one shifted against it is refused."""
    kv4, kv = _kv4(api), _kv(api)
    for shift in (-4, 4):
        assert _load(api, kv4, kv, len_out=kv4.len + shift) == api.SI_ERR_INVALID_ARG
        assert _load(api, kv4, kv, first=FAKE, len_out=FAKE + shift) == api.SI_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("with_first", [False, True])
def test_number_of_entries_in_the_array_of_the_lengths(api, with_first):
    """si_kv4_load writes len_out over src->len, or over `first`, which all of its blocks read: after they have."""
    B, H, D, cap = 3, 2, 64, 4096
    lens, first, n = [4096, 2500, 1], [4000, 17, 0], 3000
    for alias in ("len", "first") if with_first else ("len",):
        made = k4.Made(api, B, H, D, cap, 32, "bf16", lens, seed=1)
        start = torch.tensor(first, **I32) if with_first else None
        want = [torch.full((B, H, cap, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
        count = torch.zeros(B, **I32)
        api.si_kv4_load(made.cache, api.KVCache(want[0], want[1], count), start, n, count)
        out = made.length if alias == "len" else start
        status = torch.zeros(1, **I32)
        api.si_kv4_load(made.cache, api.KVCache(want[2], want[3], out), start, n, out, status)
        assert status.item() == 0 and out.tolist() == count.tolist() == [min(n, m - (f if with_first else 0)) for m, f in zip(lens, first)]
        assert torch.equal(want[0].view(torch.int16), want[2].view(torch.int16)) and torch.equal(want[1].view(torch.int16), want[3].view(torch.int16))
