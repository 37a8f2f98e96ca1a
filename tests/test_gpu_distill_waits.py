"""Streamed distillation whose waits give up: every value is whole or NaN, the status
says so, and the next call is whole again."""
import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
TIMEOUT = _abi.ISO_ERR_TIMEOUT


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


@pytest.fixture
def limit():
    """Sets the time after which a wait gives up."""
    L = _abi.lib()
    before = L.iso_distill_wait_ns(-1)
    assert before == 2000000000
    yield lambda ns: L.iso_distill_wait_ns(ns)
    torch.cuda.synchronize()
    L.iso_distill_wait_ns(before)


def _same_or_nan(got, want, what):
    ok = torch.isnan(got) | (got == want)
    assert bool(ok.all()), (what, int((~ok).sum()))
    return bool(torch.isnan(got).any())


# clusters of one CTA and of several, rows enough for each to come back to its stages
@pytest.mark.parametrize("T,V,K,dtype", [(4000, 32000, 64, BF), (3000, 16000, 200, F32), (2600, 60000, 64, F32), (1300, 152064, 64, BF)])
@pytest.mark.parametrize("form", ["joint", "in place", "loss", "gradient"])
def test_a_give_up_leaves_each_value_whole_or_nan(T, V, K, dtype, form, limit):
    g = torch.Generator(DEV).manual_seed(V)
    z = (torch.randn(T, V, generator=g, device=DEV) * 3).to(dtype)
    ids, t = torch.randint(0, V, (T, K), generator=g, device=DEV), torch.randn(T, K, generator=g, device=DEV)
    ids[::11] = -1
    d = torch.randn(T, generator=g, device=DEV)
    lse = iso.distill(z, ids, t)[1]

    def call():
        if form == "loss":
            return iso.distill(z, ids, t, status=True)
        if form == "gradient":
            return iso.distill_grad(d, z, ids, t, lse, status=True)
        x = z.clone() if form == "in place" else z
        return iso.distill(x, ids, t, dloss=d, out=x if form == "in place" else None, status=True)
    *want, st = call()
    assert int(st) == 0 and all(bool(torch.isfinite(w).all()) for w in want)
    limit(0)
    seen = set()
    for _ in range(40):
        *got, st = call()
        nan = [_same_or_nan(a, b, form) for a, b in zip(got, want)]
        seen.add(int(st))
        assert int(st) in (0, TIMEOUT) and any(nan) == (int(st) == TIMEOUT)
        del got
    if form != "loss" or V <= 32000:             # (the loss alone is streamed where one CTA holds a row)
        assert TIMEOUT in seen
    limit(2000000000)
    *again, st = call()
    assert int(st) == 0 and all(torch.equal(a, b) for a, b in zip(again, want))
