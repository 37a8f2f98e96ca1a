"""Attention whose waits give up, forward and backward: with a limit of 0 any wait does
that is not over at its first look.  A head's row is whole or NaN, the status says so,
and the next call is whole again."""
import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
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
    before = L.iso_attn_wait_ns(-1)
    yield lambda ns: L.iso_attn_wait_ns(ns)
    torch.cuda.synchronize()
    L.iso_attn_wait_ns(before)


def _rows(got, want, heads):
    """Whether some rows of heads are NaN; each is NaN throughout, or as wanted."""
    got, want = (t.view(t.shape[0], heads, -1) for t in (got, want))
    nan = torch.isnan(got).all(2)
    assert bool((nan | (got == want).all(2)).all())
    return nan


@pytest.mark.parametrize("n,m,heads,kv,D,seqs", [
    (3000, 3000, 8, 2, 128, None), (700, 700, 4, 4, 64, (0, 1, 300, 301, 700)), (1, 40000, 12, 2, 128, None),
    (300, 5000, 14, 2, 96, None), (2048, 2048, 12, 2, 64, None)])
def test_a_give_up_leaves_each_row_whole_or_nan(n, m, heads, kv, D, seqs, limit):
    g = torch.Generator(DEV).manual_seed(n + m)
    q, do = (torch.randn(n, heads * D, generator=g, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(m, kv * D, generator=g, device=DEV).bfloat16() for _ in range(2))
    ends = None if seqs is None else torch.tensor(seqs, dtype=torch.int32, device=DEV)
    out, lse = iso.attn(q, k, v, heads, kv, seqs=ends)
    grads = iso.attn_grad(do, q, k, v, out, lse, heads, kv, seqs=ends)
    limit(0)
    seen = [set(), set()]
    for _ in range(30):
        o, l, st = iso.attn(q, k, v, heads, kv, seqs=ends, status=True)
        nan = _rows(o, out, heads)
        assert torch.equal(torch.isnan(l), nan.t()) and bool((nan.t() | (l == lse)).all())
        assert int(st) == (TIMEOUT if bool(nan.any()) else 0)
        seen[0].add(int(st))
        *got, st = iso.attn_grad(do, q, k, v, out, lse, heads, kv, seqs=ends, status=True)
        nan = [bool(_rows(a, b, h).any()) for a, b, h in zip(got, grads, (heads, kv, kv))]
        assert int(st) == (TIMEOUT if any(nan) else 0)
        seen[1].add(int(st))
    assert all(TIMEOUT in s for s in seen)
    limit(2000000000)
    o, l, st = iso.attn(q, k, v, heads, kv, seqs=ends, status=True)
    *got, st2 = iso.attn_grad(do, q, k, v, o, l, heads, kv, seqs=ends, status=True)
    assert int(st) == int(st2) == 0 and all(torch.equal(a, b) for a, b in zip((o, l, *got), (out, lse, *grads)))
