"""Attention over finite scores of any size: keys that a channel of their own, against
a one in every query, puts at b or 2 b (as a padded batch masks keys by a large negative
number).  The rows of the larger number share the weight evenly, whatever b is.

Bounds: out is off by its sum's roundings, (m + 16) 2^-24 of the mean |v|, and its own,
2^-8 |out| (bfloat16) or 2^-24.  A weight of bfloat16 calls is e^(S - m) times 2 to the
rounding of m log2 e, which is the same in every weight and in their sum, but leaves
no weight a power of two: rounded to bfloat16 each is off by 2^-8, so out by 2^-8 of
the mean |v| more.  lse is off by four roundings of itself."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("b", [-1.0, -3e6, -1e9, -1e10, 1e10, -7e15, 3e20, -1e30, 1e30])
@pytest.mark.parametrize("n,m,heads,kv,D,every", [(300, 300, 4, 2, 64, 3), (40, 700, 2, 1, 128, 1), (1, 9000, 4, 1, 128, 2), (130, 130, 2, 2, 40, 5)])
def test_scores_of_any_size(n, m, heads, kv, D, every, b, dtype):
    g = torch.Generator(DEV).manual_seed(m)
    q, k = torch.zeros(n, heads * D, device=DEV, dtype=dtype), torch.zeros(m, kv * D, device=DEV, dtype=dtype)
    v = torch.randn(m, kv * D, generator=g, device=DEV).to(dtype)
    q[:, ::D] = 1
    at = torch.where(torch.arange(m, device=DEV) % every == 0, b, 2 * b).to(dtype)     # every = 1: b throughout
    k[:, ::D] = at[:, None]
    out, lse, st = iso.attn(q, k, v, heads, kv, status=True)
    assert int(st) == 0
    at, V, got, got_lse = at.double().cpu().numpy(), v.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    E = 2.0 ** -8 if dtype == BF else U
    for i in {0, 1, n // 2, n - 1} & set(range(n)):
        keys = at[:i + m - n + 1]
        w = np.exp(np.maximum((keys - keys.max()) * D ** -0.5, -1e3))
        for h in range(heads):
            c = slice(h // (heads // kv) * D, (h // (heads // kv) + 1) * D)
            want, mag = w @ V[:len(keys), c] / w.sum(), w @ np.abs(V[:len(keys), c]) / w.sum()
            tol = (m + 16) * U * mag + E * np.abs(want) + (2.0 ** -8 * mag if dtype == BF else 0)
            assert (np.abs(got[i, h * D:(h + 1) * D] - want) <= tol).all(), (i, h)
            ref = keys.max() * D ** -0.5 + math.log(w.sum())
            assert abs(got_lse[h, i] - ref) <= 4 * U * abs(ref) + (m / 64 + 32) * U + 2.0 ** -21
