"""Rows of one distillation call stay apart: each has the bits that it has in a call
that takes the rows in another order."""
import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


# streamed by clusters of one CTA (24000 bf16 or 12000 binary32 entries on), by larger
# ones, held in registers; one slot, and as many as a warp takes, all of few ids, so that
# the teacher's side takes longer than the row
@pytest.mark.parametrize("T,V,K,few,dtype", [
    (700, 32000, 1, 0, BF), (2000, 32000, 256, 3, BF), (2000, 24008, 256, 0, BF), (900, 16000, 256, 3, F32),
    (2600, 60000, 256, 3, F32), (1300, 152064, 200, 3, BF), (300, 9000, 256, 3, BF)])
def test_rows_in_another_order_keep_their_bits(T, V, K, few, dtype):
    g = torch.Generator(DEV).manual_seed(V + K)
    z = (torch.randn(T, V, generator=g, device=DEV) * 3).to(dtype)
    z += torch.randn(T, 1, generator=g, device=DEV).to(dtype) * 20          # rows of their own maximum
    ids = torch.randint(0, V, (T, K), generator=g, device=DEV)
    if few:
        ids = ids[:, :few].gather(1, torch.randint(0, few, (T, K), generator=g, device=DEV))
    ids[::7] = -1
    t, d = torch.randn(T, K, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)
    want = iso.distill(z, ids, t, 1.5, dloss=d)
    alone = iso.distill(z, ids, t, 1.5)
    grad = iso.distill_grad(d, z, ids, t, want[1], 1.5)
    order = torch.randperm(T, generator=g, device=DEV)
    a, i, w, e = z[order], ids[order].contiguous(), t[order].contiguous(), d[order].contiguous()
    for got, ref in zip((*iso.distill(a, i, w, 1.5, dloss=e), *iso.distill(a, i, w, 1.5),
                         iso.distill_grad(e, a, i, w, want[1][order].contiguous(), 1.5)), (*want, *alone, grad)):
        assert torch.isfinite(ref).all()
        assert torch.equal(got, ref[order])
    assert (want[0][::7] == 0).all() and (want[2][::7] == 0).all()
