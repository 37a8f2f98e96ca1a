"""The training-step kernels at the sizes where their outer loops turn: many
tiles a pair of CTAs, long windows, every number of sorting passes, element
offsets past 2^31.  References are binary64 on the GPU (its products and sums
are torch's); bounds are those of test_gpu_train.py."""
import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
ROUND = {BF: 2.0 ** -8, F32: U}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rand(seed, *shape, dtype=BF):
    return torch.randn(*shape, generator=_gen(seed), device=DEV).to(dtype)


def _within(got, ref, tol, what):
    d = (got.double() - ref).abs()
    assert bool((d <= tol).all()), f"{what}: {int((d > tol).sum())} outside, worst {float((d / tol).nan_to_num(nan=9e9).max()):.3g} of the bound"


# ---------------------------------------------------------------------------
# weight gradient: 340 tiles for 76 pairs of CTAs, three chains each
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,M,N", [(2100, 5000, 4104), (2100, 4999, 4101)])
def test_wgrad_of_many_tiles(T, M, N, dtype, out, accumulate):
    x, dy = _rand(1, T, N), _rand(2, T, M, dtype=dtype)
    p = iso.act_pack(x)
    xh, d = iso.act_unpack(p, dtype=F32).double(), dy.double()
    ref, mag = d.t() @ xh, d.abs().t() @ xh.abs()
    base = _rand(3, M, N, dtype=out)
    if accumulate:
        got = iso.act_wgrad(dy, p, out=base.clone(), accumulate=True)
        ref = ref + base.double()
    else:
        got = iso.act_wgrad(dy, p, dtype=out)
    eps = 4 * U * (8 + np.sqrt(T))
    _within(got, ref, eps * mag + ROUND[out] * (1 + 2 * U) * (ref.abs() + eps * mag) + U * ref.abs() + 2.0 ** -126, "wgrad")
    again = iso.act_wgrad(dy, p, out=base.clone(), accumulate=True) if accumulate else iso.act_wgrad(dy, p, dtype=out)
    assert torch.equal(got, again)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("T,M", [(5, 40), (40, 300), (700, 129)])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 6, 7, 8, 31, 33, 127, 130, 254, 255, 257, 1022])
def test_wgrad_writes_its_columns_alone(N, T, M, out):
    """G as a range of columns of a wider buffer, its rows on 16-byte boundaries
    or off them."""
    x, dy = _rand(14, T, N), _rand(15, T, M)
    p = iso.act_pack(x)
    want = iso.act_wgrad(dy, p, dtype=out)
    xh = iso.act_unpack(p, dtype=F32).double()
    ref, mag = dy.double().t() @ xh, dy.double().abs().t() @ xh.abs()
    eps = 4 * U * (8 + np.sqrt(T))
    _within(want, ref, eps * mag + ROUND[out] * (1 + 2 * U) * (ref.abs() + eps * mag) + U * ref.abs() + 2.0 ** -126, "wgrad")
    for ld, at in (((N + 15) // 8 * 8, 8), ((N + 15) // 8 * 8, 3), (N + 9, 8)):
        buf = torch.full(((M + 1) * ld + 16,), -3.0, dtype=out, device=DEV)
        view = torch.as_strided(buf, (M, N), (ld, 1), at)
        iso.act_wgrad(dy, p, out=view)
        assert torch.equal(view, want)
        view.fill_(-3.0)
        assert bool((buf == -3.0).all()), (ld, at)


# ---------------------------------------------------------------------------
# embedding gradient
# ---------------------------------------------------------------------------
def _check_embed_grad(dy, ids, V, pad, out, scale, what):
    keep = ids != pad
    k, rows = ids[keep].long(), dy[keep].double()
    ref = torch.zeros(V, dy.shape[1], dtype=torch.float64, device=DEV).index_add_(0, k, rows * scale)
    mag = torch.zeros_like(ref).index_add_(0, k, (rows * scale).abs())
    n_v = torch.bincount(k, minlength=V)[:, None]
    err = (n_v + 4) * U * mag
    dy = torch.where(keep[:, None], dy, torch.full_like(dy, float("nan")))     # what padding stands on is not read
    if dy.shape[1] % 8:
        assert dy.is_contiguous()
    got = iso.embed_grad(dy, ids, V, scale=scale, pad_id=pad, dtype=out)
    _within(got, ref, err + ROUND[out] * (1 + 2 * U) * (ref.abs() + err), what)
    base = _rand(9, V, dy.shape[1], dtype=out)
    added = iso.embed_grad(dy, ids, out=base.clone(), scale=scale, pad_id=pad, accumulate=True)
    tot = ref + base.double()
    _within(added, tot, err + ROUND[out] * (1 + 2 * U) * (tot.abs() + err) + U * tot.abs(), what + ", added")
    none = (n_v == 0).squeeze(1)
    assert torch.equal(added[none], base[none])


def _runs(T, V, lengths):
    """Ids in runs of the given lengths in turn, their tokens shuffled."""
    ids = torch.repeat_interleave(torch.arange(V), torch.tensor([lengths[i % len(lengths)] for i in range(V)]))[:T]
    assert len(ids) == T
    return ids[torch.randperm(T, generator=torch.Generator().manual_seed(5))].to(DEV)


@pytest.mark.parametrize("dtype,out", [(BF, F32), (F32, BF)])
@pytest.mark.parametrize("T,C,lengths", [
    (20000, 2056, [1, 31, 32, 33, 63, 64, 65, 200]),      # windows of 64; runs that end at, before and after items 32 and 64
    (20000, 2055, [1, 31, 32, 33, 63, 64, 65, 200]),      # the same by rows off 16-byte boundaries
    (24000, 4104, [3, 250, 256, 600, 1, 128, 129]),       # windows of 128
    (32768, 7000, [7]), (32768, 7000, [255, 1, 257]),     # windows of 256
])
def test_embed_grad_of_long_windows(T, C, lengths, dtype, out):
    V = 0
    while sum(lengths[i % len(lengths)] for i in range(V)) < T:
        V += 1
    ids = _runs(T, V, lengths)
    _check_embed_grad(_rand(6, T, C, dtype=dtype), ids, V, 2, out, 1.5, "long windows")


# rows: 2^18 takes three passes, 2^27 four; a short list takes one CTA (beside it the zeros, or, above 32 MB of
# them, a kernel after it), a longer one the cluster
@pytest.mark.parametrize("i64", [False, True])
@pytest.mark.parametrize("T", [33, 256, 257, 1500, 2048, 2049, 9000])
@pytest.mark.parametrize("V,C", [(300000, 40), (300000, 24), ((1 << 27) + 5, 1), (511, 64), (512, 64)])
def test_embed_grad_of_every_number_of_passes(V, C, T, i64):
    g = _gen(T)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    ids[::3] = torch.randint(V - 20, V, (len(ids[::3]),), generator=g, device=DEV)      # repeated and high
    ids[::5] = V - 7                                                                    # padding
    ids = ids if i64 else ids.int()
    dy = _rand(7, T, C)
    if V < 1 << 20:
        _check_embed_grad(dy, ids, V, V - 7, F32, 0.5, "passes")
        return
    got = iso.embed_grad(dy, ids, V, scale=0.5, pad_id=V - 7, dtype=BF)
    u, inv = torch.unique(ids.long(), return_inverse=True)
    ref = torch.zeros(len(u), C, dtype=torch.float64, device=DEV).index_add_(0, inv, dy.double() * 0.5)
    mag = torch.zeros_like(ref).index_add_(0, inv, (dy.double() * 0.5).abs())
    ref[u == V - 7] = 0
    err = (torch.bincount(inv)[:, None] + 4) * U * mag
    _within(got[u], ref, err + ROUND[BF] * (1 + 2 * U) * (ref.abs() + err), "passes")
    assert int((got != 0).sum()) == int((got[u] != 0).sum())


# ---------------------------------------------------------------------------
# rows whose offsets pass 2^31 elements
# ---------------------------------------------------------------------------
def test_offsets_past_32_bits():
    rows, ld = 20, 120_000_000                       # row 19 starts 2.3e9 elements in
    wide = torch.empty(rows * ld, dtype=BF, device=DEV)

    def far(cols, at):
        return torch.as_strided(wide, (rows, cols), (ld, 1), at)
    x, dy = _rand(11, rows, 320), _rand(12, rows, 264)
    far(320, 0).copy_(x)
    far(264, 320).copy_(dy)
    fx, fdy, out = far(320, 0), far(264, 320), far(320, 1024)
    p = iso.act_pack(x)
    q = iso.act_pack(fx)
    assert torch.equal(p.codes, q.codes) and torch.equal(p.exps, q.exps)
    assert torch.equal(iso.act_unpack(p, out=out), iso.act_unpack(p))
    for n in (4, rows):                              # few tokens, and the tensor cores reading in place
        assert torch.equal(iso.act_wgrad(fdy[-n:], p.rows(rows - n, rows)), iso.act_wgrad(dy[-n:], p.rows(rows - n, rows)))
    pt = iso.act_pack(dy[:, :40].contiguous())
    assert torch.equal(iso.act_wgrad(x[:, :rows].contiguous(), pt, out=far(40, 2048)),
                       iso.act_wgrad(x[:, :rows].contiguous(), pt, dtype=BF))
    h, a, b = iso.swiglu_pack(fx, out, out=far(320, 4096))
    h2, a2, b2 = iso.swiglu_pack(x, iso.act_unpack(p))
    assert torch.equal(h, h2) and torch.equal(a.codes, a2.codes) and torch.equal(b.codes, b2.codes)
    got = iso.swiglu_grad(fx, a, b, out=(far(320, 8192), far(320, 8512), far(320, 8832)))
    assert all(torch.equal(u, v) for u, v in zip(got, iso.swiglu_grad(x, a, b)))
    ids = torch.tensor([19, 0, 7, 19, 18] * 10, device=DEV)
    assert torch.equal(iso.embed(fx, ids), iso.embed(x, ids))
    dv = _rand(13, 50, 320)
    for n in (10, 50):                               # one kernel, and the sort and the rest
        want = iso.embed_grad(dv[:n], ids[:n], rows, dtype=BF)
        assert torch.equal(iso.embed_grad(dv[:n], ids[:n], out=far(320, 16384)), want)
        base = far(320, 0).clone()
        assert torch.equal(iso.embed_grad(dv[:n], ids[:n], out=far(320, 0), accumulate=True),
                           iso.embed_grad(dv[:n], ids[:n], out=base, accumulate=True))
        far(320, 0).copy_(x)
