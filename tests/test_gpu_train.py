"""GPU parity of the training-step operators (8-bit activation checkpoints,
the weight and SwiGLU gradients from them, the embedding and its gradient)
against oracle/train_step.py in binary64.

Bounds, from the arithmetic:
* checkpoints: codes, exponents and decoded values are exact;
* weight gradient: exact products, binary32 sums of T terms: within
  eps_T sum |dy| |x_hat|, eps_T = 4 * 2^-24 (8 + sqrt T), and one rounding to
  the output's type (the accumulated value's included);
* SwiGLU: exp within 2 ulp (bfloat16 outputs: the fast exponential, whose
  error grows by 1.2 ulp per unit of |g|) and a dozen binary32 roundings of
  terms of size M = |u s g| or |dh u s| (1 + |g|), and one rounding;
* embedding: scale * value is one binary32 rounding (none for scale 1) and one
  to the output's type;
* embedding gradient: binary32 sums of n_v rows: (n_v + 4) 2^-24 |scale| sum |dy|,
  and one rounding.
"""
import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from oracle import train_step as R
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: U}   # half an ulp, relative
TINY = 2.0 ** -126
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _act(seed, T, C, dtype, ld=None, off=0):
    """Activations with outlier channels, as rows of a wider buffer."""
    g = _gen(seed)
    x = torch.randn(T, C, generator=g) * torch.exp(torch.randn(T, 1, generator=g))
    x[:, ::37] *= 30
    buf = torch.full((max(T, 1) * (ld or C) + off + 8,), 7.0, dtype=dtype, device=DEV)
    view = torch.as_strided(buf, (T, C), (ld or C, 1), off)
    view.copy_(x.to(dtype))
    return view


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, tol, what):
    got, ref = _np(got), np.asarray(ref)
    assert got.shape == ref.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    ok = np.isnan(ref) | (np.abs(got - ref) <= tol)
    assert ok.all(), f"{what}: {int((~ok).sum())} of {ok.size} outside, worst {np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-300)):.3g} of the bound"


LAYOUTS = [(1, 1, None, 0), (1, 33, None, 0), (3, 31, 31, 0), (5, 64, 64, 0), (17, 200, 203, 1), (4, 1536, 1536, 0),
           (33, 257, 264, 8), (130, 1000, 1024, 0), (2, 8960, 8960, 4)]


# ---------------------------------------------------------------------------
# checkpoints
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,C,ld,off", LAYOUTS)
def test_pack_and_unpack_are_exact(T, C, ld, off, dtype):
    x = _act(11, T, C, dtype, ld, off)
    p = iso.act_pack(x)
    codes, exps = R.act_encode(_np(x))
    assert np.array_equal(p.codes.cpu().numpy(), codes)
    G = exps.shape[1]
    assert np.array_equal(p.exps.cpu().numpy()[:, :G], exps) and (p.exps[:, G:] == 1).all()
    ref = R.act_decode(codes, exps, C)
    for out_dtype in (BF, F32):
        assert np.array_equal(_np(iso.act_unpack(p, dtype=out_dtype)), ref)
    # into a strided, unaligned view: nothing outside it is written
    buf = torch.full((T, C + 5), -3.0, dtype=dtype, device=DEV)
    iso.act_unpack(p, out=buf[:, 2:2 + C])
    assert np.array_equal(_np(buf[:, 2:2 + C]), ref)
    assert (buf[:, :2] == -3).all() and (buf[:, 2 + C:] == -3).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pack_edges_of_the_format(dtype):
    big = torch.finfo(dtype).max
    tiny = 2.0 ** -133 if dtype == BF else 2.0 ** -149       # the least subnormal
    rows = [[0.0] * 32, [-0.0] * 32, [127.0] + [0.5, 1.5, 2.5, -0.5, -1.5] + [0.0] * 26,
            [127.0 * 2 ** -20, 2.0 ** -21] + [1e-8] * 30, [big, -big] + [1.0] * 30, [tiny] * 32,
            [127.0 * 2.0 ** -126, 2.0 ** -126, 2.0 ** -127, 3 * 2.0 ** -127] + [0.0] * 28,
            [float("nan")] + [1.0] * 31, [float("inf")] + [1.0] * 31, [1.0] * 31 + [float("-inf")],
            [128.0] + [64.0, 1.0] * 15 + [3.0]]
    x = torch.tensor(rows, dtype=dtype, device=DEV)
    p = iso.act_pack(x)
    codes, exps = R.act_encode(_np(x))
    assert np.array_equal(p.codes.cpu().numpy(), codes) and np.array_equal(p.exps.cpu().numpy()[:, :1], exps)
    out = _np(iso.act_unpack(p))
    assert np.array_equal(out, R.act_decode(codes, exps, 32), equal_nan=True)


def test_pack_rows_are_a_checkpoint():
    x = _act(12, 50, 130, BF)
    p = iso.act_pack(x)
    assert p.shape == (50, 130) and p.nbytes == 50 * (160 + 8)
    part = iso.act_unpack(p.rows(7, 31))
    assert torch.equal(part, iso.act_unpack(p)[7:31])
    dy = _act(13, 24, 40, BF)
    assert torch.equal(iso.act_wgrad(dy, p.rows(7, 31)), iso.act_wgrad(dy, iso.act_pack(x[7:31])))


# ---------------------------------------------------------------------------
# weight gradient
# ---------------------------------------------------------------------------
def _check_wgrad(dy, x, out_dtype, base=None, what=""):
    T = dy.shape[0]
    p = iso.act_pack(x)
    out = None if base is None else base.clone()
    got = iso.act_wgrad(dy, p, out=out, dtype=out_dtype, accumulate=base is not None)
    xv, d = torch.from_numpy(R.act_values(_np(x))), torch.from_numpy(_np(dy))
    ref = (d.t() @ xv).numpy()
    mag = (d.abs().t() @ xv.abs()).numpy()
    if base is not None:
        ref = ref + _np(base)
    eps = 4 * U * (8 + np.sqrt(T))
    _close(got, ref, eps * mag + ROUND[out_dtype] * (1 + 2 * U) * (np.abs(ref) + eps * mag) + U * np.abs(ref) + TINY,
           f"wgrad {what}")
    return got


@pytest.mark.parametrize("dtype,out", [(BF, F32), (BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("T,M,N,gap", [(1, 8, 32, 0), (1, 1, 1, 0), (2, 129, 257, 0), (63, 64, 96, 0), (64, 128, 256, 0),
                                       (65, 130, 100, 0), (333, 1120, 451, 3), (1000, 200, 72, 8), (257, 63, 33, 1),
                                       (2049, 300, 290, 0)])
def test_wgrad_matches_binary64(T, M, N, gap, dtype, out):
    x = _act(21, T, N, dtype, N + gap)
    dy = _act(22, T, M + gap, dtype)[:, :M] * 0.01 if gap == 0 else _act(22, T, M + gap, dtype)[:, :M]
    _check_wgrad(dy, x, out, what=f"{T}x{M}x{N}")


@pytest.mark.parametrize("T,M,N", [(8192, 256, 128), (5000, 1536, 256), (300, 2304, 1800), (129, 4000, 96)])
def test_wgrad_longer(T, M, N):
    _check_wgrad(_act(23, T, M, BF), _act(24, T, N, BF), F32, what="longer")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_wgrad_accumulates_into_a_strided_out(dtype):
    x, dy = _act(25, 200, 150, BF), _act(26, 200, 140, BF)
    buf = torch.randn(140, 163, generator=_gen(27)).to(DEV, dtype)
    keep = buf.clone()
    out = buf[:, 5:155]
    p = iso.act_pack(x)
    iso.act_wgrad(dy, p, out=out, accumulate=True)
    fresh = _check_wgrad(dy, x, dtype, base=keep[:, 5:155].contiguous())
    assert torch.equal(out, fresh)
    assert torch.equal(buf[:, :5], keep[:, :5]) and torch.equal(buf[:, 155:], keep[:, 155:])


def test_wgrad_same_bits_again_and_over_slices():
    x, dy = _act(28, 3000, 500, BF), _act(29, 3000, 700, BF)
    p = iso.act_pack(x)
    a = iso.act_wgrad(dy, p)
    for _ in range(3):
        assert torch.equal(a, iso.act_wgrad(dy, p))
    # micro-batches: rows [0, 1000) and [1000, 3000) of one checkpoint
    g = iso.act_wgrad(dy[:1000], p.rows(0, 1000))
    iso.act_wgrad(dy[1000:], p.rows(1000, 3000), out=g, accumulate=True)
    xv, d = torch.from_numpy(R.act_values(_np(x))), torch.from_numpy(_np(dy))
    tol = 8 * U * (8 + np.sqrt(3000)) * (d.abs().t() @ xv.abs()).numpy()
    _close(g, (d.t() @ xv).numpy(), tol, "micro-batches")


def test_wgrad_without_tokens():
    dy, x = torch.empty(0, 40, dtype=BF, device=DEV), torch.empty(0, 64, dtype=BF, device=DEV)
    out = torch.full((40, 64), 5.0, device=DEV)
    p = iso.act_pack(x)
    assert torch.equal(iso.act_wgrad(dy, p, out=out.clone(), accumulate=True), out)
    assert not iso.act_wgrad(dy, p, out=out.clone()).any()
    assert iso.act_wgrad(torch.empty(5, 0, dtype=BF, device=DEV), iso.act_pack(torch.ones(5, 64, device=DEV))).shape == (0, 64)


def test_wgrad_non_finite():
    x, dy = _act(30, 70, 96, BF), _act(31, 70, 50, BF)
    x[3, 40] = float("inf")          # its group of the checkpoint is NaN: columns 32 .. 63 of G
    dy[5, 7] = float("nan")          # row 7 of G
    dy[6, 9] = float("inf")          # row 9: Inf or NaN
    g = _np(iso.act_wgrad(dy, iso.act_pack(x)))
    bad = ~np.isfinite(g)
    want = np.zeros_like(bad)
    want[:, 32:64] = True
    want[[7, 9]] = True
    assert np.array_equal(bad, want)
    f = _np(iso.act_wgrad(dy.float(), iso.act_pack(x)))
    assert np.array_equal(~np.isfinite(f), want)
    inf_row = np.isinf(g[9]) & ~np.isnan(g[9])
    assert np.array_equal(np.isinf(f[9]), inf_row) and inf_row.any()


# ---------------------------------------------------------------------------
# SwiGLU
# ---------------------------------------------------------------------------
def _exp_err(g, dtype):
    return (16 + (2.5 * np.abs(g) if dtype == BF else 0)) * U


def _check_swiglu(gate, up, dh):
    dtype = gate.dtype
    h, gp, up_p = iso.swiglu_pack(gate, up)
    assert torch.equal(gp.codes, iso.act_pack(gate).codes) and torch.equal(up_p.exps, iso.act_pack(up).exps)
    g, u, d = _np(gate), _np(up), _np(dh)

    def tol(ref, M, g):
        return ROUND[dtype] * np.abs(ref) + (1 + ROUND[dtype]) * _exp_err(g, dtype) * M + TINY * (1 + np.abs(u)) * (1 + np.abs(g)) * 2

    ref = R.swiglu(g, u)
    _close(h, ref, tol(ref, np.abs(ref), g), "h")
    dg, du, hh = iso.swiglu_grad(dh, gp, up_p)
    g, u = R.act_values(g), R.act_values(u)
    rg, ru = R.swiglu_grad(d, g, u)
    s = R.sigmoid(g)
    _close(hh, R.swiglu(g, u), tol(R.swiglu(g, u), np.abs(R.swiglu(g, u)), g), "h again")
    _close(du, ru, tol(ru, np.abs(ru), g), "d_up")
    _close(dg, rg, tol(rg, np.abs(d * u * s) * (1 + np.abs(g)), g), "d_gate")
    two = iso.swiglu_grad(dh, gp, up_p, need_h=False)
    assert two[2] is None and torch.equal(two[0], dg) and torch.equal(two[1], du)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,C,ld,off", LAYOUTS)
def test_swiglu_matches_binary64(T, C, ld, off, dtype):
    _check_swiglu(_act(41, T, C, dtype, ld, off), _act(42, T, C, dtype, ld, off), _act(43, T, C, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_swiglu_wide_range(dtype):
    g = torch.linspace(-120, 120, 4096).reshape(16, 256).to(DEV, dtype)
    u = torch.randn(16, 256, generator=_gen(44)).to(DEV, dtype)
    _check_swiglu(g, u, torch.ones_like(u))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("C", [96, 333])
def test_swiglu_halves_of_one_buffer(C, dtype):
    both = _act(45, 37, 2 * C, dtype)
    dh = _act(46, 37, C, dtype)
    h, gp, up_p = iso.swiglu_pack(both[:, :C], both[:, C:])
    h2, gp2, up2 = iso.swiglu_pack(both[:, :C].contiguous(), both[:, C:].contiguous())
    assert torch.equal(h, h2) and torch.equal(gp.codes, gp2.codes) and torch.equal(up_p.codes, up2.codes)
    d_both = torch.empty(37, 2 * C, dtype=dtype, device=DEV)
    iso.swiglu_grad(dh, gp, up_p, out=(d_both[:, :C], d_both[:, C:]), need_h=False)
    dg, du, _ = iso.swiglu_grad(dh, gp2, up2)
    assert torch.equal(d_both, torch.cat([dg, du], 1))


def test_swiglu_non_finite_stays_in_its_group():
    g, u = _act(47, 4, 96, F32), _act(48, 4, 96, F32)
    g[1, 40], u[2, 5] = float("nan"), float("inf")
    h, gp, up_p = iso.swiglu_pack(g, u)
    assert torch.isnan(h).sum() == 1 and (~torch.isfinite(h)).sum() == 2
    dg, du, hh = iso.swiglu_grad(torch.ones_like(g), gp, up_p)
    want = torch.zeros(4, 96, dtype=torch.bool, device=DEV)
    want[1, 32:64] = True
    assert torch.equal(~torch.isfinite(du), want)
    want[2, :32] = True
    assert torch.equal(~torch.isfinite(dg), want) and torch.equal(~torch.isfinite(hh), want)


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def _ids(seed, T, V, i64, pad):
    u = torch.rand(T, generator=_gen(seed), dtype=torch.float64)
    ids = ((V + 1.0) ** u - 1).long().clamp(0, V - 1)
    ids = torch.randperm(V, generator=_gen(seed + 1))[ids]
    if pad is not None and T:
        ids[::7] = pad
    return ids.to(DEV, torch.int64 if i64 else torch.int32)


CASES = [(0, 10, 8), (1, 1, 1), (1, 500, 256), (31, 7, 40), (32, 1000, 33), (33, 3, 264), (100, 50000, 96), (1000, 513, 130),
         (4097, 300, 72), (9000, 20000, 24)]


@pytest.mark.parametrize("i64", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("T,V,C", CASES)
def test_embed_matches(T, V, C, dtype, out, i64):
    table = _act(51, V, C, dtype, C + (3 if C % 2 else 0))
    pad = V - 1 if V > 1 else None
    ids = _ids(52, T, V, i64, pad)
    for scale in (1.0, 11.3):
        got, st = iso.embed(table, ids, scale=scale, pad_id=pad, dtype=out, status=True)
        ref = R.embed(_np(table), ids.cpu().numpy(), float(np.float32(scale)), -1 if pad is None else pad)
        # table rows of the type's own values: scale 1 is exact unless rounded down to bfloat16
        tol = 0.0 if scale == 1.0 and out in (dtype, F32) else (ROUND[out] * (1 + 2 * U) + U) * np.abs(ref)
        _close(got, ref, tol, "embed")
        assert int(st) == 0


@pytest.mark.parametrize("i64", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("T,V,C", CASES)
def test_embed_grad_matches(T, V, C, dtype, out, i64):
    dy = _act(53, T, C, dtype, C + (3 if C % 2 else 0))
    pad = V - 1 if V > 1 else None
    ids = _ids(54, T, V, i64, pad)
    scale = 7.25
    n_v = np.bincount(ids.cpu().numpy(), minlength=V)[:V, None]
    ref = R.embed_grad(_np(dy), ids.cpu().numpy(), V, scale, -1 if pad is None else pad)
    mag = R.embed_grad(np.abs(_np(dy)), ids.cpu().numpy(), V, scale, -1 if pad is None else pad)
    err = (n_v + 4) * U * mag
    got, st = iso.embed_grad(dy, ids, V, scale=scale, pad_id=pad, dtype=out, status=True)
    _close(got, ref, err + ROUND[out] * (1 + 2 * U) * (np.abs(ref) + err), "embed_grad")
    assert int(st) == 0
    assert torch.equal(got, iso.embed_grad(dy, ids, V, scale=scale, pad_id=pad, dtype=out))
    # added to a strided gradient; rows without tokens and the gap keep their bits
    buf = torch.randn(V, C + 3, generator=_gen(55)).to(DEV, out)
    keep = buf.clone()
    iso.embed_grad(dy, ids, out=buf[:, 1:1 + C], scale=scale, pad_id=pad, accumulate=True)
    base = _np(keep[:, 1:1 + C])
    _close(buf[:, 1:1 + C], base + ref, err + ROUND[out] * (1 + 2 * U) * (np.abs(base + ref) + err) + U * np.abs(base + ref), "added")
    none = torch.from_numpy((mag.sum(1) == 0)).to(DEV)
    assert torch.equal(buf[none], keep[none])
    assert torch.equal(buf[:, :1], keep[:, :1]) and torch.equal(buf[:, 1 + C:], keep[:, 1 + C:])
    # written over a strided gradient
    iso.embed_grad(dy, ids, out=buf[:, 1:1 + C], scale=scale, pad_id=pad)
    assert torch.equal(buf[:, 1:1 + C], got)
    assert torch.equal(buf[:, :1], keep[:, :1]) and torch.equal(buf[:, 1 + C:], keep[:, 1 + C:])


@pytest.mark.parametrize("T", [64, 1000, 20000])
def test_embed_grad_one_frequent_token(T):
    dy = _act(56, T, 200, BF)
    ids = torch.full((T,), 3, dtype=torch.int64, device=DEV)
    got = iso.embed_grad(dy, ids, 9)
    ref, mag = _np(dy).sum(0), np.abs(_np(dy)).sum(0)
    # windows of 32, then their sums: a chain of 32 and one of T / 32
    _close(got[3], ref, (32 + T / 32 + 4) * U * mag, "frequent token")
    assert not got[:3].any() and not got[4:].any()
    # runs that start and end at window edges and inside them
    ids = (torch.arange(T, device=DEV) // 48).clamp(max=8)
    got = iso.embed_grad(dy, ids, 9)
    for v in range(9):
        rows = _np(dy)[(ids == v).cpu().numpy()]
        _close(got[v], rows.sum(0), (len(rows) + 4) * U * np.abs(rows).sum(0), f"run {v}")


def test_embed_ids_outside_the_table():
    table, dy = _act(57, 20, 64, F32), _act(58, 5, 64, F32)
    ids = torch.tensor([3, 20, -1, 7, -5], device=DEV)
    out, st = iso.embed(table, ids, status=True)
    assert int(st) == _abi.ISO_ERR_INDEX
    assert torch.equal(out[0], table[3]) and torch.equal(out[3], table[7]) and not out[[1, 2, 4]].any()
    g, st = iso.embed_grad(dy, ids, 20, status=True)
    assert int(st) == _abi.ISO_ERR_INDEX
    assert torch.equal(g[3], dy[0]) and torch.equal(g[7], dy[3]) and int((g != 0).any(1).sum()) == 2
    ids = torch.tensor([3, -1, -1, 7, 3], device=DEV)        # -1 is padding unless pad_id says otherwise
    _, st = iso.embed(table, ids, status=True)
    assert int(st) == 0
    g, st = iso.embed_grad(dy, ids, 20, status=True)
    assert int(st) == 0 and torch.equal(g[3], dy[0] + dy[4])
    _, st = iso.embed(table, ids, pad_id=19, status=True)
    assert int(st) == _abi.ISO_ERR_INDEX
    # only padding, and an empty table
    g = iso.embed_grad(dy, torch.full((5,), 2, device=DEV), 20, pad_id=2)
    assert not g.any()
    _, st = iso.embed(torch.empty(0, 64, device=DEV), ids, status=True)
    assert int(st) == _abi.ISO_ERR_INDEX


def test_gradients_are_adjoint_on_the_gpu():
    """<embed(E), dY> = <E, embed_grad(dY)>, and the weight gradient against
    differences of the layer's output."""
    E, dy = _act(61, 40, 96, F32), _act(62, 300, 96, F32)
    ids = _ids(63, 300, 40, True, None)
    a = (_np(iso.embed(E, ids, scale=3.0)) * _np(dy)).sum()
    b = (_np(E) * _np(iso.embed_grad(dy, ids, 40, scale=3.0))).sum()
    mag = 3 * (np.abs(_np(E))[ids.cpu().numpy()] * np.abs(_np(dy))).sum()
    assert abs(a - b) <= 320 * U * mag
    x, d = _act(64, 90, 70, F32), _act(65, 90, 50, F32)
    p = iso.act_pack(x)
    G, xh = _np(iso.act_wgrad(d, p)), _np(iso.act_unpack(p))
    D = np.random.default_rng(66).normal(size=(50, 70))
    lhs, rhs = (G * D).sum(), (_np(d) * (xh @ D.T)).sum()       # the derivative along D
    assert abs(lhs - rhs) <= 4 * U * (8 + np.sqrt(90)) * (np.abs(_np(d)).T @ np.abs(xh) * np.abs(D)).sum()


# ---------------------------------------------------------------------------
# streams, graphs, refusals
# ---------------------------------------------------------------------------
def test_another_stream_and_capture():
    x, dy = _act(71, 512, 640, BF), _act(72, 512, 384, BF)
    ids = _ids(73, 512, 1000, True, None)
    want = (iso.act_wgrad(dy, iso.act_pack(x)), iso.embed_grad(dy, ids, 1000))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p = iso.act_pack(x, stream=s)
    got = (iso.act_wgrad(dy, p, stream=s), iso.embed_grad(dy, ids, 1000, stream=s))
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws, out, grad = iso.Workspace(DEV), torch.empty_like(want[0]), torch.empty_like(want[1])
    pack = iso.act_pack(x)
    ws.get(max(iso.act_wgrad_workspace_size(dy, pack, out), iso.embed_grad_workspace_size(512, 384)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        iso.act_pack(x, out=pack)
        iso.act_wgrad(dy, pack, out=out, workspace=ws)
        iso.embed_grad(dy, ids, out=grad, workspace=ws)
    x.copy_(_act(74, 512, 640, BF))
    out.zero_()
    grad.fill_(9.0)
    g.replay()
    assert torch.equal(grad, want[1])
    assert torch.equal(out, iso.act_wgrad(dy, iso.act_pack(x)))


def test_both_forms_of_a_call_agree():
    """A call that allocates its outputs and one that is given them."""
    def new(*shape, dtype=BF):
        return torch.empty(*shape, dtype=dtype, device=DEV)
    x, y, dy = _act(75, 40, 136, BF), _act(76, 40, 136, BF), _act(77, 40, 56, BF)
    ids, table = _ids(78, 40, 90, False, 89), _act(79, 90, 136, BF)
    p, q = iso.act_pack(x), iso.act_pack(x, out=iso.ActPack.empty(40, 136))
    assert torch.equal(p.codes, q.codes) and torch.equal(p.exps[:, :5], q.exps[:, :5]) and p.shape == q.shape == (40, 136)
    assert torch.equal(iso.act_unpack(p), iso.act_unpack(q, out=new(40, 136)))
    assert torch.equal(iso.act_wgrad(dy, p, dtype=BF), iso.act_wgrad(dy, q, out=new(56, 136)))
    h, a, b = iso.swiglu_pack(x, y)
    h2, a2, b2 = iso.swiglu_pack(x, y, out=new(40, 136), packs=(iso.ActPack.empty(40, 136), iso.ActPack.empty(40, 136)))
    assert torch.equal(h, h2) and torch.equal(a.codes, a2.codes) and torch.equal(b.codes, b2.codes)
    for u, v in zip(iso.swiglu_grad(x, a, b), iso.swiglu_grad(x, a2, b2, out=[new(40, 136) for _ in range(3)])):
        assert torch.equal(u, v)
    assert torch.equal(iso.embed(table, ids, 2.0, 89), iso.embed(table, ids, 2.0, 89, out=new(40, 136)))
    assert torch.equal(iso.embed_grad(x, ids, 90, 2.0, 89),
                       iso.embed_grad(x, ids, scale=2.0, pad_id=89, out=new(90, 136, dtype=F32)))


def test_refusals():
    x, dy = _act(81, 8, 64, BF), _act(82, 8, 32, BF)
    p = iso.act_pack(x)
    ids = torch.zeros(8, dtype=torch.int64, device=DEV)
    with pytest.raises(ValueError):
        iso.act_pack(x.t())
    with pytest.raises(ValueError):
        iso.act_pack(x.cpu())
    with pytest.raises(TypeError):
        iso.act_pack(x.half())
    with pytest.raises(ValueError):
        iso.act_pack(x[0])
    with pytest.raises(ValueError):
        iso.act_pack(x[:1].expand(8, 64))
    with pytest.raises(iso.IsoError) as e:
        iso.act_pack(x, out=iso.ActPack.empty(8, 96))
    assert e.value.code == _abi.ISO_ERR_SHAPE
    with pytest.raises(iso.IsoError) as e:
        iso.act_wgrad(dy[:7], p)
    assert e.value.code == _abi.ISO_ERR_SHAPE
    with pytest.raises(ValueError):
        iso.act_wgrad(dy, p, accumulate=True)
    with pytest.raises(TypeError):
        iso.act_wgrad(dy, p, dtype=torch.float16)
    buf = torch.zeros(32, 96, dtype=BF, device=DEV)
    with pytest.raises(iso.IsoError) as e:                      # the gradient over its own input
        iso.act_wgrad(buf[:8, :32], p, out=buf[:, 31:95])
    assert e.value.code == _abi.ISO_ERR_ARG
    with pytest.raises(iso.IsoError) as e:
        iso.swiglu_pack(x, _act(83, 8, 64, F32))
    assert e.value.code == _abi.ISO_ERR_DTYPE
    with pytest.raises(iso.IsoError) as e:
        iso.swiglu_pack(x, x.clone(), out=x)
    assert e.value.code == _abi.ISO_ERR_ARG
    with pytest.raises(iso.IsoError) as e:
        iso.swiglu_grad(dy, p, p)
    assert e.value.code == _abi.ISO_ERR_SHAPE
    with pytest.raises(TypeError):
        iso.embed(x, ids.float())
    with pytest.raises(ValueError):
        iso.embed(x, ids, scale=float("nan"))
    with pytest.raises(ValueError):
        iso.embed_grad(dy, ids[:5], 4)
    with pytest.raises(ValueError):
        iso.embed_grad(dy, ids)
    with pytest.raises(iso.IsoError) as e:
        iso.embed(x, ids, out=torch.empty(8, 63, dtype=BF, device=DEV))
    assert e.value.code == _abi.ISO_ERR_SHAPE
    with pytest.raises(iso.IsoError) as e:
        iso.embed_grad(dy, ids, out=dy)
    assert e.value.code == _abi.ISO_ERR_ARG
