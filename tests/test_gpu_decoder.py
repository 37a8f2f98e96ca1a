"""GPU parity of rotary positions, attention with its gradient and distillation
with its gradient against oracle/decoder_step.py in binary64.

Bounds, from the arithmetic (U = 2^-24, E = eps / 2 of the outputs' type: 2^-8
for bfloat16, U for float32):
* rotary: the angle as a binary32 number of half turns is off by at most U pi,
  its sine and cosine by 2 ulp more, products and the sum by three roundings:
  10 U (|u| + |w|), and E of the value;
* attention: a score is a sum of D products, off by at most c = (D + 8) U scale
  sum |q||k| (twice that on the tensor cores, whose additions cut bits off
  instead of rounding); a weight by its score, the roundings of score and maximum
  and the exponential, (3 |S| + 3 |lse| + 8) U, and the rescalings, 3 U a tile of
  64 keys; bfloat16 on the tensor cores: 2^-8 more for the weight's rounding.
  With r_ij the sum of these, out is off by sum_j P_ij (|v_j| + |out_i|) (r_ij +
  (m + 8) U) and E of the value, lse by the largest r_ij without the weight's
  rounding, (m + 8) U and U |lse|;
* its gradients, from the out and lse that the call is given: dS_ij by P_ij
  (r_ij |dP - delta| + (D + 8) U (sum |dout||v| + sum |dout||out|) + 4 U (|dP| +
  |delta|)) and 2^-8 |dS| for its rounding; then sums over n terms, (n + 8) U of
  their magnitudes (twice on the tensor cores), and E of the value;
* distillation: scores off by U (|z| / tau + |lse|), exponentials by 4 U (the
  hardware's: 2^-21), sums of V terms kept as one per thread and joined:
  (V / 128 + 32) U relative at most.
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_19331_gb300 as iso
from oracle import decoder_step as R
from paper_2607_19331_gb300 import _abi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
E = {BF: 2.0 ** -8, F32: U}
TINY = 1e-30


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    torch.cuda.set_device(0)
    _abi.lib()


def _np(t):
    return t.detach().double().cpu().numpy()


def _rand(seed, rows, cols, dtype, ld=None, off=0, scale=1.0):
    """Rows of a wider buffer, whose other entries are NaN."""
    g = torch.Generator().manual_seed(seed)
    ld = ld or cols
    buf = torch.full((rows * ld + off + 16,), math.nan, dtype=dtype, device=DEV)
    view = torch.as_strided(buf, (rows, cols), (ld, 1), off)
    view.copy_((torch.randn(rows, cols, generator=g) * scale).to(dtype))
    return view


def _close(got, ref, tol, what):
    got, ref, tol = _np(got) if isinstance(got, torch.Tensor) else got, np.asarray(ref), np.asarray(tol)
    assert got.shape == ref.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    with np.errstate(invalid="ignore"):
        ok = np.isnan(ref) | (got == ref) | (np.abs(got - ref) <= tol + TINY)
        worst = np.nanmax(np.where(ok, 0, np.abs(got - ref) / np.maximum(tol, TINY)), initial=0)
    assert ok.all(), f"{what}: {int((~ok).sum())} of {ok.size} outside, worst {worst:.3g} of the bound"


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def _rope_tol(x, D, n, neighbours, dtype):
    """|u| + |w| of each channel's pair."""
    a = np.abs(_np(x)).reshape(x.shape[0], -1, D)
    mag = np.zeros_like(a)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if neighbours else (slice(0, n), slice(n, 2 * n))
    mag[:, :, first] = mag[:, :, second] = a[:, :, first] + a[:, :, second]
    return 10 * U * mag.reshape(x.shape)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H,D,rot,sections,pairs,ld,off", [
    (1, 14, 128, 128, None, "halves", None, 0), (7, 3, 128, 128, (32, 16, 16), "halves", None, 0),
    (5, 2, 80, 80, (20, 20), "neighbours", None, 0), (33, 1, 64, 32, None, "halves", 72, 8),
    (33, 2, 64, 32, None, "neighbours", 200, 8), (4, 3, 10, 6, (1, 1, 0, 1), "halves", 31, 1),
    (4, 3, 7, 4, None, "neighbours", 22, 1), (3, 5, 6, 0, None, "halves", None, 0), (70, 40, 16, 16, None, "halves", None, 0),
    (2, 1, 300, 256, (64, 64), "halves", None, 0)])
def test_rope(T, H, D, rot, sections, pairs, ld, off, dtype):
    plan = iso.rope_plan(D, base=1e4, sections=sections, rot_dim=rot, pairs=pairs)
    x = _rand(1, T, H * D, dtype, ld, off)
    g = torch.Generator().manual_seed(2)
    p = torch.randint(-50, 200000, (plan.axes, T), generator=g)
    p[:, 0] = 0
    freq, axis = list(plan.freq)[:rot // 2], list(plan.axis)[:rot // 2]
    tol = _rope_tol(x, D, rot // 2, pairs == "neighbours", dtype)
    for inverse, call in ((False, iso.rope), (True, iso.rope_grad)):
        ref = R.rope(_np(x), p.numpy(), D, freq, axis, pairs == "neighbours", inverse)
        for pos in (p.to(DEV), p.to(DEV, torch.int32)):
            y = call(x, pos, plan)
            _close(y, ref, tol + E[dtype] * np.abs(ref), "rope")
        if plan.axes == 1:
            assert torch.equal(call(x, p.to(DEV)[0], plan), y)
        # into a strided view, and in place: the same bits, nothing beside it
        buf = torch.full((T, H * D + 5), -3.0, dtype=dtype, device=DEV)
        call(x, p.to(DEV), plan, out=buf[:, 2:2 + H * D])
        assert torch.equal(buf[:, 2:2 + H * D], y) and (buf[:, :2] == -3).all() and (buf[:, 2 + H * D:] == -3).all()
        z = _rand(1, T, H * D, dtype, ld, off)
        assert call(z, p.to(DEV), plan, out=z) is z and torch.equal(z, y)


def test_rope_far_positions():
    """Angles are as exact far out as near: positions around 2^40, where binary64
    holds the product's fraction to 2^-12 only, against exact rational turns."""
    from fractions import Fraction
    D, T = 8, 6
    turns = [Fraction(1, 3), Fraction(1, 7), Fraction(12345, 1 << 20), Fraction(1, 1 << 30)]
    freq = [float(t) * 2 * math.pi for t in turns]
    plan = iso.RopePlan(D, freq, [0] * 4, 1)
    pos = [(1 << 40) + 5, -(1 << 40) - 1, 3 << 30, 7, 0, (1 << 62) // 3]
    x = _rand(3, T, D, F32)
    y = _np(iso.rope(x, torch.tensor(pos, device=DEV), plan))
    v = _np(x)
    # 1 / (2 pi) to 60 digits for the frequency that the binary64 angle stands for
    inv = Fraction(159154943091895335768883763372514362034459645740456448747667, 10 ** 60)
    for t in range(T):
        for i in range(4):
            a = float((Fraction(freq[i]) * inv * pos[t]) % 1) * 2 * math.pi
            slack = 2 * math.pi * (2.0 ** -30 + abs(pos[t]) * 2.0 ** -63)
            u, w = v[t, i], v[t, i + 4]
            tol = (10 * U + slack) * (abs(u) + abs(w))
            assert abs(y[t, i] - (u * math.cos(a) - w * math.sin(a))) <= tol
            assert abs(y[t, i + 4] - (u * math.sin(a) + w * math.cos(a))) <= tol


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _on_tensor_cores(D, dtype, *mats):
    es = 2 if dtype == BF else 4
    return dtype == BF and D % 8 == 0 and all(m.data_ptr() % 16 == 0 and m.stride(0) * es % 16 == 0 for m in mats)


class Case:
    """Packed sequences with padding behind them; what is no query or key is NaN."""

    def __init__(self, lens, klens=None, heads=2, kv=1, D=64, causal=True, window=0, dtype=BF, pad=0, gap=0, off=0,
                 seed=0, scale=None, amp=1.0):
        self.lens, self.klens = lens, lens if klens is None else klens
        self.heads, self.kv, self.D, self.causal, self.window, self.dtype = heads, kv, D, causal, window, dtype
        T, M = sum(lens) + pad, sum(self.klens) + pad
        self.scale = D ** -0.5 if scale is None else scale
        if klens is None and not off:
            qkv = _rand(seed, T, (heads + 2 * kv) * D, dtype, (heads + 2 * kv) * D + gap, scale=amp)
            self.q, self.k, self.v = qkv.split([heads * D, kv * D, kv * D], 1)
        else:
            self.q = _rand(seed, T, heads * D, dtype, heads * D + gap, off, amp)
            self.k = _rand(seed + 1, M, kv * D, dtype, kv * D + gap, off, amp)
            self.v = _rand(seed + 2, M, kv * D, dtype, kv * D + gap, off)
        self.dout = _rand(seed + 3, T, heads * D, dtype, heads * D + gap, off)
        for t, n in ((self.q, sum(lens)), (self.k, sum(self.klens)), (self.v, sum(self.klens)), (self.dout, sum(lens))):
            t[n:] = math.nan
        packed = len(lens) > 1 or pad
        ends = lambda c: torch.tensor(np.cumsum([0] + c), dtype=torch.int32, device=DEV)      # noqa: E731
        self.args = dict(heads=heads, kv_heads=kv, scale=scale, causal=causal, window=window,
                         seqs=ends(lens) if packed else None, kv_seqs=ends(klens) if packed and klens is not None else None)
        self.tc = _on_tensor_cores(D, dtype, self.q, self.k, self.v)

    def parts(self):
        """(query head, key head, query rows, key rows, seen) of every head and sequence."""
        q0 = k0 = 0
        for n, m in zip(self.lens, self.klens):
            seen = R.sees(n, m, self.causal, self.window)
            for h in range(self.heads):
                yield h, h // (self.heads // self.kv), slice(q0, q0 + n), slice(k0, k0 + m), seen
            q0, k0 = q0 + n, k0 + m

    def head(self, t, h, rows):
        return _np(t)[rows, h * self.D:(h + 1) * self.D]

    def relative(self, q, k, lse, seen):
        """r_ij of the module's bounds, without the weight's rounding."""
        mag = self.scale * np.abs(q) @ np.abs(k).T
        S = np.abs(self.scale * q @ k.T)
        top = np.where(np.isfinite(lse), np.abs(lse), 0)[:, None]
        tiles = seen.shape[1] // 64 + 1
        return (2 if self.tc else 1) * (self.D + 8) * U * mag + (3 * S + 3 * top + 8 + 3 * tiles) * U + (2.0 ** -21 if self.tc else 0)

    def check_forward(self, out, lse, only=None):
        """``only``: the rows to look at (a mask over the queries)."""
        used = np.zeros(self.q.shape[0], bool)
        got, got_lse = _np(out), _np(lse)
        P8 = 2.0 ** -8 if self.tc else 0.0
        for h, g, rows, keys, seen in self.parts():
            used[rows] = True
            q, k, v = self.head(self.q, h, rows), self.head(self.k, g, keys), self.head(self.v, g, keys)
            ref, ref_lse, P = R.attn(q, k, v, self.scale, seen)
            r = self.relative(q, k, ref_lse, seen) * seen
            n = (2 if self.tc else 1) * (seen.shape[1] + 8) * U
            w = P * (r + P8 + n)
            tol = w @ np.abs(v) + w.sum(1, keepdims=True) * np.abs(ref) + E[self.dtype] * np.abs(ref)
            at = slice(None) if only is None else only[rows]
            _close(got[rows, h * self.D:(h + 1) * self.D][at], ref[at], tol[at], f"out of head {h}")
            top = r.max(1, initial=0) + n + 2 * U * np.where(np.isfinite(ref_lse), np.abs(ref_lse), 0)
            _close(got_lse[h, rows][at], ref_lse[at], top[at], f"lse of head {h}")
        return used

    def check_backward(self, out, lse, dq, dk, dv, only=None):
        """``only``: the rows to look at (masks over the queries and the keys)."""
        D, two = self.D, 2 if self.tc else 1
        P8 = 2.0 ** -8 if self.tc else 0.0
        refs = [np.zeros(m.shape) for m in (self.q, self.k, self.v)]
        tols = [np.zeros(m.shape) for m in (self.q, self.k, self.v)]
        for h, g, rows, keys, seen in self.parts():
            cols, kcols = slice(h * D, (h + 1) * D), slice(g * D, (g + 1) * D)
            q, k, v = self.head(self.q, h, rows), self.head(self.k, g, keys), self.head(self.v, g, keys)
            do, o, l = self.head(self.dout, h, rows), self.head(out, h, rows), _np(lse)[h, rows]
            a, b, c = R.attn_grad(do, q, k, v, o, l, self.scale, seen)
            refs[0][rows, cols], refs[1][keys, kcols], refs[2][keys, kcols] = (
                a, refs[1][keys, kcols] + b, refs[2][keys, kcols] + c)
            P = np.where(seen, np.exp(np.where(seen, self.scale * q @ k.T - np.where(np.isfinite(l), l, 0)[:, None], 0)), 0)
            dP, delta = do @ v.T, (do * o).sum(1, keepdims=True)
            r = self.relative(q, k, l, seen)
            dS = np.abs(P * (dP - delta))
            mag = np.abs(do) @ np.abs(v).T + (np.abs(do) * np.abs(o)).sum(1, keepdims=True)
            e = P * (r * np.abs(dP - delta) + two * (D + 8) * U * mag + 4 * U * (np.abs(dP) + np.abs(delta)))
            e = e + P8 * (dS + e)
            n, m = (two * (x + 8) * U for x in seen.shape)
            tols[0][rows, cols] = self.scale * (e + m * dS) @ np.abs(k)
            # (sums over the query heads: each one's own terms)
            tols[1][keys, kcols] += self.scale * (e + (n + 8 * self.heads * U) * dS).T @ np.abs(q)
            tols[2][keys, kcols] += (P * (r + P8 + n + 8 * self.heads * U)).T @ np.abs(do)
        for what, got, ref, tol in zip(("dq", "dk", "dv"), (dq, dk, dv), refs, tols):
            rows = sum(self.lens if what == "dq" else self.klens)
            at = slice(0, rows) if only is None else only[0 if what == "dq" else 1]
            _close(_np(got)[at], ref[at], (tol + E[self.dtype] * (np.abs(ref) + tol))[at], what)

    def run(self):
        out, lse = iso.attn(self.q, self.k, self.v, **self.args)
        used = self.check_forward(out, lse)
        assert (out[torch.from_numpy(~used).to(DEV)] == 0).all() and (lse[:, torch.from_numpy(~used).to(DEV)] == 0).all()
        grads = iso.attn_grad(self.dout, self.q, self.k, self.v, out, lse, **self.args)
        self.check_backward(out, lse, *grads)
        assert (grads[0][sum(self.lens):] == 0).all() and all((g[sum(self.klens):] == 0).all() for g in grads[1:])
        return out, lse, grads


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,klens,heads,kv,D,causal,window,pad", [
    ([1], None, 1, 1, 16, True, 0, 0), ([1], [300], 4, 2, 64, True, 0, 0), ([1], [1], 1, 1, 128, False, 0, 0),
    ([64], None, 2, 2, 64, True, 0, 0), ([65], None, 2, 1, 64, True, 0, 0), ([127], None, 1, 1, 128, True, 0, 0),
    ([129], None, 3, 1, 128, True, 0, 0), ([300], None, 2, 1, 96, False, 0, 0),
    ([200, 1, 0, 63, 130], None, 4, 2, 64, True, 0, 7), ([3, 5, 2], None, 6, 3, 40, False, 0, 1),
    ([10], [4], 2, 1, 64, True, 0, 0), ([140, 5, 0, 9], [20, 0, 7, 300], 2, 1, 128, True, 0, 3),
    ([33, 70], [500, 71], 2, 2, 72, False, 0, 2), ([400], None, 2, 1, 64, True, 1, 0), ([400], None, 2, 1, 128, True, 100, 0),
    ([270], [600], 2, 1, 64, True, 130, 0), ([150], None, 1, 1, 64, True, 1000, 0), ([260], [100], 1, 1, 128, True, 30, 0)])
def test_attention_and_gradients(lens, klens, heads, kv, D, causal, window, pad, dtype):
    Case(lens, klens, heads, kv, D, causal, window, dtype, pad).run()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,gap,off", [(1, 0, 0), (33, 0, 0), (64, 3, 0), (64, 0, 1), (8, 8, 8), (100, 4, 4)])
def test_attention_of_odd_heads_strides_and_addresses(D, gap, off, dtype):
    Case([90, 40], [95, 130], 2, 1, D, dtype=dtype, gap=gap, off=off, pad=2).run()


@pytest.mark.parametrize("n,m", [(1, 1), (1, 700), (90, 1)])
def test_a_single_row_of_any_stride(n, m):
    """One query, or one key, out of rows off 16-byte boundaries."""
    q, do = (_rand(i, max(n, 2), 128, BF, 131 if n == 1 else 128) for i in (1, 2))
    k, v = (_rand(i, max(m, 2), 64, BF, 67 if m == 1 else 64) for i in (3, 4))
    c = Case([n], [m], 2, 1, 64)
    c.q, c.dout, c.k, c.v, c.tc = q[:n], do[:n], k[:m], v[:m], True
    c.run()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("amp,scale", [(8.0, None), (1.0, 2.0), (0.01, None)])
def test_attention_of_sharp_and_flat_weights(amp, scale, dtype):
    Case([180], None, 2, 1, 64, dtype=dtype, amp=amp, scale=scale).run()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_seen_has_no_part(D, dtype):
    """NaN and infinities in keys, values and gradients that a query does not see,
    within the tiles that it does: the rows that do not see them are those of
    the inputs without them, within the same bounds (the tensor cores' rows are
    done over in binary32, which these hold for too)."""
    c = Case([200, 150], None, 2, 1, D, dtype=dtype, pad=4)
    out, lse = iso.attn(c.q, c.k, c.v, **c.args)
    k, v, q, do = (t.clone() for t in (c.k, c.v, c.q, c.dout))
    for t, bad in ((k, math.nan), (v, math.inf)):
        t[120] = bad                      # token 120 of the first sequence
        t[200 + 149] = -bad               # the last one of the second
    rows = np.zeros(354, bool)
    rows[:120] = rows[200:349] = True
    got, got_lse = iso.attn(c.q, k, v, **c.args)
    c.check_forward(got, got_lse, rows)
    assert not torch.isfinite(got[120:200].float()).all(1).any()
    dq, _, _ = iso.attn_grad(c.dout, c.q, k, v, out, lse, **c.args)
    # a token's q and dout reach the keys that it sees, and no later ones
    later = np.zeros(354, bool)
    later[41:350] = True
    q[40], do[40] = math.nan, math.inf
    _, dk, dv = iso.attn_grad(do, q, c.k, c.v, out, lse, **c.args)
    c.check_backward(out, lse, dq, dk, dv, (rows, later))
    assert not torch.isfinite(dv[:41].float()).all(1).any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_writes_its_rows_and_nothing_else(dtype):
    c = Case([70, 0, 61], [70, 9, 66], 2, 1, 64, dtype=dtype, pad=5)
    out, lse = iso.attn(c.q, c.k, c.v, **c.args)
    grads = iso.attn_grad(c.dout, c.q, c.k, c.v, out, lse, **c.args)

    def frame(t):
        buf = torch.full((t.shape[0], t.shape[1] + 16), 5.0, dtype=t.dtype, device=DEV)
        return buf, buf[:, 8:8 + t.shape[1]]
    buf, o = frame(out)
    l = torch.full_like(lse, 5.0)
    assert iso.attn(c.q, c.k, c.v, out=o, lse=l, **c.args)[0] is o
    assert torch.equal(o[:131], out[:131]) and torch.equal(l[:, :131], lse[:, :131])
    assert (buf[:, :8] == 5).all() and (buf[:, -8:] == 5).all() and (buf[131:] == 5).all() and (l[:, 131:] == 5).all()
    bufs, views = zip(*(frame(g) for g in grads))
    iso.attn_grad(c.dout, c.q, c.k, c.v, out, lse, grads=views, **c.args)
    for b, view, g, n in zip(bufs, views, grads, (131, 145, 145)):
        assert torch.equal(view[:n], g[:n]) and (b[:, :8] == 5).all() and (b[:, -8:] == 5).all() and (b[n:] == 5).all()


def test_bad_offsets_are_reported():
    """Each stays within the rows: the kernels clamp what they read."""
    c = Case([64, 64], None, 2, 1, 64, pad=4)
    for bad in ([0, 64, 200], [-5, 64, 128], [0, 100, 50]):
        c.args["seqs"] = torch.tensor(bad, dtype=torch.int32, device=DEV)
        out, lse, st = iso.attn(c.q, c.k, c.v, status=True, **c.args)
        assert int(st) == _abi.ISO_ERR_INDEX
        *_, st = iso.attn_grad(c.dout, c.q, c.k, c.v, out, lse, status=True, **c.args)
        assert int(st) == _abi.ISO_ERR_INDEX
    c.args["seqs"] = torch.tensor([0, 64, 128], dtype=torch.int32, device=DEV)
    assert int(iso.attn(c.q, c.k, c.v, status=True, **c.args)[2]) == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradient_by_differences_of_the_forward_pass(dtype):
    """<gradient, change> against the change of sum out dout (binary64, from the
    oracle) along a random direction: second order in the step of 1e-4, E and the
    weights' rounding for the rest."""
    c = Case([60, 33], None, 2, 1, 64, dtype=dtype)
    out, lse, grads = c.run()
    rng = np.random.default_rng(3)
    moves = [rng.normal(size=t.shape) for t in (c.q, c.k, c.v)]

    def value(h):
        q, k, v = (_np(t) + h * m for t, m in zip((c.q, c.k, c.v), moves))
        total = 0.0
        for hd, g, rows, keys, seen in c.parts():
            sl, kl = slice(hd * 64, hd * 64 + 64), slice(g * 64, g * 64 + 64)
            o, _, _ = R.attn(q[rows, sl], k[keys, kl], v[keys, kl], c.scale, seen)
            total += (o * _np(c.dout)[rows, sl]).sum()
        return total
    want = (value(1e-4) - value(-1e-4)) / 2e-4
    terms = [(_np(g) * m) for g, m in zip(grads, moves)]
    spread = math.sqrt(sum((np.abs(t) ** 2).sum() for t in terms))
    tol = (8 * 2.0 ** -8 if dtype == BF else 1e-4) * spread
    assert abs(sum(t.sum() for t in terms) - want) <= tol


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------
def _distill_case(seed, T, V, K, dtype, ld=None, off=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    z = _rand(seed, T, V, dtype, ld, off, spread)
    ids = torch.randint(0, V, (T, K), generator=g)
    ids[torch.rand(T, K, generator=g) < 0.2] = -1
    if K > 2:
        ids[:, 1] = ids[:, 0]                    # the same entry twice
    t = (torch.randn(T, K, generator=g) * 2).to(dtype)
    dloss = torch.randn(T, generator=g)
    return z, ids, t, dloss


def _check_distill(z, ids, t, tau, dloss, loss, lse, grad, what=""):
    dtype, V = z.dtype, z.shape[1]
    Z, I, W, G = _np(z), ids.cpu().numpy(), _np(t), _np(dloss)
    rl, rs, rg = R.distill(Z, I, W, tau, G)
    fast = 2.0 ** -21 if dtype == BF else 0.0
    n = (V / 128 + 64) * U + fast
    with np.errstate(invalid="ignore"):
        score = U * 3 * (np.abs(Z) / tau + np.abs(np.where(np.isfinite(rs), rs, 0))[:, None])
        score = np.where(np.isfinite(score), score, 0)
        far = score.max(1, initial=0)
        e_lse = far + n + 2 * U * np.abs(np.where(np.isfinite(rs), rs, 0))
        if lse is not None:
            _close(lse, rs, e_lse, what + " lse")
            # sum p = 1: log p, the score and lse each off by their own
            top = np.abs(W).max(1, initial=0) / tau
            mag = np.array([np.abs(Z[r, [i for i in I[r] if 0 <= i < V]]).max(initial=0, where=np.isfinite(
                Z[r, [i for i in I[r] if 0 <= i < V]])) for r in range(len(Z))]) / tau
            e = tau ** 2 * (e_lse + U * 8 * (top + mag + np.abs(np.where(np.isfinite(rs), rs, 0)) + 8 + I.shape[1]))
            _close(loss, rl, e + 4 * U * np.abs(np.where(np.isfinite(rl), rl, 0)), what + " loss")
        if grad is not None:
            q = np.where(np.isfinite(Z), np.exp(np.where(np.isfinite(Z), Z, 0) / tau - np.where(np.isfinite(rs), rs, 0)[:, None]), 0)
            e = np.abs(G * tau)[:, None] * (q * (score + e_lse[:, None] + 8 * U + fast)
                                            + U * 16 * (2 + I.shape[1] / 8) * (np.abs(rg / np.where(G == 0, 1, G * tau)[:, None] - q) + q))
            e = np.where(np.isfinite(e), e, 0)
            _close(grad, rg, e + E[dtype] * np.where(np.isfinite(rg), np.abs(rg), 0) + 1e-36, what + " gradient")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,K,tau,ld,off", [
    (1, 1, 1, 1.0, None, 0), (3, 5, 3, 1.0, None, 0), (4, 7, 9, 2.0, 9, 1), (2, 500, 1, 0.5, None, 0),
    (5, 1000, 20, 1.0, None, 0), (5, 1001, 20, 1.0, None, 0), (3, 4099, 64, 2.0, 4107, 3), (2, 8200, 200, 1.0, None, 8),
    (160, 5000, 10, 1.0, None, 0), (3, 20011, 30, 0.7, None, 0), (2, 40960, 16, 1.0, None, 0), (1, 151936, 64, 1.0, None, 0),
    (40, 152064, 8, 1.0, None, 0), (2, 400001, 5, 1.0, None, 0)])
def test_distillation(T, V, K, tau, ld, off, dtype):
    z, ids, t, dloss = _distill_case(7, T, V, K, dtype, ld, off)
    d, i, w = dloss.to(DEV), ids.to(DEV), t.to(DEV)
    loss, lse, grad = iso.distill(z, i, w, tau, dloss=d)
    _check_distill(z, ids, t, tau, dloss, loss, lse, grad, "joint")
    # (without a gradient to place, another kernel with another order of sums may run)
    l2, s2 = iso.distill(z, i.int(), w, tau)
    _check_distill(z, ids, t, tau, dloss, l2, s2, None, "loss alone")
    g2 = iso.distill_grad(d, z, i, w, lse, tau)
    _check_distill(z, ids, t, tau, dloss, None, None, g2, "apart")
    # other alignment than the logits', and nothing written beside it
    buf = torch.full((T, V + 6), -3.0, dtype=dtype, device=DEV)
    l3, s3, g3 = iso.distill(z, i, w, tau, dloss=d, out=buf[:, 3:3 + V])
    _check_distill(z, ids, t, tau, dloss, l3, s3, g3, "aside")
    assert (buf[:, :3] == -3).all() and (buf[:, 3 + V:] == -3).all()
    # over the logits
    for joint in (True, False):
        z4 = z.clone()
        g4 = iso.distill(z4, i, w, tau, dloss=d, out=z4)[2] if joint else iso.distill_grad(d, z4, i, w, lse, tau, out=z4)
        assert g4 is z4
        _check_distill(z, ids, t, tau, dloss, None, None, g4, "in place")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,K,ld,off", [(700, 4200, 3, None, 0), (640, 20011, 20, 20015, 3), (333, 60000, 128, None, 0), (161, 152064, 5, None, 8),
                                           (700, 30001, 20, 30004, 3), (2500, 52000, 5, None, 0)])
def test_distillation_of_many_long_rows(T, V, K, ld, off, dtype):
    """Rows for every cluster to go through several of them; the last ones of
    another number, rows off 16-byte boundaries, in place."""
    z, ids, t, dloss = _distill_case(17, T, V, K, dtype, ld, off)
    z[5, 7], z[T - 1, V - 1], z[T // 2] = math.nan, math.inf, -math.inf
    ids[9], ids[T - 2] = -1, -1
    d, i, w = dloss.to(DEV), ids.to(DEV), t.to(DEV)
    same = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV) if off == 0 else None
    loss, lse, grad = iso.distill(z, i, w, 1.3, dloss=d, out=same)
    rows = sorted(set(list(range(0, T, 37)) + [5, 9, T // 2, T - 2, T - 1]))

    def check(loss, lse, grad, what):
        pick = lambda x: None if x is None else x[rows]                       # noqa: E731
        _check_distill(z[rows], ids[rows], t[rows], 1.3, dloss[rows], pick(loss), pick(lse), pick(grad), what)
    check(loss, lse, grad, "joint")
    l2, s2 = iso.distill(z, i, w, 1.3)
    check(l2, s2, None, "loss alone")
    g2 = iso.distill_grad(d, z, i, w, lse, 1.3)
    check(None, None, g2, "apart")
    for joint in (True, False):
        z4 = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV).copy_(z)
        g4 = iso.distill(z4, i, w, 1.3, dloss=d, out=z4)[2] if joint else iso.distill_grad(d, z4, i, w, lse, 1.3, out=z4)
        assert torch.equal(g4.nan_to_num(7.0), (grad if joint and off == 0 else g4).nan_to_num(7.0))
        check(None, None, g4, "in place")
    # every other row as it is in a call of its own kind of rows: nothing of one row in another
    assert torch.equal(iso.distill(z, i, w, 1.3)[1].nan_to_num(7.0), s2.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [50, 3000, 30000])
def test_distillation_of_infinities_nan_and_empty_rows(V, dtype):
    z, ids, t, dloss = _distill_case(8, 8, V, 4, dtype)
    ids[ids < 0] = 3
    z[0, :V // 2] = -math.inf                 # a masked half
    ids[0], ids[0, 0] = V - 1, V - 2
    z[1] = -math.inf                          # nothing left
    z[2, 5], z[3, 6] = math.nan, math.inf
    ids[4] = -1                               # no used slot
    t[5] = -math.inf                          # used slots without weight
    t[6, 0], ids[6, 0], z[6, 9] = -math.inf, 9, -math.inf      # no weight where the student has none
    ids[7, 2:] = 9
    z[7, 9] = -math.inf                       # weight where the student has none: infinite loss
    loss, lse, grad = iso.distill(z, ids.to(DEV), t.to(DEV), dloss=dloss.to(DEV))
    _check_distill(z, ids, t, 1.0, dloss, loss, lse, grad)
    assert math.isinf(float(loss[7])) and torch.isfinite(grad[7]).all() and (grad[4:6] == 0).all()
    g2 = iso.distill_grad(dloss.to(DEV), z, ids.to(DEV), t.to(DEV), lse)
    _check_distill(z, ids, t, 1.0, dloss, None, None, g2)


def test_distillation_ids_outside_the_vocabulary():
    z, ids, t, dloss = _distill_case(9, 4, 300, 5, BF)
    *_, st = iso.distill(z, ids.to(DEV), t.to(DEV), status=True)
    assert int(st) == 0
    ids[2, 3], ids[3, 0] = 300, -2
    loss, lse, grad, st = iso.distill(z, ids.to(DEV), t.to(DEV), dloss=dloss.to(DEV), status=True)
    assert int(st) == _abi.ISO_ERR_INDEX
    _check_distill(z, ids, t, 1.0, dloss, loss, lse, grad)
    _, st = iso.distill_grad(dloss.to(DEV), z, ids.to(DEV), t.to(DEV), lse, status=True)
    assert int(st) == _abi.ISO_ERR_INDEX


# ---------------------------------------------------------------------------
# the calls in a program
# ---------------------------------------------------------------------------
def test_empty_calls():
    x = torch.empty(0, 64, dtype=BF, device=DEV)
    k = torch.empty(5, 64, dtype=BF, device=DEV).zero_()
    plan = iso.rope_plan(64)
    assert iso.rope(x, torch.empty(0, dtype=torch.int64, device=DEV), plan).shape == (0, 64)
    out, lse = iso.attn(x, k, k, 1)
    assert out.shape == (0, 64) and lse.shape == (1, 0)
    dq, dk, dv = iso.attn_grad(x, x, k, k, out, lse, 1)
    assert dq.shape == (0, 64) and (dk == 0).all() and (dv == 0).all()
    q = torch.ones(3, 64, dtype=BF, device=DEV)
    out, lse = iso.attn(q, x, x, 1)
    assert (out == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = iso.attn_grad(q, q, x, x, out, lse, 1)
    assert (dq == 0).all() and dk.shape == (0, 64)
    z = torch.empty(0, 9, device=DEV)
    loss, lse, g = iso.distill(z, torch.empty(0, 2, dtype=torch.int64, device=DEV), torch.empty(0, 2, device=DEV),
                               dloss=torch.empty(0, device=DEV))
    assert loss.shape == (0,) and g.shape == (0, 9)
    loss, lse = iso.distill(torch.ones(2, 9, device=DEV), torch.empty(2, 0, dtype=torch.int64, device=DEV),
                            torch.empty(2, 0, device=DEV))
    assert (loss == 0).all() and torch.allclose(lse, torch.full_like(lse, 1 + math.log(9)))


def test_the_same_bits_again_on_another_stream_and_captured():
    c = Case([200, 57], None, 4, 2, 64, pad=3)
    z, ids, t, dloss = _distill_case(5, 20, 9001, 12, BF)
    ids, t, dloss = ids.to(DEV), t.to(DEV), dloss.to(DEV)
    plan, pos = iso.rope_plan(64), torch.arange(c.q.shape[0], device=DEV)

    def calls(stream=None):
        r = iso.rope(c.q, pos, plan, stream=stream)
        out, lse = iso.attn(c.q, c.k, c.v, stream=stream, **c.args)
        return (r, out, lse) + iso.attn_grad(c.dout, c.q, c.k, c.v, out, lse, stream=stream, **c.args) + iso.distill(
            z, ids, t, dloss=dloss, stream=stream)

    def same(a, b):
        return all(torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in zip(a, b))
    want = calls()
    assert same(calls(), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = calls(s)
    s.synchronize()
    assert same(got, want)
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            held = calls()
        for x in held:
            x.fill_(9.0)
        g.replay()
        g.replay()
    torch.cuda.synchronize()
    # (zeros of rows without a sequence are written within the graph too)
    assert same(held, want)


def test_refusals_on_the_device():
    c = Case([20], None, 2, 1, 64)
    with pytest.raises(ValueError, match="lse must have shape"):
        iso.attn_grad(c.dout, c.q, c.k, c.v, c.q.clone(), torch.zeros(2, 19, device=DEV), **c.args)
    with pytest.raises(_abi.IsoError):
        iso.attn(c.q, c.k, c.v[:-1], **c.args)
    with pytest.raises(ValueError, match="positions must have shape"):
        iso.rope(c.q, torch.zeros(3, 20, dtype=torch.int64, device=DEV), iso.rope_plan(64))
    with pytest.raises(_abi.IsoError):
        iso.rope(c.q, torch.zeros(20, dtype=torch.int64, device=DEV), iso.rope_plan(80))
    z, ids, t, dloss = _distill_case(5, 4, 30, 3, BF)
    with pytest.raises(ValueError, match="ids must"):
        iso.distill(z, ids.to(DEV)[:, :2].contiguous(), t.to(DEV))
    with pytest.raises(ValueError, match="needs dloss"):
        iso.distill(z, ids.to(DEV), t.to(DEV), out=z)
