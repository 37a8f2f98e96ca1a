"""The calls between the embedding and the loss where their outer loops turn and
where indexes pass 32 bits, against plain torch operations in binary64 on the
device.  The bounds are those of test_gpu_decoder with every factor at its
largest: of bfloat16 outputs an error of 2^-8 of the value and, for the weights'
rounding, 2^-8 of the sum of the terms' magnitudes (a 50th of it beside the
random signs); relative to a row's largest magnitude 0.02 covers both."""
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


def _rand(seed, *shape, dtype=BF):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def _reference(q, k, v, do, kept, heads, kv, spans, causal=True, window=0):
    """(out, lse, dq, dk, dv) in binary64, the gradients from the (out, lse) kept,
    as attn_grad takes them; spans: (q0, nq, k0, nk)."""
    D, G = q.shape[1] // heads, heads // kv
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(heads, len(q), dtype=torch.float64, device=DEV)
    grads = [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in (q, k, v)]
    for q0, nq, k0, nk in spans:
        if not nq or not nk:
            continue
        i, j = torch.arange(nk - nq, nk, device=DEV)[:, None], torch.arange(nk, device=DEV)[None]
        sees = (j <= i) & (j > i - window if window else True) if causal else torch.ones(nq, nk, dtype=torch.bool, device=DEV)
        for h in range(heads):
            a, b = slice(h * D, h * D + D), slice(h // G * D, h // G * D + D)
            x, y, w, d = (t.double() for t in (q[q0:q0 + nq, a], k[k0:k0 + nk, b], v[k0:k0 + nk, b], do[q0:q0 + nq, a]))
            S = torch.where(sees, x @ y.t() * D ** -0.5, -torch.inf)
            l = torch.logsumexp(S, 1)
            out[q0:q0 + nq, a], lse[h, q0:q0 + nq] = torch.exp(S - l[:, None]) @ w, l
            P = torch.exp(S - kept[1][h, q0:q0 + nq, None].double())
            delta = (d * kept[0][q0:q0 + nq, a].double()).sum(1, keepdim=True)
            dS = P * (d @ w.t() - delta) * D ** -0.5
            grads[0][q0:q0 + nq, a] = dS @ y
            grads[1][k0:k0 + nk, b] += dS.t() @ x
            grads[2][k0:k0 + nk, b] += P.t() @ d
    return (out, lse, *grads)


def _near(got, ref, what, tol, floor=0.0):
    """floor: what the error may be beside a gradient that cancels."""
    top = tol * ref.abs().amax(1, keepdim=True) + floor + 1e-30
    worst = ((got.double() - ref).abs() / top).max()
    assert bool(torch.isfinite(got).all()) and float(worst) <= 1, f"{what}: {float(worst):.3g} of the bound"


def _cancelled(x, v, do, heads, kv):
    """dP - delta is two sums of D binary32 products, each off by at most 2 (D + 8) U
    |dout||v| (on the tensor cores, whose additions cut bits off), and where a query
    sees one key, or keys alike, nothing is left beside that: of a term of dq, scale
    max |k| times it, of dk scale max |q| (sums of such terms have weights that add
    up to 1 for dq; for dk the queries that see few keys are few)."""
    D = v.shape[1] // kv
    norms = [t.double().unflatten(1, (-1, D)).norm(dim=2).max() for t in (do, v)]
    return float(4 * (D + 8) * 2.0 ** -24 * D ** -0.5 * norms[0] * norms[1] * x.double().abs().max())


def _check(q, k, v, do, heads, kv, spans, **args):
    dtype = q.dtype
    tol = 0.02 if dtype == BF else 1e-4
    out, lse = iso.attn(q, k, v, heads, kv, **args)
    grads = iso.attn_grad(do, q, k, v, out, lse, heads, kv, **args)
    ref = _reference(q, k, v, do, (out, lse), heads, kv, spans, args.get("causal", True), args.get("window", 0))
    _near(out, ref[0], "out", tol)
    assert float((lse.double() - ref[1]).abs().max()) <= 1e-4
    for name, g, r, x in zip(("dq", "dk", "dv"), grads, ref[2:], (k, q, None)):
        _near(g, r, name, tol, 0.0 if x is None else _cancelled(x, v, do, heads, kv))


@pytest.mark.parametrize("T,heads,kv,D,window", [(1500, 2, 1, 128, 0), (2049, 7, 1, 64, 0), (1300, 28, 4, 128, 0), (3000, 2, 2, 128, 700),
                                                 (1111, 6, 2, 72, 333)])
def test_many_tiles(T, heads, kv, D, window):
    qkv = _rand(1, T, (heads + 2 * kv) * D)
    q, k, v = qkv.split([heads * D, kv * D, kv * D], 1)
    _check(q, k, v, _rand(2, T, heads * D), heads, kv, [(0, T, 0, T)], window=window)


@pytest.mark.parametrize("heads,kv", [(1, 1), (12, 2), (28, 4)])
def test_parts_of_the_keys_and_of_the_heads(heads, kv):
    """Few queries over many keys (the keys in parts), and a short sequence of
    many query heads a key head (their sums in parts)."""
    D = 128
    for n, m in ((1, 5000), (3, 4097), (130, 2500), (500, 500)):
        q, do, k, v = _rand(n, n, heads * D), _rand(n + 1, n, heads * D), _rand(n + 2, m, kv * D), _rand(n + 3, m, kv * D)
        _check(q, k, v, do, heads, kv, [(0, n, 0, m)])


def test_many_sequences():
    """More sequences than a warp looks at in one go, empty ones among them, keys
    kept before some."""
    lens = [(7 * i) % 41 * (i % 5 != 0) for i in range(150)]
    kept = [(11 * i) % 67 for i in range(150)]
    spans, q0, k0 = [], 0, 0
    for n, m in zip(lens, kept):
        spans.append((q0, n, k0, n + m))
        q0, k0 = q0 + n, k0 + n + m
    ends = [torch.tensor([s[i] for s in spans] + [e], dtype=torch.int32, device=DEV) for i, e in ((0, q0), (2, k0))]
    _check(_rand(1, q0, 256), _rand(2, k0, 128), _rand(3, k0, 128), _rand(4, q0, 256), 4, 2, spans, seqs=ends[0], kv_seqs=ends[1])
    _check(_rand(1, q0, 80, dtype=F32), _rand(2, k0, 40, dtype=F32), _rand(3, k0, 40, dtype=F32), _rand(4, q0, 80, dtype=F32), 4, 2, spans,
           seqs=ends[0], kv_seqs=ends[1])


@pytest.mark.parametrize("D", [128, 33])
def test_rows_past_32_bits(D):
    """A cache whose entries lie beyond 2^31 elements (8.6 GB), two sequences at its
    end and one at its start."""
    kv, heads = 8, 8
    rows = (1 << 31) // (kv * D) + 3000
    k = torch.zeros(rows, kv * D, dtype=BF, device=DEV)
    v = torch.zeros(rows, kv * D, dtype=BF, device=DEV)
    spans = [(0, 40, 0, 300), (40, 0, 300, rows - 1800), (40, 130, rows - 1500, 900), (170, 5, rows - 600, 600)]
    for _, _, k0, nk in spans:
        if nk < 2000:
            k[k0:k0 + nk], v[k0:k0 + nk] = _rand(k0 % 97, nk, kv * D), _rand(k0 % 89, nk, kv * D)
    q, do = _rand(5, 175, heads * D), _rand(6, 175, heads * D)
    seqs = torch.tensor([0, 40, 40, 170, 175], dtype=torch.int32, device=DEV)
    kv_seqs = torch.tensor([0, 300, rows - 1500, rows - 600, rows], dtype=torch.int32, device=DEV)
    out, lse = iso.attn(q, k, v, heads, kv, seqs=seqs, kv_seqs=kv_seqs)
    dq, dk, dv = iso.attn_grad(do, q, k, v, out, lse, heads, kv, seqs=seqs, kv_seqs=kv_seqs)
    # the same sequences one after the other, close together
    parts = [(0, 40, 0, 300), (40, 130, rows - 1500, 900), (170, 5, rows - 600, 600)]
    ks, vs = (torch.cat([t[a:a + n] for _, _, a, n in parts]) for t in (k, v))
    ref = _reference(q, ks, vs, do, (out, lse), heads, kv, [(0, 40, 0, 300), (40, 130, 300, 900), (170, 5, 1200, 600)])
    _near(out, ref[0], "out", 0.02)
    _near(dq, ref[2], "dq", 0.02, _cancelled(ks, vs, do, heads, kv))
    for name, got, r, floor in (("dk", dk, ref[3], _cancelled(q, vs, do, heads, kv)), ("dv", dv, ref[4], 0.0)):
        _near(torch.cat([got[a:a + n] for _, _, a, n in parts]), r, name, 0.02, floor)
        assert not got[300:rows - 1500].any()


def test_logits_past_32_bits():
    """16384 rows of 152064 entries (5 GB): rows past 2^31 elements, in place."""
    T, V, K = 16384, 152064, 8
    z = torch.zeros(T, V, dtype=BF, device=DEV)
    rows = torch.tensor([0, 3, 8191, 14121, 14122, 14123, T - 1], device=DEV)
    z[rows] = _rand(1, len(rows), V) * 2
    ids = torch.randint(0, V, (T, K), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    t, w = _rand(3, T, K), torch.rand(T, device=DEV) + 0.5
    logits = z[rows].double()
    loss, lse, grad = iso.distill(z, ids, t, dloss=w, out=z)
    p = torch.softmax(t[rows].double(), 1)
    ref_lse = torch.logsumexp(logits, 1)
    ref = torch.exp(logits - ref_lse[:, None])
    ref.scatter_add_(1, ids[rows], -p)
    ref *= w[rows].double()[:, None]
    assert grad is z and float((lse[rows].double() - ref_lse).abs().max()) <= 1e-5
    assert bool(((grad[rows].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2e-6 * ref.abs().amax(1, keepdim=True)).all())
    ref_loss = (p * (p.log() - logits.gather(1, ids[rows]) + ref_lse[:, None])).sum(1)
    assert float((loss[rows].double() - ref_loss).abs().max()) <= 1e-4
    flat = torch.log(torch.tensor(float(V), dtype=torch.float64))
    assert abs(float(lse[1]) - float(flat)) <= 1e-5


@pytest.mark.parametrize("K", [129, 700, 2048])
def test_many_slots(K):
    V, T = 5000, 6
    z, t, w = _rand(1, T, V, dtype=F32), _rand(2, T, K, dtype=F32), torch.rand(T, device=DEV)
    ids = torch.randint(0, V // 3, (T, K), device=DEV)
    loss, lse, grad = iso.distill(z, ids, t, dloss=w)
    p = torch.softmax(t.double(), 1)
    ref = torch.softmax(z.double(), 1).scatter_add_(1, ids, -p) * w.double()[:, None]
    # sums of up to K probabilities: K 2^-24 of the largest mass
    assert float((grad.double() - ref).abs().max()) <= (K + 64) * 2.0 ** -24 * float(ref.abs().max())
    log_q = torch.log_softmax(z.double(), 1).gather(1, ids)
    assert float((loss.double() - (p * (p.log() - log_q)).sum(1)).abs().max()) <= 1e-5
    with pytest.raises(_abi.IsoError):
        iso.distill(z, torch.zeros(T, 2049, dtype=torch.int64, device=DEV), torch.zeros(T, 2049, device=DEV))


def test_rotary_of_many_rows_and_heads():
    """Rows past 2^31 elements, and more heads than a block takes at once."""
    plan = iso.rope_plan(128)
    x = torch.zeros((1 << 31) // 4096 + 5000, 4096, dtype=BF, device=DEV)
    x[-3:] = _rand(1, 3, 4096)
    pos = torch.arange(len(x), device=DEV, dtype=torch.int32)
    want = iso.rope(x[-3:].clone(), pos[-3:], plan)
    assert torch.equal(iso.rope(x, pos, plan, out=x)[-3:], want)
    y = _rand(2, 3, 300 * 128)
    p = torch.tensor([5, 0, 77], device=DEV)
    got = iso.rope(y, p, plan)
    assert all(torch.equal(got[:, h * 128:(h + 1) * 128], iso.rope(y[:, h * 128:(h + 1) * 128], p, plan)) for h in (0, 1, 150, 299))
