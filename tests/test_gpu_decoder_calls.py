"""How the calls between the embedding and the loss live with a program around
them, on the GPU: captured in graphs, made by several threads, given outputs and
workspaces, with waits that give up, and refused in both of their forms."""
import threading

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
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(DEV, dtype)


def _inputs(seed=0, T=300, heads=4, kv=2, D=64, dtype=BF):
    qkv = _rand(seed, T, (heads + 2 * kv) * D, dtype=dtype)
    q, k, v = qkv.split([heads * D, kv * D, kv * D], 1)
    return q, k, v, _rand(seed + 1, T, heads * D, dtype=dtype)


def test_capture_without_a_workspace_and_two_graphs():
    """Replays after larger calls on the captured stream, of two graphs in either
    order: right results, and nothing written outside the graphs' own memory."""
    q, k, v, do = _inputs()
    one, rows = _rand(9, 1, 256), _rand(8, 6000, 2 * 128)
    want = iso.attn(q, k, v, 4, 2)
    grads = iso.attn_grad(do, q, k, v, *want, 4, 2)
    split = iso.attn(one, rows[:, :128], rows[:, 128:], 4, 2)          # parts of the keys, joined
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(t) for t in (*want, *grads, *split)]

    def first():
        iso.attn(q, k, v, 4, 2, out=outs[0], lse=outs[1])
        iso.attn_grad(do, q, k, v, *want, 4, 2, grads=outs[2:5])

    def second():
        iso.attn(one, rows[:, :128], rows[:, 128:], 4, 2, out=outs[5], lse=outs[6])
        iso.attn_grad(do, q, k, v, *want, 4, 2, grads=outs[2:5])
    with torch.cuda.stream(s):
        first(), second()
        torch.cuda.synchronize()
        graphs = []
        for f in (first, second):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                f()
            graphs.append(g)
        big = _inputs(5, T=5000)
        o = iso.attn(*big[:3], 4, 2)
        iso.attn_grad(big[3], *big[:3], *o, 4, 2)
        others = [torch.full((n,), 7, dtype=torch.uint8, device=DEV) for n in [1 << 20] * 64 + [4 << 20] * 16]
        for order in ((0, 1), (1, 0)):
            for t in outs:
                t.fill_(9.0)
            for i in order:
                graphs[i].replay()
            graphs[order[0]].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, (*want, *grads, *split)))
    assert all(bool((t == 7).all()) for t in others)


def test_calls_of_several_threads_on_one_stream():
    q, k, v, do = _inputs(3, T=700)
    z, ids, t = _rand(4, 50, 20000), torch.randint(0, 20000, (50, 9), device=DEV), _rand(5, 50, 9)
    w = torch.rand(50, device=DEV)
    out, lse = iso.attn(q, k, v, 4, 2)
    want = iso.attn_grad(do, q, k, v, out, lse, 4, 2) + iso.distill(z, ids, t, dloss=w)
    got, failed = {}, []

    def call(i):
        try:
            torch.cuda.set_device(0)
            for _ in range(10):
                got[i] = iso.attn_grad(do, q, k, v, *iso.attn(q, k, v, 4, 2), 4, 2) + iso.distill(z, ids, t, dloss=w)
        except BaseException as e:        # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=call, args=(i,)) for i in range(4)]
    [x.start() for x in threads]
    [x.join() for x in threads]
    torch.cuda.synchronize()
    assert not failed and all(all(torch.equal(a, b) for a, b in zip(got[i], want)) for i in range(4))


def test_a_callers_workspace_and_status():
    q, k, v, do = _inputs(6, T=500)
    ws = iso.Workspace(torch.device(DEV))
    want = iso.attn(q, k, v, 4, 2)
    out, lse, st = iso.attn(q, k, v, 4, 2, workspace=ws, status=True)
    assert int(st) == 0 and torch.equal(out, want[0]) and torch.equal(lse, want[1])
    *g, st = iso.attn_grad(do, q, k, v, out, lse, 4, 2, workspace=ws, status=True)
    assert int(st) == 0 and all(torch.equal(a, b) for a, b in zip(g, iso.attn_grad(do, q, k, v, out, lse, 4, 2)))


def test_a_give_up_leaves_each_row_whole_or_nan():
    """With a limit of 0 a wait gives up at its second look at the clock.  Rows of
    a head are complete or NaN, the status says so, and the next calls are whole
    again."""
    L = _abi.lib()
    q, k, v, do = _inputs(7, T=3000, heads=8, kv=2, D=128)
    out, lse = iso.attn(q, k, v, 8, 2)
    grads = iso.attn_grad(do, q, k, v, out, lse, 8, 2)
    before = L.iso_attn_wait_ns(0)
    assert before == 2000000000 and L.iso_attn_wait_ns(-1) == 0
    try:
        o2, l2, st = iso.attn(q, k, v, 8, 2, status=True)
        *g2, st2 = iso.attn_grad(do, q, k, v, out, lse, 8, 2, status=True)
        torch.cuda.synchronize()
    finally:
        L.iso_attn_wait_ns(before)
    assert int(st) in (0, _abi.ISO_ERR_TIMEOUT) and int(st2) in (0, _abi.ISO_ERR_TIMEOUT)
    for got, ref, heads in ((o2, out, 8), *zip(g2, grads, (8, 2, 2))):
        got, ref = got.view(3000, heads, 128), ref.view(3000, heads, 128)
        nan = torch.isnan(got).all(2)
        assert bool((nan | (got == ref).all(2)).all())
    if int(st) == 0:
        assert torch.equal(o2, out)
    else:
        assert torch.isnan(o2).any()
    again = iso.attn_grad(do, q, k, v, *iso.attn(q, k, v, 8, 2), 8, 2)
    assert all(torch.equal(a, b) for a, b in zip(again, grads))


def test_both_forms_of_a_call_refuse_alike():
    """The common form goes through the host module, the one with a stream through
    ctypes: the same errors with the same texts."""
    q, k, v, do = _inputs(8, T=20)
    lse, s = torch.zeros(4, 20, device=DEV), torch.cuda.current_stream()
    plan, pos = iso.rope_plan(64), torch.zeros(20, dtype=torch.int64, device=DEV)
    z, ids, t, w = _rand(1, 20, 50), torch.zeros(20, 3, dtype=torch.int64, device=DEV), _rand(2, 20, 3), torch.ones(20, device=DEV)
    ends = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    bad = [
        lambda **a: iso.rope(q[0], pos, plan, **a), lambda **a: iso.rope(q.half(), pos, plan, **a),
        lambda **a: iso.rope(q.cpu(), pos, plan, **a), lambda **a: iso.rope(q.t(), pos, plan, **a),
        lambda **a: iso.rope(q, pos.float(), plan, **a), lambda **a: iso.rope(q, pos[:-1], plan, **a),
        lambda **a: iso.rope(q, pos.cpu(), plan, **a), lambda **a: iso.rope(q[:, :100], pos, plan, **a),
        lambda **a: iso.rope(q, torch.zeros(40, dtype=torch.int64, device=DEV)[::2], plan, **a),
        lambda **a: iso.rope(q, pos.expand(3, 20), iso.rope_plan(64, sections=(16, 8, 8)), **a),
        lambda **a: iso.rope_grad(q, pos[:3], plan, **a),
        lambda **a: iso.attn(q, k, v, 3, 2, **a), lambda **a: iso.attn(q, k, v, 4, 3, **a), lambda **a: iso.attn(q, k, v, 0, **a),
        lambda **a: iso.attn(q, k, v, 4, 2, window=-1, **a), lambda **a: iso.attn(q, k, v, 4, 2, causal=False, window=3, **a),
        lambda **a: iso.attn(q, k, v, 4, 2, scale=0.0, **a), lambda **a: iso.attn(q, k, v, 4, 2, scale=float("nan"), **a),
        lambda **a: iso.attn(q, k, v, 4, 2, seqs=ends.long(), **a), lambda **a: iso.attn(q, k, v, 4, 2, seqs=ends.cpu(), **a),
        lambda **a: iso.attn(q, k, v, 4, 2, seqs=ends, kv_seqs=torch.zeros(3, dtype=torch.int32, device=DEV), **a),
        lambda **a: iso.attn(q, k, v, 4, 2, kv_seqs=ends, **a), lambda **a: iso.attn(q, k[:-1], v[:-1], 4, 2, seqs=ends, **a),
        lambda **a: iso.attn(q, k.float(), v, 4, 2, **a), lambda **a: iso.attn(q, k, v[:, :64], 4, 2, **a),
        lambda **a: iso.attn_grad(do, q, k, v, do, lse[:, :-1], 4, 2, **a), lambda **a: iso.attn_grad(do, q, k, v, do, lse.double(), 4, 2, **a),
        lambda **a: iso.attn_grad(do[:-1], q, k, v, do, lse, 4, 2, **a), lambda **a: iso.attn_grad(do.float(), q, k, v, do, lse, 4, 2, **a),
        lambda **a: iso.distill(z, ids[:, :2], t, **a), lambda **a: iso.distill(z, ids.float(), t, **a),
        lambda **a: iso.distill(z, ids.t().contiguous().t(), t, **a), lambda **a: iso.distill(z, ids, t, temperature=0, **a),
        lambda **a: iso.distill(z, ids, t, dloss=w[:-1], **a), lambda **a: iso.distill(z, ids, t, dloss=w.double(), **a),
        lambda **a: iso.distill(z, ids, t[:-1], **a), lambda **a: iso.distill_grad(w, z, ids, t, w[:-1], **a),
        lambda **a: iso.distill_grad(w.cpu(), z, ids, t, w, **a), lambda **a: iso.distill_grad(w, z, ids, t, w, temperature=-1.0, **a)]
    for i, call in enumerate(bad):
        errors = []
        for form in ({}, {"stream": s}):
            with pytest.raises((TypeError, ValueError, _abi.IsoError)) as e:
                call(**form)
            errors.append((e.type, str(e.value)))
        assert errors[0] == errors[1], (i, errors)
