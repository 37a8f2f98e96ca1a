"""How the training-step calls live with a program around them, on the GPU:
captured in graphs and made by several threads, without a workspace of the
caller's."""
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


def test_capture_without_a_workspace():
    """A replay after a larger call on the captured stream: right results, and
    nothing written outside the graph's own memory."""
    x, dy = _rand(1, 700, 256), _rand(2, 700, 384)
    ids = torch.randint(0, 5000, (700,), generator=torch.Generator().manual_seed(3)).to(DEV)
    p = iso.act_pack(x)
    want = iso.act_wgrad(dy, p), iso.embed_grad(dy, ids, 5000)
    out, grad = torch.empty_like(want[0]), torch.empty_like(want[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def calls():
        iso.act_wgrad(dy, p, out=out)
        iso.embed_grad(dy, ids, out=grad)
    with torch.cuda.stream(s):
        calls()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            calls()
        # larger calls on the same stream, then tensors in whatever memory is free now
        big = _rand(4, 6000, 512)
        iso.act_wgrad(_rand(5, 6000, 640, dtype=F32), iso.act_pack(big), out=torch.empty(640, 512, device=DEV))
        iso.embed_grad(big, torch.zeros(6000, dtype=torch.int64, device=DEV), out=torch.empty(10, 512, device=DEV))
        others = [torch.full((n,), 7, dtype=torch.uint8, device=DEV) for n in [1 << 20] * 64 + [4 << 20] * 16]
        out.zero_()
        grad.fill_(9.0)
        g.replay()
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(grad, want[1])
    assert all(bool((t == 7).all()) for t in others)


def test_threads_accumulating_on_one_stream():
    """Four threads, each with inputs and gradients of its own, all on the
    default stream."""
    n = 4
    x = [_rand(10 + i, 400, 320) for i in range(n)]
    dy = [_rand(20 + i, 400, 192, dtype=F32) for i in range(n)]
    ids = [torch.randint(0, 300, (400,), generator=torch.Generator().manual_seed(30 + i)).to(DEV) for i in range(n)]
    packs = [iso.act_pack(t) for t in x]
    want = []
    for i in range(n):
        G, E = torch.zeros(192, 320, device=DEV), torch.zeros(300, 192, device=DEV)
        for _ in range(20):
            iso.act_wgrad(dy[i], packs[i], out=G, accumulate=True)
            iso.embed_grad(dy[i], ids[i], out=E, accumulate=True)
        want.append((G, E))
    got = [(torch.zeros(192, 320, device=DEV), torch.zeros(300, 192, device=DEV)) for _ in range(n)]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(n, timeout=60), []

    def work(i):
        try:
            torch.cuda.set_device(0)
            start.wait()
            for _ in range(20):
                iso.act_wgrad(dy[i], packs[i], out=got[i][0], accumulate=True)
                iso.embed_grad(dy[i], ids[i], out=got[i][1], accumulate=True)
        except BaseException as e:        # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not failed
    for (G, E), (wG, wE) in zip(got, want):
        assert torch.equal(G, wG) and torch.equal(E, wE)


@pytest.fixture
def no_patience():
    """Waits of the weight gradient's kernel that give up at once: what the
    hardware has not delivered by a wait's second look at the clock counts as
    not coming."""
    L = _abi.lib()
    limit = L.iso_act_wgrad_wait_ns(0)
    assert limit == 2_000_000_000 and L.iso_act_wgrad_wait_ns(-1) == 0
    yield
    torch.cuda.synchronize()
    L.iso_act_wgrad_wait_ns(limit)


GIVE_UPS = [
    # tokens, M, N, dY, G: many tiles a CTA pair with several chains each, parts of the tokens, binary32 parts of dY
    (2100, 5000, 4104, BF, F32), (2100, 5000, 4104, BF, BF), (8192, 256, 128, BF, F32), (8192, 1536, 1536, BF, BF),
    (1500, 2000, 1000, F32, F32),
]


@pytest.mark.parametrize("T,M,N,dtype,out", GIVE_UPS)
def test_a_give_up_leaves_sums_or_nan(no_patience, T, M, N, dtype, out):
    x, dy = _rand(41, T, N), _rand(42, T, M, dtype=dtype)
    p = iso.act_pack(x)
    base = _rand(43, M, N, dtype=out)
    _abi.lib().iso_act_wgrad_wait_ns(2_000_000_000)
    want = iso.act_wgrad(dy, p, dtype=out), iso.act_wgrad(dy, p, out=base.clone(), accumulate=True)
    assert not any(bool(w.isnan().any()) for w in want)
    torch.cuda.synchronize()
    _abi.lib().iso_act_wgrad_wait_ns(0)
    gave_up = 0
    for _ in range(5):
        g, st = iso.act_wgrad(dy, p, dtype=out, status=True)
        h = iso.act_wgrad(dy, p, out=base.clone(), accumulate=True)
        silent = iso.act_wgrad(dy, p, dtype=out)          # no status: the gradient itself says it
        for got, ref in ((g, want[0]), (h, want[1]), (silent, want[0])):
            assert bool(((got == ref) | got.isnan()).all())
        assert int(st) == (_abi.ISO_ERR_TIMEOUT if bool(g.isnan().any()) else _abi.ISO_OK)
        gave_up += int(st) != 0
    # whether a short call runs out is up to its copies' timing; a kernel of 100 us does
    assert gave_up or T * M * N < 4e10
    _abi.lib().iso_act_wgrad_wait_ns(2_000_000_000)
    assert torch.equal(iso.act_wgrad(dy, p, dtype=out), want[0])


def _refusal(f):
    try:
        f()
    except Exception as e:
        return type(e), getattr(e, "code", None)
    return None


def test_both_forms_of_a_call_refuse_alike():
    """The form that allocates its outputs and the one that is given them (or a
    status, or a stream that is not the current one)."""
    x, i8 = _rand(51, 8, 64), torch.zeros(8, dtype=torch.int64, device=DEV)
    p, s = iso.act_pack(x), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, f32 = torch.empty(8, 64, dtype=BF, device=DEV), torch.empty(64, 64, device=DEV)
    packs = iso.ActPack.empty(8, 64), iso.ActPack.empty(8, 64)
    bad = [None, [1.0], x.cpu(), x.half(), x[0], x.t(), x[:1].expand(8, 64)]
    ids = [None, [1], i8.float(), i8.cpu(), torch.zeros(8, 2, dtype=torch.int64, device=DEV)[:, 0]]
    pairs = []
    for b in bad:
        pairs += [(lambda b=b: iso.act_pack(b), lambda b=b: iso.act_pack(b, out=packs[0])),
                  (lambda b=b: iso.act_wgrad(b, p), lambda b=b: iso.act_wgrad(b, p, out=f32)),
                  (lambda b=b: iso.swiglu_pack(b, x), lambda b=b: iso.swiglu_pack(b, x, out=out)),
                  (lambda b=b: iso.swiglu_pack(x, b), lambda b=b: iso.swiglu_pack(x, b, packs=packs)),
                  (lambda b=b: iso.swiglu_grad(b, p, p), lambda b=b: iso.swiglu_grad(b, p, p, out=(out, out.clone(), out.clone()))),
                  (lambda b=b: iso.embed(b, i8), lambda b=b: iso.embed(b, i8, status=True)),
                  (lambda b=b: iso.embed_grad(b, i8, 9), lambda b=b: iso.embed_grad(b, i8, 9, status=True))]
    for b in ids:
        pairs += [(lambda b=b: iso.embed(x, b), lambda b=b: iso.embed(x, b, status=True)),
                  (lambda b=b: iso.embed_grad(x, b, 9), lambda b=b: iso.embed_grad(x, b, 9, status=True))]
    for b in [torch.float16, 5]:
        pairs += [(lambda b=b: iso.embed(x, i8, dtype=b), lambda b=b: iso.embed(x, i8, dtype=b, status=True)),
                  (lambda b=b: iso.act_wgrad(x, p, dtype=b), lambda b=b: iso.act_wgrad(x, p, dtype=b, status=True)),
                  (lambda b=b: iso.embed_grad(x, i8, 9, dtype=b), lambda b=b: iso.embed_grad(x, i8, 9, dtype=b, status=True))]
    for kw in [dict(pad_id=1 << 63), dict(pad_id="a"), dict(scale=float("inf")), dict(scale=1e39), dict(scale=None)]:
        pairs += [(lambda kw=kw: iso.embed(x, i8, **kw), lambda kw=kw: iso.embed(x, i8, status=True, **kw)),
                  (lambda kw=kw: iso.embed_grad(x, i8, 9, **kw), lambda kw=kw: iso.embed_grad(x, i8, 9, status=True, **kw))]
    pairs += [(lambda: iso.embed_grad(x, i8, -1), lambda: iso.embed_grad(x, i8, -1, status=True)),
              (lambda: iso.embed_grad(x, i8[:5], 9), lambda: iso.embed_grad(x, i8[:5], 9, status=True)),
              (lambda: iso.act_wgrad(x[:7], p), lambda: iso.act_wgrad(x[:7], p, status=True)),
              (lambda: iso.act_wgrad(x, x), lambda: iso.act_wgrad(x, x, status=True)),
              (lambda: iso.swiglu_pack(x, x.float()), lambda: iso.swiglu_pack(x, x.float(), out=out)),
              (lambda: iso.swiglu_grad(x[:, :32], p, p), lambda: iso.swiglu_grad(x[:, :32], p, p, out=(out[:, :32], out[:, 32:]), need_h=False))]
    for n, (common, other) in enumerate(pairs):
        a, b = _refusal(common), _refusal(other)
        assert a is not None and a == b, (n, a, b)


def test_results_carry_no_graph():
    table, i8 = torch.nn.Parameter(_rand(61, 20, 64)), torch.arange(8, device=DEV)
    results = [iso.embed(table, i8), iso.embed(table, i8, status=True)[0], iso.act_unpack(iso.act_pack(table)),
               iso.swiglu_pack(table, table)[0], iso.act_wgrad(table, iso.act_pack(table)), iso.embed_grad(table[:8], i8, 20)]
    assert not any(t.requires_grad for t in results)
