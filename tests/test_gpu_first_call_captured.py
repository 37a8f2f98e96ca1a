"""A process whose first call of each operator between the embedding and the loss is
captured into a graph: what a kernel is given once (shared memory, cluster counts) is
given then too."""
import subprocess
import sys
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PROGRAM = """
import torch
import paper_2607_19331_gb300 as iso
torch.cuda.set_device(0)
dev = "cuda:0"
g = torch.Generator(dev).manual_seed(1)
rand = lambda *s, dtype=torch.bfloat16: torch.randn(*s, generator=g, device=dev).to(dtype)
q, k, v, do = rand(300, 512), rand(300, 256), rand(300, 256), rand(300, 512)
w = [x.float() for x in (q, k, v, do)]
many = rand(2500, 32000), rand(1300, 152064), rand(700, 16000, dtype=torch.float32), rand(9, 5000)
ids = [torch.randint(0, z.shape[1], (z.shape[0], 8), generator=g, device=dev) for z in many]
t = [rand(z.shape[0], 8) for z in many]
d = [rand(z.shape[0], dtype=torch.float32) for z in many]
aside = torch.empty(9, 5003, dtype=torch.bfloat16, device=dev)
pos, plan = torch.arange(300, device=dev), iso.rope_plan(128)


def calls():
    r = [iso.rope(q, pos, plan), iso.rope(w[0], pos, plan)]
    for a, b, c, e in ((q, k, v, do), w):
        o, l = iso.attn(a, b, c, 4, 2)
        r += [o, l, *iso.attn_grad(e, a, b, c, o, l, 4, 2)]
    r += iso.attn(q[:1], many[0].view(-1)[:250000 * 128].view(-1, 128)[:9000].repeat(1, 2), many[0].view(-1)[:9000 * 256].view(-1, 256), 4, 2)
    for z, i, x, y in zip(many, ids, t, d):
        loss, lse, grad = iso.distill(z, i, x, dloss=y)
        r += [loss, lse, grad, iso.distill_grad(y, z, i, x, lse)]
    return r + list(iso.distill(many[3], ids[3], t[3], dloss=d[3], out=aside[:, 3:]))


s = torch.cuda.Stream()
with torch.cuda.stream(s):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held = calls()
    graph.replay()
torch.cuda.synchronize()
held = [x.clone() for x in held]
assert all(torch.equal(a, b) for a, b in zip(held, calls())) and all(bool(torch.isfinite(a).all()) for a in held)
print("captured first")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "captured first" in p.stdout, p.stdout + p.stderr
