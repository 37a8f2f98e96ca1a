"""Host side of the training-step binding, without a GPU: what a call does
around the library, against a fake of the library's entry points."""
import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_2607_19331_gb300 as iso
from paper_2607_19331_gb300 import _abi, train
from paper_2607_19331_gb300._abi import IsoMat

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def on_host(monkeypatch):
    """CPU tensors pass as the binding's matrices and ids; returns the function
    that puts a fake in the library's place."""
    def mat(t, name):
        return IsoMat(t.data_ptr(), t.shape[0], t.shape[1], t.stride(0), train._CODES[t.dtype], 0)
    monkeypatch.setattr(train, "_mat", mat)
    monkeypatch.setattr(train, "_here", lambda *t: 7)
    monkeypatch.setattr(train, "_ids", lambda ids: (ids.data_ptr(), 1, ids.numel()))
    monkeypatch.setattr(train, "embed_grad_workspace_size", lambda n, cols: 4096)
    return lambda fake: monkeypatch.setattr(train, "lib", lambda: fake)


class FakeLibrary:
    """Records the scratch that each call is given; with ``calls`` of two, the
    first call waits inside the library until the second one is inside too."""

    def __init__(self, calls=1):
        self.scratch, self.both = [], threading.Barrier(calls, timeout=20)

    def iso_act_wgrad_workspace_size(self, dy, pack, out, nb):
        nb._obj.value = 4096
        return _abi.ISO_OK

    def _inside(self, ptr, size):
        if size < 4096:
            return _abi.ISO_ERR_WORKSPACE
        self.scratch.append((ptr.value, ptr.value + 4096))
        self.both.wait()
        return _abi.ISO_OK

    def iso_act_wgrad(self, dy, pack, out, acc, ptr, size, status, stream):
        return self._inside(ptr, size)

    def iso_embed_grad(self, dy, ids, i64, pad, scale, grad, acc, ptr, size, status, stream):
        return self._inside(ptr, size)


@pytest.mark.parametrize("name", ["act_wgrad", "embed_grad"])
def test_calls_of_two_threads_on_one_stream_do_not_share_scratch(on_host, name):
    dy, out, ids = torch.zeros(40, 8), torch.zeros(8, 64), torch.zeros(40, dtype=torch.int64)
    buf = torch.zeros(40 * 72, dtype=torch.uint8)
    pack = iso.ActPack._of((buf, buf.data_ptr(), buf.data_ptr() + 40 * 64, 40, 64, 64, 8), BF)
    grad, failed = torch.zeros(9, 8), []

    def call():
        try:
            if name == "act_wgrad":
                iso.act_wgrad(dy, pack, out=out, accumulate=True)
            else:
                iso.embed_grad(dy, ids, out=grad, accumulate=True)
        except BaseException as e:        # noqa: BLE001
            failed.append(e)
    on_host(FakeLibrary())
    call()                                # what a first call keeps, if it keeps anything
    fake = FakeLibrary(calls=2)
    on_host(fake)
    threads = [threading.Thread(target=call) for _ in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed
    (a0, a1), (b0, b1) = fake.scratch
    assert a1 <= b0 or b1 <= a0


def test_a_call_leaves_no_scratch_behind(on_host, monkeypatch):
    """Scratch that outlives its call would be written by the replay of a graph
    that captured the call, whoever has the memory by then."""
    import weakref
    made, real = [], train.Workspace

    class Recorded(real):
        def __init__(self, device=None):
            super().__init__(device)
            made.append(weakref.ref(self))
    monkeypatch.setattr(train, "Workspace", Recorded)
    on_host(FakeLibrary())
    iso.embed_grad(torch.zeros(40, 8), torch.zeros(40, dtype=torch.int64), out=torch.zeros(9, 8))
    assert len(made) == 1 and made[0]() is None
    mine = Recorded("cpu")                # the caller's own is used as it is
    iso.embed_grad(torch.zeros(40, 8), torch.zeros(40, dtype=torch.int64), out=torch.zeros(9, 8), workspace=mine)
    assert len(made) == 2 and mine.buf.numel() >= 4096


CLOCK = r"""
#include <cstdio>
#include "iso_train.cuh"
int main() {
    const uint64_t MS = 1000000, LIMIT = 2000 * MS;
    int bad = 0;
    {   // a minute away between two looks, and again
        iso::WaitClock c;
        bad |= c.look(5, LIMIT);
        for (int i = 1; i <= 50; ++i) bad |= c.look(5 + i * 60000 * MS, LIMIT);
    }
    {   // looks a millisecond apart: the limit is reached after 2 s and not before
        iso::WaitClock c;
        for (int i = 0; i <= 2000; ++i) bad |= c.look(7 + i * MS, LIMIT);
        bad |= !c.look(7 + 2001 * MS, LIMIT) << 1;
    }
    {   // always away: the wait still ends
        iso::WaitClock c;
        int looks = 0;
        while (looks < 1000 && !c.look(1 + (uint64_t)looks * 1000 * MS, LIMIT)) ++looks;
        bad |= (looks >= 1000) << 2;
    }
    std::printf("%d\n", bad);
    return bad;
}
"""


def test_a_wait_does_not_count_the_time_another_process_had_the_gpu(tmp_path):
    from paper_2607_19331_gb300 import build
    (tmp_path / "clock.cu").write_text(CLOCK)
    exe = str(tmp_path / "clock")
    subprocess.run([build.nvcc(), *build.ARCH, *build.FLAGS, "-o", exe, str(tmp_path / "clock.cu")], check=True)
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


SMALL_GPU = r"""
extern "C" int cudaGetDevice(int* d) { *d = 0; return 0; }
extern "C" int cudaDeviceGetAttribute(int* v, int, int) { *v = 20; return 0; }
"""
SIZES = """
import ctypes, sys
L = ctypes.CDLL(sys.argv[1])
nb = ctypes.c_size_t()
for n, cols in ((33, 64), (4097, 72), (32768, 3584), (300000, 1536)):
    assert L.iso_embed_grad_workspace_size(ctypes.c_int64(n), ctypes.c_int64(cols), ctypes.byref(nb)) == 0
    print(nb.value)
"""


def test_the_embedding_gradients_windows_depend_on_the_sizes_alone(tmp_path):
    """The order of its sums is that of its windows, and its workspace holds two
    rows a window: the same on a device that reports 20 SMs."""
    from paper_2607_19331_gb300 import build
    lib = build.build()
    (tmp_path / "gpu.cpp").write_text(SMALL_GPU)
    shim = str(tmp_path / "gpu.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-o", shim, str(tmp_path / "gpu.cpp")], check=True)

    def sizes(**env):
        run = subprocess.run([sys.executable, "-c", SIZES, lib], capture_output=True, text=True,
                             env={**os.environ, **env}, check=True)
        return run.stdout.split()
    here = sizes()
    assert len(here) == 4 and sizes(LD_PRELOAD=shim) == here


@pytest.fixture
def fake_build(monkeypatch, tmp_path):
    """build.build() with a recorder in the compilers' place; a command whose
    text holds ``fails`` fails."""
    from paper_2607_19331_gb300 import build
    ran, state = [], {"fails": None}

    def run(cmd, **kw):
        ran.append(cmd)
        if state["fails"] and any(state["fails"] in c for c in cmd):
            return subprocess.CompletedProcess(cmd, 1, "", "no")
        out = cmd[cmd.index("-o") + 1]
        with open(out, "w"):
            pass
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build.subprocess, "check_call", lambda cmd: run(cmd))
    for name in ("LIB", "BINDING", "STAMP"):
        if hasattr(build, name):
            monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    return build, ran, state


def test_the_library_builds_without_torch(fake_build, monkeypatch):
    build, ran, _ = fake_build
    monkeypatch.setitem(sys.modules, "torch", None)
    assert os.path.exists(build.build())
    assert all("nvcc" in cmd[0] for cmd in ran) and not os.path.exists(build.BINDING)


def test_the_library_is_there_when_the_host_module_fails(fake_build):
    build, ran, state = fake_build
    state["fails"] = "train_binding.cpp"
    with pytest.raises(RuntimeError, match="compilation failed"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.BINDING)


def test_the_host_module_follows_the_torch(fake_build, monkeypatch):
    build, ran, _ = fake_build
    build.build()
    n = len(ran)
    build.build()
    assert len(ran) == n                                  # nothing to do
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    build.build()
    assert len(ran) == n + 2                              # its compilation and link, nothing else
    build.build()
    assert len(ran) == n + 2


def test_a_host_module_of_another_torch_is_not_loaded(monkeypatch):
    from paper_2607_19331_gb300 import build
    build.build()
    monkeypatch.setattr(train, "_native", None)
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    with pytest.raises(RuntimeError, match="9.9.9"):
        train._load_native()
    assert train._native is None
