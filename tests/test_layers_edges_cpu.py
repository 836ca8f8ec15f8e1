"""Host-only checks of distillation's workspace, of overlapping arguments and of how the operators are reached, without touching a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2509_11254_b200 import binding, build

    build.build_library()
    return binding.lib()


def test_distillation_workspace_is_bounded_in_entries(L):
    """Beside what the cross entropy of the same size holds and 8 bytes per token: the entries of a piece (16 bytes each) and its blocks of 32 rows and 32 columns, within a fixed size
    however many tokens there are and however long their lists."""
    a, b = C.c_size_t(), C.c_size_t()
    for grad in (0, 1):
        for T in (1 << 14, 1 << 17, 1 << 20, 1 << 24):
            for V in (40, 1000, 32000, 131072):
                for K in (1, 64, 1000, 1024):
                    assert L.psgd_distill_workspace(T, V, 64, K, grad, C.byref(a)) == 0 and L.psgd_xent_workspace(T, V, 64, grad, C.byref(b)) == 0
                    # (4 bytes per block of at most 2^32 logits, 4 per token of a piece, float32 sums of the weight gradient once there are several pieces, partial tiles)
                    assert a.value <= b.value + 8 * T + (1 << 30) + 4 * (1 << 22) + (1 << 27) + 4 * min(T, 1 << 25) + 4 * V * 64 + (1 << 26), (T, V, K, grad)


P, STEP = 1 << 32, 1 << 30         # made-up device addresses, far apart: only refusals are looked at where there is a GPU


def launches(code):
    """What a call answers that got as far as a launch on a machine without a GPU."""
    return code == -4


def over(places, out, fixed=()):
    """Every way to put the outputs `out` of {name: (address, bytes)} over another place: over its beginning, its last bytes, and so that it begins within."""
    for name in out:
        for other, (at, size) in places.items():
            if other == name or (name, other) in fixed or (other, name) in fixed:
                continue
            mine = places[name][1]
            for to in {at, at + size - 16, at - mine + 16}:
                yield name, other, (to + 15) // 16 * 16


def test_norm_outputs_over_anything_are_refused(L):
    """Vectors and the 8-bit form as well as matrices, T = 8 rows of 64."""
    import torch

    gpu = torch.cuda.is_available()
    size = dict(x=1024, r=1024, w=256, b=256, s=1024, y=1024, mean=32, rstd=32, q=512, scales=16)
    at = {k: (P + i * STEP, n) for i, (k, n) in enumerate(size.items())}

    def forward(**kw):
        p = {k: kw.get(k, v[0]) for k, v in at.items()}
        return L.psgd_norm_forward(p["x"], 64, 1, p["r"], 64, p["w"], p["b"], 0, 1e-5, 1, 8, 64, p["s"], 64, p["y"], 64, 1, p["mean"], p["rstd"], p["q"], p["scales"], None)

    assert gpu or launches(forward())
    for name, other, to in over(at, ("s", "y", "mean", "rstd", "q", "scales")):
        assert forward(**{name: to}) == -1, (name, other)
    n = C.c_size_t()
    assert L.psgd_norm_workspace(8, 64, C.byref(n)) == 0
    size = dict(dy=1024, x=1024, w=256, mean=32, rstd=32, add=1024, dx=1024, dw=256, db=256, ws=512)        # (of the workspace at least two sums per column are used)
    back = {k: (P + i * STEP, m) for i, (k, m) in enumerate(size.items())}

    def backward(**kw):
        p = {k: kw.get(k, v[0]) for k, v in back.items()}
        return L.psgd_norm_backward(p["dy"], 64, 1, p["x"], 64, 1, p["w"], 0, p["mean"], p["rstd"], p["add"], 64, 8, 64, p["dx"], 64, p["dw"], p["db"], p["ws"] // 256 * 256, n.value, None)

    assert gpu or launches(backward())
    for name, other, to in over(back, ("dx", "dw", "db")):
        assert backward(**{name: to}) == -1, (name, other)
    for other, (to, _) in back.items():
        assert other == "ws" or backward(ws=to) == -1, other


def test_rotary_outputs_over_angles_are_refused(L):
    import torch

    size = dict(q=4096, k=4096, oq=4096, ok=4096, positions=64, frequencies=256)      # 8 tokens of 4 heads of 64 values
    at = {k: (P + i * STEP, n) for i, (k, n) in enumerate(size.items())}

    def call(**kw):
        p = {k: kw.get(k, v[0]) for k, v in at.items()}
        return L.psgd_rotary(p["q"], 256, 64, 4, p["oq"], 256, 64, p["k"], 256, 64, 4, p["ok"], 256, 64, p["positions"], p["frequencies"], 8, 64, 64, 0, 0, 1.0, 1, None)

    assert torch.cuda.is_available() or launches(call())
    for name, other, to in over(at, ("oq", "ok"), fixed=(("oq", "q"), ("ok", "k"))):
        assert call(**{name: to}) == -1, (name, other)


def test_gradients_over_labels_and_weights_are_refused(L):
    """They are read for later pieces of the tokens after earlier ones' gradients are written."""
    import torch

    T, V, D, K = 8, 40, 64, 16
    size = dict(H=T * D * 2, W=V * D * 2, labels=T * 8, weight=T * 4, logits=T * K * 4, index=T * K * 8, dH=T * D * 2, dW=V * D * 2)
    at = {k: (P + i * STEP, n) for i, (k, n) in enumerate(size.items())}
    free = P + 20 * STEP
    n = C.c_size_t()

    def xent(**kw):
        p = {k: kw.get(k, v[0]) for k, v in at.items()}
        assert L.psgd_xent_workspace(T, V, D, 1, C.byref(n)) == 0
        return L.psgd_xent_grad(p["H"], D, p["W"], D, p["labels"], p["weight"], -100, T, V, D, free, free + 256, free + 512, p["dH"], D, p["dW"], D, None, free + 4096, n.value, None)

    def distill(**kw):
        p = {k: kw.get(k, v[0]) for k, v in at.items()}
        assert L.psgd_distill_workspace(T, V, D, K, 1, C.byref(n)) == 0
        return L.psgd_distill_grad(p["H"], D, p["W"], D, p["logits"], K, 0, p["index"], K, K, 1.0, p["weight"], T, V, D, free, free + 256, free + 512, p["dH"], D, p["dW"], D, None,
                                   free + 4096, n.value, None)

    assert torch.cuda.is_available() or launches(xent()) and launches(distill())
    for call, unused in ((xent, ("logits", "index")), (distill, ("labels",))):
        for name, other, to in over({k: v for k, v in at.items() if k not in unused}, ("dH", "dW")):
            assert call(**{name: to}) == -1, (name, other)


# ---- how the operators are built and reached ----------------------------------------------------------------------
class Compilers:
    """In the place of subprocess.Popen: writes what a compiler would write (of _call.so, what it was compiled against), or fails; keeps the commands."""

    def __init__(self, works):
        self.works, self.commands = works, []

    def __call__(self, command, **kw):
        import types

        self.commands.append(command)
        works = self.works(command)
        if works is None:
            raise FileNotFoundError(command[0])
        if works:
            from paper_2509_11254_b200 import build

            with open(command[command.index("-o") + 1], "w") as f:
                f.write(build.call_tag() + "\0" if command[0] == "cxx" else "")
        return types.SimpleNamespace(communicate=lambda: ("said", None), returncode=0 if works else 1)


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    from paper_2509_11254_b200 import build

    for name in ("LIB", "CALL", "OBJ_DIR"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    return build


def test_library_needs_nvcc_alone(elsewhere, monkeypatch):
    """Without torch, and where the C++ compiler of _call.so is missing or fails, the library is built all the same."""
    import os

    b = elsewhere
    monkeypatch.setattr(b, "nvcc_path", lambda: "nvcc")
    monkeypatch.setenv("CXX", "cxx")
    with monkeypatch.context() as m:
        run = Compilers(lambda c: True)
        m.setattr(b.subprocess, "Popen", run)
        m.setattr(b.importlib.util, "find_spec", lambda name: None)
        assert b.needs_build() and b.build_library() == b.LIB and os.path.exists(b.LIB) and not os.path.exists(b.CALL)
        assert len(run.commands) == len(b.SRCS) + 1 and all(c[0] == "nvcc" for c in run.commands)
        assert not b.needs_build()
    for works in (None, False):
        os.remove(b.LIB)
        with monkeypatch.context() as m:
            m.setattr(b.subprocess, "Popen", Compilers(lambda c: True if c[0] == "nvcc" else works))
            with pytest.warns(RuntimeWarning, match="_call.so could not be built"):
                assert b.build_library() == b.LIB
            assert os.path.exists(b.LIB) and not os.path.exists(b.CALL)
            # the library is there: only the other one is tried again
            again = Compilers(lambda c: True)
            m.setattr(b.subprocess, "Popen", again)
            b.build_library()
            assert os.path.exists(b.CALL) and all(c[0] == "cxx" for c in again.commands) and not b.needs_build()
            os.remove(b.CALL)
    with monkeypatch.context() as m:
        m.setattr(b.subprocess, "Popen", Compilers(lambda c: c[0] != "nvcc"))
        with pytest.raises(RuntimeError, match="nvcc failed"):
            b.build_library(force=True)


def test_operators_do_without_the_short_way(monkeypatch, tmp_path):
    """_call.so missing, compiled against another torch, or impossible to load: a warning, once, and the calls that there are without it."""
    import sys
    import types
    import warnings

    import torch

    import paper_2509_11254_b200 as p
    from paper_2509_11254_b200 import build, training

    build.build_library()
    x, w, at = torch.zeros(4, 8), torch.ones(8), torch.arange(4)
    h, z, i = x.bfloat16(), x[:, :2].contiguous(), torch.zeros(4, 2, dtype=torch.int64)
    calls = [lambda: p.layer_norm_forward(x, w), lambda: p.layer_norm_backward(x, x, w, None, x[:, 0]), lambda: p.rotary_forward(x.view(4, 1, 8), None, at, p.rotary_frequencies(8, device="cpu")),
             lambda: p.linear_distillation(h, h, z, i), lambda: p.linear_distillation_grad(h, h, z, i)]

    def without():
        monkeypatch.setattr(training, "_call", None)
        with pytest.warns(RuntimeWarning, match="_call.so cannot be used") as seen:
            for call in calls:
                with pytest.raises(p.PSGDError, match="must be a CUDA tensor"):
                    call()
        assert len(seen) == 1 and seen[0].filename == __file__

    tag, data = build.call_tag().encode(), open(build.CALL, "rb").read()
    assert torch.__version__ in build.call_tag() and build.call_fits()
    other = tmp_path / "_call.so"
    monkeypatch.setattr(build, "CALL", str(other))
    assert not build.call_fits() and build.needs_call()
    without()
    other.write_bytes(data.replace(tag, tag.replace(b"torch 2", b"torch 1")))
    assert not build.call_fits() and build.needs_call()
    without()
    other.write_bytes(data)
    assert build.call_fits() and not build.needs_call()
    monkeypatch.setitem(sys.modules, "paper_2509_11254_b200._call", None)
    monkeypatch.delattr(p, "_call", raising=False)
    without()
    monkeypatch.undo()
    monkeypatch.setattr(training, "_call", None)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert isinstance(training._plain(), types.ModuleType)


def test_no_exception_leaves_where_a_kernel_is_opted_in(tmp_path):
    """C entry points raise the shared memory of their kernels on the way: a failed allocation there must not end the process."""
    import os
    import subprocess

    from paper_2509_11254_b200 import build

    src = tmp_path / "new.cpp"
    src.write_text("""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "psgd_host.cuh"
static bool full = false;
static int asked = 0;
void* operator new(size_t n) {
    if (full) { ++asked; throw std::bad_alloc(); }
    return malloc(n);
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }
int main() {
    static int kernel;
    set_smem_attr(&kernel, 1 << 16);
    full = true;
    static int other;
    set_smem_attr(&other, 1 << 16);
    full = false;
    printf("asked %d\\n", asked);
}
""")
    cuda = os.path.dirname(os.path.dirname(build.nvcc_path()))
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(os.path.dirname(build.__file__), "csrc"), "-I" + os.path.join(cuda, "include"), "-o", str(tmp_path / "new"), str(src),
                    "-L" + os.path.join(cuda, "lib64"), "-lcudart", "-Wl,-rpath," + os.path.join(cuda, "lib64")], check=True, capture_output=True)
    r = subprocess.run([str(tmp_path / "new")], capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout.split()[1]) > 0
