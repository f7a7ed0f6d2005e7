"""C ABI and binding of the logits operators and the expert layer, checked
without a GPU: every refusal happens before any HIP call, so dummy pointers are
never followed."""

import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

from paper_2211_17111_amd import bevpool as bp
from paper_2211_17111_amd import build as b
from paper_2211_17111_amd import logits as lg
from paper_2211_17111_amd import rows

OK, EINVAL, EOVERFLOW, EDTYPE, EWORKSPACE = 0, -1, -2, -3, -4
P = 0x1000
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    rows.load_library()
    return lg.load_library()


def test_exports_every_declared_symbol(lib):
    header = os.path.join(os.path.dirname(bp.HEADER_PATH), "bevpool_logits.h")
    names = set(bp.declared_symbols(header))
    assert names == set(lg._ARGTYPES)
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_c():
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no host C compiler")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(bp.HEADER_PATH), "-x", "c", "-fsyntax-only",
                    "-"], input=b'#include "bevpool_logits.h"\n', check=True,
                   env={k: v for k, v in os.environ.items() if k != "LD_PRELOAD"})


def _sizes_refused(f):
    assert f(T=-1) == EINVAL
    assert f(T=1 << 31) == EOVERFLOW
    assert f(V=0, k=1) == EINVAL
    assert f(V=(1 << 20) + 1) == EOVERFLOW
    assert f(k=-1) == EINVAL
    assert f(V=5, k=6) == EINVAL
    assert f(dt=3) == EDTYPE
    assert f(dt=-1) == EDTYPE


def _rows_refused(f):
    _sizes_refused(f)
    assert f(stride=-1) == EINVAL
    for scale in (0.0, -1.0, float("inf"), float("nan"), 1e-60):  # (the last is 0 in float32)
        assert f(scale=scale) == EINVAL, scale
    assert f(kt=2) == EDTYPE
    assert f(x=None) == EINVAL


def test_logprobs_refusals(lib):
    n = ctypes.c_size_t()

    def size(T=4, V=100, k=3, dt=0, out=ctypes.byref(n)):
        return lib.bevpool_logprobs_workspace_size(T, V, k, dt, out)

    def fwd(T=4, V=100, k=3, dt=0, x=P, stride=100, scale=1.0, kt=0, ids=P, stats=P, lp=P, lse=P, h=P, top=P, ti=P, ws=P,
            wsb=1 << 40):
        return lib.bevpool_logprobs_forward(T, V, k, dt, x, stride, scale, kt, ids, stats, lp, lse, h, top, ti, ws, wsb,
                                            None)

    def bwd(T=4, V=100, k=3, dt=0, x=P, stride=100, scale=1.0, kt=0, ids=P, stats=P, h=P, ti=P, gl=P, gz=P, gh=P, gt=P,
            out=P):
        return lib.bevpool_logprobs_backward(T, V, k, dt, x, stride, scale, kt, ids, stats, h, ti, gl, gz, gh, gt, out,
                                             None)

    _sizes_refused(size)
    _rows_refused(fwd)
    _rows_refused(bwd)
    for f in (size, fwd, bwd):
        assert f(k=65) == EOVERFLOW
    assert size(out=None) == EINVAL
    assert size() == OK
    for name in ("ids", "stats", "top", "ti"):
        assert fwd(**{name: None}) == EINVAL, name
    for name in ("ids", "stats", "h", "ti", "out"):
        assert bwd(**{name: None}) == EINVAL, name
    none = dict(x=None, ids=None, stats=None, h=None, ti=None)
    assert fwd(T=0, lp=None, lse=None, top=None, ws=None, wsb=0, **none) == OK
    assert bwd(T=0, gl=None, gz=None, gh=None, gt=None, out=None, **none) == OK


def test_distill_refusals(lib):
    n = ctypes.c_size_t()

    def size(T=4, V=100, k=3, dt=0, out=ctypes.byref(n)):
        return lib.bevpool_distill_workspace_size(T, V, k, dt, out)

    def fwd(T=4, V=100, k=3, dt=0, x=P, stride=100, scale=1.0, kt=0, ids=P, q=P, loss=P, stats=P, ws=P, wsb=1 << 40):
        return lib.bevpool_distill_forward(T, V, k, dt, x, stride, scale, kt, ids, q, 1, loss, stats, ws, wsb, None)

    def bwd(T=4, V=100, k=3, dt=0, g=P, x=P, stride=100, scale=1.0, kt=0, ids=P, q=P, stats=P, out=P):
        return lib.bevpool_distill_backward(T, V, k, dt, g, x, stride, scale, kt, ids, q, 1, stats, out, None)

    def step(T=4, V=100, k=3, dt=0, g=P, x=P, stride=100, scale=1.0, kt=0, ids=P, q=P, loss=P, stats=P, out=P, ws=P,
             wsb=1 << 40):
        return lib.bevpool_distill_step(T, V, k, dt, g, x, stride, scale, kt, ids, q, 1, loss, stats, out, ws, wsb, None)

    _sizes_refused(size)
    for f in (fwd, bwd, step):
        _rows_refused(f)
        for name in ("ids", "q", "stats"):
            assert f(**{name: None}) == EINVAL, name
    for f in (size, fwd, bwd, step):
        assert f(k=0) == EINVAL
        assert f(V=1000, k=257) == EOVERFLOW
    for f in (fwd, step):
        assert f(loss=None) == EINVAL
    for f in (bwd, step):
        assert f(g=None) == EINVAL and f(out=None) == EINVAL
    assert size(out=None) == EINVAL
    assert size() == OK


def test_workspaces_are_checked(lib):
    """Where a call needs scratch, too little of it is refused."""
    n = ctypes.c_size_t()
    for T, V, k in ((1, 1 << 20, 64), (3, 200000, 5), (1000, 100, 2)):
        for dt in (0, 1, 2):
            assert lib.bevpool_logprobs_workspace_size(T, V, k, dt, ctypes.byref(n)) == OK
            if n.value:
                for ws, wsb in ((None, 1 << 40), (P, n.value - 1)):
                    assert lib.bevpool_logprobs_forward(T, V, k, dt, P, V, 1.0, 0, P, P, P, P, P, P, P, ws, wsb,
                                                        None) == EWORKSPACE
            assert lib.bevpool_distill_workspace_size(T, V, k, dt, ctypes.byref(n)) == OK
            if n.value:
                for ws, wsb in ((None, 1 << 40), (P, n.value - 1)):
                    assert lib.bevpool_distill_forward(T, V, k, dt, P, V, 1.0, 0, P, P, 1, P, P, ws, wsb,
                                                       None) == EWORKSPACE
                    assert lib.bevpool_distill_step(T, V, k, dt, P, P, V, 1.0, 0, P, P, 1, P, P, P, ws, wsb,
                                                    None) == EWORKSPACE


def test_expert_layer_refusals(lib):
    n = ctypes.c_size_t()

    def size(T=4, k=2, C=8, F=6, E=5, dt=0, out=ctypes.byref(n)):
        return lib.bevpool_expert_layer_workspace_size(T, k, C, F, E, dt, out)

    def fwd(T=4, k=2, C=8, F=6, E=5, dt=0, dw=0, x=P, stride=8, up=P, down=P, w=P, ids=P, out=P, ws=P, wsb=1 << 40):
        return lib.bevpool_expert_layer_forward(T, k, C, F, E, dt, dw, x, stride, up, down, w, ids, out, ws, wsb, None)

    for f in (size, fwd):
        assert f(T=-1) == EINVAL
        assert f(T=1 << 40) == EOVERFLOW
        assert f(T=513) == EOVERFLOW
        assert f(k=0) == EINVAL
        assert f(T=2, k=(1 << 31) - 1) == EOVERFLOW
        for name in ("C", "F"):
            assert f(**{name: 0}) == EINVAL
            assert f(**{name: (1 << 16) + 1}) == EOVERFLOW
        assert f(E=0) == EINVAL
        assert f(E=1025) == EOVERFLOW
        assert f(dt=3) == EDTYPE
    assert size(out=None) == EINVAL
    assert size(T=0) == OK and size(T=512) == OK and n.value >= 1024 * 6 * 4
    assert fwd(dt=1, dw=2) == EDTYPE
    assert fwd(dw=9) == EDTYPE
    assert fwd(stride=-1) == EINVAL
    for name in ("x", "up", "down", "w", "ids", "out"):
        assert fwd(**{name: None}) == EINVAL, name
    assert fwd(ws=None) == EWORKSPACE
    assert fwd(wsb=8) == EWORKSPACE
    assert fwd(T=0, x=None, up=None, down=None, w=None, ids=None, out=None) == OK


def test_binding_refuses_cpu_tensors():
    x, ids, g = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4)
    r = lg.Logprobs(None, g, None, None, None, torch.zeros(4, 2))
    for call in (lambda: lg.logprobs_forward(x), lambda: lg.logprobs_backward(x, r, grad_lse=g), lambda: lg.logprobs(x),
                 lambda: lg.distill_forward(x, ids, torch.zeros(4, 2)), lambda: lg.distill(x, ids, torch.zeros(4, 2)),
                 lambda: lg.distill_backward(g, x, ids, torch.zeros(4, 2), torch.zeros(4, 2)),
                 lambda: lg.distill_step(g, x, ids, torch.zeros(4, 2)),
                 lambda: rows.expert_layer_forward(x, torch.zeros(3, 10, 8), torch.zeros(3, 8, 5), torch.zeros(4, 2), ids)):
        with pytest.raises(ValueError):
            call()


def test_teacher_that_needs_a_gradient_is_refused():
    with pytest.raises(ValueError):
        lg.distill(torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2, requires_grad=True))


@pytest.mark.skipif("BEVPOOL_LIBRARY" in os.environ, reason="runs the others under the sanitizers itself")
def test_validation_under_sanitizers():
    """The checks above with AddressSanitizer and UndefinedBehaviorSanitizer on the host code."""
    library, runtime = b.build_sanitized(), b.sanitizer_runtime()
    env = dict(os.environ, LD_PRELOAD=runtime, BEVPOOL_LIBRARY=library, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "not gpu", "-p", "no:cacheprovider",
                          os.path.join(ROOT, "tests", "test_logits_abi.py")], cwd=ROOT, env=env, stdout=subprocess.PIPE,
                         stderr=subprocess.STDOUT, text=True, timeout=900)
    out = res.stdout
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert res.returncode == 0 and " passed" in out, out[-4000:]


def test_scales_whose_exponents_overflow_are_refused(lib):
    """scale log2 e has to be finite in float32; the largest such scale and the smallest number are taken."""
    def calls(scale):
        rows = (0, 100, 3, 0)
        at = (P, 100, scale, 0, P)
        yield lib.bevpool_logprobs_forward(*rows, *at, P, P, P, P, P, P, None, 0, None)
        yield lib.bevpool_logprobs_backward(*rows, *at, P, P, P, P, P, P, P, P, None)
        yield lib.bevpool_distill_forward(*rows, *at, P, 1, P, P, None, 0, None)
        yield lib.bevpool_distill_backward(*rows, P, *at, P, 1, P, P, None)
        yield lib.bevpool_distill_step(*rows, P, *at, P, 1, P, P, P, None, 0, None)

    for scale in (2.36e38, 3.4e38):
        assert list(calls(scale)) == [EINVAL] * 5, scale
    for scale in (2.35e38, 2.0 ** 127, 1e-45):
        assert list(calls(scale)) == [OK] * 5, scale
