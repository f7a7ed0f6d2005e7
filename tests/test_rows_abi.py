"""C ABI and binding of the row operators, checked without a GPU: every
refusal happens before any HIP call, so dummy pointers are never followed."""

import ctypes

import pytest
import torch

from paper_2211_17111_amd import bevpool as bp
from paper_2211_17111_amd import rows

OK, EINVAL, EOVERFLOW, EDTYPE, EWORKSPACE = 0, -1, -2, -3, -4
P = 0x1000
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return rows.load_library()


def test_exports_every_declared_symbol(lib):
    import os
    header = os.path.join(os.path.dirname(bp.HEADER_PATH), "bevpool_rows.h")
    names = set(bp.declared_symbols(header))
    assert names == set(rows._ARGTYPES)
    for n in names:
        assert hasattr(lib, n), n


def test_header_is_c():
    """The header compiles as C and its constants are the binding's."""
    import os
    import re
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no host C compiler")
    inc = os.path.dirname(bp.HEADER_PATH)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", inc, "-x", "c", "-fsyntax-only", "-"],
                   input=b'#include "bevpool_rows.h"\n', check=True,
                   env={k: v for k, v in os.environ.items() if k != "LD_PRELOAD"})
    text = open(os.path.join(inc, "bevpool_rows.h")).read()
    assert int(re.search(r"#define BEVPOOL_BF16 (\d+)", text).group(1)) == rows.BEVPOOL_BF16
    for name in ("BEVPOOL_KEY_I32", "BEVPOOL_KEY_I64"):
        assert int(re.search(name + r" = (\d+)", text).group(1)) == getattr(rows, name)


def _sort(lib, n=100, n_keys=8, kt=0, keys=P, order=P, position=P, offsets=P, ws=P, wsb=1 << 30):
    return lib.bevpool_sort_keys(n, n_keys, kt, keys, order, position, offsets, ws, wsb, None)


def test_sort_keys_refusals(lib):
    assert _sort(lib, n=-1) == EINVAL
    assert _sort(lib, n=1 << 31) == EOVERFLOW
    assert _sort(lib, n_keys=0) == EINVAL
    assert _sort(lib, n_keys=(1 << 31) - 1) == EOVERFLOW
    assert _sort(lib, kt=2) == EDTYPE
    for name in ("keys", "order", "position", "offsets"):
        assert _sort(lib, **{name: None}) == EINVAL
        assert name.encode() in lib.bevpool_last_error()
    assert _sort(lib, n=100000, ws=None) == EWORKSPACE
    assert _sort(lib, n=100000, wsb=8) == EWORKSPACE
    n = ctypes.c_size_t()
    assert lib.bevpool_sort_keys_workspace_size(10, 10, None) == EINVAL
    assert lib.bevpool_sort_keys_workspace_size(-1, 10, ctypes.byref(n)) == EINVAL
    assert lib.bevpool_sort_keys_workspace_size(0, 10, ctypes.byref(n)) == OK and n.value == 0
    assert lib.bevpool_sort_keys_workspace_size((1 << 31) - 1, (1 << 31) - 2, ctypes.byref(n)) == OK
    assert n.value > 4 * 4 * ((1 << 31) - 1)  # two buffers of keys and slots


def test_route_refusals(lib):
    def fwd(T=4, E=8, k=2, dt=0, logits=P, stride=8, w=P, ids=P):
        return lib.bevpool_route_forward(T, E, k, dt, logits, stride, 1, w, ids, None)

    def bwd(T=4, E=8, k=2, dt=0, g=P, logits=P, stride=8, w=P, ids=P, re=0, out=P):
        return lib.bevpool_route_backward(T, E, k, dt, g, logits, stride, w, ids, re, out, None)

    for f in (fwd, bwd):
        assert f(T=-1) == EINVAL
        assert f(T=1 << 31) == EOVERFLOW
        assert f(T=1 << 30, k=2) == EOVERFLOW
        assert f(E=0, k=1) == EINVAL
        assert f(E=1025) == EOVERFLOW
        assert f(k=0) == EINVAL
        assert f(k=9) == EINVAL
        assert f(E=200, k=65) == EOVERFLOW
        assert f(dt=3) == EDTYPE
        assert f(dt=-1) == EDTYPE
        assert f(stride=-1) == EINVAL
        assert f(logits=None) == EINVAL
        assert f(w=None) == EINVAL
        assert f(ids=None) == EINVAL
    assert bwd(g=None) == EINVAL
    assert bwd(out=None) == EINVAL


def test_dispatch_refusals(lib):
    def fwd(T=4, k=2, C=8, K=5, dt=0, x=P, stride=8, kt=0, ids=P, order=P, pos=P, off=P, out=P, ws=P, wsb=1 << 30):
        return lib.bevpool_dispatch_forward(T, k, C, K, dt, x, stride, kt, ids, order, pos, off, out, ws, wsb, None)

    def rows_(T=4, k=2, C=8, dt=0, x=P, stride=8, pos=P, kept=P, out=P):
        return lib.bevpool_dispatch_rows(T, k, C, dt, x, stride, pos, kept, out, None)

    def bwd(T=4, k=2, C=8, dt=0, x=P, stride=8, pos=P, kept=P, out=P):
        return lib.bevpool_dispatch_backward(T, k, C, dt, x, stride, pos, kept, out, None)

    for f in (fwd, rows_, bwd):
        assert f(T=-1) == EINVAL
        assert f(T=1 << 31) == EOVERFLOW
        assert f(T=BIG) == EOVERFLOW
        assert f(T=1 << 29, k=8) == EOVERFLOW
        assert f(k=0) == EINVAL
        assert f(C=0) == EINVAL
        assert f(C=(1 << 20) + 1) == EOVERFLOW
        assert f(dt=3) == EDTYPE
        assert f(stride=-8) == EINVAL
        for name in ("x", "pos", "out"):
            assert f(**{name: None}) == EINVAL, name
    for name in ("ids", "order", "off"):
        assert fwd(**{name: None}) == EINVAL, name
    assert fwd(K=0) == EINVAL
    assert fwd(kt=7) == EDTYPE
    assert fwd(T=100000, ws=None) == EWORKSPACE
    assert fwd(T=100000, wsb=1) == EWORKSPACE
    assert rows_(kept=None) == EINVAL
    assert bwd(kept=None) == EINVAL


def test_combine_refusals(lib):
    def fwd(T=4, k=2, C=8, di=0, do=0, dw=0, x=P, stride=8, w=P, pos=P, kept=P, out=P):
        return lib.bevpool_combine_forward(T, k, C, di, do, dw, x, stride, w, pos, kept, out, None)

    def bwd(T=4, k=2, C=8, di=0, do=0, dw=0, g=P, gs=8, x=P, stride=8, w=P, pos=P, kept=P, gi=P, gw=P):
        return lib.bevpool_combine_backward(T, k, C, di, do, dw, g, gs, x, stride, w, pos, kept, gi, gw, None)

    for f in (fwd, bwd):
        assert f(T=-1) == EINVAL
        assert f(T=1 << 31) == EOVERFLOW
        assert f(k=-2) == EINVAL
        assert f(C=0) == EINVAL
        assert f(di=3) == EDTYPE
        assert f(do=1) == EDTYPE               # float32 in, float16 out
        assert f(di=1, do=2) == EDTYPE
        assert f(di=1, dw=2) == EDTYPE
        assert f(dw=5) == EDTYPE
        assert f(stride=-1) == EINVAL
        for name in ("x", "w", "pos", "kept"):
            assert f(**{name: None}) == EINVAL, name
    assert fwd(out=None) == EINVAL
    assert bwd(g=None) == EINVAL
    assert bwd(gs=-1) == EINVAL
    # no output wanted, or no rows: nothing to do, and nothing is launched
    assert bwd(gi=None, gw=None, x=None, w=None) == OK
    assert bwd(T=0, g=None, x=None, w=None, pos=None, kept=None, gi=None, gw=None) == OK
    assert fwd(T=0, x=None, w=None, pos=None, kept=None, out=None) == OK


def test_embed_refusals(lib):
    def fwd(n=4, V=10, C=8, di=0, do=0, t=P, stride=8, kt=1, ids=P, out=P):
        return lib.bevpool_embed_forward(n, V, C, di, do, t, stride, kt, ids, 1.0, out, None)

    def bwd(n=4, V=10, C=8, di=0, do=0, t=P, stride=8, kt=1, ids=P, out=P, ws=P, wsb=1 << 30):
        return lib.bevpool_embed_backward(n, V, C, di, do, t, stride, kt, ids, 1.0, out, ws, wsb, None)

    for f in (fwd, bwd):
        assert f(n=-1) == EINVAL
        assert f(n=1 << 31) == EOVERFLOW
        assert f(V=0) == EINVAL
        assert f(V=BIG) == EOVERFLOW
        assert f(C=0) == EINVAL
        assert f(C=1 << 21) == EOVERFLOW
        assert f(di=4) == EDTYPE
        assert f(do=4) == EDTYPE
        assert f(di=1, do=2) == EDTYPE
        assert f(kt=2) == EDTYPE
        assert f(stride=-1) == EINVAL
        for name in ("t", "ids", "out"):
            assert f(**{name: None}) == EINVAL, name
    assert fwd(do=1) == EDTYPE  # (the gradient may be narrower than a float32 grad_out)
    assert bwd(ws=None) == EWORKSPACE
    assert bwd(wsb=16) == EWORKSPACE
    n = ctypes.c_size_t()
    assert lib.bevpool_embed_backward_workspace_size(5, 5, 0, ctypes.byref(n)) == EINVAL
    assert lib.bevpool_embed_backward_workspace_size(5, 5, 8, None) == EINVAL
    # more blocks than a launch holds (an expanded gradient could ask for it)
    assert lib.bevpool_embed_backward_workspace_size((1 << 31) - 1, 5, 1 << 20, ctypes.byref(n)) == EOVERFLOW
    assert bwd(n=(1 << 31) - 1, C=1 << 20) == EOVERFLOW
    assert lib.bevpool_embed_backward_workspace_size(0, 5, 8, ctypes.byref(n)) == OK and n.value > 0


def test_binding_refuses_cpu_tensors():
    x, ids = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    plan = rows.KeyOrder(ids.view(-1), ids.view(-1), torch.zeros(6, dtype=torch.int32), 5)
    for call in (lambda: rows.sort_keys(ids, 5), lambda: rows.route_forward(x, 2),
                 lambda: rows.dispatch_forward(x, ids, 5), lambda: rows.dispatch_backward(x, plan, 2),
                 lambda: rows.combine_forward(x, torch.zeros(2, 2), plan),
                 lambda: rows.embed_forward(x, ids), lambda: rows.embed_backward(x, ids, 4)):
        with pytest.raises(ValueError):
            call()
