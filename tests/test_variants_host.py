"""CPU: planning and refusals of the windowed and the tree attention and of the page calls (the pointers passed here
are never dereferenced)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2511_20982_amd import attn as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "masked_harness.cpp")
FAKE = 0x1000  # a non-null, aligned device address


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("masked") / "masked_harness")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", SRC, "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("cus,xcds", [(256, 8), (64, 4), (32, 8), (80, 1)])
def test_plans(harness, cus, xcds):
    res = subprocess.run([harness, str(cus), str(xcds), "300"], capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr


def i32(*a):
    return np.array(a, np.int32)


def p(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def masked(kind, shape=(8, 2, 128, "bf16"), fp8=False, cu=i32(0, 3, 10), pre=i32(40, 0), n=2, stride=8, pages=20, ptr=FAKE,
           how=None, ws=FAKE, ws_bytes=1 << 30, k_scale=FAKE, **over):
    """Status of a call whose arguments are fine but for those given."""
    sh = A.make_shape(*shape)
    if "page_size" in over:
        sh.page_size = over["page_size"]
    if "head_dim" in over:
        sh.head_dim = over["head_dim"]
    at = {x: over.get(x, ptr) for x in ("q", "k", "v", "pt", "cu_dev", "pre_dev", "out", "lse", "mask")}
    how = how if how is not None else ((16, 2) if kind == "window" else (at["mask"], 1))
    f = getattr(A.lib(), f"dopd_{kind}_attn" + ("_fp8" if fp8 else ""))
    scales = (k_scale, ptr) if fp8 else ()
    return f(C.byref(sh), at["q"], at["k"], at["v"], *scales, pages, at["pt"], stride, at["cu_dev"], p(cu), at["pre_dev"],
             p(pre), n, *how, at["out"], at["lse"], ws, ws_bytes, None)


KINDS = [("window", False), ("window", True), ("tree", False), ("tree", True)]


@pytest.mark.parametrize("kind,fp8", KINDS)
def test_masked_refusals(kind, fp8):
    ok = (8, 2, 128, "fp8" if fp8 else "bf16")
    bad = lambda status, **kw: masked(kind, **{"shape": ok, "fp8": fp8, **kw}) == status  # noqa: E731
    assert bad(A.DOPD_ERR_INVALID_SHAPE, shape=(8, 3, 128, ok[3]))
    assert bad(A.DOPD_ERR_UNSUPPORTED, head_dim=96) and bad(A.DOPD_ERR_UNSUPPORTED, page_size=32)
    assert bad(A.DOPD_ERR_UNSUPPORTED, shape=(8, 2, 128, "bf16" if fp8 else "fp8"))
    if fp8:
        assert bad(A.DOPD_ERR_UNSUPPORTED, shape=(8, 2, 128, "fp32")) and bad(A.DOPD_ERR_NULL_POINTER, k_scale=None)
    for name in ("q", "k", "v", "pt", "cu_dev", "pre_dev", "out"):
        assert bad(A.DOPD_ERR_NULL_POINTER, **{name: None}), name
    assert bad(A.DOPD_ERR_NULL_POINTER, cu=None) and bad(A.DOPD_ERR_NULL_POINTER, pre=None)
    for name in ("q", "k", "v", "out"):
        assert bad(A.DOPD_ERR_INVALID_SHAPE, **{name: FAKE + 8}), name
    for kw in (dict(n=-1), dict(stride=-1), dict(pages=-1), dict(cu=i32(1, 3, 10)), dict(cu=i32(0, 3, 2)), dict(pre=i32(-1, 0)),
               dict(stride=2), dict(pre=i32(2 ** 30, 0), stride=2 ** 30), dict(pre=i32(2 ** 31 - 1, 0), stride=2 ** 30)):
        assert bad(A.DOPD_ERR_INVALID_SHAPE, **kw), kw
    assert bad(A.DOPD_OK, n=0) and bad(A.DOPD_OK, cu=i32(0, 0, 0), q=None, out=None)
    if kind == "window":
        for how in ((0, 0), (-3, 0), (5, -1)):
            assert bad(A.DOPD_ERR_INVALID_SHAPE, how=how), how
    else:
        assert bad(A.DOPD_ERR_NULL_POINTER, mask=None)
        for words in (0, -1, 33):
            assert bad(A.DOPD_ERR_INVALID_SHAPE, how=(FAKE, words)), words
        assert bad(A.DOPD_ERR_INVALID_SHAPE, cu=i32(0, 33, 34), how=(FAKE, 1), stride=100)
    # a call that is split needs its workspace
    long = dict(pre=i32(9000, 0), stride=600, how=(8000, 2) if kind == "window" else None)
    assert bad(A.DOPD_ERR_NULL_POINTER, ws=None, **long)
    assert bad(A.DOPD_ERR_WORKSPACE_TOO_SMALL, ws_bytes=0, **long)
    assert bad(A.DOPD_ERR_INVALID_SHAPE, ws=FAKE + 16, **long)
    # rows whose packed index would not fit the kernels' division
    assert bad(A.DOPD_ERR_INVALID_SHAPE, shape=(4096, 1, 128, ok[3]), cu=i32(0, 1000, 1000), stride=10 ** 6, how=(FAKE, 32) if kind == "tree" else None)


def test_workspace_sizes():
    sh = A.make_shape(8, 2, 128)
    cu, pre = i32(0, 1, 41), i32(9000, 70)
    assert A.dopd_window_workspace_size(sh, cu, pre, 2, 64) == 256  # short windows are not split
    wide = A.dopd_window_workspace_size(sh, cu, pre, 2, 8000, 4)
    tree = A.dopd_tree_workspace_size(sh, cu, pre, 2)
    assert wide > 256 and tree > 256 and wide % 256 == 0 and tree % 256 == 0
    assert A.dopd_tree_workspace_size(A.make_shape(8, 2, 128, "fp8"), cu, pre, 2) == tree
    assert A.dopd_tree_workspace_size(A.make_shape(8, 2, 128, "fp32"), cu, pre, 2) == 256
    assert A.dopd_tree_workspace_size(sh, i32(0), i32(0)[:0], 0) == 256
    for call in (lambda: A.dopd_tree_workspace_size(A.make_shape(8, 3, 128), cu, pre, 2),
                 lambda: A.dopd_tree_workspace_size(sh, None, pre, 2), lambda: A.dopd_tree_workspace_size(sh, cu, pre, -1),
                 lambda: A.dopd_tree_workspace_size(sh, i32(0, 1025), i32(0), 1),
                 lambda: A.dopd_window_workspace_size(sh, cu, i32(-1, 0), 2, 5),
                 lambda: A.dopd_window_workspace_size(sh, cu, pre, 2, 0), lambda: A.dopd_window_workspace_size(sh, cu, pre, 2, 5, -1)):
        assert call() == 0
    with pytest.raises(A.DopdError):
        A.window_workspace(sh, cu, pre, 2, 0, device="cpu")
    with pytest.raises(A.DopdError):
        A.tree_workspace(A.make_shape(8, 3, 128), cu, pre, 2, device="cpu")


def copy(shape=(8, 2, 128, "bf16"), layers=1, k=FAKE, v=FAKE, pages=10, src=FAKE, dst=FAKE, n=1):
    sh = A.make_shape(*shape)
    return A.lib().dopd_kv_copy_pages(C.byref(sh), layers, k, v, pages, src, dst, n, None)


def compact(shape=(8, 2, 128, "bf16"), layers=1, k=FAKE, v=FAKE, pages=10, pt=FAKE, stride=4, pre=FAKE, acc=FAKE, cnt=FAKE, most=2, n=1):
    sh = A.make_shape(*shape)
    return A.lib().dopd_kv_compact(C.byref(sh), layers, k, v, pages, pt, stride, pre, acc, cnt, most, n, None)


@pytest.mark.parametrize("call,pointers,counts,nothing", [
    (copy, ("k", "v", "src", "dst"), ("layers", "pages", "n"), ("layers", "n")),
    (compact, ("k", "v", "pt", "pre", "acc", "cnt"), ("layers", "pages", "stride", "most", "n"), ("layers", "most", "n"))])
def test_page_call_refusals(call, pointers, counts, nothing):
    assert call(shape=(8, 3, 128, "bf16")) == A.DOPD_ERR_INVALID_SHAPE
    for name in pointers:
        assert call(**{name: None}) == A.DOPD_ERR_NULL_POINTER, name
    for name in ("k", "v"):
        assert call(**{name: FAKE + 4}) == A.DOPD_ERR_INVALID_SHAPE, name
    for name in counts:
        assert call(**{name: -1}) == A.DOPD_ERR_INVALID_SHAPE, name
    for name in nothing:
        assert call(**{name: 0}) == A.DOPD_OK, name
    assert call(layers=2 ** 31 - 1, n=2 ** 31 - 1) == A.DOPD_ERR_INVALID_SHAPE
    assert call(shape=(2 ** 30, 2 ** 30, 128, "fp32")) == A.DOPD_ERR_INVALID_SHAPE
