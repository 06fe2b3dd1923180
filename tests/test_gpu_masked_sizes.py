"""GPU: windowed and tree attention where one kernel takes over from another, against the fp64 reference: requests of
1 to 129 packed rows in every type, calls of one size and of several, contexts that several workgroups share, large
scores, scales of any sign, and calls that repeat bit for bit."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(require_gpu):
    pass


import torch  # noqa: E402

from paper_2511_20982_amd import attn as A  # noqa: E402
from tests import gpu_util as G  # noqa: E402
from tests import masked_util as U  # noqa: E402


def window(c, size, sinks, what=""):
    U.check(U.run(c, ("window", size, sinks)), U.window_reference(c, size, sinks), c,
            f"window {size} sinks {sinks} {c['hq']}/{c['hkv']} d {c['d']} {c['dtype']} {what}")


def tree(c, seed, what="", empty=0.0):
    new = np.diff(c["cu"])
    mask = U.tree_masks(np.random.default_rng(seed), new, max(1, (int(new.max()) + 31) // 32), empty)
    U.check(U.run(c, ("tree", mask)), U.tree_reference(c, mask), c, f"tree {c['hq']}/{c['hkv']} d {c['d']} {c['dtype']} {what}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("new,hq,hkv", [(16, 2, 2), (17, 2, 2), (4, 8, 2), (11, 6, 2), (2, 16, 1), (32, 4, 2), (13, 5, 1),
                                        (64, 2, 2), (65, 2, 2), (43, 3, 1), (128, 1, 1), (129, 1, 1), (7, 64, 2)])
def test_rows_around_each_kernel_s_limit(new, hq, hkv, d, dtype):
    """One size a call; prefixes on both sides of pages, tiles of 32 keys and the ring's five tiles."""
    for prefix in ([0, 15, 16, 17], [31, 32, 33, 97], [128, 159, 160, 161, 191, 192, 193]):
        c = U.case(1000 + new + prefix[0], prefix, [new] * len(prefix), hq, hkv, d, dtype)
        window(c, 70, 3)
        tree(c, 7)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("new,hq,hkv", [(1, 8, 1), (3, 8, 1), (6, 8, 1), (12, 8, 1), (40, 8, 1)])
def test_long_contexts_of_each_size(new, hq, hkv, d, dtype):
    """Few requests whose contexts several workgroups share; windows that begin and end inside tiles."""
    c = U.case(1100 + new, [2900, 1777, 3], [new, new, new], hq, hkv, d, dtype)
    window(c, 2001, 37)
    window(c, 6000, 0)
    tree(c, 8, empty=0.2)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
def test_calls_that_hold_all_sizes(d, dtype):
    """Every class with a share of its own, then one class after the other with little to do."""
    heavy = [1500, 900, 1200], [1, 5, 60]
    c = U.case(1200, heavy[0] * 2 + [700, 0, 1000], heavy[1] * 2 + [0, 3, 1], 16, 2, d, dtype)
    window(c, 800, 5)
    tree(c, 9)
    for prefix, new in (([1400, 40, 30], [60, 2, 5]), ([1400, 40, 30], [5, 2, 60]), ([1400, 40, 30], [1, 5, 60])):
        c = U.case(1210 + new[0], prefix, new, 16, 2, d, dtype)
        window(c, 1000, 5, str(new))
        tree(c, 10, str(new))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 2.0])
@pytest.mark.parametrize("new", [1, 5, 30])
def test_scales_of_each_size(new, scale, dtype):
    """2.0: scores so far apart that the running maximum moves in the middle of a context."""
    c = U.case(1300 + new, [600, 90], [new, new], 16, 2, 128, dtype)
    c["scale"] = scale
    window(c, 300, 2, f"scale {scale}")
    tree(c, 11, f"scale {scale}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("new", [1, 6, 61])
def test_a_call_repeats_bit_for_bit(new, dtype):
    """Also where workgroups share contexts: partial results are joined in one order."""
    c = U.case(1400 + new, [2500, 1200, 60], [new] * 3, 8, 1, 128, dtype)
    mask = U.tree_masks(np.random.default_rng(12), [new] * 3, 2)
    for how in (("window", 1900, 4), ("tree", mask)):
        first = U.run(c, how)
        for _ in range(3):
            out, lse = U.run(c, how)
            assert np.array_equal(out, first[0]) and np.array_equal(lse, first[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("new", [2, 6, 40])
def test_a_tree_call_captured_and_replayed(new, dtype):
    """New rows, masks and cache contents in the captured buffers, eager work between the replays."""
    prefix = [2000, 300, 17]
    rng = np.random.default_rng(13)
    masks = [U.tree_masks(rng, [new] * 3, 2) for _ in range(3)]
    c = U.case(1500, prefix, [new] * 3, 8, 1, 128, dtype)
    sign = c["k"].dtype.type(0x80 if dtype == "fp8" else 0x8000)
    cases = [c, dict(c, k=c["k"] ^ sign), dict(c, q=np.ascontiguousarray(c["q"][::-1]), v=c["v"] ^ sign)]
    dev = U.on_device(c)
    words = A.to_device(masks[0].view(np.int32))
    sh = U.shape_of(c)
    size = A.dopd_tree_workspace_size(sh, c["cu"], c["prefix"], 3)
    ws, out = torch.empty(size, dtype=torch.uint8, device=U.DEV), torch.empty_like(dev["q"])
    lse = torch.empty(c["q"].shape[:2], device=U.DEV)
    scales = (dev["ks"], dev["vs"]) if dtype == "fp8" else ()
    name = A.dopd_tree_attn_fp8 if dtype == "fp8" else A.dopd_tree_attn

    def call():
        name(sh, dev["q"], dev["k"], dev["v"], *scales, c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["cu"], c["cu"],
             dev["prefix"], c["prefix"], 3, words, masks[0].shape[1], out, lse, ws, size)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for x, mask in zip(cases, masks):
        fresh = U.on_device(x)
        for k in ("q", "k", "v"):
            dev[k].copy_(fresh[k])
        words.copy_(A.to_device(mask.view(np.int32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = G.widen(A.to_host(out)), lse.cpu().numpy().astype(np.float64)
        U.check(got, U.tree_reference(x, mask), x, f"replay {new} {dtype}")
        call()
        torch.cuda.synchronize()
        assert np.array_equal(G.widen(A.to_host(out)), got[0])
