"""GPU: page copies and the compaction of accepted drafts, bit by bit, and the calls
around them as a server makes them: drafted, verified, compacted, forked."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(require_gpu):
    pass


import torch  # noqa: E402

from oracle import masked as M  # noqa: E402
from paper_2511_20982_amd import attn as A  # noqa: E402
from paper_2511_20982_amd import inputs as I  # noqa: E402
from tests import gpu_util as G  # noqa: E402
from tests import masked_util as U  # noqa: E402

NP = {"bf16": np.uint16, "fp32": np.float32, "fp8": np.uint8}


def pools(rng, layers, pages, hkv, d, dtype):
    t = NP[dtype]
    make = lambda shape: rng.integers(0, 256, shape + (t().itemsize,), dtype=np.uint8).view(t)[..., 0]  # noqa: E731
    k, v = make((layers, pages, hkv, 16, d)), make((layers, pages, hkv, d, 16))
    if dtype == "fp32":  # (any bits but NaN, whose payloads a host copy need not keep)
        k, v = np.nan_to_num(k), np.nan_to_num(v)
    return k, v


def same(t, want):
    got = A.to_host(t)
    return np.array_equal(got.view(np.uint8), want.view(np.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("layers,hkv,d,copies", [(1, 1, 64, 1), (3, 5, 64, 7), (2, 8, 128, 40), (1, 32, 128, 3)])
def test_copy_pages(layers, hkv, d, copies, dtype):
    rng = np.random.default_rng(hkv + copies)
    pages = 2 * copies + 9
    k, v = pools(rng, layers, pages, hkv, d, dtype)
    perm = rng.permutation(pages).astype(np.int32)
    dst, src = perm[:copies].copy(), rng.choice(perm[copies:], copies).astype(np.int32)
    if copies > 3:  # what a padded list holds, and ids outside the pool
        dst[1], src[2], dst[3] = -1, pages, 2 ** 31 - 1
    kd, vd = A.to_device(k), A.to_device(v)
    A.dopd_kv_copy_pages(A.make_shape(hkv, hkv, d, dtype), layers, kd, vd, pages, A.to_device(src), A.to_device(dst), copies)
    want = M.copy_pages(k, v, src, dst)
    assert same(kd, want[0]) and same(vd, want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("layers,hkv,d", [(1, 1, 64), (3, 5, 64), (2, 8, 128)])
def test_compact(layers, hkv, d, dtype):
    rng = np.random.default_rng(layers + hkv)
    nodes, most = 50, 21
    prefix = np.array([0, 5, 15, 16, 31, 100, 250, 7], np.int32)
    n = len(prefix)
    pt, pages = I.allocate_pages(rng, prefix + nodes)
    k, v = pools(rng, layers, pages, hkv, d, dtype)
    count = np.array([0, 1, most, 9, 3, 20, 5, most], np.int32)
    path = np.full((n, most), -7, np.int32)  # (what is not accepted is not looked at)
    for r, m in enumerate(count):
        path[r, :m] = np.sort(rng.choice(nodes, m, replace=False))
    path[7] = np.arange(most)  # already in place
    kd, vd = A.to_device(k), A.to_device(v)
    args = (A.make_shape(hkv, hkv, d, dtype), layers, kd, vd, pages, A.to_device(pt), pt.shape[1], A.to_device(prefix),
            A.to_device(path))
    A.dopd_kv_compact(*args, A.to_device(count), most, n)
    want = M.compact(k, v, pt, prefix, path, count)
    assert same(kd, want[0]) and same(vd, want[1])


def test_compact_leaves_out_what_lies_outside():
    """Counts below 0 or above the list, positions past the table, pages outside the pool, steps backwards."""
    rng = np.random.default_rng(4)
    prefix = np.array([0, 10, 20, 30, 30, 30], np.int32)
    pt, pages = I.allocate_pages(rng, prefix + 18)
    pt = np.concatenate([pt, np.full((len(prefix), 1), -1, np.int32)], 1)
    k, v = pools(rng, 2, pages, 2, 64, "bf16")
    path = np.tile(np.array([1, 3], np.int32), (6, 1))
    count = np.array([-5, 9, 2, 2, 2, 2], np.int32)
    path[2] = [1, 10 ** 6]           # past the table
    path[3] = [1, 2 ** 31 - 1]
    path[4] = [1, 40]                # an entry of -1
    path[5] = [-3, 0]                # no path: nothing moves backwards
    kd, vd = A.to_device(k), A.to_device(v)
    A.dopd_kv_compact(A.make_shape(2, 2, 64), 2, kd, vd, pages, A.to_device(pt), pt.shape[1], A.to_device(prefix),
                      A.to_device(path), A.to_device(count), 2, 6)
    take = np.array([0, 2, 1, 1, 1, 0], np.int32)
    want = M.compact(k, v, pt, prefix, path, take)
    assert same(kd, want[0]) and same(vd, want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_draft_verify_compact_and_fork(dtype):
    """Drafts written behind the prefix, verified as a tree, the accepted path compacted, the request forked: the
    cache then holds what a request that had those tokens from the start holds, and attends alike."""
    rng = np.random.default_rng(77)
    hq, hkv, d, nodes = 8, 2, 128, 12
    prefix = np.array([37, 100, 0], np.int32)
    fresh = "fp32" if dtype == "fp32" else "bf16"
    n = len(prefix)
    c = U.case(78, prefix, [nodes] * n, hq, hkv, d, dtype)
    mask = U.tree_masks(rng, [nodes] * n, 1)
    dev = U.on_device(c)
    U.check(U.run(c, ("tree", mask), dev), U.tree_reference(c, mask), c, "verify")
    # accepted: the path of a draft, from its mask
    paths = [np.nonzero(np.unpackbits(mask[r * nodes + leaf: r * nodes + leaf + 1].view(np.uint8), bitorder="little"))[0]
             for r, leaf in enumerate((11, 9, 10))]
    most = max(len(p) for p in paths)
    acc, count = np.zeros((n, most), np.int32), np.array([len(p) for p in paths], np.int32)
    for r, p in enumerate(paths):
        acc[r, :len(p)] = p
    sh = U.shape_of(c)
    A.dopd_kv_compact(sh, 1, dev["k"], dev["v"], c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["prefix"],
                      A.to_device(acc), A.to_device(count), most, n)
    k2, v2 = M.compact(c["k"][None], c["v"][None], c["pt"], prefix, acc, count)
    assert same(dev["k"], k2[0]) and same(dev["v"], v2[0])
    # the first request forks: its last page is copied, the others are shared
    length = prefix + count
    spare = sorted(set(range(c["k"].shape[0])) - set(c["pt"].ravel().tolist()))[0]
    last = (length[0] - 1) // 16
    A.dopd_kv_copy_pages(sh, 1, dev["k"], dev["v"], c["k"].shape[0], A.to_device(c["pt"][0, last:last + 1].copy()),
                         A.to_device(np.array([spare], np.int32)), 1)
    fork = c["pt"][0].copy()
    fork[last] = spare
    k2, v2 = M.copy_pages(k2, v2, [c["pt"][0, last]], [spare])
    # one windowed decode step of all four continuations (their last token's row)
    step = dict(c, k=k2[0], v=v2[0], pt=np.concatenate([c["pt"], fork[None]]),
                prefix=np.append(length, length[0]).astype(np.int32) - 1, cu=I.cu_from_lens([1] * (n + 1)),
                q=I.normal(rng, (n + 1, hq, d), fresh))
    got = U.run(step, ("window", 21, 2), {**U.on_device(step), "k": dev["k"], "v": dev["v"]})
    U.check(got, U.window_reference(step, 21, 2), step, "decode of the fork")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_another_stream_and_a_captured_graph(dtype):
    """On a side stream, and captured and replayed with new contents of the same buffers, eager work in between."""
    c = U.case(90, [2000, 60, 5], [1, 30, 2], 8, 2, 128, dtype)
    ref = U.window_reference(c, 700, 4)
    side = torch.cuda.Stream()
    U.check(U.run(c, ("window", 700, 4), stream=side), ref, c, "side stream")
    dev, sh, n = U.on_device(c), U.shape_of(c), 3
    out, lse = torch.zeros_like(dev["q"]), torch.zeros(c["q"].shape[:2], device="cuda")
    ws = A.window_workspace(sh, c["cu"], c["prefix"], n, 700, 4)
    scales = (dev["ks"], dev["vs"]) if dtype == "fp8" else ()
    call = A.dopd_window_attn_fp8 if dtype == "fp8" else A.dopd_window_attn
    path, count = A.to_device(np.array([[0], [29], [1]], np.int32)), A.to_device(np.array([1, 1, 1], np.int32))

    def step():
        call(sh, dev["q"], dev["k"], dev["v"], *scales, c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["cu"], c["cu"],
             dev["prefix"], c["prefix"], n, 700, 4, out, lse, ws)
        A.dopd_kv_compact(sh, 1, dev["k"], dev["v"], c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["prefix"], path,
                          count, 1, n)

    k0, v0, q0 = dev["k"].clone(), dev["v"].clone(), dev["q"].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        dev["k"].copy_(k0)
        dev["v"].copy_(v0)
        dev["q"].copy_(q0 if i % 2 == 0 else q0.flip(0))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        seen = out.clone(), lse.clone(), dev["k"].clone(), dev["v"].clone()
        dev["k"].copy_(k0)
        dev["v"].copy_(v0)
        out.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(seen, (out, lse, dev["k"], dev["v"])):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f"replay {i}"
    assert same(dev["k"], M.compact(c["k"][None], c["v"][None], c["pt"], c["prefix"], np.array([[0], [29], [1]]), [1, 1, 1])[0][0])


def test_two_calls_at_once_on_two_streams():
    c = U.case(91, [3000, 900], [1, 40], 8, 2, 128, "bf16")
    mask = U.tree_masks(np.random.default_rng(1), [1, 40], 2)
    want = U.run(c, ("window", 1000, 4)), U.run(c, ("tree", mask))
    dev, sh = U.on_device(c), U.shape_of(c)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.zeros_like(dev["q"]) for _ in range(2)]
    ws = A.window_workspace(sh, c["cu"], c["prefix"], 2, 1000, 4), A.tree_workspace(sh, c["cu"], c["prefix"], 2)
    m = A.to_device(mask.view(np.int32))
    table = (c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["cu"], c["cu"], dev["prefix"], c["prefix"], 2)
    torch.cuda.synchronize()
    for _ in range(5):
        A.dopd_window_attn(sh, dev["q"], dev["k"], dev["v"], *table, 1000, 4, outs[0], None, ws[0], stream=streams[0])
        A.dopd_tree_attn(sh, dev["q"], dev["k"], dev["v"], *table, m, 2, outs[1], None, ws[1], stream=streams[1])
    torch.cuda.synchronize()
    for got, (w, _) in zip(outs, want):
        assert np.array_equal(G.widen(A.to_host(got)), w)
