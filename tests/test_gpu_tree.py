"""GPU: tree attention over the paged cache against the fp64 reference."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(require_gpu):
    pass


from tests import gpu_util as G  # noqa: E402
from tests import masked_util as U  # noqa: E402

PREFIX = [0, 1, 15, 16, 17, 63, 64, 65, 200, 777, 0, 40, 129]
NODES = [9, 1, 16, 30, 64, 33, 100, 128, 1, 7, 0, 31, 2]


def both(c, mask, what=""):
    U.check(U.run(c, ("tree", mask)), U.tree_reference(c, mask), c,
            f"tree {c['hq']}/{c['hkv']} d {c['d']} {c['dtype']} {what}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (8, 2), (7, 1), (32, 1)])
def test_ragged_batch(hq, hkv, d, dtype):
    c = U.case(800 + hq + d, PREFIX, NODES, hq, hkv, d, dtype)
    both(c, U.tree_masks(np.random.default_rng(hq), NODES, 4))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("nodes,words", [(1, 1), (2, 3), (31, 1), (32, 1), (33, 2), (65, 5), (300, 10)])
def test_mask_words_and_arbitrary_masks(nodes, words, dtype):
    """Any bits, those past the request's drafts among them."""
    rng = np.random.default_rng(nodes)
    pre = [0, 30, 64, 97]
    c = U.case(810 + nodes, pre, [nodes] * len(pre), 4, 2, 64, dtype)
    both(c, rng.integers(0, 2 ** 32, (nodes * len(pre), words), dtype=np.uint32), f"{nodes} nodes")


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 2)])
def test_rows_that_see_nothing(hq, hkv, dtype):
    """No cached token and an empty mask: 0, and an lse of -inf; beside ordinary rows."""
    n, pre = [5, 1, 40, 70, 3], [0, 0, 0, 0, 20]
    c = U.case(820, pre, n, hq, hkv, 128, dtype)
    mask = U.tree_masks(np.random.default_rng(3), n, 3, empty=0.5)
    mask[5] = 0  # the second request's only draft
    out, lse = U.run(c, ("tree", mask))
    ref = U.tree_reference(c, mask)
    assert np.isneginf(ref[1]).any() and (out[np.isneginf(ref[1])] == 0).all()
    U.check((out, lse), ref, c, "rows that see nothing")
    mask[:] = 0
    both(c, mask, "no row sees a draft")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
def test_long_contexts_split_over_workgroups(d, dtype):
    both(U.case(830, [3000, 1500, 20, 0], [2, 2, 1, 2], 8, 1, d, dtype), U.tree_masks(np.random.default_rng(5), [2, 2, 1, 2], 1))
    both(U.case(831, [2500, 70], [21, 40], 16, 2, d, dtype), U.tree_masks(np.random.default_rng(6), [21, 40], 2))


def test_a_chain_is_a_chunk_and_one_draft_a_decode_step():
    c = U.case(840, [100, 7, 640], [50, 3, 20], 8, 2, 128, "bf16")
    n = np.diff(c["cu"])
    mask = np.concatenate([np.packbits(np.tril(np.ones((64, 64), bool))[:m], axis=1, bitorder="little").view("<u4") for m in n])
    out, lse = U.run(c, ("tree", mask.astype(np.uint32)))
    chunk, chunk_lse = G.gpu_prefill_paged(U.shape_of(c), c["q"], c["k"], c["v"], c["pt"], c["cu"], c["prefix"])
    # each is within u(bf16) W + u(bf16) |ref| of the reference, so twice that of the other
    want, _, weighted, _ = U.tree_reference(c, mask.astype(np.uint32))
    assert (np.abs(out - chunk) <= 2 * 1.01 * U.UBF * (weighted + np.abs(want)) + 1e-5).all()
    assert np.max(np.abs(lse - chunk_lse)) < 2e-2
    c = U.case(841, [100, 7, 640], [1, 1, 1], 8, 2, 128, "bf16")
    out, _ = U.run(c, ("tree", np.ones((3, 1), np.uint32)))
    dec, _ = G.gpu_decode(U.shape_of(c), c["q"], c["k"], c["v"], c["pt"], (c["prefix"] + 1).astype(np.int32))
    want, _, weighted, _ = U.tree_reference(c, np.ones((3, 1), np.uint32))
    assert (np.abs(out - dec) <= 2 * 1.01 * U.UBF * (weighted + np.abs(want)) + 1e-5).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("nodes,hq,hkv", [(6, 8, 8), (40, 8, 2)])
def test_non_finite_drafts_reach_only_rows_that_see_them(nodes, hq, hkv, dtype, bad):
    if dtype == "fp8" and np.isinf(bad):
        pytest.skip("E4M3 has no infinities")
    pre = 45
    c = U.case(850, [pre, pre], [nodes, nodes], hq, hkv, 128, dtype)
    value = {"fp32": np.float32(bad), "bf16": np.uint16(0x7FC0 if np.isnan(bad) else 0x7F80), "fp8": np.uint8(0x7F)}[dtype]
    mask = U.tree_masks(np.random.default_rng(9), [nodes, nodes], 2)
    for r, j in ((0, nodes // 2), (1, 1)):
        page, slot = c["pt"][r, (pre + j) // 16], (pre + j) % 16
        c["v"][page, :, 3, slot] = value
        if r == 1:
            c["k"][page, 0, slot, :] = np.abs(c["k"][page, 0, slot, :]) if dtype == "fp32" else value
    out, _ = U.run(c, ("tree", mask))
    want, want_lse, weighted, products = U.tree_reference(c, mask)
    ok = np.isfinite(want)
    assert 0 < ok.sum() < ok.size
    assert np.array_equal(np.isfinite(out), ok)
    clean = [np.where(np.isfinite(x), x, 0) for x in (weighted, products)]
    U.check((np.where(ok, out, 0), None), (np.where(ok, want, 0), np.where(np.isfinite(want_lse), want_lse, 0), *clean), c, "bad drafts")
