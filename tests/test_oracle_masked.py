"""CPU: the fp64 reference of the windowed and the tree attention (oracle/masked.py) against the C oracle, the
dense formulation and closed forms; of the page calls against plain rearrangements; and planted mistakes."""
import numpy as np
import pytest

import oracle
from oracle import masked as M
from paper_2511_20982_amd import inputs as I
from tests import masked_util as U

PREFIX, NEW = [0, 5, 40, 33], [7, 1, 20, 0]


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_a_window_of_everything_is_the_chunk_oracle(dtype):
    c = U.case(1, PREFIX, NEW, 4, 2, 64, dtype)
    args = (c["q"], c["k"], c["v"])
    table = (c["pt"], c["cu"], c["prefix"], c["scale"])
    if dtype == "fp8":
        want, want_lse = oracle.prefill_paged_e4m3(*args, c["ks"], c["vs"], *table)
    else:
        want, want_lse = oracle.prefill_paged(*args, *table)
    chain = np.tile(np.packbits(np.tril(np.ones((32, 32), bool)), axis=1, bitorder="little").view("<u4"), (4, 1))
    chain = np.concatenate([chain[:n] for n in NEW])
    for out, lse, weighted, _ in (U.window_reference(c, 10 ** 6, 0), U.window_reference(c, 1, 10 ** 6), U.tree_reference(c, chain)):
        assert np.abs(out - want).max() < 1e-12 and np.abs(lse - want_lse).max() < 1e-12
        assert (weighted >= np.abs(out) - 1e-12).all()


def dense(c, hidden):
    """Softmax over all positions of the first request with the hidden ones at -inf, values by einsum."""
    end = int(c["prefix"][0] + c["cu"][1])
    at = np.arange(end)
    k = M.widen(c["k"][c["pt"][0, at // 16], :, at % 16, :])
    v = M.widen(c["v"][c["pt"][0, at // 16], :, :, at % 16])
    g = c["hq"] // c["hkv"]
    q = M.widen(c["q"][: c["cu"][1]])
    s = c["scale"] * np.einsum("ihd,jhd->ihj", q, np.repeat(k, g, 1))
    s[np.broadcast_to(hidden[:, None], s.shape)] = -np.inf
    p = np.exp(s - s.max(2, keepdims=True))
    return np.einsum("ihj,jhd->ihd", p / p.sum(2, keepdims=True), np.repeat(v, g, 1))


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (9, 30), (16, 1)])
def test_window_against_the_dense_formulation(window, sinks):
    c = U.case(2, [21], [13], 6, 3, 64, "fp32")
    j, p = np.arange(34)[None], 21 + np.arange(13)[:, None]
    hidden = ~((j <= p) & ((p - j < window) | (j < sinks)))
    assert np.abs(U.window_reference(c, window, sinks)[0] - dense(c, hidden)).max() < 1e-12


def test_tree_against_the_dense_formulation():
    c = U.case(3, [21], [40], 6, 3, 64, "fp32")
    mask = U.random_tree(np.random.default_rng(0), 40, 3)
    hidden = np.zeros((40, 61), bool)
    for i in range(40):
        for j in range(40):
            hidden[i, 21 + j] = not (int(mask[i, j // 32]) >> (j % 32)) & 1
    assert np.abs(U.tree_reference(c, mask)[0] - dense(c, hidden)).max() < 1e-12


def test_a_window_of_one_returns_its_own_value():
    c = U.case(4, [10], [5], 2, 2, 64, "fp32")
    out = U.window_reference(c, 1, 0)[0]
    at = 10 + np.arange(5)
    v = c["v"][c["pt"][0, at // 16], :, :, at % 16]
    assert np.array_equal(out, v.astype(np.float64))


def test_a_row_that_sees_nothing():
    c = U.case(5, [0, 3], [2, 2], 2, 2, 64, "fp32")
    out, lse, weighted, _ = U.tree_reference(c, np.array([[0], [2], [0], [0]], np.uint32))
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all() and np.isfinite(lse[1:]).all() and (weighted[0] == 0).all()


def test_page_calls():
    rng = np.random.default_rng(6)
    k, v = rng.random((2, 6, 3, 16, 8)), rng.random((2, 6, 3, 8, 16))
    k2, v2 = M.copy_pages(k, v, [1, 1, 9], [4, 0, 2])
    assert np.array_equal(k2[:, [4, 0, 1, 2]], k[:, [1, 1, 1, 2]]) and np.array_equal(v2[:, [4, 0, 3]], v[:, [1, 1, 3]])
    pt = np.array([[3, 5]], np.int32)
    k2, v2 = M.compact(k, v, pt, [14], np.array([[1, 3, 4, 9]]), [3])
    rows = lambda x: np.concatenate([x[:, 3], x[:, 5]], 2)  # noqa: E731
    assert np.array_equal(rows(k2)[:, :, 14:17], rows(k)[:, :, [15, 17, 18]]) and np.array_equal(rows(k2)[:, :, :14], rows(k)[:, :, :14])
    cols = lambda x: np.concatenate([x[:, 3], x[:, 5]], 3)  # noqa: E731
    assert np.array_equal(cols(v2)[..., 14:17], cols(v)[..., [15, 17, 18]]) and np.array_equal(cols(v2)[..., 17:], cols(v)[..., 17:])


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_the_bounds_catch_planted_mistakes(dtype):
    """One key too many or too few at either end of the window, one sink too few, a wrong draft: all outside the
    bounds the kernels are held to."""
    c = U.case(7, [60, 20], [9, 30], 4, 2, 128, dtype)
    ref = U.window_reference(c, 12, 3)
    right = [np.float32(ref[0]).astype(np.float64), np.float32(ref[1]).astype(np.float64)]
    if dtype != "fp32":
        right[0] = M.widen(I.f32_to_bf16_bits(ref[0].astype(np.float32)))
    U.check(right, ref, c, "right")
    for window, sinks in ((13, 3), (11, 3), (12, 2), (12, 4)):
        with pytest.raises(AssertionError):
            U.check(U.window_reference(c, window, sinks)[:2], ref, c, "planted")
    mask = U.tree_masks(np.random.default_rng(1), [9, 30], 1)
    ref = U.tree_reference(c, mask)
    mask[20] ^= 2
    with pytest.raises(AssertionError):
        U.check(U.tree_reference(c, mask)[:2], ref, c, "planted")
