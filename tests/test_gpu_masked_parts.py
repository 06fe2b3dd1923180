"""GPU: windowed and tree attention in calls whose contexts several workgroups share, where what one part of a row's keys
holds has to survive the merge of the parts: NaN in Q and in K; and values of V near the largest finite ones, whose sums
stay finite as long as the weights are formed against the largest score."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(require_gpu):
    pass


from paper_2511_20982_amd import attn as A  # noqa: E402
from tests import masked_util as U  # noqa: E402

PREFIX = [3000, 1777, 20]
NAN = {"bf16": np.uint16(0x7FC0), "fp8": np.uint8(0x7F)}
HOWS = ["window", "tree"]
# one packed row group of each kernel: 8, 48 and 320 rows of a KV head
SIZES = [1, 6, 40]


def calls(c, kind, seed=21):
    """The call, and its reference, of a case that is split over workgroups (its partial results need a workspace)."""
    new, n = np.diff(c["cu"]), len(c["prefix"])
    if kind == "window":
        how = ("window", 2000, 37)
        size = A.dopd_window_workspace_size(U.shape_of(c), c["cu"], c["prefix"], n, *how[1:])
        ref = lambda: U.window_reference(c, *how[1:])  # noqa: E731
    else:
        how = ("tree", U.tree_masks(np.random.default_rng(seed), new, max(1, (int(new.max()) + 31) // 32)))
        size = A.dopd_tree_workspace_size(U.shape_of(c), c["cu"], c["prefix"], n)
        ref = lambda: U.tree_reference(c, how[1])  # noqa: E731
    assert size > 256
    return how, ref


@pytest.mark.parametrize("kind", HOWS)
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("new", SIZES)
def test_nan_in_a_row_of_q(new, d, dtype, kind):
    """Every part of the row has scores of NaN alone; the other rows of the request and of the call are as they were."""
    c = U.case(1600 + new, PREFIX, [new] * 3, 8, 1, d, dtype)
    c["q"][new // 2, 3, 5] = NAN["bf16"]
    c["q"][2 * new, 7, 0] = NAN["bf16"]
    how, ref = calls(c, kind)
    got, want = U.run(c, how), ref()
    assert np.isnan(want[1]).sum() == 2
    U.check(got, want, c, f"NaN in Q, {new} {d} {dtype} {kind}")
    assert np.isnan(got[1][np.isnan(want[1])]).all()


@pytest.mark.parametrize("backwards", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("new", SIZES)
def test_nan_in_all_keys_of_some_parts(new, dtype, backwards):
    """K is NaN up to (or from) every 32nd position in turn, so that at some of them each part is NaN or finite as a
    whole: the rows, which see all cached tokens, are NaN."""
    c = U.case(1620, [2500], [new], 8, 1, 128, dtype)
    how, _ = calls(c, "tree")
    dev = U.on_device(c)
    out, lse = U.run(c, how, dev)
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    bits = A.to_device(np.full((16, 128), NAN[dtype]))
    tiles = range(2500 // 32)
    for t in reversed(tiles) if backwards else tiles:
        for page in c["pt"][0, 2 * t:2 * t + 2]:
            dev["k"][int(page), 0] = bits
        out, lse = U.run(c, how, dev)
        assert np.isnan(out).all() and np.isnan(lse).all(), f"{new} {dtype}: NaN in tile {t} and those before it in turn"


def steep(new, prefix, value, low):
    """Rows of a KV head with g = 8 whose scores are 0 in the 32-key tiles `low` and 9.6875 (14 octaves up) in the others,
    over V of value .. 2 value, of one sign in each dim."""
    n = len(prefix)
    c = U.case(1640, prefix, [new] * n, 8, 1, 128, "bf16")
    c["scale"] = 1.0
    bits = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731
    c["q"][:] = 0
    c["q"][:, :, 0] = bits(1.0)
    rng = np.random.default_rng(5)
    for r, pre in enumerate(prefix):
        at = np.arange(pre + new)
        page, slot = c["pt"][r, at // 16], at % 16
        k = np.zeros((len(at), 1, 128), np.float32)
        k[:, 0, 0] = np.where(np.isin(at // 32, low), 0.0, 9.6875)
        v = np.where(np.arange(128) % 3, 1.0, -1.0) * (1 + rng.random((len(at), 1, 128)) * 0.99) * value
        c["k"][page, :, slot, :] = bits(k)
        c["v"][page, :, :, slot] = bits(v)
    return c


@pytest.mark.parametrize("new", SIZES)
def test_large_values_under_rising_scores(new):
    """Items that run whole: 2^14 times the weights of the first tile, times V of 2^112, times 130 keys are beyond fp32."""
    c = steep(new, [130, 75], 2.0 ** 112, [0])
    assert A.dopd_window_workspace_size(U.shape_of(c), c["cu"], c["prefix"], 2, 10 ** 6, 0) == 256
    ref = U.window_reference(c, 10 ** 6, 0)
    assert np.isfinite(ref[0]).all()
    U.check(U.run(c, ("window", 10 ** 6, 0)), ref, c, f"V of 2^112, {new}")


@pytest.mark.parametrize("new", [1, 6, 16])
def test_large_values_in_parts_that_start_low(new):
    """Every part's first tile is far below the rest of it, so that its weights (formed against the first tile) are up to
    2^14: V of 2^105 leaves each part finite, and the sum of the parts as they stand beyond fp32."""
    prefix, rows, seg = 3000, {1: 16, 6: 64, 16: 128}[new], {1: 8, 6: 8, 16: 20}[new]
    c = steep(new, [prefix], 1.0, [0])
    size = A.dopd_window_workspace_size(U.shape_of(c), c["cu"], c["prefix"], 1, 10 ** 6, 0)
    parts = size // (2 * rows * (128 + 2) * 4)
    units = seg + (prefix + new + 31) // 32
    first = [max(0, i * (units // parts) + min(i, units % parts) - seg) for i in range(parts)]
    assert parts >= 8 and len(set(first)) >= 8
    c = steep(new, [prefix], 2.0 ** 105, first)
    ref = U.window_reference(c, 10 ** 6, 0)
    assert np.isfinite(ref[0]).all()
    U.check(U.run(c, ("window", 10 ** 6, 0)), ref, c, f"V of 2^105 in {parts} parts, {new}")
