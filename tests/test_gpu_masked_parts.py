"""GPU: windowed and tree attention in calls whose contexts several workgroups share, where what one part of a row's keys
holds has to survive the merge of the parts, and only that: NaN in Q and in K, values that are not finite where some rows
or none see them, freed pages, rows that see nothing in any part or in some, and values of V near the largest finite
ones, whose sums stay finite as long as the weights are formed against the largest score."""
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


def finite_part(got, ref, c, what):
    """Finite where the reference is, and right there (bounds from the finite values)."""
    (out, lse), (want, want_lse, weighted, products) = got, ref
    ok, ok_lse = np.isfinite(want), np.isfinite(want_lse)
    assert 0 < ok.sum() < ok.size
    assert np.array_equal(np.isfinite(out), ok), f"{what}: {np.argwhere(np.isfinite(out) != ok)[:4]}"
    assert np.array_equal(np.isfinite(lse), ok_lse), what
    zero = lambda x, at: np.where(at, x, 0)  # noqa: E731
    U.check((zero(out, ok), zero(lse, ok_lse)), (zero(want, ok), zero(want_lse, ok_lse), zero(weighted, np.isfinite(weighted)),
                                                 zero(products, np.isfinite(products))), c, what)


@pytest.mark.parametrize("kind", HOWS)
@pytest.mark.parametrize("dtype,bad", [("bf16", np.nan), ("bf16", np.inf), ("fp8", np.nan)])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("new", [2, 6, 40])
def test_non_finite_values_in_parts_reach_only_rows_that_see_them(new, d, dtype, bad, kind):
    """V at the first position that the first row sees and others do not (windows), between the sinks and the window,
    inside the window, and at drafts that some rows see; K at a draft of its own request."""
    c = U.case(1660 + new, PREFIX, [new] * 3, 16, 2, d, dtype)
    value = np.uint16(0x7F80) if np.isinf(bad) else NAN[dtype]
    how, _ = calls(c, kind)
    if kind == "tree":
        c["v"][c["pt"][1, 700 // 16], 0, 3, 700 % 16] = value  # (all rows of that request see it)
        spots = [(0, 3000 + new // 2), (1, 1777 + new - 1)]
    else:
        spots = [(0, 3000 - 2000 + 1), (0, 500), (0, 3000 + new - 1)]
    for r, at in spots:
        c["v"][c["pt"][r, at // 16], :, 5, at % 16] = value
    last = 20 + new - 1
    if not np.isinf(bad):
        c["k"][c["pt"][2, last // 16], 1, last % 16, 7] = value
    how, ref = calls(c, kind)  # (the same mask)
    finite_part(U.run(c, how), ref(), c, f"{new} {d} {dtype} {bad} {kind}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("new", SIZES)
def test_freed_pages_between_parts(new, dtype):
    """Long contexts whose pages between the sinks and the window went back to the pool (entries of -1, and of a page
    full of NaN)."""
    window, sinks = 2000, 37
    c = U.case(1680 + new, [6000, 3500, 2100], [new] * 3, 8, 2, 128, dtype)
    how, ref = calls(c, "window")
    want = ref()
    freed = sorted(set(range(c["k"].shape[0])) - set(c["pt"].ravel().tolist()))[0]
    c["k"][freed], c["v"][freed] = NAN[dtype], NAN[dtype]
    count = 0
    for r, pre in enumerate(c["prefix"]):
        for t in range(c["pt"].shape[1]):
            if 16 * t >= sinks and 16 * t + 15 < pre - window + 1:
                c["pt"][r, t] = freed if t % 2 else -1
                count += 1
    assert count > 300
    U.check(U.run(c, how), want, c, f"freed pages {new} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
def test_rows_that_see_nothing_in_any_part(d, dtype):
    """Trees of hundreds of drafts without a cached token, split over workgroups: rows with an empty mask, rows that see
    the drafts of one part alone, rows that see all."""
    new = [700, 333]
    c = U.case(1690, [0, 0], new, 2, 1, d, dtype)
    rng = np.random.default_rng(3)
    bits = np.zeros((sum(new), 704), bool)
    for r, start in ((0, 0), (1, 700)):
        for i in range(new[r]):
            kind, at = i % 4, int(rng.integers(0, new[r]))
            if kind == 1:
                bits[start + i, at] = True
            elif kind == 2:
                bits[start + i, at:at + 40] = True  # (bits from n on are ignored)
            elif kind == 3:
                bits[start + i] = rng.random(704) < 0.5
    mask = np.packbits(bits, axis=1, bitorder="little").view("<u4").astype(np.uint32)
    assert A.dopd_tree_workspace_size(U.shape_of(c), c["cu"], c["prefix"], 2) > 256
    out, lse = U.run(c, ("tree", mask))
    ref = U.tree_reference(c, mask)
    empty = np.isneginf(ref[1])
    assert empty.sum() >= 2 * 250 and (out[empty] == 0).all()
    U.check((out, lse), ref, c, f"rows that see nothing {d} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_more_requests_than_a_wave_has_lanes(dtype):
    """150 requests of all sizes: the kernels look their items up 64 requests at a time."""
    rng = np.random.default_rng(8)
    prefix = rng.integers(0, 300, 150)
    prefix[[3, 70, 149]] = [2600, 1900, 2200]
    new = rng.choice([0, 1, 1, 1, 2, 5, 9, 40], 150)
    new[[3, 70, 149]] = [1, 9, 40]
    c = U.case(1695, prefix, new, 8, 2, 64, dtype)
    U.check(U.run(c, ("window", 1500, 4)), U.window_reference(c, 1500, 4), c, f"150 requests, window {dtype}")
    mask = U.tree_masks(rng, new, 2, 0.1)
    U.check(U.run(c, ("tree", mask)), U.tree_reference(c, mask), c, f"150 requests, tree {dtype}")


def steep(new, prefix, value, low, rise=9.6875):
    """Rows of a KV head with g = 8 whose scores are 0 in the 32-key tiles `low` and 9.6875 (14 octaves up) in the others,
    or `rise`, over V of value .. 2 value, of one sign in each dim."""
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
        k[:, 0, 0] = np.where(np.isin(at // 32, low), 0.0, rise)
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


@pytest.mark.parametrize("rise", [9.6875, 10.375, 11.0625, 13.8125, 14.5, 40.0, -40.0])
@pytest.mark.parametrize("prefix", [130, 3000])
@pytest.mark.parametrize("new", [1, 6, 16])
def test_scores_that_rise_around_the_limit_of_the_weights(new, prefix, rise):
    """By 14, 15, 16, 20, 21 and 58 octaves (8 and 16 keys of a lane sum to 2^17 .. 2^25 and to inf), and down by 58, in
    calls that run whole and in parts."""
    c = steep(new, [prefix], 1.0, [0, 3, 4, 41], rise)
    U.check(U.run(c, ("window", 10 ** 6, 0)), U.window_reference(c, 10 ** 6, 0), c, f"{new} {prefix} {rise}")


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("new", [1, 6, 40])
def test_a_scale_of_nan_reaches_only_rows_that_see_something(new, d):
    """A KV head with a k_scale of NaN: its rows are NaN, but those that see nothing have 0 and -inf."""
    c = U.case(1698, [0, 300, 0], [new] * 3, 16, 2, d, "fp8")
    c["ks"][1] = np.nan
    mask = U.tree_masks(np.random.default_rng(2), [new] * 3, 2)
    mask[:new:2] = 0
    out, lse = U.run(c, ("tree", mask))
    ref = U.tree_reference(c, mask)
    assert np.isneginf(ref[1]).any() and np.isnan(ref[1]).any()
    U.check((out, lse), ref, c, f"k_scale of NaN {new} {d}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("prefix", [75, 3000])
@pytest.mark.parametrize("new", [1, 6, 40])
def test_scores_that_are_all_minus_infinity(new, prefix, dtype):
    """Of one KV head's rows, in calls that run whole and in parts; the other head's rows are ordinary."""
    c = U.case(1699, [prefix], [new], 16, 2, 128, dtype)
    one, low = (np.float32(1), np.float32(-np.inf)) if dtype == "fp32" else (np.uint16(0x3F80), np.uint16(0xFF80))
    c["q"][:, 8:, 9] = one
    at = np.arange(prefix + new)
    c["k"][c["pt"][0, at // 16], 1, at % 16, 9] = low
    out, lse = U.run(c, ("window", 10 ** 6, 0))
    assert (out[:, 8:] == 0).all() and np.isneginf(lse[:, 8:]).all()
    want, want_lse, weighted, products = U.window_reference(c, 10 ** 6, 0)
    first = lambda x: np.ascontiguousarray(x[:, :8])  # noqa: E731
    U.check((first(out), first(lse)), tuple(map(first, (want, want_lse, weighted, products))), c, f"{new} {prefix} {dtype}")
