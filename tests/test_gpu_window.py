"""GPU: windowed attention with sinks over the paged cache against the fp64 reference."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(require_gpu):
    pass


from tests import masked_util as U  # noqa: E402

PREFIX = [0, 1, 15, 16, 17, 63, 64, 65, 200, 777, 0, 40, 129, 500]
CHUNK = [9, 1, 16, 30, 64, 65, 128, 129, 1, 140, 0, 33, 2, 1]


def both(c, window, sinks, what=""):
    U.check(U.run(c, ("window", window, sinks)), U.window_reference(c, window, sinks), c,
            f"window {window} sinks {sinks} {c['hq']}/{c['hkv']} d {c['d']} {c['dtype']} {what}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (8, 2), (7, 1), (32, 1)])
def test_ragged_batch(hq, hkv, d, dtype):
    c = U.case(900 + hq + d, PREFIX, CHUNK, hq, hkv, d, dtype)
    for window, sinks in ((1, 0), (100, 4)):
        both(c, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("window,sinks", [(1, 1), (5, 0), (16, 16), (17, 3), (64, 70), (65, 130), (333, 17), (5000, 4)])
def test_windows_and_sinks(window, sinks, dtype):
    both(U.case(910, [0, 3, 400, 61, 1000, 700], [40, 1, 1, 90, 2, 150], 8, 2, 128, dtype), window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [128, 64])
def test_decode_steps_split_over_workgroups(d, dtype):
    """Few long contexts, more than one workgroup each; a wide group on the other kernel."""
    both(U.case(920, [3000, 1500, 20], [1, 1, 1], 8, 2, d, dtype), 2000, 4)
    both(U.case(921, [2500], [3], 32, 1, d, dtype), 1900, 20)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_window_of_the_whole_context_is_causal_attention(dtype):
    c = U.case(930, [0, 5, 300], [20, 1, 130], 4, 4, 64, dtype)
    ref = U.window_reference(c, 10 ** 6, 0)
    for window, sinks in ((2 ** 31 - 1, 0), (450, 2 ** 31 - 1), (1, 450)):
        U.check(U.run(c, ("window", window, sinks)), ref, c, f"{window} {sinks}")


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(scale):
    c = U.case(931, [0, 70, 5], [12, 90, 1], 4, 2, 128, "bf16")
    c["scale"] = scale
    both(c, 33, 2, f"scale {scale}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("new", [1, 2, 40])
def test_freed_pages_are_not_read(new, dtype):
    """Pages between the sinks and the window go back to the pool: their entries name a page full of NaN."""
    c = U.case(940, [700, 100], [new, new], 8, 2, 128, dtype)
    window, sinks = 90, 20
    ref = U.window_reference(c, window, sinks)
    freed = [set(range(c["k"].shape[0])) - set(c["pt"].ravel().tolist())][0].pop()
    c["k"][freed], c["v"][freed] = c["k"].dtype.type(0), c["v"].dtype.type(0)
    nan = {"bf16": 0x7FC0, "fp8": 0x7F, "fp32": np.nan}[dtype]
    c["k"][freed], c["v"][freed] = nan, nan
    for r, pre in enumerate(c["prefix"]):
        for t in range(c["pt"].shape[1]):
            if 16 * t >= sinks and 16 * t + 15 < pre - window + 1:
                c["pt"][r, t] = freed
    U.check(U.run(c, ("window", window, sinks)), ref, c, "freed pages")


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,hq,hkv", [(3, 8, 8), (4, 8, 2), (70, 8, 2), (12, 32, 1)])
def test_non_finite_values_reach_only_rows_that_see_them(new, hq, hkv, dtype, bad):
    window, sinks, pre = 50, 2, 130
    c = U.case(950, [pre, pre], [new, new], hq, hkv, 128, dtype)
    value = np.float32(bad) if dtype == "fp32" else np.uint16({"nan": 0x7FC0, "inf": 0x7F80, "-inf": 0xFF80}[str(bad)])
    for r, pos in ((0, pre - window + 1), (0, pre + new - 1), (1, pre + new // 2)):
        page, slot = c["pt"][r, pos // 16], pos % 16
        c["v"][page, 0, 5, slot] = value
        if r == 1 and not np.isneginf(bad):
            c["k"][page, hkv - 1, slot, 7] = value
    out, lse = U.run(c, ("window", window, sinks))
    want, want_lse, _, _ = ref = U.window_reference(c, window, sinks)
    ok = np.isfinite(want)
    assert 0 < ok.sum() < ok.size
    assert np.array_equal(np.isfinite(out), ok)
    out, want = np.where(ok, out, 0), np.where(ok, want, 0)
    lse = np.where(np.isfinite(want_lse), lse, want_lse)
    clean = tuple(np.where(np.isfinite(x), x, 0) for x in ref[2:])
    U.check((out, None), (want, want_lse, *clean), c, "non-finite values")
    assert np.max(np.abs(np.where(np.isfinite(want_lse), lse - want_lse, 0))) < 1e-4


def test_lse_may_be_left_out_and_an_empty_call_touches_nothing():
    c = U.case(960, [30, 5], [20, 1], 4, 2, 64, "bf16")
    ref = U.window_reference(c, 9, 1)
    U.check(U.run(c, ("window", 9, 1), with_lse=False), ref, c, "no lse")
    c = U.case(961, [3, 4], [0, 0], 4, 2, 64, "bf16")
    U.run(c, ("window", 9, 1))
