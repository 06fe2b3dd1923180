"""Helpers for the tests of the windowed and the tree attention: cases over pools
whose dead slots hold NaN, the calls, and the error bounds.

Bounds (u(t) half a rounding step of type t: bf16 2^-8, fp32 2^-24).  With W = sum p |v| / sum p and P the largest
sum of absolute products in a score of the row, both in log units:
  a score is off by at most e_s = d u(fp32) P (products and sums in fp32) + 4 u(fp32) (P + |lse|) (scale, maximum);
  a weight by a factor of 1 + 2 e_s + 8 u(fp32) (exponential), and for bf16 by 1 + u(bf16) more (rounded for the MFMA);
  sums of n weights by n u(fp32) (any order), the merge of parts and the division by 32 u(fp32) more;
  the output of bf16 is rounded once more.
So |out - ref| <= W (2 (2 e_s + 8 u + n u + 32 u) + [u(bf16)]) + [u(bf16) (|ref| + what precedes)], and
|lse - ref| <= 2 e_s + (8 + n + 32) u + 4 u |lse|.
"""
from __future__ import annotations

import numpy as np
import torch

import oracle
from oracle import masked as M
from paper_2511_20982_amd import attn as A
from paper_2511_20982_amd import inputs as I
from tests import gpu_util as G

U32, UBF = 2.0 ** -24, 2.0 ** -8
DEV = "cuda"


def case(seed, prefix, new, hq, hkv, d, dtype, spread=1.0):
    """Pools with prefix + new tokens of each request (NaN in every other slot) and the new rows of Q."""
    rng = np.random.default_rng(seed)
    prefix, new = np.asarray(prefix, np.int32), np.asarray(new, np.int32)
    total = prefix + new
    pt, pages = I.allocate_pages(rng, np.maximum(total, 1))
    fresh = "fp32" if dtype == "fp32" else "bf16"
    kp, vp = I.empty_pools(pages, hkv, d, fresh)
    _, kf, vf = I.prefill_batch(rng, total, hq, hkv, d, fresh)
    kp, vp = oracle.kv_write(kf, vf, kp, vp, pt, I.cu_from_lens(total), np.zeros(len(total), np.int32))
    q = I.normal(rng, (int(new.sum()), hq, d), fresh)
    c = dict(q=q, k=kp, v=vp, pt=pt, cu=I.cu_from_lens(new), prefix=prefix, hq=hq, hkv=hkv, d=d, dtype=dtype, ks=None,
             vs=None, scale=1.0 / np.sqrt(d))
    if dtype == "fp8":
        c["ks"] = (0.02 + 0.01 * rng.random(hkv)).astype(np.float32)
        c["vs"] = (0.02 + 0.01 * rng.random(hkv)).astype(np.float32)
        c["k"], c["v"] = G.quantize_pools(kp, vp, c["ks"], c["vs"])  # (NaN stays NaN: code 0x7f)
    return c


def reference(c, sees):
    return M.attention(c["q"], c["k"], c["v"], c["pt"], c["cu"], c["prefix"], c["scale"], sees, c["ks"], c["vs"])


def window_reference(c, window, sinks):
    return reference(c, lambda r, i: M.window_sees(int(c["prefix"][r]) + i, window, sinks))


def tree_reference(c, mask):
    n = np.diff(c["cu"])
    return reference(c, lambda r, i: M.tree_sees(int(c["prefix"][r]), int(n[r]), mask[int(c["cu"][r]) + i]))


def check(got, ref, c, what):
    """got, ref: (out, lse) and what `attention` returns."""
    out, lse = got
    want, want_lse, weighted, products = ref
    u = U32
    most = int((c["prefix"] + np.diff(c["cu"])).max()) if len(c["prefix"]) else 0
    empty = np.isneginf(want_lse)
    flat = np.where(np.isfinite(want_lse), want_lse, 0.0)
    e_s = c["d"] * u * products + 4 * u * (products + np.abs(flat))
    rel = 2 * (2 * e_s + (8 + most + 32) * u)
    tol = weighted * (rel[..., None] + (0 if c["dtype"] == "fp32" else UBF))
    if c["dtype"] != "fp32":
        tol = tol + UBF * (np.abs(want) + tol)
    finite = np.isfinite(want)
    assert np.array_equal(np.isfinite(out), finite), f"{what}: {np.argwhere(np.isfinite(out) != finite)[:4]} finite or not"
    err = np.where(finite, np.abs(np.where(finite, out, 0) - np.where(finite, want, 0)), 0)
    tol = np.where(finite, tol, 1)
    bad = np.argwhere(err > tol + 1e-30)
    assert len(bad) == 0, f"{what}: {len(bad)} outputs off, first at {bad[0]}: {err[tuple(bad[0])]:.3e} > {tol[tuple(bad[0])]:.3e}"
    if lse is None:
        return
    assert np.array_equal(np.isneginf(lse), empty), f"{what}: lse of rows that see nothing"
    ok = np.isfinite(want_lse)
    assert np.array_equal(np.isfinite(lse), ok), f"{what}: lse finite or not"
    err = np.abs(np.where(ok, lse, 0) - flat)
    tol = 2 * e_s + (8 + most + 32) * u + 4 * u * np.abs(flat)
    assert (err[ok] <= tol[ok]).all(), f"{what}: lse off by {err[ok].max():.3e}, bound {tol[ok].min():.3e}"


def on_device(c):
    """The case's arrays on the GPU."""
    dev = {k: A.to_device(c[k]) for k in ("q", "k", "v", "pt", "cu", "prefix")}
    if c["ks"] is not None:
        dev["ks"], dev["vs"] = A.to_device(c["ks"]), A.to_device(c["vs"])
    return dev


def shape_of(c):
    return A.make_shape(c["hq"], c["hkv"], c["d"], c["dtype"], c["scale"])


def run(c, how, dev=None, with_lse=True, stream=None):
    """how: ("window", window, sinks) or ("tree", mask).  The output is guarded, the workspace full of 0xff."""
    dev = dev or on_device(c)
    sh = shape_of(c)
    out, obuf, margin = G.guarded(dev["q"].shape, dev["q"].dtype)
    lse = torch.full(c["q"].shape[:2], float("nan"), device=DEV) if with_lse else None
    n = len(c["prefix"])
    if how[0] == "window":
        size = A.dopd_window_workspace_size(sh, c["cu"], c["prefix"], n, how[1], how[2])
        extra = how[1:]
    else:
        size = A.dopd_tree_workspace_size(sh, c["cu"], c["prefix"], n)
        extra = (A.to_device(how[1].view(np.int32)), how[1].shape[1])
    assert size >= 256 and size % 256 == 0
    wbuf = torch.full((size + 4096 + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    off = (-wbuf.data_ptr()) % 256
    ws = wbuf[off:off + size]
    scales = (dev["ks"], dev["vs"]) if c["dtype"] == "fp8" else ()
    name = f"dopd_{how[0]}_attn" + ("_fp8" if c["dtype"] == "fp8" else "")
    torch.cuda.synchronize()
    getattr(A, name)(sh, dev["q"], dev["k"], dev["v"], *scales, c["k"].shape[0], dev["pt"], c["pt"].shape[1], dev["cu"],
                     c["cu"], dev["prefix"], c["prefix"], n, *extra, out, lse, ws, size, stream=stream)
    torch.cuda.synchronize()
    assert bool((wbuf[off + size:] == 0xFF).all()), "wrote past its workspace"
    assert G.canary_intact(obuf, margin, out.numel() * out.element_size()), "wrote past the output"
    return G.widen(A.to_host(out)), (lse.cpu().numpy().astype(np.float64) if with_lse else None)


def random_tree(rng, n, words=None, empty=0.0):
    """Mask words of a random tree of n drafts (a share `empty` of the rows sees no draft at all)."""
    words = words or max(1, (n + 31) // 32)
    bits = np.zeros((n, 32 * words), bool)
    for i in range(n):
        p = int(rng.integers(-1, i)) if i else -1
        if p >= 0:
            bits[i] = bits[p]
        bits[i, i] = True
    bits[rng.random(n) < empty] = False
    return np.packbits(bits, axis=1, bitorder="little").view("<u4").astype(np.uint32)


def tree_masks(rng, lens, words, empty=0.0):
    lens = [int(n) for n in lens]
    return np.concatenate([random_tree(rng, n, words, empty) for n in lens if n] or [np.zeros((0, words), np.uint32)])
