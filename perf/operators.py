"""What the attention variants of the paged cache and the calls that rearrange its pages are timed on.

A case is a dict of plain values; ``op`` names the operator:

* ``window``  -- causal attention over the paged cache in which a token sees the last ``window`` positions and the
  first ``sinks`` ones (a decode step is a chunk of one token);
* ``tree``    -- the tokens of a drafted tree attend to the whole cached prefix and to their ancestors in the tree;
* ``copy``    -- whole pages copied to other pages of the pools, in every layer;
* ``compact`` -- the accepted tokens of a drafted tree moved to the places right behind the prefix, in every layer.

Request lengths and tree shapes follow the case alone (its length law and ``lengths`` seed); values, page orders,
scales, the pages copied and the tokens accepted follow the seed given to ``prepare``.

The plain forms gather the keys that a call can see into padded arrays and work in float32; ``exact`` goes through
the requests one by one in float64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # true: run() calls the library, false: it computes the plain forms

PAGE = 16  # tokens of a cache page
DEV = "cuda"
TORCH_TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.uint8}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # A lightly loaded instance decodes four short conversations of a model with windowed layers: latency alone.
        dict(name="window_small", op="window", dtype="bf16", hq=64, hkv=8, d=128, n=4, chunk=1, law="uniform", lo=100,
             hi=500, window=256, sinks=4, lengths=31),
        # High-concurrency decode, long and short contexts mixed: the longest see a window and the first tokens.
        dict(name="window_decode_70b", op="window", dtype="bf16", hq=64, hkv=8, d=128, n=256, chunk=1, law="bimodal",
             lo=100, hi=500, long_lo=4096, long_hi=16384, window=4096, sinks=4, lengths=32),
        # A full chunked-prefill call of windowed layers, 16 prompts behind prefixes of different lengths.
        dict(name="window_chunk", op="window", dtype="bf16", hq=32, hkv=32, d=128, n=16, chunk=512, law="lognormal",
             median=1000, sigma=1.0, lo=0, hi=8192, window=1024, sinks=16, lengths=33),
        # Two long prompts' chunks over an E4M3 cache, a wide window that ends inside pages.
        dict(name="window_chunk_fp8", op="window", dtype="fp8", hq=64, hkv=8, d=128, n=2, chunk=1021, law="uniform",
             lo=7000, hi=9000, window=4001, sinks=4, lengths=34),
        # A few small trees, fp32 throughout, head_dim 64: the smallest attention call.
        dict(name="tree_small_fp32", op="tree", dtype="fp32", hq=8, hkv=2, d=64, n=4, nodes=7, law="uniform", lo=5,
             hi=120, lengths=35),
        # Speculative decode of a 70B-shaped GQA layer: trees of 8 drafts over ordinary contexts.
        dict(name="tree_batch", op="tree", dtype="bf16", hq=64, hkv=8, d=128, n=64, nodes=8, law="lognormal",
             median=2048, sigma=0.7, lo=64, hi=16384, lengths=36),
        # The same for a 7B-shaped MHA layer, 16 drafts a tree (one MFMA column block per head).
        dict(name="tree_mha_7b", op="tree", dtype="bf16", hq=32, hkv=32, d=128, n=32, nodes=16, law="lognormal",
             median=1024, sigma=0.8, lo=16, hi=4096, lengths=37),
        # Large ragged trees over an E4M3 cache: as much arithmetic as a chunk of a prefill.
        dict(name="tree_wide_fp8", op="tree", dtype="fp8", hq=64, hkv=8, d=128, n=16, nodes=61, law="uniform",
             lo=2000, hi=8000, lengths=38),
        # One conversation forks: its last page is copied in one layer's pools (E4M3).
        dict(name="copy_small_fp8", op="copy", dtype="fp8", hq=64, hkv=8, d=128, layers=1, copies=3, pages=256),
        # A batch of sampled continuations forks, and a pool is defragmented: 700 pages in all 28 layers.
        dict(name="copy_28_layers", op="copy", dtype="bf16", hq=28, hkv=4, d=128, layers=28, copies=700, pages=4096),
        # The drafts that one request accepted, one layer.
        dict(name="compact_small", op="compact", dtype="bf16", hq=64, hkv=8, d=128, layers=1, n=1, nodes=7, most=4,
             law="uniform", lo=100, hi=500, lengths=39),
        # A whole batch's accepted drafts in all 28 layers.
        dict(name="compact_28_layers", op="compact", dtype="bf16", hq=28, hkv=4, d=128, layers=28, n=192, nodes=16,
             most=6, law="lognormal", median=256, sigma=0.7, lo=16, hi=1024, lengths=40),
    ]


HEADS = ((32, 32, 128), (64, 8, 128), (28, 4, 128), (32, 8, 128), (16, 16, 64), (32, 8, 64), (8, 2, 64))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("window", "window", "window", "tree", "tree", "tree", "copy", "compact"))
    hq, hkv, d = rng.choice(HEADS)
    c = dict(op=op, hq=hq, hkv=hkv, d=d, dtype=rng.choice(("bf16", "bf16", "fp8", "fp32")))
    if op == "copy":
        c.update(layers=_log(rng, 1, 28), copies=_log(rng, 1, 700))
        c["pages"] = 2 * c["copies"] + _log(rng, 64, 2048)
        while _cost(c) > _most():
            c["copies"] = max(1, c["copies"] * 2 // 3)
        return c
    c.update(lengths=rng.randrange(1 << 30), law="lognormal", sigma=rng.uniform(0.1, 1.0))
    if op == "compact":
        c.update(n=_log(rng, 1, 192), layers=_log(rng, 1, 28), nodes=_log(rng, 2, 64), median=_log(rng, 16, 512), lo=1,
                 hi=1024)
        c["most"] = min(c["nodes"], _log(rng, 1, 12))
    elif op == "tree":
        c.update(n=_log(rng, 1, 64), nodes=_log(rng, 1, 128), median=_log(rng, 32, 6000), lo=1, hi=16384)
    elif rng.random() < 0.5:  # decode steps
        c.update(n=_log(rng, 1, 256), chunk=1, median=_log(rng, 64, 8000), lo=0, hi=16384)
    else:
        c.update(n=_log(rng, 1, 16), chunk=_log(rng, 2, 1024), median=_log(rng, 64, 6000), lo=0, hi=8192)
    if op == "window":
        c.update(window=_log(rng, 16, 4096), sinks=rng.choice((0, 1, 4, 4, 16, 37)))
    if c["dtype"] == "fp32":  # the parity type: small calls
        c["n"], c["hi"] = min(c["n"], 8), 512
        c.update({k: min(c[k], 64) for k in ("chunk", "nodes") if k in c})
    while _cost(c) > _most() and c["n"] > 1:
        c["n"] = max(1, c["n"] * 2 // 3)
    return c


def _most():
    return max(_cost(c) for c in listed())


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


# ---------------------------------------------------------------- lengths, trees and work
def _lens(c):
    """Cached tokens of the case's requests before the call (for decode steps: before the step's own token)."""
    r = np.random.default_rng(c["lengths"])
    n = c["n"]
    if c["law"] == "lognormal":
        v = np.exp(r.normal(math.log(c["median"]), c["sigma"], n))
        return np.clip(np.rint(v), c["lo"], c["hi"]).astype(np.int64)
    v = r.integers(c["lo"], c["hi"] + 1, n)
    if c["law"] == "bimodal":
        at = r.permutation(n)[: round(0.2 * n)]
        v[at] = r.integers(c["long_lo"], c["long_hi"] + 1, len(at))
    return v.astype(np.int64)


def _new(c):
    """New tokens of each request: the chunk, or its drafted tree (the nodes of a case, a few requests with fewer)."""
    if c["op"] == "window":
        return np.full(c["n"], c["chunk"], np.int64)
    r = np.random.default_rng(c["lengths"] + 1)
    few = r.integers(1, c["nodes"] + 1, c["n"])
    return np.where(r.random(c["n"]) < 0.15, few, c["nodes"]).astype(np.int64)


def _sees(c):
    """[nodes][nodes] truth values: which drafts a draft of the case's tree sees (itself and its ancestors).  A node
    hangs from one of the few before it, so that paths grow as drafting by depth makes them; smaller trees are the
    first nodes of it."""
    r = np.random.default_rng(c["lengths"] + 2)
    sees = np.zeros((c["nodes"], c["nodes"]), bool)
    for i in range(c["nodes"]):
        p = i - 1 - int(r.integers(0, 5))
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def _words(c):
    return (c["nodes"] + 31) // 32


def work(case):
    c = case
    size = {"bf16": 2, "fp32": 4, "fp8": 1}[c["dtype"]]
    fresh = 4 if c["dtype"] == "fp32" else 2
    row = c["hkv"] * c["d"]  # elements of one token's K or V
    if c["op"] == "copy":  # every page read once and written once, K and V
        return {"bytes": 4 * c["layers"] * c["copies"] * PAGE * row * size + 8 * c["copies"], "flops": 0}
    pre, new = _lens(c), _new(c)
    if c["op"] == "compact":  # of each request up to `most` tokens, half of them on average
        moved = int(np.minimum(new, c["most"]).sum()) / 2
        return {"bytes": 4 * c["layers"] * moved * row * size, "flops": 0}
    total = int(new.sum())
    if c["op"] == "window":
        w, s = c["window"], c["sinks"]
        end = pre + new
        low = np.maximum(0, pre - w + 1)
        keys = int((end - low + np.minimum(low, s)).sum())
        p = np.concatenate([a + np.arange(b) for a, b in zip(pre, new)])
        seen = float((np.minimum(p + 1, w) + np.clip(p + 1 - w, 0, s)).sum())
        masks = 0
    else:
        keys = int((pre + new).sum())
        depth = np.cumsum(_sees(c).sum(1))
        seen = float((pre * new).sum() + depth[new - 1].sum())
        masks = 4 * total * _words(c)
    return {"bytes": 2 * keys * row * size + 2 * total * c["hq"] * c["d"] * fresh + 4 * total * c["hq"] + masks +
            4 * keys // PAGE, "flops": 4 * c["d"] * c["hq"] * seen}


# ---------------------------------------------------------------- inputs
def _i32(a):
    """An int32 host array and its device copy."""
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, torch.from_numpy(a).to(DEV)


def _tables(g, lens):
    """Page table of requests of `lens` tokens over a pool a quarter larger than they need, in random page order."""
    need = (lens + PAGE - 1) // PAGE
    pages = max(1, int(math.ceil(1.25 * need.sum())))
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = np.arange(max(1, int(need.max())))[None, :]
    start = np.cumsum(need) - need
    pt = perm[torch.from_numpy(np.where(at < need[:, None], start[:, None] + at, 0)).to(DEV)]
    pt[torch.from_numpy(at >= need[:, None]).to(DEV)] = -1
    return pt.contiguous(), pages


def _pools(g, c, pages, lead=()):
    """K and V pools full of N(0, 1), or of its codes under scales that put the largest values near the top code."""
    ks, vs = lead + (pages, c["hkv"], PAGE, c["d"]), lead + (pages, c["hkv"], c["d"], PAGE)
    if c["dtype"] != "fp8":
        return tuple(torch.randn(x, generator=g, device=DEV, dtype=TORCH_TYPE[c["dtype"]]) for x in (ks, vs)) + (None, None)
    scales = [(0.8 + 0.4 * torch.rand(c["hkv"], generator=g, device=DEV)) * (5.5 / 448.0) for _ in range(2)]

    def codes(shape, scale):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        x = x / scale.view(c["hkv"], 1, 1).to(torch.bfloat16)
        return x.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    return codes(ks, scales[0]), codes(vs, scales[1]), scales[0], scales[1]


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(op=c["op"], fp8=c["dtype"] == "fp8", hq=c["hq"], hkv=c["hkv"], d=c["d"])
    if c["op"] == "copy":
        s["pages"], s["layers"] = c["pages"], c["layers"]
        s["k"], s["v"], _, _ = _pools(g, c, c["pages"], (c["layers"],))
        perm = torch.randperm(c["pages"], generator=g, device=DEV).to(torch.int32)
        s["dst"] = perm[: c["copies"]].contiguous()
        rest = perm[c["copies"]:]  # a page may be copied to several (a fork into several continuations)
        s["src"] = rest[torch.randint(len(rest), (c["copies"],), generator=g, device=DEV)].contiguous()
    else:
        pre, new = _lens(c), _new(c)
        s["n"] = c["n"]
        s["pre_h"], s["pre"] = _i32(pre)
        s["pt"], s["pages"] = _tables(g, pre + new)
        if c["op"] == "compact":
            s["layers"], s["most"] = c["layers"], c["most"]
            s["k"], s["v"], _, _ = _pools(g, c, s["pages"], (c["layers"],))
            r = np.random.default_rng(seed)
            count = r.integers(0, np.minimum(new, c["most"]) + 1)
            path = np.zeros((c["n"], c["most"]), np.int64)
            for i, m in enumerate(count):
                path[i, :m] = np.sort(r.permutation(new[i])[:m])
            (_, s["count"]), (_, s["path"]) = _i32(count), _i32(path)
        else:
            fresh = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
            s["k"], s["v"], s["ks"], s["vs"] = _pools(g, c, s["pages"])
            s["cu_h"], s["cu"] = _i32(np.concatenate([[0], np.cumsum(new)]))
            t = int(s["cu_h"][-1])
            s["q"] = torch.randn((t, c["hq"], c["d"]), generator=g, device=DEV, dtype=fresh)
            s["out"] = torch.zeros((t, c["hq"], c["d"]), device=DEV, dtype=fresh)
            s["lse"] = torch.zeros((t, c["hq"]), device=DEV)
            if c["op"] == "window":
                s["window"], s["sinks"] = c["window"], c["sinks"]
            else:
                bits = np.zeros((c["nodes"], 32 * _words(c)), bool)
                bits[:, : c["nodes"]] = _sees(c)
                rows = np.packbits(bits, axis=1, bitorder="little").view("<u4")
                rows = np.concatenate([rows[:m] for m in new])
                s["mask"], s["words"] = _i32(rows.view(np.int32))[1], _words(c)
    if own:
        from paper_2511_20982_amd import attn as A
        s["A"], s["shape"] = A, A.make_shape(c["hq"], c["hkv"], c["d"], c["dtype"])
        if c["op"] == "window":
            s["ws"] = A.window_workspace(s["shape"], s["cu_h"], s["pre_h"], s["n"], c["window"], c["sinks"])
        elif c["op"] == "tree":
            s["ws"] = A.tree_workspace(s["shape"], s["cu_h"], s["pre_h"], s["n"])
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    s = state
    if own:
        return _call(s)
    if s["op"] == "copy":
        return _plain_copy(s)
    return _plain_compact(s) if s["op"] == "compact" else _plain_attention(s)


def _stored(s):
    """The pools as the values they hold."""
    return [p.view(torch.float8_e4m3fn) if s["fp8"] else p for p in (s["k"], s["v"])]


def _call(s):
    A, sh = s["A"], s["shape"]
    if s["op"] == "copy":
        A.dopd_kv_copy_pages(sh, s["layers"], s["k"], s["v"], s["pages"], s["src"], s["dst"], len(s["src"]))
        return _stored(s)
    table = (s["pages"], s["pt"], s["pt"].shape[1])
    if s["op"] == "compact":
        A.dopd_kv_compact(sh, s["layers"], s["k"], s["v"], *table, s["pre"], s["path"], s["count"], s["most"], s["n"])
        return _stored(s)
    rows = (s["cu"], s["cu_h"], s["pre"], s["pre_h"], s["n"])
    how = (s["window"], s["sinks"]) if s["op"] == "window" else (s["mask"], s["words"])
    scales = (s["ks"], s["vs"]) if s["fp8"] else ()
    call = {("window", False): A.dopd_window_attn, ("window", True): A.dopd_window_attn_fp8,
            ("tree", False): A.dopd_tree_attn, ("tree", True): A.dopd_tree_attn_fp8}[s["op"], s["fp8"]]
    call(sh, s["q"], s["k"], s["v"], *scales, *table, *rows, *how, s["out"], s["lse"], s["ws"])
    return s["out"], s["lse"]


# ---------------------------------------------------------------- plain forms
def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]
    return _stored(s)


def _plain_compact(s):
    at = torch.arange(s["most"], device=DEV)
    live = at < s["count"][:, None]
    to = s["pre"][:, None].long() + at
    to = torch.where(live, to, s["pre"][:, None].long())
    fr = torch.where(live, s["pre"][:, None].long() + s["path"], to)
    page = lambda pos: torch.gather(s["pt"], 1, pos // PAGE).long()  # noqa: E731
    some = live[:, :1]  # what is not live goes where the request's first accepted token goes, with its value
    for pool, tokens in ((s["k"], 3), (s["v"], 4)):
        rows = pool.movedim(tokens, 2)  # [layers, pages, slot, hkv, d]
        old = rows[:, page(to), to % PAGE]
        new = rows[:, page(fr), fr % PAGE]
        spare = torch.where(some[None, :, :, None, None], new[:, :, :1], old)
        new = torch.where(live[None, :, :, None, None], new, spare)
        rows[:, page(to), to % PAGE] = new
    return _stored(s)


def _gathered(s, pos):
    """K and V [request, head, key, d] in float32 of the cached positions `pos` [request, key]."""
    page, slot = torch.gather(s["pt"], 1, pos // PAGE).long(), pos % PAGE
    k, v = s["k"][page, :, slot], s["v"][page, :, :, slot]  # [request, key, head, d]
    if s["fp8"]:
        k, v = (x.view(torch.float8_e4m3fn) for x in (k, v))
    k, v = k.float().transpose(1, 2), v.float().transpose(1, 2)
    if s["fp8"]:
        k, v = k * s["ks"].view(-1, 1, 1), v * s["vs"].view(-1, 1, 1)
    return k.contiguous(), v.contiguous()


def _plain_attention(s):
    n, hkv, g, d = s["n"], s["hkv"], s["hq"] // s["hkv"], s["d"]
    pre, cu = s["pre"].long(), s["cu"].long()
    new = cu[1:] - cu[:-1]
    total, most = len(s["q"]), int((s["cu_h"][1:] - s["cu_h"][:-1]).max())
    row = torch.arange(total, device=DEV)
    req = torch.searchsorted(cu, row, right=True) - 1
    i = row - cu[req]
    last = (pre + new - 1)[:, None]
    p = pre[:, None] + torch.arange(most, device=DEV)  # [request, token]: its position
    if s["op"] == "window":
        w, sinks = s["window"], s["sinks"]
        low = (pre - w + 1).clamp(min=0)[:, None]
        sink, near = torch.arange(sinks, device=DEV)[None], low + torch.arange(min(w, int(s["pre_h"].max()) + 1) + most - 1, device=DEV)
        pos = torch.cat([sink.expand(n, -1), near], 1)
        real = torch.cat([(sink < low).expand(n, -1), near <= last], 1)
        key, at = pos[:, None], p[:, :, None]
        seen = real[:, None] & (key <= at) & ((key > at - w) | (key < sinks))
    else:
        pos = torch.arange(int((s["pre_h"] + s["cu_h"][1:] - s["cu_h"][:-1]).max()), device=DEV)[None].expand(n, -1)
        draft = pos - pre[:, None]  # [request, key]: which draft a key is
        mask = torch.zeros((n, most, s["words"]), dtype=torch.int32, device=DEV)
        mask[req, i] = s["mask"]
        at = draft.clamp(0, 32 * s["words"] - 1)
        bits = torch.gather(mask, 2, (at // 32)[:, None].expand(-1, most, -1)) >> (at % 32)[:, None].int()
        seen = (draft < 0)[:, None] | ((bits & 1 == 1) & (pos <= last)[:, None])
    pos = torch.minimum(pos, last).contiguous()
    k, v = _gathered(s, pos)
    q = torch.zeros((n, most, s["hq"], d), device=DEV)
    q[req, i] = s["q"].float()
    q = q.view(n, most, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * most, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(n, hkv, g, most, -1) * (1.0 / math.sqrt(d))
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)  # (a row that sees nothing: 0 everywhere)
    e = torch.exp(x - top)
    total_e = e.sum(-1, keepdim=True)
    out = torch.matmul(e.view(n, hkv, g * most, -1), v).view(n, hkv, g, most, d) / total_e.clamp(min=1e-30)
    lse = (top + torch.log(total_e)).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(n, most, s["hq"], d)[req, i]
    return out.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(n, most, s["hq"])[req, i]


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    c = case
    if c["op"] in ("copy", "compact"):  # bits that move: nothing is computed
        return None
    s = prepare(c, seed)
    pre, new, g = _lens(c), _new(c), c["hq"] // c["hkv"]
    sees = None if c["op"] == "window" else torch.from_numpy(_sees(c)).to(DEV)
    outs, lses = [], []
    for r in range(c["n"]):
        m, end, start = int(new[r]), int(pre[r] + new[r]), int(s["cu_h"][r])
        pages = s["pt"][r, : (end + PAGE - 1) // PAGE].long()
        k, v = s["k"][pages], s["v"][pages]
        if c["dtype"] == "fp8":
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        k = k.double().permute(1, 0, 2, 3).reshape(c["hkv"], -1, c["d"])[:, :end]
        v = v.double().permute(1, 0, 3, 2).reshape(c["hkv"], -1, c["d"])[:, :end]
        if c["dtype"] == "fp8":
            k, v = k * s["ks"].double().view(-1, 1, 1), v * s["vs"].double().view(-1, 1, 1)
        hidden = torch.zeros((m, end), dtype=torch.bool, device=DEV)
        if c["op"] == "window":
            j, p = torch.arange(end, device=DEV), int(pre[r]) + torch.arange(m, device=DEV)[:, None]
            hidden |= (j > p) | ((p - j >= c["window"]) & (j >= c["sinks"]))
        else:
            hidden[:, int(pre[r]):] = ~sees[:m, :m]
        o = torch.empty((m, c["hq"], c["d"]), dtype=torch.float64, device=DEV)
        z = torch.empty((m, c["hq"]), dtype=torch.float64, device=DEV)
        for h in range(c["hq"]):
            y = s["q"][start: start + m, h].double() @ k[h // g].T.contiguous() / math.sqrt(c["d"])
            y = y.masked_fill(hidden, -math.inf)
            z[:, h] = torch.logsumexp(y, 1)
            o[:, h] = torch.exp(y - z[:, h: h + 1]) @ v[h // g]
        outs.append(o)
        lses.append(z)
    return torch.cat(outs), torch.cat(lses)
