"""Operators on the paged KV cache, as cases to time and compare: rotary positions with the cache append, attention
with modified scores and masks (and the weights that the cached keys received), eviction by those weights.

A case is a dict of plain values: the operator, heads, element type of the cache, the request lengths (drawn from the
case's ranges with its own length seed, so that the amount of work is a property of the case) and the operator's own
settings.  Where ``own`` is false ``run`` computes the plain form in elementary torch operations, else it calls the
framework's kernels.  Requests with one new row come first, then those with a chunk of new rows.
"""
from __future__ import annotations

import math
import types

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16
SCALES = (0.5, 0.25)  # k_scale, v_scale of an 8-bit cache


def _case(op, heads, *, dec=(0, 0, 0), pre=(0, 0, 0, 0, 0), kv="bf16", lens=1, **more):
    """heads: query heads, KV heads, head_dim; dec: requests with one new row, shortest and longest context; pre:
    requests with a chunk, shortest and longest chunk, shortest and longest context before it."""
    return {"op": op, "nq": heads[0], "nkv": heads[1], "hd": heads[2], "n_dec": dec[0], "ctx_lo": dec[1],
            "ctx_hi": dec[2], "n_pre": pre[0], "chunk_lo": pre[1], "chunk_hi": pre[2], "prefix_lo": pre[3],
            "prefix_hi": pre[4], "kv": kv, "lens": lens, **more}


def _rotary(heads, rdim, layout, scaling, factor, far, **kw):
    """rdim: rotated dims; far: positions run up to this much ahead of the cache slots (0: they are the slots)."""
    return _case("rotary", heads, rdim=rdim, layout=layout, scaling=scaling, factor=factor, far=far, **kw)


def _attend(heads, *, cap=0.0, bias=False, window=0, docs=0, pad=False, two_way=False, weights=False, wrows=0, **kw):
    """cap: tanh cap of the scores; bias: distance bias; docs: mean document length of a document mask; pad: padding
    rows, which see nothing; two_way: half of each chunk and all before it is seen by every row; weights: accumulate
    what each key receives from the last wrows rows (0: all)."""
    return _case("attend", heads, cap=cap, bias=bias, window=window, docs=docs, pad=pad, two_way=two_way,
                 weights=weights, wrows=wrows, **kw)


def _evict(heads, keep, sink, recent, **kw):
    return _case("evict", heads, keep=keep, sink=sink, recent=recent, **kw)


_8B, _70B, _30B, _TINY = (32, 8, 128), (64, 8, 128), (32, 4, 128), (4, 2, 64)


def listed():
    return [
        # one user decoding after an eviction: a single row, its position far ahead of its slot (latency)
        dict(_rotary(_8B, 128, "half", "wavelength", 8.0, 100000, dec=(1, 700, 700)), name="rot_one"),
        # a full decode batch into an 8-bit cache, half of each head rotated in neighbouring pairs
        dict(_rotary(_70B, 64, "interleaved", "linear", 4.0, 60000, dec=(256, 64, 512), kv="fp8"), name="rot_dec256_fp8"),
        # the prompts of one prefill iteration, frequencies stretched for a long context
        dict(_rotary(_8B, 128, "half", "yarn", 16.0, 0, pre=(7, 700, 1600, 0, 512)), name="rot_pre7"),
        # one user decoding with capped scores (latency)
        dict(_attend(_8B, cap=50.0, dec=(1, 1500, 1500)), name="att_one_cap"),
        # an ordinary decode batch with capped scores that keeps account of the weights its keys receive
        dict(_attend(_8B, cap=30.0, weights=True, dec=(64, 512, 4096)), name="att_dec64_weights"),
        # few requests with very long contexts, distance bias, 8-bit cache
        dict(_attend(_70B, bias=True, dec=(13, 20000, 120000), kv="fp8"), name="att_dec13_long_bias"),
        # drafted tokens to verify: some rows each over long contexts, half of them behind a window
        dict(_attend(_30B, window=4096, pre=(24, 3, 9, 2000, 16000)), name="att_verify24_window"),
        # packed documents with padding at the end of each row of a prompt batch, weights from every row
        dict(_attend((32, 8, 64), docs=300, pad=True, weights=True, pre=(6, 900, 2000, 0, 0)), name="att_docs6_weights"),
        # one chunk of a long prompt with capped scores: the largest
        dict(_attend(_8B, cap=50.0, pre=(1, 4096, 4096, 32768, 32768)), name="att_chunk_32k_cap"),
        # a few short requests, two thirds kept (latency)
        dict(_evict(_TINY, 200, 4, 32, dec=(3, 250, 330)), name="evict_small"),
        # a running batch cut back to its budget, 8-bit cache, ragged, some requests still under it
        dict(_evict(_8B, 4000, 4, 256, dec=(32, 3900, 4700), kv="fp8"), name="evict_batch32_fp8"),
        # prompts just read, cut to a sixteenth
        dict(_evict(_70B, 4096, 16, 512, dec=(4, 40000, 66000)), name="evict_prompts4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1, 1 << 30)
    heads = rng.choice([_8B, _70B, _30B, _TINY, (32, 8, 64), (16, 16, 64), (24, 12, 128)])
    kv = rng.choice(["bf16", "bf16", "fp8"])
    op = rng.choice(["rotary", "rotary", "attend", "attend", "attend", "attend", "evict", "evict"])
    if op == "rotary":
        dec, pre = (0, 0, 0), (0, 0, 0, 0, 0)
        if rng.random() < 0.7:
            hi = _log(rng, 1, 1500)
            dec = (_log(rng, 1, 256), rng.randrange(0, hi + 1), hi)
        if not dec[0] or rng.random() < 0.4:
            hi = _log(rng, 2, 1600)
            pre = (rng.randrange(1, 7), max(2, hi // rng.choice([1, 3, 10])), hi, 0, rng.choice([0, _log(rng, 1, 1000)]))
        rdim = rng.choice([heads[2], heads[2] // 2, heads[2] // 4, 48])
        scaling = rng.choice(["none", "linear", "ntk", "wavelength", "yarn"])
        return _rotary(heads, rdim, rng.choice(["half", "interleaved"]), scaling,
                       1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]), rng.choice([0, _log(rng, 10, 500000)]),
                       dec=dec, pre=pre, kv=kv, lens=lens)
    if op == "evict":
        n = _log(rng, 1, 48)
        hi = max(2, min(_log(rng, 40, 70000), int(1.6e6 / n / heads[1])))
        keep = max(1, int(hi * rng.choice([0.06, 0.25, 0.5, 0.9])))
        sink = rng.randrange(0, min(keep, 16) + 1)
        recent = rng.randrange(0, (keep - sink) // 2 + 1)
        return _evict(heads, keep, sink, recent, dec=(n, max(1, hi // rng.choice([1, 2, 8])), hi), kv=kv, lens=lens)
    dec, pre = (0, 0, 0), (0, 0, 0, 0, 0)
    mode = rng.choice(["dec", "dec", "pre", "few", "mixed"])
    if mode in ("dec", "mixed"):
        n = _log(rng, 1, 128)
        hi = max(1, min(_log(rng, 20, 100000), int(9e6 / n / heads[1])))
        dec = (n, max(0, hi // rng.choice([1, 4, 32])), hi)
    if mode == "few":  # a few rows each, over contexts of any length
        n = _log(rng, 1, 32)
        hi = max(1, min(_log(rng, 20, 60000), int(6e6 / n / heads[1])))
        pre = (n, 2, rng.randrange(2, 17), hi // rng.choice([1, 4, 32]), hi)
    elif mode in ("pre", "mixed"):
        n = rng.randrange(1, 6)
        hi = _log(rng, 2, 2000)
        px = rng.choice([0, 0, _log(rng, 16, 4000)])
        pre = (n, max(2, hi // rng.choice([1, 4, 16])), hi, px // 4, px)
    weights = rng.random() < 0.4
    return _attend(heads, cap=rng.choice([0.0, 20.0, 50.0]), bias=rng.random() < 0.3,
                   window=rng.choice([0, 0, _log(rng, 1, 8000)]), docs=rng.choice([0, 0, _log(rng, 10, 2000)]),
                   pad=rng.random() < 0.3, two_way=rng.random() < 0.25, weights=weights,
                   wrows=rng.choice([0, 0, 32]) if weights else 0, dec=dec, pre=pre, kv=kv, lens=lens)


# ---------------------------------------------------------------------------
# lengths and masks (properties of the case)
# ---------------------------------------------------------------------------
def _lens(case):
    """(contexts, new rows) of the requests."""
    rng = np.random.default_rng([case["lens"], case["n_dec"], case["n_pre"]])
    dec = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, case["n_dec"])
    chunk = rng.integers(case["chunk_lo"], case["chunk_hi"] + 1, case["n_pre"])
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, case["n_pre"])
    return np.concatenate([dec, prefix]), np.concatenate([np.ones_like(dec), chunk])


def _masks(case, c, n):
    """first_key per row (or None) and prefix length per request (or None)."""
    rng = np.random.default_rng([case["lens"], 5])
    first = None
    if case["docs"] or case["pad"]:
        rows = []
        for ci, ni in zip(c, n):
            pos = np.arange(ci, ci + ni)
            f = np.zeros(ni, np.int64)
            if case["docs"]:
                starts = np.flatnonzero(rng.random(ci + ni) < 1.0 / case["docs"])
                starts = np.concatenate([[0], starts])
                f = starts[np.searchsorted(starts, pos, side="right") - 1]
            if case["pad"]:
                f = np.where(np.arange(ni) >= ni - rng.integers(0, max(1, ni // 4) + 1), ci + ni, f)
            rows.append(f)
        first = np.concatenate(rows).astype(np.int32)
    prefix = (c + n // 2).astype(np.int32) if case["two_way"] else None
    return first, prefix


def _intervals(case, c, n, first, prefix):
    """[lo, hi) of the keys that each row sees."""
    seq = np.repeat(np.arange(len(c)), n)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(c, n)])
    lo, hi = np.zeros_like(pos), pos + 1
    if case["window"]:
        lo = np.maximum(lo, pos - case["window"] + 1)
    if first is not None:
        lo = np.maximum(lo, first)
    if prefix is not None:
        hi = np.maximum(hi, prefix[seq])
    return seq, pos, lo, np.maximum(hi, lo)


def work(case):
    c, n = _lens(case)
    nq, nkv, hd, es = case["nq"], case["nkv"], case["hd"], 1 if case["kv"] == "fp8" else 2
    T = float(n.sum())
    if case["op"] == "rotary":
        nb = T * (nq * case["rdim"] * 4.0 + 2 * nkv * hd * (2 + es))
        return {"bytes": nb, "flops": 3.0 * T * (nq + nkv) * case["rdim"]}
    if case["op"] == "evict":
        k = np.minimum(c, case["keep"])
        return {"bytes": float(nkv * (4.0 * c.sum() + k.sum() * (4.0 * hd * es + 8.0))), "flops": float(nkv * c.sum())}
    seq, _, lo, hi = _intervals(case, c, n, *_masks(case, c, n))
    seen = 0.0
    for i in range(len(c)):
        at = (seq == i) & (hi > lo)
        seen += float(hi[at].max() - lo[at].min()) if at.any() else 0.0
    nb = seen * 2 * nkv * hd * es + T * nq * (hd * 4.0 + 4.0)
    if case["weights"]:
        nb += seen * nkv * 8.0
    return {"bytes": nb, "flops": 4.0 * nq * hd * float((hi - lo).sum())}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _pool(g, case, tokens, extra=1):
    """K and V pages with every slot filled, block tables of the requests (padding names the last page, which no
    request has)."""
    need = -(-tokens // PAGE)
    pages = int(need.sum()) + extra
    shape = (pages, case["nkv"], PAGE, case["hd"])
    kv = []
    for s in SCALES:
        t = torch.randn(shape, generator=g, device=DEV)
        kv.append((t / s).to(torch.float8_e4m3fn).view(torch.uint8) if case["kv"] == "fp8" else t.to(torch.bfloat16))
    order = torch.randperm(pages - 1, generator=g, device=DEV).to(torch.int32)
    width = max(1, int(need.max()))
    at = np.cumsum(need) - need
    idx = at[:, None] + np.minimum(np.arange(width), np.maximum(need[:, None] - 1, 0))
    table = order[torch.from_numpy(np.minimum(idx, max(0, pages - 2))).to(DEV)] if pages > 1 else None
    live = torch.from_numpy(np.arange(width)[None] < need[:, None]).to(DEV)
    last = torch.full((len(tokens), width), pages - 1, dtype=torch.int32, device=DEV)
    return kv[0], kv[1], last if table is None else torch.where(live, table, last).contiguous()


def _group(c, n, row0, seq0):
    """Index tensors of the requests of one group, their rows padded to the longest."""
    if not len(c):
        return None
    m = int(n.max())
    j = np.minimum(np.arange(m)[None], n[:, None] - 1)
    start = row0 + np.cumsum(n) - n
    real = np.arange(m)[None] < n[:, None]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    return {"rows": dev(start[:, None] + j), "pos": dev(c[:, None] + j), "flat": dev(np.flatnonzero(real.ravel())),
            "c": dev(c), "len": dev(c + n), "seqs": slice(seq0, seq0 + len(c)), "at": slice(row0, row0 + int(n.sum())),
            "real": dev(real), "n": dev(n)}


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c, n = _lens(case)
    nq, nkv, hd, T = case["nq"], case["nkv"], case["hd"], int(n.sum())
    st = {"case": case, "c": c.astype(np.int32), "n": n.astype(np.int32)}
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    if case["op"] == "evict":
        st["k"], st["v"], st["bt"] = _pool(g, case, c)
        k = np.minimum(c, case["keep"])
        st["keep"] = k.astype(np.int32)
        st["dk"], st["dv"], st["dbt"] = _pool(g, case, k)
        # what attention leaves behind: most keys little, some much
        st["acc"] = torch.exp(2.0 * torch.randn(st["k"].shape[:3], generator=g, device=DEV))
        st["dacc"] = torch.zeros(st["dk"].shape[:3], device=DEV)
        st["kept"] = torch.full((len(c), nkv, int(k.max())), -1, dtype=torch.int32, device=DEV)
        st["len"], st["budget"] = dev(c), dev(k)
        st["pair_s"] = dev(np.repeat(np.arange(len(c)), k))
        st["pair_j"] = dev(np.concatenate([np.arange(x) for x in k]))
        return st
    st["k"], st["v"], st["bt"] = _pool(g, case, c + n)
    st["qkv"] = torch.randn(T, (nq + 2 * nkv) * hd, generator=g, device=DEV)
    seq = np.repeat(np.arange(len(c)), n)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(c, n)])
    if case["op"] == "rotary":
        st["qkv"] = st["qkv"].to(torch.bfloat16)
        st["seq"], st["slot"], st["positions"] = dev(seq), dev(pos), None
        if case["far"]:
            ahead = torch.randint(0, case["far"] + 1, (len(c),), generator=g, device=DEV)
            st["positions"] = (st["slot"] + ahead[st["seq"]]).to(torch.int32)
        return st
    # queries a few times larger than unit: scores that a cap and a mask matter for
    st["qkv"][:, :nq * hd] *= 4.0
    st["qkv"] = st["qkv"].to(torch.bfloat16)
    first, prefix = _masks(case, c, n)
    st["first"] = None if first is None else dev(first)
    st["prefix"], st["prefix_dev"] = prefix, None if prefix is None else dev(prefix)
    st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, nq + 1, device=DEV) / nq) if case["bias"] else None
    st["acc"] = torch.rand(st["k"].shape[:3], generator=g, device=DEV) if case["weights"] else None
    d = case["n_dec"]
    st["dec"] = _group(c[:d], n[:d], 0, 0)
    st["pre"] = _group(c[d:], n[d:], d, d)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _own_prepare(st)
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _theta():
    return 5e5


def _inv_freq(case):
    """The rotation per position of each pair, 64 bits."""
    R, f, theta, length = case["rdim"], case["factor"], _theta(), 8192.0
    t = torch.arange(R // 2, dtype=torch.float64, device=DEV)
    if case["scaling"] == "ntk":
        theta = theta * f ** (R / (R - 2.0))
    inv = theta ** (-2.0 * t / R)
    if case["scaling"] == "linear":
        inv = inv / f
    if case["scaling"] == "wavelength":  # long waves stretched, short ones kept, a ramp between 1/4 and 1 of the length
        turns = length * inv / (2 * math.pi)
        mix = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        inv = inv * mix + inv / f * (1 - mix)
    if case["scaling"] == "yarn":  # the ramp runs over the pair index, between 32 turns and 1 turn in the length
        at = [R * math.log(length / (b * 2 * math.pi)) / (2 * math.log(theta)) for b in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        ramp = ((t - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        inv = inv * (1 - ramp) + inv / f * ramp
    return inv


def _codes(x, scale):
    return (x.to(torch.bfloat16).float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(t):
    """A cache as numbers of its own type."""
    return t.view(torch.float8_e4m3fn) if t.dtype == torch.uint8 else t


def _plain_rotary(st):
    case = st["case"]
    nq, nkv, hd, R = case["nq"], case["nkv"], case["hd"], case["rdim"]
    T = st["qkv"].shape[0]
    x = st["qkv"].view(T, nq + 2 * nkv, hd)
    pos = st["slot"] if st["positions"] is None else st["positions"]
    ang = pos.double()[:, None] * _inv_freq(case)
    co, si = ang.cos().float()[:, None], ang.sin().float()[:, None]
    qk = x[:, :nq + nkv].float()
    if case["layout"] == "half":
        a, b = qk[..., :R // 2], qk[..., R // 2:R]
        rot = torch.cat([a * co - b * si, a * si + b * co], -1)
    else:
        a, b = qk[..., 0:R:2], qk[..., 1:R:2]
        rot = torch.stack([a * co - b * si, a * si + b * co], -1).reshape(T, nq + nkv, R)
    x[:, :nq, :R] = rot[:, :nq].to(torch.bfloat16)
    k = torch.cat([rot[:, nq:], qk[:, nq:, R:]], -1)
    v = x[:, nq + nkv:].float()
    page, slot = st["bt"][st["seq"], st["slot"] // PAGE].long(), st["slot"] % PAGE
    if case["kv"] == "fp8":
        k, v = _codes(k, SCALES[0]), _codes(v, SCALES[1])
    st["k"][page, :, slot] = k.to(st["k"].dtype)
    st["v"][page, :, slot] = v.to(st["v"].dtype)
    return {"qkv": st["qkv"], "k": _values(st["k"]), "v": _values(st["v"])}


def _dense(st, name, bt, scale):
    """[requests, kv heads, keys, hd] in 32 bits of the requests with these block tables."""
    t = _values(st[name][bt.long()])
    S, P, nkv, _, hd = t.shape
    t = t.permute(0, 2, 1, 3, 4).reshape(S, nkv, P * PAGE, hd).float()
    return t * scale if st["case"]["kv"] == "fp8" else t


def _plain_group(st, g, out, lse):
    case = st["case"]
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    G = nq // nkv
    bt = st["bt"][g["seqs"]]
    k, v = _dense(st, "k", bt, SCALES[0]), _dense(st, "v", bt, SCALES[1])
    S, m = g["rows"].shape
    L = k.shape[2]
    q = st["qkv"][:, :nq * hd].float()[g["rows"]].view(S, m, nkv, G, hd).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(S, nkv, G * m, hd), k.transpose(2, 3)).view(S, nkv, G, m, L)
    s = s * (1.0 / math.sqrt(hd))
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    key = torch.arange(L, device=DEV)
    if case["bias"]:
        dist = (g["pos"][:, :, None] - key).abs().float()
        s = s - st["slopes"].view(1, nkv, G, 1, 1) * dist[:, None, None]
    lo, hi = torch.zeros_like(g["pos"]), g["pos"] + 1
    if case["window"]:
        lo = torch.maximum(lo, g["pos"] - case["window"] + 1)
    if st["first"] is not None:
        lo = torch.maximum(lo, st["first"].long()[g["rows"]])
    if st["prefix_dev"] is not None:
        hi = torch.maximum(hi, st["prefix_dev"].long()[g["seqs"]][:, None])
    seen = ((key >= lo[:, :, None]) & (key < hi[:, :, None]))[:, None, None]
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(s - base)
    total = p.sum(-1, keepdim=True)
    share = 1.0 / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(S, nkv, G * m, L), v).view(S, nkv, G, m, hd) * share
    rows = lambda t: t.permute(0, 3, 1, 2, 4).reshape(S * m, nq, -1)[g["flat"]]  # noqa: E731
    out[g["at"]] = rows(o).reshape(-1, nq * hd).to(torch.bfloat16)
    lse[g["at"]] = rows(base + torch.log(total)).reshape(-1, nq)
    if case["weights"]:
        counts = g["real"]
        if case["wrows"]:
            counts = counts & (torch.arange(m, device=DEV) >= (g["n"] - case["wrows"])[:, None])
        got = (p * (share * counts[:, None, None, :, None])).sum((2, 3))
        old = st["acc"][bt.long()].permute(0, 2, 1, 3).reshape(S, nkv, L)
        new = torch.where(key < g["c"][:, None, None], old, torch.zeros_like(old)) + got
        new = torch.where(key < g["len"][:, None, None], new, old)
        st["acc"][bt.long()] = new.view(S, nkv, L // PAGE, PAGE).permute(0, 2, 1, 3)


def _plain_attend(st):
    case = st["case"]
    T = st["qkv"].shape[0]
    out = torch.empty(T, case["nq"] * case["hd"], dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(T, case["nq"], device=DEV)
    if st["dec"]:
        _plain_group(st, st["dec"], out, lse)
    if st["pre"]:
        _plain_group(st, st["pre"], out, lse)
    return {"out": out, "lse": lse, "weights": st["acc"]}


def _plain_evict(st):
    case = st["case"]
    nkv = case["nkv"]
    bt = st["bt"].long()
    S, P = bt.shape
    c, budget = st["len"][:, None, None], st["budget"][:, None, None]
    score = st["acc"][bt].permute(0, 2, 1, 3).reshape(S, nkv, P * PAGE)
    key = torch.arange(P * PAGE, device=DEV)
    score = score.masked_fill((key < case["sink"]) | (key >= c - case["recent"]), math.inf)
    score = score.masked_fill(key >= c, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1]  # equal ones: the lower key first
    width = st["kept"].shape[2]
    order = order[..., :width]
    live = torch.arange(width, device=DEV) < budget
    kept = torch.sort(torch.where(live, order, torch.full_like(order, 1 << 40)), dim=-1)[0]
    st["kept"].copy_(torch.where(live, kept, st["kept"].long()))
    s, j, h = st["pair_s"][:, None], st["pair_j"][:, None], torch.arange(nkv, device=DEV)
    at = kept.permute(0, 2, 1)[st["pair_s"], st["pair_j"]]
    page, dpage = bt[s, at // PAGE], st["dbt"].long()[s, j // PAGE]
    st["dk"][dpage, h, j % PAGE] = st["k"][page, h, at % PAGE]
    st["dv"][dpage, h, j % PAGE] = st["v"][page, h, at % PAGE]
    st["dacc"][dpage, h, j % PAGE] = st["acc"][page, h, at % PAGE]
    return {"k": _values(st["dk"]), "v": _values(st["dv"]), "weights": st["dacc"], "kept": st["kept"]}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own_prepare(st):
    from paper_2606_00516_amd import binding as B

    case = st["case"]
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    T = max(1, int(st["n"].sum()))
    shape = types.SimpleNamespace(hidden=nq * hd, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, ffn=8, rms_eps=1e-5,
                                  rope_theta=_theta())
    scales = SCALES if case["kv"] == "fp8" else None
    st["B"], st["h"] = B, B.Handle(shape, len(st["c"]), T)
    st["kv"] = B.kv_struct(st["k"], st["v"], st["bt"], scales)
    if case["op"] == "evict":
        st["dkv"] = B.kv_struct(st["dk"], st["dv"], st["dbt"], scales)
        st["ws"] = B.alloc_workspace(B.eb_op_kv_evict_workspace_bytes(st["h"], st["c"], st["keep"]))
        return
    st["batch"] = B.HostBatch(st["c"], st["n"])
    if case["op"] == "rotary":
        st["rot"] = B.rotary(theta=_theta(), rotary_dim=case["rdim"], layout=case["layout"], scaling=case["scaling"],
                             factor=case["factor"], original_len=8192, magnitude=1.0)
        st["ws"] = B.alloc_workspace(B.eb_op_rotary_kv_append_workspace_bytes(st["h"], st["batch"]))
        return
    st["mod"] = B.score_mod(softcap=case["cap"], slopes=st["slopes"], window=case["window"], first_key=st["first"],
                            prefix_lens=st["prefix"])
    st["out"] = torch.empty(T, nq * hd, dtype=torch.bfloat16, device=DEV)
    st["lse"] = torch.empty(T, nq, device=DEV)
    st["ws"] = B.alloc_workspace(B.eb_op_attention_mod_workspace_bytes(st["h"], st["batch"], st["mod"], case["weights"]))


def _own_run(st):
    case, B = st["case"], st["B"]
    if case["op"] == "rotary":
        B.eb_op_rotary_kv_append(st["h"], st["rot"], st["qkv"], st["kv"], st["batch"], positions=st["positions"],
                                 ws=st["ws"])
        return {"qkv": st["qkv"], "k": _values(st["k"]), "v": _values(st["v"])}
    if case["op"] == "attend":
        B.eb_op_attention_mod(st["h"], st["qkv"], st["kv"], st["batch"], st["mod"], out=st["out"], lse=st["lse"],
                              kv_weights=st["acc"], weight_rows=case["wrows"], ws=st["ws"])
        return {"out": st["out"], "lse": st["lse"], "weights": st["acc"]}
    B.eb_op_kv_evict(st["h"], st["kv"], st["acc"], st["c"], st["keep"], st["dkv"], dst_weights=st["dacc"],
                     sink=case["sink"], recent=case["recent"], kept=st["kept"], ws=st["ws"])
    return {"k": _values(st["dk"]), "v": _values(st["dv"]), "weights": st["dacc"], "kept": st["kept"]}


def run(st):
    if own:
        return _own_run(st)
    return {"rotary": _plain_rotary, "attend": _plain_attend, "evict": _plain_evict}[st["case"]["op"]](st)


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits, request by request
# ---------------------------------------------------------------------------
def _exact_freq(case):
    """As _inv_freq, pair by pair in plain numbers."""
    R, f, theta, length, got = case["rdim"], case["factor"], _theta(), 8192.0, []
    for t in range(R // 2):
        base = theta * f ** (R / (R - 2.0)) if case["scaling"] == "ntk" else theta
        w = math.exp(-2.0 * t / R * math.log(base))
        if case["scaling"] == "linear":
            w /= f
        elif case["scaling"] == "wavelength":
            wave = 2 * math.pi / w
            if wave > length:
                w /= f
            elif wave > length / 4:
                mix = (length / wave - 1.0) / 3.0
                w = (1 - mix) * w / f + mix * w
        elif case["scaling"] == "yarn":
            index = lambda turns: R * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
            lo, hi = max(0, math.floor(index(32.0))), min(R - 1, math.ceil(index(1.0)))
            keep = 1.0 - min(1.0, max(0.0, (t - lo) / max(hi - lo, 1e-3)))
            w = w / f * (1 - keep) + w * keep
        got.append(w)
    return torch.tensor(got, dtype=torch.float64, device=DEV)


def _exact_rotary(st):
    case = st["case"]
    nq, nkv, hd, R = case["nq"], case["nkv"], case["hd"], case["rdim"]
    x = st["qkv"].double().view(-1, nq + 2 * nkv, hd).clone()
    w = _exact_freq(case)
    kc, vc = _values(st["k"]).double(), _values(st["v"]).double()
    ks, vs = SCALES if case["kv"] == "fp8" else (1.0, 1.0)
    row = 0
    for i, (c, n) in enumerate(zip(st["c"].tolist(), st["n"].tolist())):
        at = torch.arange(c, c + n, device=DEV)
        p = at if st["positions"] is None else st["positions"][row:row + n]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), p.double()[:, None, None] * w)
        part = x[row:row + n, :nq + nkv, :R]
        if case["layout"] == "half":
            z = torch.complex(part[..., :R // 2].contiguous(), part[..., R // 2:].contiguous()) * turn
            part.copy_(torch.cat([z.real, z.imag], -1))
        else:
            z = torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) * turn
            part.copy_(torch.view_as_real(z).reshape(part.shape))
        page = st["bt"][i].long()[at // PAGE]
        kc[page, :, at % PAGE] = x[row:row + n, nq:nq + nkv] / ks
        vc[page, :, at % PAGE] = x[row:row + n, nq + nkv:] / vs
        row += n
    x[:, nq:nq + nkv] = st["qkv"].double().view(x.shape)[:, nq:nq + nkv]  # the row keeps its keys as they came
    return {"qkv": x.reshape(st["qkv"].shape), "k": kc.clamp(-448, 448) if case["kv"] == "fp8" else kc,
            "v": vc.clamp(-448, 448) if case["kv"] == "fp8" else vc}


def _exact_attend(st):
    case = st["case"]
    c, n = st["c"].astype(np.int64), st["n"].astype(np.int64)
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    G = nq // nkv
    first, prefix = _masks(case, c, n)
    _, _, lo, hi = _intervals(case, c, n, first, prefix)
    lo, hi = (torch.from_numpy(a).to(DEV) for a in (lo, hi))
    T = int(n.sum())
    out = torch.zeros(T, nq, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((T, nq), -math.inf, dtype=torch.float64, device=DEV)
    acc = None if st["acc"] is None else st["acc"].double()
    ks, vs = SCALES if case["kv"] == "fp8" else (1.0, 1.0)
    q = st["qkv"].double()
    row = 0
    for i in range(len(c)):
        L = int(c[i] + n[i])
        pages = st["bt"][i, :-(-L // PAGE)].long()
        key = torch.arange(L, device=DEV)
        got = torch.zeros(nkv, L, dtype=torch.float64, device=DEV)
        step = max(1, int(6e8 / L / G))
        for h in range(nkv):
            K = _values(st["k"])[pages, h].double().reshape(-1, hd)[:L] * ks
            V = _values(st["v"])[pages, h].double().reshape(-1, hd)[:L] * vs
            for r in range(0, int(n[i]), step):
                at = torch.arange(row + r, row + min(int(n[i]), r + step), device=DEV)
                Q = q[at][:, h * G * hd:(h + 1) * G * hd].view(-1, G, hd)
                s = (Q @ K.t()) / math.sqrt(hd)
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["bias"]:
                    far = (key[None] - (at - row + int(c[i]))[:, None]).abs()
                    s = s - far[:, None].double() * st["slopes"][h * G:(h + 1) * G, None].double()
                sees = (key[None] >= lo[at][:, None]) & (key[None] < hi[at][:, None])
                s = torch.where(sees[:, None], s, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
                z = torch.logsumexp(s, -1)
                w = torch.where(sees[:, None], torch.exp(s - z[..., None]), torch.zeros((), dtype=torch.float64, device=DEV))
                lse[at, h * G:(h + 1) * G] = z
                out[at, h * G:(h + 1) * G] = w @ V
                counts = (at - row) >= (int(n[i]) - case["wrows"] if case["wrows"] else 0)
                got[h] += (w * counts[:, None, None]).sum((0, 1))
        if acc is not None:
            old = torch.where(key < int(c[i]), acc[pages].permute(1, 0, 2).reshape(nkv, -1)[:, :L], torch.zeros_like(got))
            acc[pages[key // PAGE], :, key % PAGE] = (old + got).t()
        row += int(n[i])
    return {"out": out.reshape(T, nq * hd), "lse": lse, "weights": acc}


def _exact_evict(st):
    case = st["case"]
    acc, bt, dbt = st["acc"].double().cpu().numpy(), st["bt"].cpu().numpy(), st["dbt"].cpu().numpy()
    dacc = st["dacc"].double().cpu().numpy()
    k, v, dk, dv = (_values(st[x]).double() for x in ("k", "v", "dk", "dv"))
    kept = st["kept"].cpu().numpy().copy()
    for i, (c, b) in enumerate(zip(st["c"].tolist(), st["keep"].tolist())):
        t = np.arange(c)
        pg, sl = bt[i][t // PAGE], t % PAGE
        must = (t < case["sink"]) | (t >= c - case["recent"])
        for h in range(case["nkv"]):
            order = np.lexsort((t, -acc[pg, h, sl], ~must))
            at = np.sort(order[:b])
            j = np.arange(b)
            kept[i, h, :b] = at
            dacc[dbt[i][j // PAGE], h, j % PAGE] = acc[pg[at], h, sl[at]]
            to, frm = (torch.from_numpy(a.astype(np.int64)).to(DEV) for a in (dbt[i][j // PAGE], pg[at]))
            ds, fs = (torch.from_numpy(a).to(DEV) for a in (j % PAGE, sl[at]))
            dk[to, h, ds], dv[to, h, ds] = k[frm, h, fs], v[frm, h, fs]
    return {"k": dk, "v": dv, "weights": torch.from_numpy(dacc), "kept": torch.from_numpy(kept)}


def exact(case, seed):
    st = _inputs(case, seed)
    return {"rotary": _exact_rotary, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](st)
