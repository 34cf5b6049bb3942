"""The operators on the paged cache in plain 64-bit numpy, and small inputs for
them.  Written from the definitions in include/eb_layer.h."""
from __future__ import annotations

import dataclasses
import math
import types

import numpy as np
import torch

PAGE = 16


def f64(t: torch.Tensor) -> np.ndarray:
    """Values of a bf16 / fp32 tensor, or of 8-bit codes (uint8)."""
    t = t.detach().cpu()
    if t.dtype == torch.uint8:
        t = t.view(torch.float8_e4m3fn)
    return t.to(torch.float64).numpy()


def shape(nq, nkv, hd, qk_norm=False):
    return types.SimpleNamespace(hidden=nq * hd, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, ffn=8, rms_eps=1e-5,
                                 rope_theta=1e4, qk_norm=qk_norm)


@dataclasses.dataclass
class Cache:
    k: torch.Tensor          # [pages, nkv, 16, hd]
    v: torch.Tensor
    bt: torch.Tensor         # int32 [S, width]
    scales: tuple            # (k_scale, v_scale) or None

    def cuda(self):
        return Cache(self.k.cuda(), self.v.cuda(), self.bt.cuda(), self.scales)


def make_cache(lens, nkv, hd, fp8=False, seed=0, spare=3, poison=True, width=None):
    """Pages for these lengths in random order; slots past a request's end and
    spare pages hold NaN (poison) where they can."""
    g = torch.Generator().manual_seed(seed)
    lens = np.asarray(lens)
    need = -(-lens // PAGE)
    pages = int(need.sum()) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    w = width or max(1, int(need.max()) if len(need) else 1)
    bt = torch.full((len(lens), w), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        bt[i, :n] = order[at:at + n]
        at += int(n)
    scales = (0.5, 0.25) if fp8 else None
    out = []
    for s in (0.5, 0.25):
        t = torch.randn(pages, nkv, PAGE, hd, generator=g)
        t = (t / s).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else t.to(torch.bfloat16)
        if poison:
            bad = torch.ones(pages, PAGE, dtype=torch.bool)
            for i, n in enumerate(lens):
                p = np.arange(int(n))
                bad[bt[i][torch.from_numpy(p // PAGE)].long(), torch.from_numpy(p % PAGE)] = False
            t.permute(0, 2, 1, 3)[bad] = 0x7F if fp8 else math.nan
        out.append(t)
    return Cache(out[0], out[1], bt, scales)


def gather(t: torch.Tensor, bt_row: torch.Tensor, n: int, scale=1.0) -> np.ndarray:
    """[n, nkv, hd] values of a request's first n slots."""
    p = np.arange(n)
    return f64(t)[bt_row.cpu().numpy()[p // PAGE], :, p % PAGE] * scale


# ------------------------------------------------------------------ rotary
def frequencies(R, theta, scaling="none", factor=1.0, length=0, low=0.0, high=0.0):
    theta = float(np.float32(theta))
    factor = float(np.float32(factor))
    if scaling == "ntk":
        theta = theta * factor ** (R / (R - 2))
    t = np.arange(R // 2)
    w = theta ** (-2.0 * t / R)
    if scaling == "linear":
        return w / factor
    if scaling == "wavelength":
        low, high = (1.0, 4.0) if low == high == 0 else (low, high)
        wave = 2 * np.pi / w
        mix = np.clip((length / wave - low) / (high - low), 0, 1)
        return w * mix + w / factor * (1 - mix)
    if scaling == "yarn":
        low, high = (1.0, 32.0) if low == high == 0 else (low, high)
        index = lambda n: R * np.log(length / (2 * np.pi * n)) / (2 * np.log(theta))  # noqa: E731
        a, b = max(np.floor(index(high)), 0), min(np.ceil(index(low)), R - 1)
        g = np.clip((t - a) / max(b - a, 1e-3), 0, 1)
        return w * (1 - g) + w / factor * g
    return w


def rotate(x, pos, R, freq, layout="half", magnitude=1.0):
    """x [rows, heads, hd] at positions pos, in 64 bits."""
    x = np.array(x, np.float64)
    ang = np.asarray(pos, np.float64)[:, None, None] * freq
    c, s = np.cos(ang) * magnitude, np.sin(ang) * magnitude
    i, j = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    a, b = x[..., i].copy(), x[..., j].copy()
    x[..., i], x[..., j] = a * c - b * s, a * s + b * c
    return x


# --------------------------------------------------------------- attention
def visible(c, n, window=0, prefix=0, first=None):
    """bool [n, c + n]: which keys each new row sees."""
    p = c + np.arange(n)[:, None]
    t = np.arange(c + n)[None]
    lo = np.zeros((n, 1), np.int64)
    if window:
        lo = np.maximum(lo, p - window + 1)
    if first is not None:
        lo = np.maximum(lo, np.asarray(first, np.int64)[:, None])
    return (t >= lo) & (t < np.maximum(p + 1, prefix))


def attend(q, k, v, see, c, scale=None, softcap=0.0, slopes=None):
    """q [n, nq, hd], k, v [c + n, nkv, hd] -> out [n, nq, hd], lse [n, nq], p [n, nq, c + n]."""
    n, nq, hd = q.shape
    nkv = k.shape[1]
    scale = 1 / math.sqrt(hd) if not scale else float(np.float32(scale))
    out, lse, pr = np.zeros((n, nq, hd)), np.full((n, nq), -np.inf), np.zeros((n, nq, k.shape[0]))
    dist = np.abs(c + np.arange(n)[:, None] - np.arange(k.shape[0])[None])
    with np.errstate(all="ignore"):
        for h in range(nq):
            kh = h // (nq // nkv)
            s = (q[:, h] @ k[:, kh].T) * scale
            if softcap:
                s = softcap * np.tanh(s / softcap)
            if slopes is not None:
                s = s - float(slopes[h]) * dist
            for r in range(n):
                m = see[r]
                if not m.any():
                    continue
                top = s[r, m].max()
                e = np.exp(s[r, m] - top)
                lse[r, h] = top + np.log(e.sum())
                pr[r, h, m] = e / e.sum()
                out[r, h] = (e / e.sum()) @ v[m, kh]
    return out, lse, pr


def attend_batch(sh, qkv, cache, ctx, chk, window=0, prefix=None, first=None, weights=None, weight_rows=0, **kw):
    """Reference of a whole call: out [T, nq hd], lse [T, nq], weights after it."""
    nq, nkv, hd = sh.n_q_heads, sh.n_kv_heads, sh.head_dim
    q = f64(qkv)[:, :nq * hd].reshape(-1, nq, hd)
    out, lse = np.zeros((len(q), nq * hd)), np.zeros((len(q), nq))
    w = None if weights is None else f64(weights).copy()
    row = 0
    for i, (c, n) in enumerate(zip(ctx, chk)):
        c, n = int(c), int(n)
        ks, vs = cache.scales or (1.0, 1.0)
        k, v = gather(cache.k, cache.bt[i], c + n, ks), gather(cache.v, cache.bt[i], c + n, vs)
        see = visible(c, n, window, 0 if prefix is None else int(prefix[i]),
                      None if first is None else first[row:row + n])
        o, z, p = attend(q[row:row + n], k, v, see, c, **kw)
        out[row:row + n], lse[row:row + n] = o.reshape(n, -1), z
        if w is not None:
            j0 = max(0, n - weight_rows) if weight_rows else 0
            got = p[j0:].sum(0).reshape(nkv, nq // nkv, c + n).sum(1)   # [nkv, keys]
            t = np.arange(c + n)
            pg, sl = cache.bt[i].cpu().numpy()[t // PAGE], t % PAGE
            w[pg, :, sl] = np.where(t[:, None] < c, w[pg, :, sl], 0) + got.T
        row += n
    return out, lse, w


# ---------------------------------------------------------------- eviction
def keep_positions(w, keep, sink, recent):
    """Ascending positions that stay of a head's weights w [c]."""
    c = len(w)
    t = np.arange(c)
    must = (t < sink) | (t >= c - recent)
    key = np.where(np.isnan(w), np.inf, w)
    nan = np.isnan(w)
    order = np.lexsort((t, -key, ~nan, ~must))
    return np.sort(order[:min(keep, c)])
