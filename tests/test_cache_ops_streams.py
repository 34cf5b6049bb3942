"""Calls of the cache operators on a stream that the caller names, with the
memory that the binding makes for itself: it has to come from that stream's own
pool.  Memory of another stream's pool may have been freed there with that
stream's kernels still writing it."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R
from tests.test_gpu_cache_attention import _qkv


class _Calls:
    """The library's entries as far as the binding sees them: every call succeeds."""

    def __getattr__(self, name):
        return (lambda *a: 512) if name.endswith("_bytes") else (lambda *a: 0)


@pytest.fixture
def world(monkeypatch):
    """The binding on CPU tensors; `made` lists the stream that was current at
    each allocation, `used` the tensors marked as used by another."""
    w = types.SimpleNamespace(current=["first"], made=[], used=[])

    @contextlib.contextmanager
    def stream(s):
        w.current.append(s)
        yield
        w.current.pop()
    real = torch.empty

    def empty(*a, **kw):
        w.made.append(w.current[-1])
        kw.pop("device", None)
        return real(*a, **kw)
    monkeypatch.setattr(B, "_lib", _Calls())
    monkeypatch.setattr(B, "_dev", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: w.current[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda s, dev: None)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.used.append((t.dtype, s)))
    monkeypatch.setattr(torch, "empty", empty)
    w.h = object.__new__(B.Handle)
    w.h.h = None
    w.h.n_q_heads, w.h.n_kv_heads, w.h.head_dim, w.h.qkv_cols, w.h.page_keys = 4, 2, 64, 512, 32
    w.h.cfg = B.LayerConfig()
    w.kv = B.KvCache(256, 256, 4, 256, 4, 0, 1.0, 1.0)
    w.x = torch.zeros(1, 512, dtype=torch.bfloat16)
    w.weights = torch.zeros(4, 2, 16)
    return w


def _all(w, stream, **kw):
    b = B.HostBatch([39], [1])
    B.eb_op_rotary_kv_append(w.h, B.Rotary(), w.x, w.kv, b, stream=stream, **kw)
    B.eb_op_attention_mod(w.h, w.x, w.kv, b, stream=stream, **kw)
    B.eb_op_kv_evict(w.h, w.kv, w.weights, [40], [16], w.kv, stream=stream, **kw)


def test_own_memory_comes_from_the_stream_of_the_call(world):
    _all(world, "other")
    # three workspaces and an output; the output is the caller's to use on its own stream
    assert world.made == ["other"] * 4 and world.current == ["first"]
    assert (torch.bfloat16, "first") in world.used


def test_own_memory_on_the_current_stream(world):
    _all(world, None)
    assert world.made == ["first"] * 4 and not world.used


def test_given_workspaces_are_taken_as_they_are(world):
    ws = torch.zeros(512, dtype=torch.uint8)
    _all(world, "other", ws=ws)
    assert world.made == ["other"]   # the output alone


@pytest.mark.gpu
def test_calls_on_two_streams_with_their_own_memory():
    sh = R.shape(8, 2, 128)
    h = B.Handle(sh, 4, 300)
    ctx, chk = np.array([3000, 100, 0, 1500]), np.array([1, 80, 129, 1])
    T = int(chk.sum())
    d = [R.make_cache(ctx + chk, 2, 128, seed=k, poison=False).cuda() for k in range(2)]
    kv = [B.kv_struct(c.k, c.v, c.bt) for c in d]
    x = [_qkv(T, sh, k).cuda() for k in range(2)]
    batch, mod, s = B.HostBatch(ctx, chk), B.score_mod(softcap=20.0), torch.cuda.Stream()
    keep = np.minimum(ctx + chk, 64)
    dst = [R.make_cache(keep, 2, 128, seed=5, poison=False).cuda() for _ in range(2)]
    to = [B.kv_struct(p.k, p.v, p.bt) for p in dst]

    def made():   # what a call writes
        return torch.zeros(d[0].k.shape[:3], device="cuda"), torch.zeros(4, 2, 64, dtype=torch.int32, device="cuda")

    def go(k, w, kept, stream):
        o = B.eb_op_attention_mod(h, x[k], kv[k], batch, mod, kv_weights=w, stream=stream)
        B.eb_op_kv_evict(h, kv[k], w, ctx + chk, keep, to[k], sink=4, recent=8, kept=kept, stream=stream)
        return o
    want = []
    for k in range(2):
        w, kept = made()
        o = go(k, w, kept, None)
        torch.cuda.synchronize()
        want.append((o, w, kept))
    for _ in range(10):
        own = [made() for _ in range(4)]
        torch.cuda.synchronize()
        got = [go(i % 2, *own[i], s if i % 2 else None) for i in range(4)]   # nothing waits for anything
        torch.cuda.synchronize()
        for i in range(4):
            for a, b in zip((got[i], *own[i]), want[i % 2]):
                assert torch.equal(a, b)
