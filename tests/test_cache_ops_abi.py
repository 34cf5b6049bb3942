"""The cache operators without a GPU: what the C entries refuse, with which
status, before any work is enqueued; workspace sizes; the binding's own
checks.  Addresses are made up: no call here gets past its checks."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R

FAKE = 0x10000


@pytest.fixture(scope="module")
def handle():
    """eb_create allocates pinned memory and needs a GPU; the refusals below
    themselves launch nothing."""
    return B.Handle(R.shape(8, 2, 64), 4, 64)


def test_null_handles():
    L = B.lib()
    b = B.HostBatch([3], [1])
    kv = B.KvCache(FAKE, FAKE, 4, FAKE, 4, 0, 1.0, 1.0)
    rot, mod = B.rotary(1e4), B.score_mod()
    assert L.eb_op_rotary_kv_append(None, rot, FAKE, kv, b.c, None, FAKE, 1 << 20, None) == -1
    assert L.eb_op_attention_mod(None, FAKE, kv, b.c, mod, FAKE, None, None, 0, FAKE, 1 << 20, None) == -1
    one = np.array([3], np.int32)
    assert L.eb_op_kv_evict(None, kv, FAKE, 1, one.ctypes.data, one.ctypes.data, 0, 0, kv, None, None, 0, FAKE, 1 << 20,
                            None) == -1
    assert L.eb_op_rotary_kv_append_workspace_bytes(None, b.c) == 0
    assert L.eb_op_attention_mod_workspace_bytes(None, b.c, mod, 1) == 0
    assert L.eb_op_kv_evict_workspace_bytes(None, 1, one.ctypes.data, one.ctypes.data) == 0
    assert B.eb_last_error()


def test_struct_sizes_match_the_header():
    # laid out by the C rules: 3 int32, 5 floats, 1 int32 and padding, 2 pointers; 2 floats, pointer, int32, 2 pointers
    assert ctypes.sizeof(B.Rotary) == 56 and B.Rotary.q_norm.offset == 40
    assert ctypes.sizeof(B.ScoreMod) == 40 and B.ScoreMod.slopes.offset == 8 and B.ScoreMod.prefix_lens_host.offset == 24


def test_unknown_names():
    with pytest.raises(KeyError):
        B.rotary(1e4, layout="thirds")
    with pytest.raises(KeyError):
        B.rotary(1e4, scaling="guess")


def test_cpu_tensors_are_refused():
    with pytest.raises((ValueError, RuntimeError)):
        B.score_mod(slopes=torch.zeros(8))
    with pytest.raises(TypeError):
        B.score_mod(slopes=torch.zeros(8, dtype=torch.float64))
    with pytest.raises(TypeError):
        B.score_mod(first_key=torch.zeros(8, dtype=torch.int64))
    with pytest.raises(TypeError):
        B.score_mod(prefix_lens=[0.5])


ROTARY_BAD = [dict(rotary_dim=8), dict(rotary_dim=-16), dict(rotary_dim=80), dict(theta=1.0), dict(theta=float("nan")),
              dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=float("inf")),
              dict(scaling="yarn", factor=2.0), dict(scaling="wavelength", factor=2.0, original_len=100, low=4.0, high=2.0),
              dict(scaling="wavelength", factor=2.0, original_len=100, low=1.0), dict(magnitude=-1.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("bad", range(len(ROTARY_BAD)))
def test_rotary_refusals(handle, bad):
    L, kw = B.lib(), dict(theta=1e4)
    kw.update(ROTARY_BAD[bad])
    b, kv = B.HostBatch([3], [1]), B.KvCache(FAKE, FAKE, 4, FAKE, 4, 0, 1.0, 1.0)
    assert L.eb_op_rotary_kv_append(handle.h, B.rotary(**kw), FAKE, kv, b.c, None, FAKE, 1 << 20, None) == -2
    assert B.eb_last_error()


@pytest.mark.gpu
def test_rotary_argument_refusals(handle):
    L, rot = B.lib(), B.rotary(1e4)
    b, kv = B.HostBatch([3], [1]), B.KvCache(FAKE, FAKE, 4, FAKE, 4, 0, 1.0, 1.0)
    call = lambda rot=rot, q=FAKE, kv=kv, b=b, pos=None, ws=FAKE, n=1 << 20: L.eb_op_rotary_kv_append(  # noqa: E731
        handle.h, rot, q, kv, b.c, pos, ws, n, None)
    assert call(rot=None) == -1 and call(q=None) == -1
    assert call(q=FAKE + 2) == -2 and call(pos=FAKE + 1) == -2
    assert call(ws=None) == -6 and call(n=8) == -6 and call(ws=FAKE + 16) == -6
    assert call(b=B.HostBatch([63], [2])) == -5          # past the block table
    assert call(b=B.HostBatch([-1], [1])) == -3 and call(b=B.HostBatch([1], [0])) == -3
    assert call(b=B.HostBatch([0], [65])) == -5 and call(b=B.HostBatch([0] * 5, [1] * 5)) == -7
    assert call(kv=B.KvCache(FAKE, None, 4, FAKE, 4, 0, 1.0, 1.0)) == -1
    assert call(kv=B.KvCache(FAKE + 8, FAKE, 4, FAKE, 4, 0, 1.0, 1.0)) == -2
    assert call(kv=B.KvCache(FAKE, FAKE, 4, FAKE, 4, 1, 0.0, 1.0)) == -2
    with_norms = B.Handle(R.shape(8, 2, 64, qk_norm=True), 4, 64)
    assert L.eb_op_rotary_kv_append(with_norms.h, rot, FAKE, kv, b.c, None, FAKE, 1 << 20, None) == -1


@pytest.mark.gpu
def test_attention_refusals(handle):
    L = B.lib()
    b, kv = B.HostBatch([3, 5], [1, 4]), B.KvCache(FAKE, FAKE, 4, FAKE, 4, 0, 1.0, 1.0)

    def call(mod=None, q=FAKE, kv=kv, b=b, out=FAKE, lse=None, w=None, rows=0, ws=FAKE, n=1 << 30):
        return L.eb_op_attention_mod(handle.h, q, kv, b.c, mod, out, lse, w, rows, ws, n, None)
    for kw in (dict(scale=-1.0), dict(scale=float("nan")), dict(softcap=-2.0), dict(softcap=float("inf")),
               dict(softcap=float("nan")), dict(softcap=2000.0), dict(window=-1)):
        assert call(B.score_mod(**kw)) == -2, kw
    for p in ([0, 10], [-1, 0], [5, 0]):
        assert call(B.score_mod(prefix_lens=p)) == -3, p
    assert call(q=None) == -1 and call(out=None) == -1 and call(kv=None) == -1 and call(rows=-1) == -2
    assert call(q=FAKE + 8) == -2 and call(out=FAKE + 2) == -2 and call(w=FAKE + 4) == -2 and call(lse=FAKE + 2) == -2
    need = B.eb_op_attention_mod_workspace_bytes(handle, b)
    assert need > 0 and call(ws=None) == -6 and call(n=need - 1) == -6 and call(ws=FAKE + 128) == -6
    assert call(b=B.HostBatch([64], [1])) == -5
    assert B.eb_op_attention_mod_workspace_bytes(handle, b, None, True) > need
    assert B.eb_op_attention_mod_workspace_bytes(handle, b, B.score_mod(window=-1)) == 0
    with pytest.raises(ValueError):
        B.eb_op_attention_mod_workspace_bytes(handle, b, B.score_mod(prefix_lens=[1]))
    with pytest.raises(ValueError):
        B.eb_op_attention_mod_workspace_bytes(handle, b, B.score_mod(slopes=torch.zeros(4, device="cuda")))
    with pytest.raises(ValueError):
        B.eb_op_attention_mod_workspace_bytes(handle, b, B.score_mod(first_key=torch.zeros(4, dtype=torch.int32, device="cuda")))


@pytest.mark.gpu
def test_evict_refusals(handle):
    L = B.lib()
    kv = B.KvCache(FAKE, FAKE, 8, FAKE, 4, 0, 1.0, 1.0)
    f8 = B.KvCache(FAKE, FAKE, 8, FAKE, 4, 1, 0.5, 0.5)

    def call(lens=(40, 20), keep=(16, 16), sink=0, recent=0, src=kv, dst=kv, w=FAKE, dw=None, kept=None, stride=0, ws=FAKE,
             n=1 << 30):
        a, b = np.array(lens, np.int32), np.array(keep, np.int32)
        return L.eb_op_kv_evict(handle.h, src, w, len(a), a.ctypes.data, b.ctypes.data, sink, recent, dst, dw, kept, stride,
                                ws, n, None)
    assert call(src=None) == -1 and call(dst=None) == -1 and call(w=None) == -1
    assert call(dst=f8) == -2 and call(src=f8, dst=B.KvCache(FAKE, FAKE, 8, FAKE, 4, 1, 0.5, 0.25)) == -2
    assert call(sink=-1) == -2 and call(recent=-1) == -2
    assert call(sink=10, recent=7) == -3 and call(sink=2 ** 31 - 1, recent=2 ** 31 - 1) == -3
    assert call(lens=(-1, 3)) == -3 and call(keep=(-1, 3)) == -3
    assert call(lens=(65, 3)) == -5 and call(lens=(64, 64), keep=(64, 64), dst=B.KvCache(FAKE, FAKE, 8, FAKE, 3, 0, 1.0, 1.0)) == -5
    assert call(lens=[9] * 5, keep=[9] * 5) == -7
    assert call(kept=FAKE, stride=15) == -2 and call(kept=FAKE + 2, stride=16) == -2 and call(w=FAKE + 4) == -2
    need = B.eb_op_kv_evict_workspace_bytes(handle, [40, 20], [16, 16])
    assert call(ws=None) == -6 and call(n=need - 1) == -6
    assert call(lens=(0, 0)) == 0 and call(keep=(0, 0), w=None) == 0    # nothing to keep: nothing to do
    with pytest.raises(ValueError):
        B.eb_op_kv_evict_workspace_bytes(handle, [1, 2], [1])
