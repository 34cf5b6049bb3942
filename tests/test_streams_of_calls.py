"""The binding's entries on a stream that the caller names, with the memory that
they make themselves: outputs and workspaces come from that stream's pool, as
memory of another pool may have been freed with kernels still writing it."""
import contextlib
import types

import pytest
import torch

from paper_2606_00516_amd import binding as B


@pytest.fixture
def world(monkeypatch):
    w = types.SimpleNamespace(current=["first"], made=[], used=[])

    @contextlib.contextmanager
    def stream(s):
        w.current.append(s)
        yield
        w.current.pop()

    class Calls:
        def __getattr__(self, name):
            return lambda *a: 4096 if name.endswith("_bytes") else 0
    empty, like = torch.empty, torch.empty_like

    def noted(f):
        def make(*a, **kw):
            w.made.append(w.current[-1])
            kw.pop("device", None)
            return f(*a, **kw)
        return make
    monkeypatch.setattr(B, "_lib", Calls())
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(B, "_stream", lambda s: None)
    monkeypatch.setattr(torch, "empty", noted(empty))
    monkeypatch.setattr(torch, "empty_like", noted(like))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: w.current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.used.append((t.data_ptr(), s)))
    w.h = object.__new__(B.Handle)
    w.h.h, w.h.shape = None, types.SimpleNamespace(n_q_heads=4, n_kv_heads=2, head_dim=64, hidden=256, ffn=64)
    return w


def bf(*n):
    return torch.zeros(n, dtype=torch.bfloat16)


def _calls(h, s):
    k, v, bt = bf(4, 2, 16, 64), bf(4, 2, 16, 64), torch.zeros(1, 4, dtype=torch.int32)
    x, w, codes = bf(3, 256), {"w_qkv": bf(8, 8)}, torch.zeros(64, 256, dtype=torch.uint8)
    step = (h, w, k, v, bt, [0], [3], x)
    return {
        "decode": lambda: B.eb_layer_step_decode(*step, stream=s), "prefill": lambda: B.eb_layer_step_prefill(*step, stream=s),
        "mixed": lambda: B.eb_layer_step_mixed(*step, stream=s),
        "noalloc": lambda: B.eb_layer_step_mixed_noalloc(*step, stream=s),
        "stack": lambda: B.eb_stack_step(h, "mixed", [w], [(k, v, bt)], [0], [3], x, stream=s),
        "rmsnorm": lambda: B.eb_op_rmsnorm(h, x, bf(256), stream=s),
        "gemm": lambda: B.eb_op_gemm(x, bf(64, 256), stream=s),
        "gemm_w8": lambda: B.eb_op_gemm_w8(x, codes, torch.ones(64), stream=s),
        "pack": lambda: B.eb_pack_weight(bf(64, 32), stream=s),
        "moe": lambda: B.eb_op_moe_ffn(x, bf(16, 256), bf(16, 16, 256), bf(16, 256, 8), 2, return_routing=True, stream=s),
        "rope": lambda: B.eb_op_rope_kv_append(h, bf(3, 512), k, v, bt, [0], [3], stream=s),
        "attention": lambda: B.eb_op_attention(h, bf(3, 512), k, v, bt, [0], [3], stream=s),
        "gather": lambda: B.eb_op_gather_kv(h, k, v, bt, [0], [3], stream=s),
    }


NAMES = ["decode", "prefill", "mixed", "noalloc", "stack", "rmsnorm", "gemm", "gemm_w8", "pack", "moe", "rope", "attention",
         "gather"]


@pytest.mark.parametrize("name", NAMES)
def test_own_memory_comes_from_the_stream_of_the_call(world, name):
    got = _calls(world.h, "other")[name]()
    assert world.made and set(world.made) == {"other"} and world.current == ["first"]
    if name != "rope":   # (returns the caller's own)
        for t in got if isinstance(got, tuple) else (got,):
            assert (t.data_ptr(), "first") in world.used


@pytest.mark.parametrize("name", NAMES)
def test_own_memory_on_the_current_stream(world, name):
    _calls(world.h, None)[name]()
    assert world.made and set(world.made) == {"first"} and not world.used
