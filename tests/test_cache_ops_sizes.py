"""What the binding's calls of the cache operators compare before anything
reaches the library, whose pointers carry no sizes: norm gains with the heads,
block tables with the requests, caches with the handle.  Each of these
mistakes would read or write past a tensor."""
import pytest
import torch

from paper_2606_00516_amd import binding as B


class _NoCalls:
    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 512

        def reached(*a):
            raise AssertionError(f"{name} was called")
        return reached


@pytest.fixture
def h(monkeypatch):
    """A handle of 4 query and 2 kv heads of 64, on CPU tensors."""
    monkeypatch.setattr(B, "_lib", _NoCalls())
    dev = B._dev
    # (a CPU tensor's device is -1, which the check takes for "the current one": here it is that)
    monkeypatch.setattr(B, "_dev", lambda t, dtype, name, numel=-1, d=-1: dev(t, dtype, name, numel, -1))
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(B, "_raw_stream", lambda s, dev: None)
    monkeypatch.setattr(B, "alloc_workspace", lambda n: torch.zeros(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    x = object.__new__(B.Handle)
    x.h = None
    x.n_q_heads, x.n_kv_heads, x.head_dim, x.qkv_cols, x.page_keys = 4, 2, 64, 512, 32
    x.cfg = B.LayerConfig(qk_norm=1)
    return x


def _kv(rows=2, pages=4, nkv=2, hd=64, vpages=None, page=16):
    k = torch.zeros(pages, nkv, page, hd, dtype=torch.bfloat16)
    v = torch.zeros(vpages or pages, nkv, page, hd, dtype=torch.bfloat16)
    return B.kv_struct(k, v, torch.zeros(rows, 2, dtype=torch.int32))


def _calls(h, kv):
    x, b = torch.zeros(2, 512, dtype=torch.bfloat16), B.HostBatch([3, 5], [1, 1])
    w = torch.zeros(4, 2, 16)
    good = _kv()
    return [lambda: B.eb_op_rotary_kv_append(h, B.Rotary(), x, kv, b),
            lambda: B.eb_op_attention_mod(h, x, kv, b),
            lambda: B.eb_op_kv_evict(h, kv, w, [20, 20], [16, 16], good),
            lambda: B.eb_op_kv_evict(h, good, w, [20, 20], [16, 16], kv)]


@pytest.mark.parametrize("i", range(4))
def test_what_fits_reaches_the_library(h, i):
    for kv in (_kv(), _kv(rows=5), _kv(vpages=6)):
        with pytest.raises(AssertionError, match="was called"):
            _calls(h, kv)[i]()


@pytest.mark.parametrize("i", range(4))
def test_block_tables_with_fewer_rows_than_requests(h, i):
    for rows in (0, 1):
        with pytest.raises(ValueError, match="block_tables"):
            _calls(h, _kv(rows=rows))[i]()


@pytest.mark.parametrize("i", range(4))
@pytest.mark.parametrize("kw", [dict(hd=32), dict(nkv=1), dict(vpages=3), dict(page=8)])
def test_caches_of_another_shape(h, i, kw):
    with pytest.raises(ValueError, match="cache"):
        _calls(h, _kv(**kw))[i]()


@pytest.mark.parametrize("q,k", [(32, 64), (64, 32), (128, 64), (64, 128)])
def test_norm_gains_of_another_length(h, q, k):
    x, b = torch.zeros(2, 512, dtype=torch.bfloat16), B.HostBatch([3, 5], [1, 1])
    rot = B.rotary(1e4, q_norm=torch.ones(q, dtype=torch.bfloat16), k_norm=torch.ones(k, dtype=torch.bfloat16))
    for kv in (None, _kv()):
        with pytest.raises(ValueError, match="norm"):
            B.eb_op_rotary_kv_append(h, rot, x, kv, b)
    h.cfg.qk_norm = 0   # then they are ignored
    with pytest.raises(AssertionError, match="was called"):
        B.eb_op_rotary_kv_append(h, rot, x, _kv(), b)


def test_tensors_of_another_device(h, monkeypatch):
    kv, x, b = _kv(), torch.zeros(2, 512, dtype=torch.bfloat16), B.HostBatch([3, 5], [1, 1])
    mod = B.score_mod(slopes=torch.ones(4))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for i in range(4):
        with pytest.raises(ValueError, match="current GPU"):
            _calls(h, kv)[i]()
    with pytest.raises(ValueError, match="slopes"):
        B.eb_op_attention_mod_workspace_bytes(h, b, mod)


def test_structs_filled_by_hand_name_their_own_sizes(h):
    for i in range(4):
        with pytest.raises(AssertionError, match="was called"):
            _calls(h, B.KvCache(256, 256, 4, 256, 4, 0, 1.0, 1.0))[i]()
