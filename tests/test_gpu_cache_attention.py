"""eb_op_attention_mod against plain 64-bit attention: scores (cap, distance
bias, scale), masks (window, prefix, documents, rows that see nothing), decode
rows, chunks and both, long contexts with split keys, 8-bit caches, log-sum-exp
and the weights that the cached keys receive.

Tolerances.  Probabilities enter the second product rounded to bf16 (2^-9
relative, bf16 half steps counted as 2^-8 of the value), the output is rounded
once more (2^-8), so each output is off by at most
2^-8 sum p |v| + 2^-8 |o| plus fp32 terms far below; 2^-7 max|v| bounds both.
lse and weights stay in fp32: the scores' products are exact, their sums,
exponentials and the cap's tanh are off by a few fp32 steps of the largest
score in log2 units (at most 2^8 here, so 2^8 2^-23 = 3e-5 absolute, of lse and
relative of a weight); sums of n weights add n steps of 2^-24."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R

pytestmark = pytest.mark.gpu


def _qkv(T, sh, seed, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, (sh.n_q_heads + 2 * sh.n_kv_heads) * sh.head_dim, generator=g)
    x[:, :sh.n_q_heads * sh.head_dim] *= scale
    return x.to(torch.bfloat16)


def run(sh, ctx, chk, *, fp8=False, seed=1, window=0, prefix=None, first=None, softcap=0.0, slopes=None, scale=0.0,
        weights=False, weight_rows=0, cache=None, qkv=None, poison=True):
    ctx, chk = np.asarray(ctx), np.asarray(chk)
    T = int(chk.sum())
    cache = cache or R.make_cache(ctx + chk, sh.n_kv_heads, sh.head_dim, fp8, seed, poison=poison)
    qkv = _qkv(T, sh, seed + 1) if qkv is None else qkv
    w0 = torch.rand(cache.k.shape[:3], generator=torch.Generator().manual_seed(seed + 2)) if weights else None
    first_t = None if first is None else torch.tensor(np.asarray(first), dtype=torch.int32)
    sl = None if slopes is None else torch.tensor(slopes, dtype=torch.float32)
    ref = R.attend_batch(sh, qkv, cache, ctx, chk, window, prefix, first, w0, weight_rows, scale=scale,
                         softcap=softcap, slopes=None if sl is None else sl.numpy())
    d = cache.cuda()
    h = B.Handle(sh, len(ctx), T)
    kv, batch = B.kv_struct(d.k, d.v, d.bt, cache.scales), B.HostBatch(ctx, chk)
    mod = B.score_mod(scale, softcap, None if sl is None else sl.cuda(), window,
                      None if first_t is None else first_t.cuda(), prefix)
    lse = torch.full((T, sh.n_q_heads), 7.0, device="cuda")
    w = None if w0 is None else w0.cuda()
    out = B.eb_op_attention_mod(h, qkv.cuda(), kv, batch, mod, lse=lse, kv_weights=w, weight_rows=weight_rows)
    torch.cuda.synchronize()
    return (R.f64(out), R.f64(lse), None if w is None else R.f64(w)), ref, cache, w0


def check(got, ref, vmax=6.0):
    out, lse, w = got
    ro, rl, rw = ref
    assert np.array_equal(np.isneginf(lse), np.isneginf(rl))
    assert np.array_equal(np.isfinite(out), np.isfinite(ro))
    fine = np.isfinite(ro)
    assert np.all(np.abs(out - ro)[fine] <= 2.0 ** -7 * vmax), np.abs(out - ro)[fine].max()
    m = np.isfinite(rl)
    assert np.all(np.abs(lse - rl)[m] <= 3e-5 + 2.0 ** -22 * np.abs(rl[m])), np.abs(lse - rl)[m].max()
    if w is not None:
        assert np.allclose(w, rw, rtol=6e-5, atol=1e-6, equal_nan=True), np.nanmax(np.abs(w - rw))


HEADS = [(4, 4, 64), (4, 2, 64), (8, 2, 128), (16, 2, 128), (8, 1, 64)]
MODS = [dict(), dict(softcap=20.0), dict(slopes=True), dict(softcap=30.0, slopes=True), dict(scale=0.3)]


def _mod(m, sh):
    m = dict(m)
    if m.get("slopes"):
        m["slopes"] = [2.0 ** (-8.0 * (i + 1) / sh.n_q_heads) for i in range(sh.n_q_heads)]
    return m


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("mod", range(len(MODS)))
def test_decode(heads, fp8, mod):
    sh = R.shape(*heads)
    # one key, page edges, one split, several
    ctx = [0, 1, 14, 15, 16, 63, 127, 128, 300, 1024, 1100]
    got, ref, _, _ = run(sh, ctx, [1] * len(ctx), fp8=fp8, weights=True, **_mod(MODS[mod], sh))
    check(got, ref)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("mod", range(len(MODS)))
def test_chunks(heads, fp8, mod):
    sh = R.shape(*heads)
    ctx, chk = [0, 5, 100, 0, 700], [2, 33, 130, 17, 3]
    got, ref, _, _ = run(sh, ctx, chk, fp8=fp8, weights=True, **_mod(MODS[mod], sh))
    check(got, ref)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 129, 1000])
def test_window(window, fp8):
    sh = R.shape(8, 2, 128)
    ctx, chk = [0, 700, 100, 15, 16, 1300, 400], [1, 1, 40, 1, 1, 6, 150]
    got, ref, _, _ = run(sh, ctx, chk, fp8=fp8, window=window, weights=True, softcap=25.0)
    check(got, ref)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 1, 128)])
def test_prefix(heads):
    sh = R.shape(*heads)
    ctx, chk = [0, 40, 100, 9], [70, 65, 1, 200]
    for prefix in ([70, 0, 101, 100], [33, 105, 50, 209], [0, 41, 0, 10]):
        got, ref, _, _ = run(sh, ctx, chk, prefix=prefix, weights=True)
        check(got, ref)
    slopes = [0.1 * (i + 1) for i in range(sh.n_q_heads)]
    got, ref, _, _ = run(sh, ctx, chk, prefix=[70, 80, 20, 130], window=50, slopes=slopes, weights=True)
    check(got, ref)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [(4, 2, 64), (16, 2, 128)])
def test_documents_and_rows_that_see_nothing(heads, fp8):
    sh = R.shape(*heads)
    ctx, chk = [0, 300, 1100, 90, 0, 500], [150, 80, 1, 1, 1, 9]
    rng = np.random.default_rng(4)
    first, row = [], 0
    for c, n in zip(ctx, chk):
        p = c + np.arange(n)
        first.append(np.maximum(p - rng.integers(0, 60, n), 0))
    first[0][-20:] = 10 ** 9            # padding at the end of a chunk
    first[1][:] = 2 ** 31 - 1           # a whole chunk of it
    first[2][:] = 1101                  # a decode row that sees nothing
    first[3][:] = -5
    got, ref, _, _ = run(sh, ctx, chk, first=np.concatenate(first), fp8=fp8, weights=True)
    check(got, ref)
    assert np.all(got[0][150:230] == 0) and np.all(np.isneginf(got[1][150:231]))


@pytest.mark.parametrize("rows", [1, 7, 32, 500])
def test_weight_rows(rows):
    sh = R.shape(8, 2, 64)
    got, ref, _, _ = run(sh, [0, 200, 30], [100, 45, 1], weights=True, weight_rows=rows, window=90)
    check(got, ref)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [(8, 1, 128), (4, 4, 64)])
def test_long_contexts_split(heads, fp8):
    # more than 64 splits of a decode row, split chunks; a bias that leaves far splits nothing but zeros
    sh = R.shape(*heads)
    for kw in (dict(softcap=50.0), dict(slopes=[0.5 / (i + 1) for i in range(sh.n_q_heads)])):
        got, ref, _, _ = run(sh, [40000, 9000, 5000], [1, 1, 5], fp8=fp8, weights=True, **kw)
        check(got, ref)


def test_values_of_hidden_keys_do_not_reach_a_row():
    sh = R.shape(8, 2, 128)
    ctx, chk = [200, 300, 64], [1, 70, 130]
    cache = R.make_cache(np.add(ctx, chk), 2, 128, seed=3)
    k, v, bt = cache.k, cache.v, cache.bt
    # before the windows' reach (whole pages and inside one), and keys that only later rows see
    for i, t, x in ((0, 3, np.nan), (0, 150, np.inf), (1, 100, np.nan), (1, 330, np.inf), (2, 100, np.nan),
                    (2, 101, -np.inf)):
        v[bt[i, t // 16].long(), :, t % 16, 5] = x
    for i, t, x in ((0, 20, np.nan), (1, 60, np.inf), (2, 180, np.nan)):
        k[bt[i, t // 16].long(), :, t % 16, 9] = x
    got, ref, _, _ = run(sh, ctx, chk, cache=cache, window=45, weights=True)
    assert np.isfinite(ref[0]).any() and not np.isfinite(ref[0]).all()
    out, lse, w = got
    assert np.array_equal(np.isnan(out), np.isnan(ref[0]))
    assert np.array_equal(np.isposinf(out), np.isposinf(ref[0])) and np.array_equal(np.isneginf(out), np.isneginf(ref[0]))
    fine = np.isfinite(ref[0])
    assert np.all(np.abs(out - ref[0])[fine] <= 2.0 ** -7 * 6)


def test_bad_pages_read_as_zeros_and_get_no_weights():
    sh = R.shape(4, 2, 64)
    ctx, chk = [100, 90], [1, 40]
    cache = R.make_cache(np.add(ctx, chk), 2, 64, seed=5)
    bt = cache.bt.clone()
    bt[0, 2], bt[1, 3] = -1, cache.k.shape[0] + 7
    zeroed = R.Cache(cache.k.clone(), cache.v.clone(), cache.bt, None)
    for i, p in ((0, 2), (1, 3)):
        zeroed.k[cache.bt[i, p].long()] = 0
        zeroed.v[cache.bt[i, p].long()] = 0
    qkv = _qkv(41, sh, 9)
    ref = R.attend_batch(sh, qkv, zeroed, ctx, chk)
    h = B.Handle(sh, 2, 41)
    d = cache.cuda()
    w0 = torch.rand(cache.k.shape[:3])
    w = w0.cuda()
    btd = bt.cuda()
    out = B.eb_op_attention_mod(h, qkv.cuda(), B.kv_struct(d.k, d.v, btd), B.HostBatch(ctx, chk), kv_weights=w)
    torch.cuda.synchronize()
    assert np.all(np.abs(R.f64(out) - ref[0]) <= 2.0 ** -7 * 6)
    for i, p in ((0, 2), (1, 3)):
        assert torch.equal(w[cache.bt[i, p].long()].cpu(), w0[cache.bt[i, p].long()])


def test_plain_mod_equals_eb_op_attention_and_untouched_slots():
    sh = R.shape(8, 2, 128)
    ctx, chk = [500, 33, 0], [1, 20, 64]
    cache = R.make_cache(np.add(ctx, chk), 2, 128, seed=6)
    got, ref, _, w0 = run(sh, ctx, chk, cache=cache, weights=True, seed=6)
    check(got, ref)
    d = cache.cuda()
    h = B.Handle(sh, 3, 85)
    old = B.eb_op_attention(h, _qkv(85, sh, 7).cuda(), d.k, d.v, d.bt, ctx, chk)
    assert np.all(np.abs(R.f64(old) - got[0]) <= 2.0 ** -6)
    # weights outside the requests' slots keep their bits
    own = np.zeros(cache.k.shape[0] * 16, bool).reshape(-1, 16)
    for i, n in enumerate(np.add(ctx, chk)):
        t = np.arange(n)
        own[cache.bt[i].numpy()[t // 16], t % 16] = True
    own = np.broadcast_to(own[:, None], got[2].shape)
    assert np.array_equal(got[2][~own], R.f64(w0)[~own])


def test_row_does_not_depend_on_the_batch_and_repeats_bitwise():
    sh = R.shape(8, 2, 64)
    ctx, chk = [900, 64, 10, 2000], [1, 30, 1, 3]
    cache = R.make_cache(np.add(ctx, chk), 2, 64, seed=8)
    qkv = _qkv(35, sh, 12)
    kw = dict(cache=cache, qkv=qkv, softcap=20.0, weights=True)
    a = run(sh, ctx, chk, **kw)[0]
    b = run(sh, ctx, chk, **kw)[0]
    assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(a, b))
    row = 0
    for i, n in enumerate(chk):
        one = R.Cache(cache.k, cache.v, cache.bt[i:i + 1].contiguous(), None)
        got = run(sh, ctx[i:i + 1], chk[i:i + 1], cache=one, qkv=qkv[row:row + n].contiguous(), softcap=20.0)[0]
        assert np.array_equal(got[0], a[0][row:row + n]) and np.array_equal(got[1], a[1][row:row + n])
        row += n


def test_many_requests_use_a_table_in_the_workspace():
    sh = R.shape(4, 2, 64)
    rng = np.random.default_rng(2)
    ctx = rng.integers(0, 40, 300)
    chk = np.where(np.arange(300) % 3 == 0, rng.integers(2, 6, 300), 1)
    got, ref, _, _ = run(sh, ctx, chk, weights=True, window=20)
    check(got, ref)


def test_captured_call_replays():
    sh = R.shape(8, 2, 64)
    rng = np.random.default_rng(3)
    ctx, chk = rng.integers(0, 900, 150), np.where(np.arange(150) % 5 == 0, 9, 1)
    T = int(chk.sum())
    d = R.make_cache(ctx + chk, 2, 64, seed=4).cuda()
    h, batch = B.Handle(sh, 150, T), B.HostBatch(ctx, chk)
    kv, mod = B.kv_struct(d.k, d.v, d.bt), B.score_mod(softcap=15.0)
    qkv = _qkv(T, sh, 5).cuda()
    ws = B.alloc_workspace(B.eb_op_attention_mod_workspace_bytes(h, batch, mod, True))
    out, lse = torch.empty(T, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 8, device="cuda")
    w = torch.zeros(d.k.shape[:3], device="cuda")
    call = lambda: B.eb_op_attention_mod(h, qkv, kv, batch, mod, out, lse, w, ws=ws)  # noqa: E731
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    other = R.make_cache([50], 2, 64, seed=9).cuda()
    for k in range(3):
        qkv.copy_(_qkv(T, sh, 20 + k))
        w.zero_()
        g.replay()
        torch.cuda.synchronize()
        a, b, c = out.clone(), lse.clone(), w.clone()
        # another call of the same handle in between
        B.eb_op_attention_mod(h, _qkv(1, sh, 3).cuda(), B.kv_struct(other.k, other.v, other.bt), B.HostBatch([49], [1]))
        w.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, lse) and torch.equal(c, w)


def test_empty_batch_and_another_stream():
    sh = R.shape(4, 2, 64)
    h = B.Handle(sh, 2, 8)
    d = R.make_cache([40], 2, 64, seed=1, poison=False).cuda()
    kv = B.kv_struct(d.k, d.v, d.bt)
    out = B.eb_op_attention_mod(h, torch.empty(0, 512, dtype=torch.bfloat16, device="cuda"), kv, B.HostBatch([], []))
    assert out.shape == (0, 256)
    qkv = _qkv(1, sh, 2).cuda()
    a = B.eb_op_attention_mod(h, qkv, kv, B.HostBatch([39], [1]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = B.eb_op_attention_mod(h, qkv, kv, B.HostBatch([39], [1]), stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b)
