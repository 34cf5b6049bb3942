"""eb_op_kv_evict: the kept positions, and the copies of keys, values and weights
bit for bit, against a plain sort; and a request served across the three
operators: rotate and append, attend and count weights, evict, go on."""
import numpy as np
import pytest
import torch

from paper_2606_00516_amd import binding as B
from tests import _cache_ops as R

pytestmark = pytest.mark.gpu


def run(sh, lens, keep, sink, recent, *, fp8=False, seed=1, make=None, same_pool=False, want_kept=True, stride=None):
    lens, keep = np.asarray(lens), np.asarray(keep)
    nkv, hd = sh.n_kv_heads, sh.head_dim
    k = np.minimum(lens, keep)
    src = R.make_cache(lens, nkv, hd, fp8, seed)
    g = torch.Generator().manual_seed(seed + 3)
    w = torch.exp(3 * torch.randn(src.k.shape[:3], generator=g))
    if make is not None:
        w = make(w, src, g)
    dst = R.make_cache(k, nkv, hd, fp8, seed + 9)
    if same_pool:   # the destination's pages behind the source's in one pool
        n = src.k.shape[0]
        pool = R.Cache(torch.cat([src.k, dst.k]), torch.cat([src.v, dst.v]), src.bt, src.scales)
        w = torch.cat([w, torch.zeros(dst.k.shape[:3])])
        dst = R.Cache(pool.k, pool.v, torch.where(dst.bt >= 0, dst.bt + n, dst.bt), src.scales)
        src = pool
    ds, dd = src.cuda(), None
    if same_pool:
        dd = R.Cache(ds.k, ds.v, dst.bt.cuda(), dst.scales)
        wd = w.cuda()
        dw = wd
    else:
        dd = dst.cuda()
        wd = w.cuda()
        dw = torch.full(dst.k.shape[:3], -7.0, device="cuda")
    dw0 = dw.cpu().clone()
    h = B.Handle(sh, max(1, len(lens)), 8)
    kept = torch.full((len(lens), nkv, stride or max(1, int(k.max()) if len(k) else 1)), -3, dtype=torch.int32, device="cuda")
    got = B.eb_op_kv_evict(h, B.kv_struct(ds.k, ds.v, ds.bt, src.scales), wd, lens, keep,
                           B.kv_struct(dd.k, dd.v, dd.bt, dst.scales), dw, sink, recent, kept if want_kept else None)
    torch.cuda.synchronize()
    assert np.array_equal(got, k)
    view = torch.uint8 if fp8 else torch.int16
    bits = lambda t: t.cpu().view(view).numpy()  # noqa: E731
    ek, ev, ew = bits(dst.k).copy(), bits(dst.v).copy(), dw0.numpy().copy()
    sk, sv, sw = bits(src.k), bits(src.v), w.numpy()
    ekept = np.full(kept.shape, -3, np.int32)
    for i in range(len(lens)):
        t = np.arange(lens[i])
        pg, sl = src.bt[i].numpy()[t // 16], t % 16
        for hh in range(nkv):
            at = R.keep_positions(sw[pg, hh, sl], int(keep[i]), sink, recent)
            assert len(at) == k[i]
            ekept[i, hh, :k[i]] = at
            j = np.arange(k[i])
            to = (dst.bt[i].numpy()[j // 16], hh, j % 16)
            frm = (pg[at], hh, sl[at])
            ek[to], ev[to], ew[to] = sk[frm], sv[frm], sw[frm]
    if want_kept:
        assert np.array_equal(kept.cpu().numpy(), ekept)
    assert np.array_equal(bits(dd.k), ek) and np.array_equal(bits(dd.v), ev)
    assert np.array_equal(dw.cpu().numpy().view(np.int32), ew.view(np.int32))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (8, 8, 128)])
def test_sizes(heads, fp8):
    sh = R.shape(*heads)
    run(sh, [1, 2, 15, 16, 17, 63, 64, 65, 100, 1000, 0], [1, 1, 8, 16, 16, 3, 64, 64, 37, 999, 5], 0, 0, fp8=fp8)
    run(sh, [300, 250, 20, 33], [200, 200, 200, 20], 4, 16, fp8=fp8, stride=211)


@pytest.mark.parametrize("n", [4095, 4096, 4097, 16385, 65536, 65537, 150000])
def test_long_requests(n):
    sh = R.shape(2, 1, 64)
    run(sh, [n, n // 3], [n // 7, n // 4], 3, 100)
    run(sh, [n], [n - 1], 0, 0)


@pytest.mark.parametrize("sink,recent", [(0, 0), (10, 0), (0, 10), (20, 44), (64, 0), (0, 64)])
def test_sink_and_recent(sink, recent):
    run(R.shape(4, 2, 64), [500, 64, 65, 70, 30], [64] * 5, sink, recent)


def _ties(w, src, g):
    return (w * 2).round().clamp(0, 3)


def _zeros(w, src, g):
    w = torch.where(torch.rand(w.shape, generator=g) < 0.95, torch.zeros(()), w)
    return torch.where(torch.rand(w.shape, generator=g) < 0.3, -w, w)   # -0 as well as 0


def _odd(w, src, g):
    u = torch.rand(w.shape, generator=g)
    w = torch.where(u < 0.02, torch.full((), float("inf")), w)
    w = torch.where((u > 0.02) & (u < 0.03), torch.full((), float("nan")), w)
    w = torch.where((u > 0.03) & (u < 0.2), -w, w)
    return torch.where((u > 0.2) & (u < 0.3), torch.full((), 1e-42), w)


@pytest.mark.parametrize("make", [_ties, _zeros, _odd, lambda w, s, g: torch.ones_like(w)])
def test_equal_and_odd_weights(make):
    run(R.shape(4, 2, 64), [900, 5000, 40, 17], [450, 1234, 39, 5], 2, 3, make=make)


def test_one_pool_and_no_kept_and_many_requests():
    sh = R.shape(4, 2, 64)
    run(sh, [300, 90, 400], [100, 90, 33], 4, 8, same_pool=True, want_kept=False)
    rng = np.random.default_rng(1)
    run(sh, rng.integers(0, 90, 400), rng.integers(8, 60, 400), 3, 5)


def test_captured_call_replays():
    sh = R.shape(4, 2, 64)
    rng = np.random.default_rng(5)
    lens = rng.integers(40, 90, 400)
    keep = np.full(400, 32)
    src, dst = R.make_cache(lens, 2, 64, seed=1).cuda(), R.make_cache(keep, 2, 64, seed=2).cuda()
    h = B.Handle(sh, 400, 8)
    a, b = B.kv_struct(src.k, src.v, src.bt), B.kv_struct(dst.k, dst.v, dst.bt)
    w = torch.rand(src.k.shape[:3], device="cuda")
    kept = torch.zeros(400, 2, 32, dtype=torch.int32, device="cuda")
    ws = B.alloc_workspace(B.eb_op_kv_evict_workspace_bytes(h, lens, keep))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.eb_op_kv_evict(h, a, w, lens, keep, b, None, 1, 2, kept, ws)
    for k in range(3):
        w.copy_(torch.rand(w.shape, generator=torch.Generator().manual_seed(k)).cuda())
        g.replay()
        torch.cuda.synchronize()
        x, y = kept.clone(), dst.k.clone()
        kept.zero_()
        B.eb_op_kv_evict(h, a, w, lens, keep, b, None, 1, 2, kept)
        torch.cuda.synchronize()
        assert torch.equal(x, kept)
        assert torch.equal(y.view(torch.int16), dst.k.view(torch.int16))


@pytest.mark.parametrize("fp8", [False, True])
def test_served_across_the_operators(fp8):
    """Prompts are rotated, appended and attended to with their weights, cut back, and decoded further at their true
    positions: each step's outputs against 64-bit attention over what the cache holds, and the weights that choose
    what stays against sums of its probabilities."""
    sh = R.shape(8, 2, 64)
    nq, nkv, hd, S = 8, 2, 64, 3
    chk = np.array([150, 70, 33])
    ctx = np.zeros(3, np.int64)
    width = 12
    pool = R.make_cache([width * 16] * (2 * S), nkv, hd, fp8, seed=3, poison=False)
    rows = [pool.bt[:S].contiguous(), pool.bt[S:].contiguous()]
    d = pool.cuda()
    bts = [r.cuda() for r in rows]
    w = torch.zeros(pool.k.shape[:3], device="cuda")
    h = B.Handle(sh, S, 300)
    rot = B.rotary(1e4, 32, "interleaved", "yarn", 4.0, 128)
    mod = B.score_mod(softcap=30.0)
    g = torch.Generator().manual_seed(1)
    cur, true_pos = 0, np.zeros(3, np.int64)
    for step in range(7):
        n = chk if step == 0 else np.ones(3, np.int64)
        T = int(n.sum())
        qkv = (2 * torch.randn(T, (nq + 2 * nkv) * hd, generator=g)).to(torch.bfloat16).cuda()
        pos = torch.tensor(np.concatenate([np.arange(p, p + m) for p, m in zip(true_pos, n)]), dtype=torch.int32).cuda()
        kv, batch = B.kv_struct(d.k, d.v, bts[cur], pool.scales), B.HostBatch(ctx, n)
        before = R.f64(qkv)
        B.eb_op_rotary_kv_append(h, rot, qkv, kv, batch, pos)
        w0 = w.cpu().clone()
        lse = torch.empty(T, nq, device="cuda")
        out = B.eb_op_attention_mod(h, qkv, kv, batch, mod, lse=lse, kv_weights=w)
        torch.cuda.synchronize()
        x = before.reshape(T, -1, hd)
        f = R.frequencies(32, 1e4, "yarn", 4.0, 128)
        rq = R.rotate(x[:, :nq], pos.cpu().numpy(), 32, f, "interleaved", 0.1 * np.log(4.0) + 1)
        assert np.all(np.abs(R.f64(qkv).reshape(T, -1, hd)[:, :nq] - rq) <= 2.0 ** -8 * np.abs(rq) + 1e-4)
        now = R.Cache(d.k.cpu(), d.v.cpu(), rows[cur], pool.scales)
        ro, rl, rw = R.attend_batch(sh, qkv, now, ctx, n, weights=w0, softcap=30.0)
        assert np.all(np.abs(R.f64(out) - ro) <= 2.0 ** -7 * 12)
        assert np.all(np.abs(R.f64(lse) - rl) <= 1e-4)
        assert np.allclose(R.f64(w), rw, rtol=1e-4, atol=1e-6)
        ctx, true_pos = ctx + n, true_pos + n
        if step in (0, 3, 5):   # over the budget of 40 keys
            keep = np.full(3, 40)
            kept = torch.zeros(S, nkv, 40, dtype=torch.int32, device="cuda")
            new = B.eb_op_kv_evict(h, kv, w, ctx, keep, B.kv_struct(d.k, d.v, bts[1 - cur], pool.scales), w, 2, 8, kept)
            torch.cuda.synchronize()
            for i in range(S):
                if ctx[i] <= 40:
                    continue
                t = np.arange(ctx[i])
                for hh in range(nkv):
                    wt = w.cpu().numpy()[rows[cur][i].numpy()[t // 16], hh, t % 16]
                    assert np.array_equal(kept[i, hh].cpu().numpy(), R.keep_positions(wt, 40, 2, 8))
            ctx, cur = new.astype(np.int64), 1 - cur
