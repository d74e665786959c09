"""Eviction by accumulated attention weight against sorting on the CPU, and the
block cache's operators run together with the selection.  Needs an MI355X and
the built library."""
import numpy as np
import pytest

from paper_2606_03910_amd import workload as W
from tests import blockcache_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _say(*a):
    print("[gpu-case]", *a, flush=True)


@pytest.fixture(scope="module")
def nk():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_03910_amd import netkv
    netkv.load_library()
    return netkv


@pytest.fixture(scope="module")
def sel(nk):
    s = nk.Selector(0)
    yield s
    s.close()


def run(nk, sel, sizes, weight, keep, newest=0, n_keep=None):
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.uint64)
    hashes = np.random.default_rng(1).integers(1, 1 << 63, int(off[-1])).astype(np.uint64)
    cache = dict(hash_off=nk.to_device(off, sel.device), hashes=nk.to_device(hashes, sel.device))
    r = sel.evict(cache, nk.to_device(weight.astype(np.uint64), sel.device),
                  nk.to_device(np.asarray(keep, np.uint32), sel.device), newest, n_keep)
    sel.sync_errors()
    got = [nk.to_numpy(r[x]) for x in ("hash_off", "pos", "hashes")]
    want = R.evict(off, weight, hashes, keep, newest)
    for name, x, y in zip(("hash_off", "pos", "hashes"), got, want):
        assert x.shape == y.shape, (name, x.shape, y.shape)
        assert np.array_equal(x, y), f"{name}: {int((x != y).sum())} of {len(y)} differ"
    return cache, r


SIZES = [[1], [0, 1, 0, 2, 3], [255, 256, 257, 4096, 4095], [4097, 1, 4098], [16384, 16385, 5], [40000, 0, 3, 33000, 4096],
         [70001]]
KINDS = ["spread", "equal", "few", "zero", "top", "low"]


def draw(rng, n, kind):
    if kind == "spread":
        return np.minimum(np.exp(rng.standard_normal(n) * 8 + 20), 2.0 ** 62).astype(np.uint64)
    if kind == "equal":
        return np.full(n, 123456789012345, np.uint64)
    if kind == "few":
        return rng.integers(0, 4, n).astype(np.uint64) << np.uint64(40)
    if kind == "zero":
        return np.where(rng.random(n) < 0.7, 0, rng.integers(0, 40, n)).astype(np.uint64)
    if kind == "top":
        return (np.uint64((1 << 64) - 2) - rng.integers(0, 1 << 12, n).astype(np.uint64))
    return (np.uint64(1 << 50) + rng.integers(0, 1000, n).astype(np.uint64))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes", range(len(SIZES)))
def test_evict(nk, sel, sizes, kind):
    n = SIZES[sizes]
    _say("evict", n, kind)
    rng = np.random.default_rng(10 * sizes + len(kind))
    w = draw(rng, sum(n), kind)
    for part, newest in ((0.5, 0), (0.01, 3), (0.9, 100)):
        run(nk, sel, n, w, [int(np.ceil(part * x)) for x in n], newest)
    run(nk, sel, n, w, [0] * len(n))
    run(nk, sel, n, w, [0xFFFFFFFF] * len(n), 7)
    run(nk, sel, n, w, [1] * len(n), 0)


def test_evict_many_segments(nk, sel):
    rng = np.random.default_rng(2)
    n = rng.integers(0, 9, 5000)
    run(nk, sel, n, draw(rng, int(n.sum()), "few"), rng.integers(0, 6, 5000), 1)


def test_evict_outputs_that_are_too_small_and_bad_offsets(nk, sel):
    dev = sel.device
    off = np.array([0, 600, 5000, 9100], np.uint64)
    w = nk.to_device(np.arange(9100, dtype=np.uint64), dev)
    cache = dict(hash_off=nk.to_device(off, dev), hashes=nk.to_device(np.arange(1, 9101, dtype=np.uint64), dev))
    keep = nk.to_device(np.array([600, 4400, 2000], np.uint32), dev)
    work = torch.empty(nk.netkv_cache_evict_workspace(sel.h, 9100), dtype=torch.uint8, device=dev)
    room = torch.full((5400,), 77, dtype=torch.int64, device=dev)
    out_off = torch.empty(4, dtype=torch.uint64, device=dev)
    nk.netkv_cache_evict(sel.h, cache["hash_off"], w, cache["hashes"], keep, 0, out_off, None,
                         room[:5300].view(torch.uint64), work, dev)
    with pytest.raises(nk.NetKVError, match="eviction"):
        sel.sync_errors()
    assert (room[5300:] == 77).all() and room[0] == 1 and nk.to_numpy(out_off)[3] == 7000
    for bad in ([0, 600, 500, 9100], [0, 600, 5000, 9101], [7, 6, 5, 4]):
        cache["hash_off"] = nk.to_device(np.array(bad, np.uint64), dev)
        r = sel.evict(cache, w, keep, n_keep=10)
        with pytest.raises(nk.NetKVError, match="eviction"):
            sel.sync_errors()
        assert not nk.to_numpy(r["hash_off"]).any()
    sel.sync_errors()


def test_evict_refusals(nk, sel):
    dev = sel.device
    w = nk.to_device(np.arange(10, dtype=np.uint64), dev)
    off = nk.to_device(np.array([0, 10], np.uint64), dev)
    keep = nk.to_device(np.array([5], np.uint32), dev)
    out = torch.empty(2, dtype=torch.uint64, device=dev)
    pos = torch.empty(5, dtype=torch.uint32, device=dev)
    work = torch.empty(256, dtype=torch.uint8, device=dev)
    with pytest.raises(nk.NetKVError, match="work"):
        nk.netkv_cache_evict(sel.h, off, w, None, keep, 0, out, pos, None, work[:0], dev)
    with pytest.raises(nk.NetKVError, match="hashes"):
        nk.netkv_cache_evict(sel.h, off, w, None, keep, 0, out, None, out, work, dev)
    with pytest.raises(TypeError):
        nk.netkv_cache_evict(sel.h, off, w.view(torch.int64), None, keep, 0, out, pos, None, work, dev)
    with pytest.raises(nk.NetKVError, match="ECAPACITY"):
        nk.netkv_cache_evict_workspace(sel.h, 1 << 31)
    nk.netkv_cache_evict(sel.h, off, w, None, keep, 0, out, pos, None, work, dev)
    sel.sync_errors()
    assert nk.to_numpy(pos).tolist() == [5, 6, 7, 8, 9]


def test_evict_captured_and_on_another_stream(nk, sel):
    dev = sel.device
    rng = np.random.default_rng(4)
    n = [5000, 30, 20000]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.uint64)
    hashes = rng.integers(1, 1 << 63, sum(n)).astype(np.uint64)
    keep = np.array([700, 3, 9999], np.uint32)
    cache = dict(hash_off=nk.to_device(off, dev), hashes=nk.to_device(hashes, dev))
    kd, w = nk.to_device(keep, dev), torch.zeros(sum(n), dtype=torch.int64, device=dev)
    total = int(np.minimum(keep, n).sum())
    sel.evict(cache, w.view(torch.uint64), kd, 5, total)
    torch.cuda.synchronize()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = sel.evict(cache, w.view(torch.uint64), kd, 5, total)
    for step in range(3):
        x = draw(rng, sum(n), "spread")
        w.copy_(torch.from_numpy(x.astype(np.int64)))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        s.synchronize()
        want = R.evict(off, x, hashes, keep, 5)
        for name, y in zip(("hash_off", "pos", "hashes"), want):
            assert np.array_equal(nk.to_numpy(r[name]), y), name
        e = sel.evict(cache, w.view(torch.uint64), kd, 5, total)
        assert torch.equal(e["pos"].view(torch.int32), r["pos"].view(torch.int32))
        torch.cuda.synchronize()
    sel.sync_errors()


def test_the_operators_together(nk):
    """A decode instance of a small cluster: prompts are stored, a step's
    attention gives block weights, the pages' weights say which half stays,
    the resident set is loaded anew and the router sees it."""
    cfg = W.scaled(W.CONFIGS["c0"], n_requests=64)
    snap = W.make_snapshot(cfg, 0)
    sel = nk.Selector(0)
    sel.load_snapshot(snap)
    D, B = int(snap["n_decode"]), 16
    sel_b = dict(snap, block_tokens=B)
    sel.load_snapshot(sel_b)
    rng = np.random.default_rng(0)
    ctx = [300, 500, 129, 64]
    table, pages = R.tables(rng, ctx, B, spare=0, shared=4)
    hk, heads, dim = 2, 8, 64
    cache = nk.BlockCache.empty(sel, pages, hk, dim, B)
    # prompts in order, the shared prefix written by the first sequence alone
    # (the others' copies of it are the same pages)
    new = [300, 500 - 64, 129 - 64, 0]
    x = torch.from_numpy(rng.standard_normal((sum(new), 2 * hk, dim))).to(torch.bfloat16).cuda()

    def seqs(n):
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
        return nk.Sequences(torch.from_numpy(off).cuda().view(torch.uint64),
                            torch.tensor(ctx, dtype=torch.int32, device="cuda").view(torch.uint32),
                            torch.from_numpy(table.astype(np.int32)).cuda().view(torch.uint32), int(sum(n)), max(n))

    cache.store(seqs(new), x[:, :hk], x[:, hk:])
    step = seqs([1] * 4)
    q = torch.from_numpy(rng.standard_normal((4, heads, dim)) * 3).to(torch.bfloat16).cuda()
    o, bw = cache.attend(step, q, weights=True)
    sel.sync_errors()
    c = R.Cache(pages, hk, dim, B, rng)
    c.from_device(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    c.ks, c.vs = (t.double().cpu().numpy().reshape(pages, hk) for t in (cache.k_scale, cache.v_scale))
    ro, rw, tol, wtol = R.attend(c, table, ctx, [1] * 4, q.double().cpu().numpy(), heads, dim ** -0.5)
    assert (np.abs(o.double().cpu().numpy() - ro) <= tol + np.abs(ro) * torch.finfo(q.dtype).eps / 2 + 1e-30).all()
    assert (np.abs(bw.double().cpu().numpy() - rw) <= wtol).all()
    # every row's weights sum to one; the pages take all of them
    pw = torch.zeros(pages, dtype=torch.int64, device="cuda")
    cache.weigh(step, bw, pw.view(torch.uint64))
    assert abs(float(pw.sum()) / 2 ** 24 - 4 * heads) <= 4 * heads * 1e-5 + table.size * 2.0 ** -25
    # instance 0 holds these pages, the others nothing; it keeps half
    page_hash = rng.integers(1, 1 << 62, pages).astype(np.uint64)
    off = np.full(D + 1, pages, np.uint64)
    off[0] = 0
    full = dict(hash_off=nk.to_device(off, sel.device), hashes=nk.to_device(page_hash, sel.device))
    sel.load_evicted(full)
    req = dict(prefill=np.zeros(4, np.uint32), len_tokens=np.array(ctx, np.uint32),
               hash_off=np.concatenate([[0], np.cumsum([n // B for n in ctx])]).astype(np.uint64),
               hashes=np.concatenate([page_hash[table[s, :n // B]] for s, n in enumerate(ctx)]))
    rd = nk.requests_to_device(req, sel.device)
    j0 = nk.to_numpy(sel.select(rd, pairs=True)["pairs"]["prefix_blocks"]).reshape(4, D)
    assert j0[:, 0].tolist() == [n // B for n in ctx] and not j0[:, 1:].any()
    keep = np.zeros(D, np.uint32)
    keep[0] = pages // 2
    left = sel.evict(full, pw.view(torch.uint64), nk.to_device(keep, sel.device), n_keep=int(keep[0]))
    sel.load_evicted(left)
    j1 = nk.to_numpy(sel.select(rd, pairs=True)["pairs"]["prefix_blocks"]).reshape(4, D)
    stays = set(R.evict(np.array([0, pages], np.uint64), pw.cpu().numpy(), page_hash, [pages // 2], 0)[1].tolist())
    for s, n in enumerate(ctx):
        want = 0
        while want < n // B and int(table[s, want]) in stays:
            want += 1
        assert j1[s, 0] == want
    assert (j1[:, 0] < j0[:, 0]).any()
    sel.sync_errors()
    sel.close()
