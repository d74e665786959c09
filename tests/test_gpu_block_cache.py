"""The block cache's operators (store, read, attend, weigh) against plain forms
in 64 bits, through the C ABI.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = {"bf16": torch.bfloat16, "fp16": torch.float16}


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


def dev(x, dt):
    return torch.from_numpy(np.ascontiguousarray(x).astype(dt)).cuda()


def upload(nk, sel, c):
    p, h, d, b = c.shape
    return nk.BlockCache(sel, torch.from_numpy(c.k.copy()).cuda().view(-1), torch.from_numpy(c.device_v()).cuda().view(-1),
                         dev(c.ks, np.float32).view(-1), dev(c.vs, np.float32).view(-1), h, d, b)


def sequences(nk, n_new, ctx, table, n_tok=None, max_tok=None, off=None):
    off = np.concatenate([[0], np.cumsum(n_new)]) if off is None else off
    return nk.Sequences(dev(off, np.int64).view(torch.uint64), dev(ctx, np.int32).view(torch.uint32),
                        dev(table, np.int32).view(torch.uint32), int(np.sum(n_new)) if n_tok is None else n_tok,
                        max(n_new) if max_tok is None else max_tok)


def case(nk, sel, seed, ctx, n_new, heads, hk, dim, block, dtype, shared=0, qstd=2.0):
    rng = np.random.default_rng(seed)
    table, pages = R.tables(rng, ctx, block, shared=shared)
    c = R.Cache(pages, hk, dim, block, rng)
    for s, n in enumerate(ctx):
        for i in range(-(-n // block)):
            c.put(table[s, i], min(block, n - i * block))
    q = torch.from_numpy(rng.standard_normal((max(1, sum(n_new)), heads, dim)) * qstd).to(HALF[dtype])
    return c, table, q


def check_attend(c, table, ctx, n_new, q, got, w=None, scale=None):
    heads, dim = q.shape[1], q.shape[2]
    n = sum(n_new)
    o, rw, tol, wtol = R.attend(c, table, ctx, n_new, q.double().numpy(), heads, dim ** -0.5 if scale is None else scale)
    x = got[:n].double().cpu().numpy()
    o, tol = o[:n], tol[:n]
    fi = torch.finfo(q.dtype)
    lim = tol + np.abs(o) * fi.eps / 2 + fi.smallest_normal * fi.eps
    assert np.array_equal(np.isnan(x), np.isnan(o))
    ok = ~np.isnan(o)
    worst = float((np.abs(x - o)[ok] / lim[ok]).max()) if ok.any() else 0.0
    assert worst <= 1.0, f"out is {worst:.2f} of what it may be off"
    ww = 0.0
    if w is not None:
        y = w.double().cpu().numpy()
        assert np.array_equal(np.isnan(y), np.isnan(rw))
        ok = ~np.isnan(rw)
        ww = float((np.abs(y - rw)[ok] / wtol[ok]).max())
        assert ww <= 1.0, f"weights are {ww:.2f} of what they may be off"
    return worst, ww


SHAPES = [
    # ctx, new tokens, heads, kv heads, dim, block
    ([1], [1], 1, 1, 64, 16),
    ([1, 2, 15, 16, 17, 63, 64, 65, 127, 300], [1] * 10, 8, 2, 128, 16),
    ([700, 33, 1029], [1, 1, 1], 16, 2, 128, 32),
    ([64, 512, 513, 1500], [1, 1, 1, 1], 5, 5, 64, 512),
    ([2100, 260], [1, 1], 6, 2, 256, 128),
    ([40, 7, 333], [3, 2, 1], 15, 5, 64, 32),          # 9 rows a head
    ([40, 7, 333], [4, 1, 4], 14, 2, 128, 64),         # 28 rows
    ([90, 200, 5], [4, 2, 5], 24, 2, 128, 16),         # 60 rows
    ([70, 300], [2, 1], 32, 2, 256, 512),              # 32 rows of 256
    ([65, 300], [65, 1], 8, 2, 64, 16),                # prompts from here on
    ([200, 77, 5], [200, 77, 5], 12, 4, 128, 16),
    ([900, 140], [130, 67], 16, 2, 128, 512),
    ([150, 333], [90, 33], 4, 2, 256, 64),
    ([1200], [1], 64, 1, 128, 1024),
    ([3000, 10], [70, 1], 5, 1, 64, 128),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attend(nk, sel, shape, dtype):
    ctx, n_new, heads, hk, dim, block = SHAPES[shape]
    _say("attend", shape, dtype, ctx, n_new, heads, hk, dim, block)
    c, table, q = case(nk, sel, 100 + shape, ctx, n_new, heads, hk, dim, block, dtype)
    seqs, qd = sequences(nk, n_new, ctx, table), q.cuda()
    cache = upload(nk, sel, c)
    o, w = cache.attend(seqs, qd, weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))
    assert torch.equal(cache.attend(seqs, qd), o)          # with and without weights, and again


def test_attend_many_sequences(nk, sel):
    """More sequences than the plan takes at a time, some with no rows or no tokens."""
    rng = np.random.default_rng(5)
    n_new = [int(x) for x in rng.integers(0, 3, 1500)]
    ctx = [int(x) for x in rng.integers(0, 40, 1500)]
    c, table, q = case(nk, sel, 5, ctx, n_new, 4, 2, 64, 16, "bf16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


@pytest.mark.parametrize("n_new", [[3, 5, 1], [70, 66, 1]])
def test_attend_rows_that_see_nothing(nk, sel, n_new):
    """More rows than tokens: the first rows are zero."""
    ctx = [2, 0, 1]
    c, table, q = case(nk, sel, 6, ctx, n_new, 4, 2, 128, 16, "bf16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    check_attend(c, table, ctx, n_new, q, o, w)
    assert not o[:n_new[0] - 2].any() and not o[n_new[0]:n_new[0] + n_new[1]].any()


@pytest.mark.parametrize("block", [16, 64, 512])
@pytest.mark.parametrize("n_new", [4, 90])
def test_attend_nan_in_what_a_row_does_not_see(nk, sel, n_new, block):
    """A NaN key or value reaches the rows that see its token and no others;
    slots past the last token hold NaN throughout."""
    ctx = [100]
    c, table, q = case(nk, sel, 7, ctx, [n_new], 4, 2, 64, block, "bf16")
    tok = 100 - n_new // 2
    c.v[table[0, tok // block], 1, tok % block, 5] = 0xFF
    kt = 100 - n_new // 4
    c.k[table[0, kt // block], 0, kt % block, 9] = 0x7F
    o = upload(nk, sel, c).attend(sequences(nk, [n_new], ctx, table), q.cuda())
    sel.sync_errors()
    check_attend(c, table, ctx, [n_new], q, o)
    nan = torch.isnan(o.float())
    first = tok - (100 - n_new)                            # the row whose own token it is
    assert not nan[:first, 2:].any() and nan[first:, 2:, 5].all() and nan[:, 2:].sum() == (n_new - first) * 2
    first = kt - (100 - n_new)
    assert not nan[:first, :2].any() and nan[first:, :2].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n_new", [1, 80])
def test_attend_large_scores_and_unequal_scales(nk, sel, n_new, dtype):
    """Scores of hundreds, and value scales far apart: a row that attends to a
    block of tiny values keeps them."""
    ctx = [400, 130]
    c, table, q = case(nk, sel, 8, ctx, [n_new, 1], 4, 2, 128, 16, dtype, qstd=60.0)
    c.vs = c.vs * 2.0 ** c.rng.integers(-28, 28, c.vs.shape)
    if dtype == "fp16":
        c.vs = np.minimum(c.vs, 2.0 ** 5)
        c.vs = np.maximum(c.vs, 2.0 ** -12)
    o, w = upload(nk, sel, c).attend(sequences(nk, [n_new, 1], ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, [n_new, 1], q, o, w))


def test_attend_queries_that_are_not_finite(nk, sel):
    """They make their own row and head NaN, no other."""
    ctx, n_new = [90, 200], [2, 1]
    c, table, q = case(nk, sel, 9, ctx, n_new, 8, 2, 128, 32, "bf16")
    q[1, 3, 7] = float("nan")
    q[2, 6, 0] = float("inf")
    o = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda())
    bad = torch.isnan(o).any(2).cpu()
    assert bad[1, 3] and bad[2, 6] and bad.sum() == 2


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_attend_scale(nk, sel, scale):
    ctx, n_new = [77, 300], [1, 2]
    c, table, q = case(nk, sel, 10, ctx, n_new, 8, 4, 64, 16, "fp16", qstd=0.7)
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), scale, weights=True)
    check_attend(c, table, ctx, n_new, q, o, w, scale)


@pytest.mark.parametrize("n_new", [[1, 2, 1], [70, 3, 1]])
def test_attend_strides_and_rows_behind_the_last(nk, sel, n_new):
    """Queries and outputs inside wider rows, rows past the last sequence and
    the rest of the wide rows as they were; host bounds larger than needed."""
    ctx = [130, 20, 700]
    c, table, q = case(nk, sel, 11, ctx, n_new, 8, 2, 128, 64, "bf16")
    n = sum(n_new)
    wide = torch.full((n + 5, 20, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:n, 3:11] = q.cuda()
    out = torch.full((n + 5, 12, 128), -3.0, dtype=torch.bfloat16, device="cuda")
    table = np.concatenate([table, np.full((3, 4), 1 << 30)], 1)      # never read
    seqs = sequences(nk, n_new, ctx, table, n_tok=n + 5, max_tok=max(n_new) + 3)
    upload(nk, sel, c).attend(seqs, wide[:, 3:11], out=out[:, 2:10])
    sel.sync_errors()
    check_attend(c, table, ctx, n_new, q, out[:, 2:10])
    assert (out[n:] == -3).all() and (out[:, :2] == -3).all() and (out[:, 10:] == -3).all()


def test_attend_long_sequence_is_split(nk, sel):
    """One sequence over all of the card, beside short ones; fp32 joins."""
    ctx, n_new = [40000, 3, 900], [1, 1, 2]
    c, table, q = case(nk, sel, 12, ctx, n_new, 8, 1, 64, 512, "fp16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


def test_attend_prompt_tile_is_split(nk, sel):
    """Few rows of a prompt after a long context: split, with empty ranges
    for the first rows' tiles."""
    ctx, n_new = [9000, 600], [40, 600]
    c, table, q = case(nk, sel, 13, ctx, n_new, 4, 2, 64, 64, "bf16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


def test_attend_on_another_stream_and_device_context(nk, sel):
    ctx, n_new = [300, 50], [1, 1]
    c, table, q = case(nk, sel, 14, ctx, n_new, 8, 2, 128, 16, "bf16")
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    want = cache.attend(seqs, q.cuda())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        qd = torch.zeros_like(q, device="cuda")
        torch.cuda._sleep(2000000)
        qd.copy_(q.cuda())
        got = cache.attend(seqs, qd)
    s.synchronize()
    assert torch.equal(want, got)


def test_attend_captured(nk, sel):
    """Two graphs, each with its own workspace, replayed several times between
    eager calls, lengths changed in place."""
    ctx, n_new = [300, 50, 2000], [1, 1, 1]
    c, table, q = case(nk, sel, 15, ctx, n_new, 8, 2, 128, 16, "bf16")
    cache = upload(nk, sel, c)
    qd = q.cuda()
    lens = [dev(ctx, np.int32).view(torch.uint32) for _ in range(2)]
    off, tb = dev([0, 1, 2, 3], np.int64).view(torch.uint64), dev(table, np.int32).view(torch.uint32)
    plans = [nk.Sequences(off, x, tb, 3, 1) for x in lens]
    cache.attend(plans[0], qd, weights=True)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for p in plans:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cache.attend(p, qd, weights=True))
        graphs.append(g)
    side = torch.cuda.Stream()
    for step in range(3):
        a, b = [300 - step, 50, 2000], [17, 50 - step, 999]
        for x, v in zip(lens, (a, b)):
            x.view(torch.int32).copy_(dev(v, np.int32))
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for p, (o, w) in zip(plans, outs):
            eo, ew = cache.attend(p, qd, weights=True)
            assert torch.equal(eo, o) and torch.equal(ew, w)
        torch.cuda.synchronize()


@pytest.mark.parametrize("n_new", [1, 80])
def test_attend_invalid_sequences(nk, sel, n_new):
    """Bad pages, lengths and offsets: reported, that sequence NaN, the others
    as without it; the next check is clean."""
    ctx, new = [100, 200, 300], [n_new] * 3
    c, table, q = case(nk, sel, 16, ctx, new, 4, 2, 64, 16, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    good = cache.attend(sequences(nk, new, ctx, table), qd)
    sel.sync_errors()
    bad = table.copy()
    bad[1, 3] = c.shape[0]                                 # one past the cache
    o, w = cache.attend(sequences(nk, new, ctx, bad), qd, weights=True)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    sel.sync_errors()
    lo, hi = n_new, 2 * n_new
    assert torch.isnan(o[lo:hi]).all() and torch.equal(o[:lo], good[:lo]) and torch.equal(o[hi:], good[hi:])
    long = [100, table.shape[1] * 16 + 1, 300]             # more tokens than the table holds
    o, w = cache.attend(sequences(nk, new, long, table), qd, weights=True)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    assert torch.isnan(o[lo:hi]).all() and torch.equal(o[:lo], good[:lo]) and torch.equal(o[hi:], good[hi:])
    assert torch.isnan(w[1]).all() and not torch.isnan(w[[0, 2]]).any()
    out = torch.full_like(qd, 5.0)
    seqs = sequences(nk, new, ctx, table, off=[0, 2 * n_new, n_new, 3 * n_new + 1], max_tok=2 * n_new + 1)
    cache.attend(seqs, qd, out=out)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    seqs = sequences(nk, new, ctx, table, max_tok=n_new)
    assert torch.equal(cache.attend(seqs, qd), good)
    sel.sync_errors()


def test_empty_calls(nk, sel):
    c = R.Cache(3, 2, 64, 16, np.random.default_rng(0))
    cache = upload(nk, sel, c)
    none = nk.Sequences(dev([0], np.int64).view(torch.uint64), dev([], np.int32).view(torch.uint32),
                        torch.zeros((0, 1), dtype=torch.int32, device="cuda").view(torch.uint32), 0, 0)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert cache.attend(none, q).shape == q.shape
    cache.store(none, kv, kv)
    assert cache.read(none)[0].shape == kv.shape
    idle = sequences(nk, [0, 0], [5, 0], np.zeros((2, 1)))
    o, w = cache.attend(idle, q, weights=True)
    assert not w.any()
    cache.store(idle, kv, kv)
    cache.read(idle)
    sel.sync_errors()


# ------------------------------------------------------------------ store and read

def ref_store(c, table, ctx, n_new, k, v):
    p, hk, d, b = c.shape
    row = 0
    for s, (n, t) in enumerate(zip(n_new, ctx)):
        for blk in range((t - n) // b, -(-t // b)) if n else []:
            p0, p1 = max(t - n - blk * b, 0), min(t - blk * b, b)
            page = table[s, blk]
            r0 = row + blk * b + p0 - (t - n)
            for x, sc, new in ((c.k, c.ks, k), (c.v, c.vs, v)):
                for h in range(hk):
                    y = new[r0:r0 + p1 - p0, h]
                    fin = np.abs(y[np.isfinite(y)])
                    s1 = R.scale_for(fin.max() if fin.size else 0.0)
                    if p0:
                        s1 = max(s1, sc[page, h])
                        x[page, h, :p0] = R.nearest(R.values(x[page, h, :p0]) * (sc[page, h] / s1))
                    sc[page, h] = s1
                    x[page, h, p0:p1] = R.nearest(y / s1)
        row += n


def same_cache(cache, c, table, ctx):
    """Every held token's bytes and scales, NaN by being NaN."""
    p, h, d, b = c.shape
    got = R.Cache(p, h, d, b, np.random.default_rng(0))
    got.from_device(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    assert np.array_equal(cache.k_scale.cpu().numpy().reshape(p, h), c.ks.astype(np.float32))
    assert np.array_equal(cache.v_scale.cpu().numpy().reshape(p, h), c.vs.astype(np.float32))
    used = np.zeros((p, b), bool)
    for s, t in enumerate(ctx):
        for i in range(-(-t // b)):
            used[table[s, i], :min(b, t - i * b)] = True
    for x, y in ((got.k, c.k), (got.v, c.v)):
        x, y = x.transpose(0, 2, 1, 3)[used], y.transpose(0, 2, 1, 3)[used]
        nx, ny = (x & 127) == 127, (y & 127) == 127
        assert np.array_equal(nx, ny)
        assert np.array_equal(x[~nx], y[~ny]), f"{int((x != y).sum())} bytes differ"


STORES = [
    # ctx after, new, kv heads, dim, block
    ([1], [1], 1, 64, 16),
    ([1, 16, 17, 40, 512, 700], [1, 1, 1, 1, 1, 1], 3, 128, 16),
    ([513, 512, 70, 1], [1, 1, 1, 1], 2, 128, 512),
    ([100, 64, 65, 31], [100, 3, 65, 30], 2, 64, 32),
    ([700, 30, 1100], [650, 13, 1100], 2, 128, 512),
    ([300, 1030], [299, 517], 1, 256, 128),
    ([1030, 2050], [1030, 1027], 1, 256, 1024),
    ([90, 5, 0, 33], [9, 0, 0, 2], 2, 64, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(STORES)))
def test_store_and_read(nk, sel, shape, dtype):
    """Bytes and scales equal the definition's; other pages are untouched;
    reading gives the values back."""
    ctx, n_new, hk, dim, block = STORES[shape]
    _say("store", shape, dtype)
    rng = np.random.default_rng(200 + shape)
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, hk, dim, block, rng)
    for s, (t, n) in enumerate(zip(ctx, n_new)):
        for i in range(-(-t // block)):
            c.put(table[s, i], max(0, min(block, t - n - i * block)))
    n = sum(n_new)
    x = rng.standard_normal((n, 2 * hk, dim)) * np.exp(2 * rng.standard_normal((n, 2 * hk, 1)))
    x = torch.from_numpy(x).to(HALF[dtype])
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    before = cache.k.clone()
    xd = x.cuda()
    cache.store(seqs, xd[:, :hk], xd[:, hk:])              # slices of one tensor
    sel.sync_errors()
    f = x.double().numpy()
    ref_store(c, table, ctx, n_new, f[:, :hk], f[:, hk:])
    same_cache(cache, c, table, ctx)
    spare = np.setdiff1d(np.arange(pages), np.concatenate([table[s, :-(-t // block)] for s, t in enumerate(ctx)] or [[]]))
    assert torch.equal(cache.k.view(pages, -1)[spare], before.view(pages, -1)[spare])
    k, v = cache.read(seqs, torch.bfloat16)
    sel.sync_errors()
    row = 0
    for s, (t, m) in enumerate(zip(ctx, n_new)):
        for h in range(hk):
            for got, which in ((k, "k"), (v, "v")):
                assert np.array_equal(got[row:row + m, h].double().cpu().numpy(), c.held(table[s], t, h, which)[t - m:])
        row += m


@pytest.mark.parametrize("block", [16, 512])
def test_store_token_by_token(nk, sel, block):
    """Tokens of growing size, one a call: the open block's scale grows and
    what it holds follows; a call of all at once agrees to the rounding of
    values that became subnormal."""
    hk, dim, T = 2, 64, 37
    rng = np.random.default_rng(3)
    table, pages = R.tables(rng, [T], block)
    c = R.Cache(pages, hk, dim, block, rng)
    x = rng.standard_normal((T, 2 * hk, dim)) * 1.25 ** np.arange(T)[:, None, None]
    x = torch.from_numpy(x).to(torch.bfloat16)
    cache, xd = upload(nk, sel, c), x.cuda()
    for t in range(T):
        cache.store(sequences(nk, [1], [t + 1], table), xd[t:t + 1, :hk], xd[t:t + 1, hk:])
        f = x[t:t + 1].double().numpy()
        ref_store(c, table, [t + 1], [1], f[:, :hk], f[:, hk:])
    sel.sync_errors()
    same_cache(cache, c, table, [T])


def test_store_values_that_are_not_finite(nk, sel):
    """Stored as NaN and left out of the scale; zeros, tiny and huge values."""
    hk, dim, block = 1, 64, 32
    rng = np.random.default_rng(4)
    ctx = [32, 32, 32, 32]
    table, pages = R.tables(rng, ctx, block)
    x = rng.standard_normal((128, 2, dim))
    x[3, 0, 4], x[5, 0, 6], x[7, 1, 8] = np.nan, np.inf, -np.inf
    x[32:64] = 0
    x[64:96] *= 1e-37
    x[96:] *= 1e36
    x = torch.from_numpy(x).to(torch.bfloat16)
    c = R.Cache(pages, hk, dim, block, rng)
    cache, xd = upload(nk, sel, c), x.cuda()
    cache.store(sequences(nk, ctx, ctx, table), xd[:, :1], xd[:, 1:])
    sel.sync_errors()
    f = x.double().numpy()
    ref_store(c, table, ctx, ctx, f[:, :1], f[:, 1:])
    same_cache(cache, c, table, ctx)
    assert (c.k[table[0, 0], 0] == 0x7F).sum() == 2


def test_store_and_read_invalid(nk, sel):
    """A bad page, or more rows than tokens: left out and reported."""
    hk, dim, block = 1, 64, 16
    rng = np.random.default_rng(5)
    ctx, n_new = [20, 20, 3], [20, 20, 5]
    table, pages = R.tables(rng, ctx, block)
    bad = table.copy()
    bad[0, 1] = 0xFFFFFFF
    x = torch.from_numpy(rng.standard_normal((45, 2, dim))).to(torch.bfloat16).cuda()
    c = R.Cache(pages, hk, dim, block, rng)
    cache = upload(nk, sel, c)
    before = cache.k.clone()
    seqs = sequences(nk, n_new, ctx, bad)
    cache.store(seqs, x[:, :1], x[:, 1:])
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    assert torch.equal(cache.k.view(pages, -1)[table[2, 0]], before.view(pages, -1)[table[2, 0]])
    k = torch.full((45, 1, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    nk.netkv_kv_read(sel.h, cache.c, seqs, k, v, sel.device)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    assert (k[40:] == 9).all() and torch.isnan(k[16:20]).all() and not torch.isnan(k[20:40]).any()
    assert torch.isnan(v[16:20]).all() and not torch.isnan(v[20:40]).any()


# ------------------------------------------------------------------ weigh

def test_weigh(nk, sel):
    """Sums over pages that sequences share, to the unit; blocks past the last
    token and what is not a weight add nothing."""
    rng = np.random.default_rng(6)
    ctx = [100, 64, 1, 0, 333]
    table, pages = R.tables(rng, ctx, 16, shared=3)
    w = np.exp(3 * rng.standard_normal(table.shape)).astype(np.float32)
    pw = rng.integers(0, 1 << 40, pages)
    want = pw.copy()
    for s, n in enumerate(ctx):
        for b in range(-(-n // 16)):
            want[table[s, b]] += int(np.rint(float(w[s, b]) * 2 ** 24))
    seqs = sequences(nk, [0] * 5, ctx, table)
    got, wd = dev(pw, np.int64), torch.from_numpy(w).cuda()
    nk.netkv_kv_weigh(sel.h, seqs, 16, wd, got.view(torch.uint64), sel.device)
    sel.sync_errors()
    assert np.array_equal(got.cpu().numpy(), want)
    wd[0, 0], wd[1, 1], wd[4, 2] = float("nan"), -1.0, float("inf")
    got = dev(pw, np.int64)
    nk.netkv_kv_weigh(sel.h, seqs, 16, wd, got.view(torch.uint64), sel.device)
    with pytest.raises(nk.NetKVError, match="weight"):
        sel.sync_errors()
    for s, b in ((0, 0), (1, 1), (4, 2)):
        want[table[s, b]] -= int(np.rint(float(w[s, b]) * 2 ** 24))
    assert np.array_equal(got.cpu().numpy(), want)


# ------------------------------------------------------------------ refusals

def test_refusals(nk, sel):
    c = R.Cache(4, 2, 64, 16, np.random.default_rng(0))
    cache = upload(nk, sel, c)
    seqs = sequences(nk, [1], [5], np.zeros((1, 1)))
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    for kw in (dict(block_tokens=24), dict(block_tokens=8), dict(block_tokens=2048), dict(head_dim=96),
               dict(n_kv_heads=0), dict(n_pages=0)):
        bad = nk.netkv_kv_t.from_buffer_copy(cache.c)
        for name, v in kw.items():
            setattr(bad, name, v)
        with pytest.raises(nk.NetKVError, match="EINVAL"):
            nk.netkv_kv_attend_workspace(sel.h, bad, seqs, 4, False)
    with pytest.raises(nk.NetKVError, match="multiple of n_kv_heads"):
        cache.attend(seqs, torch.zeros((1, 3, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(nk.NetKVError, match="<= 64"):
        cache.attend(seqs, torch.zeros((1, 130, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(nk.NetKVError, match="scale"):
        cache.attend(seqs, q, float("nan"))
    with pytest.raises(TypeError):
        cache.attend(seqs, q.float())
    with pytest.raises(TypeError):
        cache.attend(seqs, q, out=torch.zeros_like(q, dtype=torch.float16))
    with pytest.raises(ValueError):
        cache.attend(seqs, q[:, :, :32])
    with pytest.raises(ValueError):
        cache.attend(seqs, torch.zeros((1, 64, 4), dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    with pytest.raises(ValueError, match="aligned"):
        cache.attend(seqs, torch.zeros(4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(1, 4, 64))
    with pytest.raises(ValueError):
        cache.attend(sequences(nk, [2], [5], np.zeros((1, 1))), q)
    with pytest.raises(nk.NetKVError, match="work"):
        nk.netkv_kv_attend(sel.h, cache.c, seqs, q, 0.1, torch.empty_like(q), None,
                           torch.empty(256, dtype=torch.uint8, device="cuda"), sel.device)
    with pytest.raises(ValueError):
        nk.Sequences(dev([0, 1], np.int64).view(torch.uint64), dev([5], np.int32).view(torch.uint32),
                     torch.zeros(3, dtype=torch.int32, device="cuda").view(torch.uint32), 1, 1)
    with pytest.raises(TypeError):
        nk.Sequences(torch.zeros(2, dtype=torch.uint64), torch.zeros(1, dtype=torch.uint32),
                     torch.zeros((1, 1), dtype=torch.uint32), 1, 1)
    with pytest.raises(TypeError, match="dtype"):
        k = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
        cache.store(seqs, k, k.half())
    torch.cuda.synchronize()
