"""Differential attention over the block cache against its plain form in 64
bits, through the C ABI.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R
from tests import diff_ref as F
from tests import rope_ref as T
from tests.test_gpu_block_cache import HALF, case, dev, ref_store, sequences, upload

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


def weights(seed, heads, dim):
    rng = np.random.default_rng(1000 + seed)
    return (0.5 + 0.3 * rng.standard_normal(heads // 2)).astype(np.float32), (1 + 0.2 * rng.standard_normal(2 * dim)).astype(np.float32)


def run(cache, seqs, qd, lam, norm=None, **kw):
    if "out" not in kw:                                    # a row left out must not hold an earlier call's answer
        kw["out"] = torch.full((qd.shape[0], qd.shape[1] // 2, 2 * qd.shape[2]), -77.0, dtype=qd.dtype, device="cuda")
    return cache.attend_diff(seqs, qd, dev(lam, np.float32), norm=None if norm is None else dev(norm, np.float32), **kw)


def check(c, table, ctx, n_new, q, got, lam, norm=None, scale=None, eps=1e-5, gain=1.0):
    n = sum(n_new)
    o, tol = F.attend(c, table, ctx, n_new, q.double().numpy(), q.shape[2] ** -0.5 if scale is None else scale,
                      lam.astype(np.float64), None if norm is None else norm.astype(np.float64), eps, gain)
    x = got[:n].double().cpu().numpy()
    o, tol = o[:n], tol[:n]
    fi = torch.finfo(q.dtype)
    lim = tol * (1 + fi.eps) + np.abs(o) * fi.eps / 2 + fi.smallest_normal * fi.eps
    assert np.array_equal(np.isnan(x), np.isnan(o))
    ok = ~np.isnan(o)
    worst = float((np.abs(x - o)[ok] / lim[ok]).max()) if ok.any() else 0.0
    assert worst <= 1.0, f"out is {worst:.2f} of what it may be off"
    return worst


SHAPES = [
    # ctx, new tokens, heads, kv heads, dim, block
    ([1], [1], 2, 2, 64, 16),
    ([1, 2, 15, 16, 17, 63, 64, 65, 127, 300], [1] * 10, 8, 2, 128, 16),
    ([700, 33, 1029], [1, 1, 1], 16, 2, 128, 32),
    ([64, 512, 513, 1500], [1, 1, 1, 1], 6, 6, 64, 512),
    ([2100, 260], [1, 1], 24, 4, 64, 128),
    ([40, 7, 333], [3, 2, 1], 18, 6, 64, 32),          # 9 rows a pair
    ([40, 7, 333], [4, 1, 4], 28, 4, 128, 64),         # 28 rows: two tiles
    ([90, 200, 5], [4, 2, 5], 48, 4, 64, 16),          # 60 rows: four tiles
    ([1200], [1], 64, 2, 64, 1024),                    # 32 rows of one token
    ([1200], [1], 128, 2, 128, 1024),                  # 64 rows of 128 dimensions: for prompts
    ([65, 300], [65, 1], 16, 4, 64, 16),               # prompts from here on
    ([200, 77, 5], [200, 77, 5], 12, 4, 128, 16),
    ([900, 140], [130, 67], 16, 2, 64, 512),
    ([900, 140], [130, 67], 16, 2, 128, 512),
    ([150, 333], [90, 33], 4, 2, 128, 64),
    ([3000, 10], [230, 1], 2, 2, 64, 128),
    ([90, 5], [3, 1], 128, 2, 64, 16),                 # 64 rows of one token
    ([90, 40], [7, 40], 128, 2, 128, 32),
    ([17, 3], [1, 2], 512, 512, 64, 16),               # more pairs than workgroup slots a range
    ([70], [60], 256, 256, 128, 64),
    ([448, 100], [1, 1], 16, 2, 128, 64),              # the longest that are not split, and one step more
    ([449, 100], [1, 1], 16, 2, 128, 64),
    ([768, 500], [2, 1], 8, 2, 64, 16),
    ([769, 500], [2, 1], 8, 2, 64, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_diff(nk, sel, shape, dtype):
    ctx, n_new, heads, hk, dim, block = SHAPES[shape]
    _say("diff", shape, dtype, ctx, n_new, heads, hk, dim, block)
    c, table, q = case(nk, sel, 600 + shape, ctx, n_new, heads, hk, dim, block, dtype)
    lam, norm = weights(shape, heads, dim)
    seqs, qd, cache = sequences(nk, n_new, ctx, table), q.cuda(), upload(nk, sel, c)
    o = run(cache, seqs, qd, lam)
    _say(check(c, table, ctx, n_new, q, o, lam))
    o = run(cache, seqs, qd, lam, norm, gain=0.4)
    _say(check(c, table, ctx, n_new, q, o, lam, norm, gain=0.4))
    assert torch.equal(run(cache, seqs, qd, lam, norm, gain=0.4), o)
    sel.sync_errors()


@pytest.mark.parametrize("dim,block", [(64, 16), (128, 16), (64, 64), (128, 512)])
def test_forms_agree_at_their_border(nk, sel, dim, block):
    """One row more takes the form for prompts."""
    rows = 192 if dim == 64 else 48
    for n in (rows - 1, rows, rows + 1):
        ctx, n_new = [n + 300], [n]
        c, table, q = case(nk, sel, 620, ctx, n_new, 2, 2, dim, block, "bf16")
        lam, norm = weights(20, 2, dim)
        _say(n, check(c, table, ctx, n_new, q, run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm), lam, norm))
    sel.sync_errors()


def test_one_map_is_plain_attention(nk, sel):
    """lambda 0 leaves the first map: its first half is attend's."""
    ctx, n_new = [300, 90], [2, 90]
    c, table, q = case(nk, sel, 621, ctx, n_new, 2, 2, 128, 32, "bf16")
    cache, seqs, qd = upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda()
    o = run(cache, seqs, qd, np.zeros(1, np.float32))
    a = cache.attend(seqs, qd)
    # both within 2^-10 and their bf16 rounding of the exact mean of |v| <= 448 * 2^-6
    assert ((o[:, 0, :128].float() - a[:, 0].float()).abs() <= 2.0 ** -7 * a[:, 0].float().abs() + 2.0 ** -9 * 7).all()


def test_many_sequences(nk, sel):
    """More sequences than a wavefront finds by itself, some with no rows or no tokens."""
    rng = np.random.default_rng(5)
    n_new = [int(x) for x in rng.integers(0, 3, 1500)]
    ctx = [int(x) for x in rng.integers(0, 40, 1500)]
    c, table, q = case(nk, sel, 622, ctx, n_new, 4, 2, 64, 16, "bf16")
    lam, norm = weights(22, 4, 64)
    o = run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm)
    sel.sync_errors()
    _say(check(c, table, ctx, n_new, q, o, lam, norm))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_new", [[3, 5, 1], [130, 66, 1]])
def test_rows_that_see_nothing(nk, sel, n_new, dim):
    """More rows than tokens: the first rows are zero, with a norm too."""
    ctx = [2, 0, 1]
    c, table, q = case(nk, sel, 623, ctx, n_new, 4, 2, dim, 16, "bf16")
    lam, norm = weights(23, 4, dim)
    for nm in (None, norm):
        o = run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, nm)
        sel.sync_errors()
        check(c, table, ctx, n_new, q, o, lam, nm)
        assert not o[:n_new[0] - 2].any() and not o[n_new[0]:n_new[0] + n_new[1]].any()


@pytest.mark.parametrize("block", [16, 64, 512])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_new", [4, 130])
def test_nan_in_what_a_row_does_not_see(nk, sel, n_new, dim, block):
    """A NaN key or value reaches the rows that see its token and no others;
    slots past the last token hold NaN throughout."""
    ctx = [200]
    c, table, q = case(nk, sel, 624, ctx, [n_new], 8, 4, dim, block, "bf16")
    lam, _ = weights(24, 8, dim)
    tok = 200 - n_new // 2
    c.v[table[0, tok // block], 1, tok % block, 5] = 0xFF          # second half of the first pair
    kt = 200 - n_new // 4
    c.k[table[0, kt // block], 2, kt % block, 9] = 0x7F            # first map of the second pair
    o = run(upload(nk, sel, c), sequences(nk, [n_new], ctx, table), q.cuda(), lam)
    sel.sync_errors()
    check(c, table, ctx, [n_new], q, o, lam)
    nan = torch.isnan(o.float())
    first = tok - (200 - n_new)                                    # the row whose own token it is
    assert not nan[:first, :2].any() and nan[first:, :2, dim + 5].all() and nan[:, :2].sum() == (n_new - first) * 2
    first = kt - (200 - n_new)
    assert not nan[:first, 2:].any() and nan[first:, 2:].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,n_new", [(64, 1), (64, 130), (128, 1), (128, 80)])
def test_large_scores_and_unequal_scales(nk, sel, dim, n_new, dtype):
    """Scores of hundreds; value scales far apart, between pages and between a
    pair's heads, by powers of two and not."""
    for kind in range(3):
        ctx = [400, 130]
        c, table, q = case(nk, sel, 625, ctx, [n_new, 1], 4, 2, dim, 16, dtype, qstd=60.0)
        far = 28 if kind == 0 else 5
        c.vs = c.vs * 2.0 ** c.rng.integers(-far, far, c.vs.shape)
        if kind == 2:
            c.vs = (c.vs * c.rng.uniform(0.5, 1.0, c.vs.shape)).astype(np.float32).astype(np.float64)
        if dtype == "fp16":
            c.vs = np.clip(c.vs, 2.0 ** -12, 2.0 ** 5)
        lam, norm = weights(25, 4, dim)
        cache, seqs, qd = upload(nk, sel, c), sequences(nk, [n_new, 1], ctx, table), q.cuda()
        _say(kind, check(c, table, ctx, [n_new, 1], q, run(cache, seqs, qd, lam), lam))
        _say(kind, check(c, table, ctx, [n_new, 1], q, run(cache, seqs, qd, lam, norm), lam, norm))
    sel.sync_errors()


@pytest.mark.parametrize("dim,n_new", [(64, 2), (64, 130), (128, 2), (128, 80)])
@pytest.mark.parametrize("e", [-126, -60, 100, 110])
def test_smallest_and_largest_scales(nk, sel, dim, n_new, e):
    """Rows near the ends of fp32: the norm neither overflows nor vanishes.
    (Without it what bf16 holds of the smallest is flushed or not, at 2^-133.)"""
    ctx = [150]
    c, table, q = case(nk, sel, 626, ctx, [n_new], 4, 2, dim, 16, "bf16")
    c.vs = np.full(c.vs.shape, 2.0 ** e)
    lam, norm = weights(26, 4, dim)
    cache, seqs = upload(nk, sel, c), sequences(nk, [n_new], ctx, table)
    for eps in (1e-5, 1e-30):
        check(c, table, ctx, [n_new], q, run(cache, seqs, q.cuda(), lam, norm, eps=eps), lam, norm, eps=float(np.float32(eps)))
    check(c, table, ctx, [n_new], q, run(cache, seqs, q.cuda(), lam), lam)


@pytest.mark.parametrize("n_new", [2, 130])
def test_scales_of_zero(nk, sel, n_new):
    """Values whose scales are all 0 are 0; of one of the heads, its half is."""
    ctx = [150]
    c, table, q = case(nk, sel, 627, ctx, [n_new], 4, 2, 64, 16, "bf16")
    lam, norm = weights(27, 4, 64)
    c.v[c.v == 0x7F] = 0
    vs = c.vs.copy()
    c.vs = np.zeros_like(vs)
    assert not run(upload(nk, sel, c), sequences(nk, [n_new], ctx, table), q.cuda(), lam, norm).any()
    c.vs = vs.copy()
    c.vs[:, 1] = 0
    o = run(upload(nk, sel, c), sequences(nk, [n_new], ctx, table), q.cuda(), lam)
    assert not o[..., 64:].any() and o[..., :64].any(-1).all()
    check(c, table, ctx, [n_new], q, o, lam)


@pytest.mark.parametrize("n_new", [1, 130])
def test_maps_that_cancel(nk, sel, n_new):
    """Equal maps and lambda 1: nothing is left but rounding, and the norm's eps
    keeps it small; lambda below 0 adds them."""
    ctx = [200]
    c, table, q = case(nk, sel, 628, ctx, [n_new], 4, 2, 64, 16, "bf16")
    c.k[:, 1] = c.k[:, 0]
    c.ks[:, 1] = c.ks[:, 0]
    q[:, 1::2] = q[:, ::2]
    cache, seqs = upload(nk, sel, c), sequences(nk, [n_new], ctx, table)
    one = np.ones(2, np.float32)
    assert not run(cache, seqs, q.cuda(), one).any()
    check(c, table, ctx, [n_new], q, run(cache, seqs, q.cuda(), -one), -one)
    lam, norm = weights(28, 4, 64)
    check(c, table, ctx, [n_new], q, run(cache, seqs, q.cuda(), one, norm, eps=1e-3), one, norm, eps=float(np.float32(1e-3)))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scale(nk, sel, scale):
    ctx, n_new = [77, 300], [1, 2]
    c, table, q = case(nk, sel, 629, ctx, n_new, 8, 4, 64, 16, "fp16", qstd=0.7)
    lam, norm = weights(29, 8, 64)
    check(c, table, ctx, n_new, q, run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm, scale=scale), lam,
          norm, scale)


def test_queries_and_weights_that_are_not_finite(nk, sel):
    """They make their own row and pair NaN, no other."""
    ctx, n_new = [90, 200], [2, 1]
    c, table, q = case(nk, sel, 630, ctx, n_new, 8, 2, 128, 32, "bf16")
    lam, _ = weights(30, 8, 128)
    q[1, 3, 7] = float("nan")
    q[2, 6, 0] = float("inf")
    lam[0] = float("nan")
    bad = torch.isnan(run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam)).any(2).cpu()
    assert bad[1, 1] and bad[2, 3] and bad[:, 0].all() and bad.sum() == 5


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_new", [[1, 2, 1], [130, 3, 1]])
def test_strides_in_place_and_rows_behind_the_last(nk, sel, n_new, dim):
    """Queries and outputs inside wider rows, rows past the last sequence and
    the rest of the wide rows as they were; host bounds larger than needed."""
    ctx = [230, 20, 700]
    c, table, q = case(nk, sel, 631, ctx, n_new, 8, 2, dim, 64, "bf16")
    lam, norm = weights(31, 8, dim)
    n = sum(n_new)
    wide = torch.full((n + 5, 20, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:n, 4:12] = q.cuda()
    out = torch.full((n + 5, 6, 2 * dim), -3.0, dtype=torch.bfloat16, device="cuda")
    table = np.concatenate([table, np.full((3, 4), 1 << 30)], 1)      # never read
    seqs, cache = sequences(nk, n_new, ctx, table, n_tok=n + 5, max_tok=max(n_new) + 3), upload(nk, sel, c)
    run(cache, seqs, wide[:, 4:12], lam, norm, out=out[:, 1:5])
    check(c, table, ctx, n_new, q, out[:, 1:5], lam, norm)
    assert (out[n:] == -3).all() and (out[:, :1] == -3).all() and (out[:, 5:] == -3).all()
    place = wide.view(n + 5, 10, 2 * dim)[:, 2:6]
    run(cache, seqs, wide[:, 4:12], lam, norm, out=place)
    assert torch.equal(place[:n], out[:n, 1:5]) and (wide[n:] == 7).all() and (wide[:, :4] == 7).all() and (wide[:, 12:] == 7).all()
    sel.sync_errors()


@pytest.mark.parametrize("dim", [64, 128])
def test_in_place_where_rows_are_split(nk, sel, dim):
    ctx, n_new = [9000, 300], [5, 1]
    c, table, q = case(nk, sel, 632, ctx, n_new, 8, 2, dim, 64, "bf16")
    lam, norm = weights(32, 8, dim)
    cache, seqs, qd = upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda()
    want = run(cache, seqs, qd, lam, norm)
    run(cache, seqs, qd, lam, norm, out=qd.view(qd.shape[0], -1, 2 * dim))
    assert torch.equal(qd.view_as(want), want)


@pytest.mark.parametrize("dim", [64, 128])
def test_long_sequence_is_split(nk, sel, dim):
    """One sequence over all of the card, beside short ones; fp32 joins."""
    ctx, n_new = [40000, 3, 900], [1, 1, 2]
    c, table, q = case(nk, sel, 633, ctx, n_new, 16, 2, dim, 512, "fp16")
    lam, norm = weights(33, 16, dim)
    o = run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm)
    sel.sync_errors()
    _say(check(c, table, ctx, n_new, q, o, lam, norm))


@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_tile_is_split(nk, sel, dim):
    """Few rows of a prompt after a long context, with empty ranges for the
    first rows' tiles."""
    ctx, n_new = [9000, 600], [70, 600]
    c, table, q = case(nk, sel, 634, ctx, n_new, 4, 2, dim, 64, "bf16")
    lam, norm = weights(34, 4, dim)
    o = run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm)
    sel.sync_errors()
    _say(check(c, table, ctx, n_new, q, o, lam, norm))


@pytest.mark.parametrize("dim,n_new,ctx,block,dtype", [(64, 1, 30000, 512, "bf16"), (128, 40, 8000, 16, "fp16")])
def test_dominant_token(nk, sel, dim, n_new, ctx, block, dtype):
    """Many equal tokens behind one that takes most of a row."""
    c, table, q = case(nk, sel, 635, [ctx], [n_new], 2, 2, dim, block, dtype, qstd=0.0)
    c.k[:] = 0
    q[..., 0] = 1.0
    c.k[table[0, 0], :, 0, 0] = 0x78                       # 256
    c.ks[:] = 2.0 ** -3
    lam, _ = weights(35, 2, dim)
    cache, seqs = upload(nk, sel, c), sequences(nk, [n_new], [ctx], table)
    for scale in (0.2, 0.3, 0.5):
        _say(scale, check(c, table, [ctx], [n_new], q, run(cache, seqs, q.cuda(), lam, scale=scale), lam, scale=scale))


@pytest.mark.parametrize("dim,n_new", [(64, 1), (64, 130), (128, 1), (128, 80)])
def test_invalid_sequences(nk, sel, dim, n_new):
    """Bad pages, lengths and offsets: reported, that sequence NaN, the others
    as without it; the next check is clean."""
    ctx, new = [200, 300, 400], [n_new] * 3
    c, table, q = case(nk, sel, 636, ctx, new, 4, 2, dim, 16, "bf16")
    lam, norm = weights(36, 4, dim)
    cache, qd = upload(nk, sel, c), q.cuda()
    go = lambda s, **kw: run(cache, s, qd, lam, norm, **kw)
    good = go(sequences(nk, new, ctx, table))
    sel.sync_errors()
    lo, hi = n_new, 2 * n_new
    bad = table.copy()
    bad[1, 3] = c.shape[0]                                 # one past the cache
    long = [200, table.shape[1] * 16 + 1, 400]             # more tokens than the table holds
    for s in (sequences(nk, new, ctx, bad), sequences(nk, new, long, table)):
        o = go(s)
        with pytest.raises(nk.NetKVError, match="block cache"):
            sel.sync_errors()
        sel.sync_errors()
        assert torch.isnan(o[lo:hi]).all()
        # how a sequence is split may depend on the others: within what its sums may be off
        check(c, table[:1], ctx[:1], new[:1], q[:lo], o[:lo], lam, norm)
        check(c, table[2:], ctx[2:], new[2:], q[hi:], o[hi:], lam, norm)
    out = torch.full((3 * n_new, 2, 2 * dim), 5.0, dtype=torch.bfloat16, device="cuda")
    go(sequences(nk, new, ctx, table, off=[0, 2 * n_new, n_new, 3 * n_new + 1], max_tok=2 * n_new + 1), out=out)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    assert torch.equal(go(sequences(nk, new, ctx, table, max_tok=n_new)), good)
    sel.sync_errors()


@pytest.mark.parametrize("n_seq", [7, 700])
def test_rows_of_two_sequences(nk, sel, n_seq):
    """Rows that an earlier sequence names are that one's; the later ones do not count."""
    off = [0, 20] * ((n_seq + 1) // 2) + [21]
    off = off[:n_seq] + [21]
    rng = np.random.default_rng(3)
    table, pages = R.tables(rng, [512] * n_seq, 512)
    table = table % 4
    c = R.Cache(4, 4, 64, 512, rng)
    for i in range(4):
        c.put(i, 512)
    q = torch.from_numpy(rng.standard_normal((21, 8, 64)) * 2).to(torch.bfloat16)
    lam, norm = weights(37, 8, 64)
    cache = upload(nk, sel, c)
    s = sequences(nk, None, [512] * n_seq, table, n_tok=21, max_tok=20, off=off)
    o = run(cache, s, q.cuda(), lam, norm)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    alone = run(cache, sequences(nk, [20], [512], table[:1]), q.cuda()[:20], lam, norm)
    assert ((o[:20].float() - alone.float()).abs() <= 2.0 ** -6 * alone.float().abs() + 2.0 ** -7).all()
    check(c, table[:1], [512], [20], q[:20], o, lam, norm)


def test_on_another_stream(nk, sel):
    ctx, n_new = [300, 50], [1, 1]
    c, table, q = case(nk, sel, 638, ctx, n_new, 8, 2, 128, 16, "bf16")
    lam, norm = weights(38, 8, 128)
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    lam, norm, qs = dev(lam, np.float32), dev(norm, np.float32), q.cuda()
    want = cache.attend_diff(seqs, qs, lam, norm=norm)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        qd = torch.zeros_like(qs)
        torch.cuda._sleep(2000000)
        qd.copy_(qs)
        got = cache.attend_diff(seqs, qd, lam, norm=norm)
    s.synchronize()
    assert torch.equal(want, got)


@pytest.mark.parametrize("dim", [64, 128])
def test_captured(nk, sel, dim):
    """Two graphs, each with its own workspace, replayed several times at once
    between eager calls, lengths changed in place."""
    ctx, n_new = [300, 50, 5000], [1, 1, 1]
    c, table, q = case(nk, sel, 639, ctx, n_new, 8, 2, dim, 16, "bf16")
    lam, norm = (dev(x, np.float32) for x in weights(39, 8, dim))
    cache, qd = upload(nk, sel, c), q.cuda()
    lens = [dev(ctx, np.int32).view(torch.uint32) for _ in range(2)]
    off, tb = dev([0, 1, 2, 3], np.int64).view(torch.uint64), dev(table, np.int32).view(torch.uint32)
    plans = [nk.Sequences(off, x, tb, 3, 1) for x in lens]
    cache.attend_diff(plans[0], qd, lam, norm=norm)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for p in plans:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cache.attend_diff(p, qd, lam, norm=norm))
        graphs.append(g)
    side = torch.cuda.Stream()
    for step in range(3):
        for x, v in zip(lens, ([300 - step, 50, 5000], [17, 50 - step, 999])):
            x.view(torch.int32).copy_(dev(v, np.int32))
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for p, o in zip(plans, outs):
            assert torch.equal(cache.attend_diff(p, qd, lam, norm=norm), o)
        torch.cuda.synchronize()


def test_prompt_captured(nk, sel):
    ctx, n_new = [700, 150], [300, 150]
    c, table, q = case(nk, sel, 640, ctx, n_new, 4, 2, 64, 32, "fp16")
    lam, norm = (dev(x, np.float32) for x in weights(40, 4, 64))
    cache, qd, seqs = upload(nk, sel, c), q.cuda(), sequences(nk, n_new, ctx, table)
    cache.attend_diff(seqs, qd, lam, norm=norm)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = cache.attend_diff(seqs, qd, lam, norm=norm)
    for step in range(3):
        qd.mul_(-0.9)
        torch.cuda.synchronize()
        o.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(cache.attend_diff(seqs, qd, lam, norm=norm), o)
    sel.sync_errors()


def test_a_step_of_a_layer(nk, sel):
    """Append with rotation, then differential attention, as a prompt, as
    single tokens and as a few at a time, in place."""
    ctx, rng = [0, 0], np.random.default_rng(90)
    table, pages = R.tables(rng, [190, 150], 16)
    c = R.Cache(pages, 4, 64, 16, rng)
    cache = upload(nk, sel, c)
    tab = T.table(190, 64, rng)
    rope = nk.Rope(sel, dev(tab, np.float32))
    lam, norm = weights(41, 8, 64)
    for n_new in ([170, 133], [1, 1], [3, 1], [1, 2]):
        ctx = [a + b for a, b in zip(ctx, n_new)]
        x = torch.from_numpy(rng.standard_normal((sum(n_new), 16, 64)) * 2).to(torch.bfloat16)
        xd, seqs = x.cuda(), sequences(nk, n_new, ctx, table)
        q = cache.append(seqs, rope, xd[:, 8:12], xd[:, 12:], xd[:, :8])
        pos = np.concatenate([np.arange(t - n, t) for t, n in zip(ctx, n_new)])[None]
        f = x.double().numpy()
        ref_store(c, table, ctx, n_new, T.rotate(f[:, 8:12], tab, pos, [0] * 32, False), f[:, 12:])
        host = q.cpu()
        run(cache, seqs, q, lam, norm, gain=0.5, out=q.view(-1, 4, 128))
        check(c, table, ctx, n_new, host, q.view(-1, 4, 128), lam, norm, gain=0.5)
    sel.sync_errors()


def test_empty_and_refusals(nk, sel):
    c = R.Cache(3, 2, 64, 16, np.random.default_rng(0))
    cache = upload(nk, sel, c)
    lam = torch.ones(2, device="cuda")
    none = nk.Sequences(dev([0], np.int64).view(torch.uint64), dev([], np.int32).view(torch.uint32),
                        torch.zeros((0, 1), dtype=torch.int32, device="cuda").view(torch.uint32), 0, 0)
    q0 = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert cache.attend_diff(none, q0, lam).shape == (0, 2, 128)
    assert cache.attend_diff(sequences(nk, [0, 0], [5, 0], np.zeros((2, 1))), q0, lam).shape == (0, 2, 128)
    seqs = sequences(nk, [2], [2], np.zeros((1, 1)))
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    cache.attend_diff(seqs, q, lam)
    norm = torch.ones(129, device="cuda")
    for bad in (dict(scale=float("nan")), dict(gain=float("inf"))):
        with pytest.raises(nk.NetKVError, match="finite"):
            cache.attend_diff(seqs, q, lam, **bad)
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(nk.NetKVError, match="eps"):
            cache.attend_diff(seqs, q, lam, norm=norm[:128], eps=eps)
    cache.attend_diff(seqs, q, lam, eps=0.0)
    with pytest.raises(nk.NetKVError, match="norm"):
        cache.attend_diff(seqs, q, lam, norm=norm[1:])
    with pytest.raises(ValueError, match="norm"):
        cache.attend_diff(seqs, q, lam, norm=norm[:127])
    with pytest.raises(ValueError, match="lam"):
        cache.attend_diff(seqs, q, lam[:1])
    with pytest.raises(TypeError, match="lam"):
        cache.attend_diff(seqs, q, lam.half())
    with pytest.raises(ValueError, match="gradient"):
        cache.attend_diff(seqs, q, lam.clone().requires_grad_())
    with pytest.raises(ValueError, match="gradient"):
        cache.attend_diff(seqs, q.clone().requires_grad_(), lam)
    with pytest.raises(nk.NetKVError, match="multiple of n_kv_heads"):
        cache.attend_diff(seqs, q[:, :3], lam)
    with pytest.raises(nk.NetKVError, match="overlap"):
        buf = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
        cache.attend_diff(seqs, buf[:2], lam, out=buf[1:].view(2, 2, 128))
    with pytest.raises(TypeError, match="dtype"):
        cache.attend_diff(seqs, q, lam, out=torch.zeros((2, 2, 128), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        cache.attend_diff(seqs, q, lam, out=torch.zeros_like(q))
    odd = upload(nk, sel, R.Cache(3, 3, 64, 16, np.random.default_rng(0)))
    with pytest.raises(nk.NetKVError, match="even"):
        odd.attend_diff(seqs, torch.zeros((2, 6, 64), dtype=torch.bfloat16, device="cuda"), torch.ones(3, device="cuda"))
    wide = upload(nk, sel, R.Cache(3, 2, 256, 16, np.random.default_rng(0)))
    with pytest.raises(nk.NetKVError, match="head_dim"):
        wide.attend_diff(seqs, torch.zeros((2, 4, 256), dtype=torch.bfloat16, device="cuda"), lam)
    with pytest.raises(nk.NetKVError, match="work"):
        nk.netkv_kv_attend_diff(sel.h, cache.c, seqs, q, 1.0, lam, None, 0.0, 1.0, torch.zeros((2, 2, 128), dtype=q.dtype, device="cuda"),
                                torch.zeros(256, dtype=torch.uint8, device="cuda"), sel.device)
    sel.sync_errors()


@pytest.mark.parametrize("n_seq,n_tok,max_tok,max_pages,block,heads,hk,dim", [
    (256, 256, 1, 8192, 16, 64, 8, 128), (256, 1792, 7, 8192, 16, 64, 8, 128), (512, 15360, 30, 8192, 16, 64, 8, 64),
    (16, 131072, 16384, 256, 512, 64, 8, 128), (2, 2048, 1024, 64, 512, 64, 16, 64), (64, 64, 1, 2048, 512, 2048, 1024, 128),
    (64, 6400, 100, 2048, 512, 2048, 1024, 64)])
def test_workspace_is_bounded(nk, sel, n_seq, n_tok, max_tok, max_pages, block, heads, hk, dim):
    kv = nk.netkv_kv_t(n_pages=1, block_tokens=block, n_kv_heads=hk, head_dim=dim, k=256, v=256, k_scale=256, v_scale=256)
    seqs = sequences(nk, None, [1] * n_seq, np.zeros((n_seq, max_pages)), n_tok=n_tok, max_tok=max_tok, off=[0] * (n_seq + 1))
    tiles = n_tok * heads // hk // 16 + n_seq
    assert nk.netkv_kv_attend_diff_workspace(sel.h, kv, seqs, heads) <= 300e6 + 48 * tiles


@pytest.mark.parametrize("n_new", [1, 130])
def test_offsets_past_32_bits(nk, sel, n_new):
    """Pages beyond 4 GiB of the cache."""
    block, hk, dim = 512, 8, 64
    n_pages = (1 << 32) // (block * hk * dim) + 2
    cache = nk.BlockCache.empty(sel, n_pages, hk, dim, block)
    rng = np.random.default_rng(91)
    small = R.Cache(2, hk, dim, block, rng)
    for i in range(2):
        small.put(i, 512)
    up = upload(nk, sel, small)
    for a, b in ((cache.k, up.k), (cache.v, up.v), (cache.k_scale, up.k_scale), (cache.v_scale, up.v_scale)):
        a.view(n_pages, -1)[-2:] = b.view(2, -1)
    q = torch.from_numpy(rng.standard_normal((n_new, 16, dim)) * 2).to(torch.bfloat16).cuda()
    lam, norm = (dev(x, np.float32) for x in weights(42, 16, dim))
    far, near = sequences(nk, [n_new], [900], np.array([[n_pages - 2, n_pages - 1]])), sequences(nk, [n_new], [900], np.array([[0, 1]]))
    assert torch.equal(cache.attend_diff(far, q, lam, norm=norm), up.attend_diff(near, q, lam, norm=norm))
    sel.sync_errors()


@pytest.mark.parametrize("n_new", [1, 70])
def test_longest_sequence(nk, sel, n_new):
    """Just under 2^31 tokens of few pages over and over: positions that use all
    of 31 bits, equal keys, so every map is the mean of the values."""
    block = 1024
    n = (1 << 31) // block - 1
    if n_new > 1:
        n //= 64                                           # rows by the prompt's form take longer
    rng = np.random.default_rng(92)
    c = R.Cache(2, 2, 64, block, rng)
    for i in range(2):
        c.put(i, block)
    c.k[:] = 0
    table = torch.zeros((1, n), dtype=torch.int32, device="cuda")
    table[0, 1::2] = 1
    seqs = nk.Sequences(dev([0, n_new], np.int64).view(torch.uint64), dev([n * block], np.int32).view(torch.uint32),
                        table.view(torch.uint32), n_new, n_new)
    q = torch.ones((n_new, 4, 64), dtype=torch.bfloat16, device="cuda")
    lam = np.array([0.25, -1.0], np.float32)
    o = run(upload(nk, sel, c), seqs, q, lam).double().cpu().numpy()
    sel.sync_errors()
    pg = np.arange(n) % 2
    v = np.concatenate([sum((pg == i).mean() * (R.values(c.v[i, m]) * c.vs[i, m]).mean(0) for i in range(2)) for m in range(2)])
    size = np.concatenate([sum((pg == i).mean() * (np.abs(R.values(c.v[i, m])) * c.vs[i, m]).mean(0) for i in range(2)) for m in range(2)])
    # weights 2^-11, fp32 sums of up to 2^31 / 64 / 4 terms a lane: 2^-24 of their magnitude for each of 2^13 steps a range
    # and its joins in the worst case, sqrt of it as rounding goes
    lim = (2.0 ** -11 + 2.0 ** -24 * 2 ** 7) * size
    for j in range(2):
        want = (1 - lam[j]) * v
        assert (np.abs(o[:, j] - want) <= (1 + abs(lam[j])) * lim + np.abs(want) * 2.0 ** -8 + 1e-30).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_many_sequences_of_prompts(nk, sel, dim):
    """More sequences than a wavefront finds by itself, some long enough to be split."""
    rng = np.random.default_rng(6)
    n_new = [int(x) for x in rng.integers(0, 3, 400)]
    ctx = [int(x) for x in rng.integers(0, 40, 400)]
    n_new[7], ctx[7], n_new[300], ctx[300], ctx[399], n_new[399] = 200, 333, 70, 3001, 1500, 1
    c, table, q = case(nk, sel, 643, ctx, n_new, 4, 2, dim, 64, "bf16")
    lam, norm = weights(43, 4, dim)
    o = run(upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda(), lam, norm)
    sel.sync_errors()
    _say(check(c, table, ctx, n_new, q, o, lam, norm))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,n_seq,n_new", [(64, 70, 1), (128, 70, 3), (128, 250, 1), (64, 33, 9)])
def test_ragged_sequences_of_long_tables(nk, sel, dim, n_seq, n_new, dtype):
    """Ranges of all lengths, the longest first; tables wider than any sequence."""
    rng = np.random.default_rng(7)
    ctx = [int(x) for x in np.exp(rng.uniform(np.log(1), np.log(3000), n_seq))]
    ctx[0], ctx[5], ctx[n_seq - 1] = 3, 3000, 2999
    new = [n_new] * n_seq
    new[3], ctx[3], ctx[4] = 0, 50, 0
    c, table, q = case(nk, sel, 645, ctx, new, 4, 2, dim, 64, dtype)
    lam, norm = weights(45, 4, dim)
    wide = np.concatenate([table, np.full((n_seq, 2048 - table.shape[1]), 1 << 30)], 1)      # never read
    o = run(upload(nk, sel, c), sequences(nk, new, ctx, wide), q.cuda(), lam, norm)
    sel.sync_errors()
    _say(check(c, table, ctx, new, q, o, lam, norm))


@pytest.mark.parametrize("dim", [64, 128])
def test_two_calls_at_once(nk, sel, dim):
    """Calls on two streams, each with its workspace, over one cache."""
    ctx, n_new = [9000, 300, 2000], [1, 1, 1]
    c, table, q = case(nk, sel, 644, ctx, n_new, 8, 2, dim, 64, "bf16")
    lam, norm = (dev(x, np.float32) for x in weights(44, 8, dim))
    cache, seqs, qs = upload(nk, sel, c), sequences(nk, n_new, ctx, table), [q.cuda(), -q.cuda()]
    want = [cache.attend_diff(seqs, x, lam, norm=norm) for x in qs]
    torch.cuda.synchronize()
    got = []
    for x in qs:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append([cache.attend_diff(seqs, x, lam, norm=norm) for _ in range(5)])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w, x) for x in g)
    sel.sync_errors()
