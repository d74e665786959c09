"""Rotary positions and the append with rotation against plain forms in 64
bits, through the C ABI.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R
from tests import rope_ref as T
from tests.test_gpu_block_cache import HALF, case, check_attend, dev, ref_store, same_cache, sequences, upload

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


def places(rng, n_axes, n, n_pos):
    return rng.integers(0, n_pos, (n_axes, n))


def u32(x):
    return dev(x, np.uint32).view(torch.uint32) if np.asarray(x).dtype != np.uint32 else dev(np.asarray(x).view(np.int32), np.int32).view(torch.uint32)


def check_rotated(got, x, tab, pos, axis, inter, transpose=False):
    """Every element within what its rounding allows."""
    f = x.double().cpu().numpy()
    want = T.rotate(f, tab, pos, axis, inter, transpose)
    with np.errstate(all="ignore"):
        size = T.rotate(np.abs(f), np.abs(tab), pos, axis, inter, False)       # lower of the pair's sums of magnitudes: taken both ways
        size = np.maximum(np.abs(size), T.rotate(np.abs(f), np.abs(tab), pos, axis, inter, True))
    fi = torch.finfo(got.dtype)
    lim = T.limit(want, fi.eps, fi.smallest_normal * fi.eps, 2 * size)
    y = got.double().cpu().numpy()
    big = ~(np.abs(want) < fi.max)                                             # NaN, infinite, or past the type
    assert np.array_equal(np.isnan(y), np.isnan(want))
    ok = ~big & ~np.isinf(y)
    worst = float((np.abs(y - want)[ok] / lim[ok]).max()) if ok.any() else 0.0
    assert worst <= 1.0, f"{worst:.3f} of what it may be off"
    edge = fi.max * (1 + fi.eps / 4)                                           # half a step past the largest
    assert not np.isinf(y[np.abs(want) < edge * (1 - 2.0 ** -20)]).any()
    assert np.isinf(y[np.abs(want) > edge * (1 + 2.0 ** -20)]).all()
    return worst


ROTATES = [
    # rows, heads, dim, rot, axes, mixed, interleaved, transpose
    (1, 1, 64, 64, 1, False, False, False),
    (1, 64, 128, 128, 1, False, True, False),
    (7, 5, 80, 80, 2, False, False, False),
    (7, 5, 80, 80, 2, True, True, True),
    (33, 3, 72, 64, 3, True, False, False),
    (300, 24, 128, 64, 1, False, True, True),
    (300, 9, 128, 48, 4, False, False, True),
    (1029, 16, 96, 96, 3, False, False, False),
    (2050, 40, 256, 256, 4, True, False, False),
    (5, 2, 1024, 256, 1, False, False, False),
    (65, 1, 24, 16, 1, False, False, False),
    (65, 2, 16, 16, 4, True, True, False),
    (3, 4099, 16, 16, 1, False, False, False),
    (257, 6, 136, 112, 2, False, True, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(ROTATES)))
def test_rotate(nk, sel, shape, dtype):
    rows, heads, dim, rot, n_axes, mixed, inter, trans = ROTATES[shape]
    _say("rotate", shape, dtype)
    rng = np.random.default_rng(300 + shape)
    tab, axis = T.table(501, rot, rng), T.axes(rot, n_axes, mixed)
    pos = places(rng, n_axes, rows, 501)
    x = torch.from_numpy(rng.standard_normal((rows, heads, dim))).to(HALF[dtype])
    rope = nk.Rope(sel, dev(tab, np.float32), axis if n_axes > 1 else None, interleaved=inter)
    xd, pd = x.cuda(), dev(pos, np.int32).view(torch.uint32)
    got = rope.rotate(xd, pd, transpose=trans)
    _say(check_rotated(got, x, tab, pos, axis, inter, trans))
    assert torch.equal(got[..., rot:], xd[..., rot:])
    # inside wider rows, and in place; rows and elements beside them as they were
    wide = torch.full((rows + 3, heads + 2, dim), 7.0, dtype=x.dtype, device="cuda")
    wide[:rows, 1:-1] = xd
    part = wide[:rows, 1:-1]
    assert rope.rotate(part, pd, out=part, transpose=trans) is part
    assert torch.equal(part, got) and (wide[rows:] == 7).all() and (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all()
    sel.sync_errors()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rotate_where_products_cancel(nk, sel, dtype):
    """Pairs whose products nearly cancel keep what is left; elements of all
    magnitudes of the type."""
    rng = np.random.default_rng(40)
    tab = T.table(4096, 128, rng)
    n = 4096
    pos = np.arange(n)[None]
    x = rng.standard_normal((n, 2, 128))
    x[:, 0, :64], x[:, 0, 64:] = tab[:, 64:], tab[:, :64]      # a cos - b sin = 0 but for the elements' rounding
    x[:, 1] *= 2.0 ** rng.integers(-30 if dtype == "bf16" else -20, 12, (n, 128))
    x = torch.from_numpy(x).to(HALF[dtype])
    rope = nk.Rope(sel, dev(tab, np.float32))
    _say(check_rotated(rope.rotate(x.cuda(), dev(pos, np.int32).view(torch.uint32)), x, tab, pos, [0] * 64, False))


@pytest.mark.parametrize("inter", [False, True])
def test_rotate_values_that_are_not_finite(nk, sel, inter):
    """They reach their own pair alone; infinities stay infinite."""
    rng = np.random.default_rng(41)
    tab = T.table(50, 64, rng)
    x = torch.from_numpy(rng.standard_normal((9, 2, 64))).to(torch.bfloat16)
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 5] = float("inf"), float("-inf"), float("nan")
    x[4, 0, 6], x[4, 0, 7], x[4, 0, 38] = 3.3e38, 3.3e38, 3.3e38
    pos = rng.integers(1, 50, (1, 9))
    got = nk.Rope(sel, dev(tab, np.float32), interleaved=inter).rotate(x.cuda(), dev(pos, np.int32).view(torch.uint32))
    check_rotated(got, x, tab, pos, [0] * 32, inter)
    bad = ~torch.isfinite(got)
    assert bad.sum() <= 10 and bad[1, 0].sum() == 2 and bad[2, 1].sum() == 2 and bad[3, 0].sum() == 2


def test_rotate_positions_past_the_table(nk, sel):
    """Reported, their axis's pairs NaN, all else as without them."""
    rng = np.random.default_rng(42)
    tab, axis = T.table(20, 64, rng), T.axes(64, 2, True)
    x = torch.from_numpy(rng.standard_normal((6, 3, 96))).to(torch.float16)
    pos = rng.integers(0, 20, (2, 6)).astype(np.uint32)
    rope = nk.Rope(sel, dev(tab, np.float32), axis)
    good = rope.rotate(x.cuda(), u32(pos))
    sel.sync_errors()
    pos[1, 2], pos[0, 4] = 20, 0xFFFFFFFF
    got = rope.rotate(x.cuda(), u32(pos))
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    sel.sync_errors()
    check_rotated(got, x, tab, pos, axis, False)
    nan = torch.isnan(got)
    assert nan.sum() == 2 * 3 * 32 and torch.equal(got[~nan], good[~nan])


def test_rotate_gradient(nk, sel):
    """The transposed rotation of g is the gradient of sum(rotate(x) g): by the
    formula, and by differences that 16 bits hold exactly."""
    rng = np.random.default_rng(43)
    tab, axis = T.table(64, 96, rng, scale=1.25), T.axes(96, 3, True)
    pos = rng.integers(0, 64, (3, 40))
    g = torch.from_numpy(rng.standard_normal((40, 4, 128))).to(torch.float16)
    rope, pd = nk.Rope(sel, dev(tab, np.float32), axis), dev(pos, np.int32).view(torch.uint32)
    d = rope.rotate(g.cuda(), pd, transpose=True)
    check_rotated(d, g, tab, pos, axis, False, True)
    # a rotation is linear: its difference along one element is its image
    for e in (0, 20, 47, 48, 95, 96, 127):
        x = torch.zeros((40, 4, 128), dtype=torch.float16, device="cuda")
        x[:, :, e] = 1.0
        y = rope.rotate(x, pd).double()
        want = (y * g.cuda().double()).sum(-1)
        # y is rounded (2^-11 of each of at most two elements), and d
        lim = 2.0 ** -11 * 1.01 * ((y * g.cuda().double()).abs().sum(-1) + want.abs()) + 2.0 ** -24
        assert ((d[:, :, e].double() - want).abs() <= lim).all()


def test_rotate_empty_and_refusals(nk, sel):
    rng = np.random.default_rng(44)
    rope = nk.Rope(sel, dev(T.table(20, 64, rng), np.float32))
    none = torch.zeros((0, 3, 64), dtype=torch.bfloat16, device="cuda")
    p0 = torch.zeros((1, 0), dtype=torch.int32, device="cuda").view(torch.uint32)
    assert rope.rotate(none, p0).shape == none.shape
    x = torch.zeros((4, 3, 64), dtype=torch.bfloat16, device="cuda")
    p = torch.zeros(4, dtype=torch.int32, device="cuda").view(torch.uint32)
    rope.rotate(x, p)
    with pytest.raises(ValueError, match="pos"):
        rope.rotate(x, p[:3])
    with pytest.raises(TypeError, match="pos"):
        rope.rotate(x, p.view(torch.int32))
    with pytest.raises(TypeError):
        rope.rotate(x.float(), p)
    with pytest.raises(ValueError, match="gradient"):
        rope.rotate(x.clone().requires_grad_(), p)
    with pytest.raises(ValueError, match="dense"):
        rope.rotate(x.transpose(0, 1), p)
    with pytest.raises(TypeError, match="dtype"):
        rope.rotate(x, p, out=x.half())
    with pytest.raises(nk.NetKVError, match="overlap"):
        buf = torch.zeros((5, 3, 64), dtype=torch.bfloat16, device="cuda")
        rope.rotate(buf[:4], p, out=buf[1:])
    with pytest.raises(nk.NetKVError, match="rot_dim"):
        rope.rotate(torch.zeros((4, 3, 48), dtype=torch.bfloat16, device="cuda"), p)
    with pytest.raises(ValueError, match="table"):
        nk.Rope(sel, torch.zeros(64, device="cuda"))
    with pytest.raises(ValueError, match="axis"):
        nk.Rope(sel, torch.zeros((4, 64), device="cuda"), [0] * 31)
    with pytest.raises(ValueError, match="axis"):
        nk.Rope(sel, torch.zeros((4, 64), device="cuda"), [4] * 32)
    with pytest.raises(nk.NetKVError, match="head_dim"):
        rope.rotate(torch.zeros((4, 1, 1032), dtype=torch.bfloat16, device="cuda"), p)
    two = nk.Rope(sel, dev(T.table(20, 64, rng), np.float32), [0, 1] * 16)
    with pytest.raises(ValueError, match="pos"):
        two.rotate(x, p)
    sel.sync_errors()


# ------------------------------------------------------------------ append

APPENDS = [
    # ctx after, new, heads, kv heads, dim, block, rot, axes, mixed, interleaved
    ([1], [1], 1, 1, 64, 16, 64, 1, False, False),
    ([1, 16, 17, 40, 512, 700], [1, 1, 1, 1, 1, 1], 6, 3, 128, 16, 128, 1, False, False),
    ([513, 512, 70, 1], [1, 1, 1, 1], 64, 2, 128, 512, 128, 1, False, True),
    ([100, 64, 65, 31], [100, 3, 65, 30], 15, 5, 64, 32, 48, 3, True, False),
    ([700, 30, 1100], [650, 13, 1100], 4, 2, 128, 512, 64, 2, False, True),
    ([300, 1030], [299, 517], 2, 1, 256, 128, 256, 1, False, False),
    ([1030, 2050], [1030, 1027], 1, 1, 256, 1024, 96, 4, True, False),
    ([90, 5, 0, 33], [9, 0, 0, 2], 0, 2, 64, 64, 16, 1, False, False),
    ([1100, 700], [1095, 513], 9, 2, 64, 1024, 32, 2, True, True),
    ([600, 90], [590, 90], 0, 3, 256, 64, 240, 1, False, True),
    ([300] * 3, [290, 0, 17], 70, 1, 128, 256, 128, 3, False, False),
    ([9, 1], [2, 1], 512, 256, 64, 16, 64, 1, False, False),
    ([90, 33, 5, 70] * 4, [60, 1, 5, 37] * 4, 7, 64, 128, 32, 64, 1, False, True),      # a wavefront a block and head
    ([17, 40, 64] * 40, [2, 40, 33] * 40, 3, 5, 256, 16, 96, 3, True, False),
    ([100] * 250, [1] * 250, 9, 4, 64, 64, 64, 1, False, False),
]


def filled(shape):
    ctx, n_new, heads, hk, dim, block, rot, n_axes, mixed, inter = shape
    rng = np.random.default_rng(500 + dim + block + len(ctx))
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, hk, dim, block, rng)
    for s, (t, n) in enumerate(zip(ctx, n_new)):
        for i in range(-(-t // block)):
            c.put(table[s, i], max(0, min(block, t - n - i * block)))
    n = sum(n_new)
    x = rng.standard_normal((n, heads + 2 * hk, dim)) * np.exp(2 * rng.standard_normal((n, heads + 2 * hk, 1)))
    return rng, c, table, x


def own_places(ctx, n_new):
    return np.concatenate([np.arange(t - n, t) for t, n in zip(ctx, n_new)])[None]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(APPENDS)))
def test_append(nk, sel, shape, dtype):
    """Bytes and scales equal the definition's, queries are rotated; pages that
    no row touches as they were."""
    ctx, n_new, heads, hk, dim, block, rot, n_axes, mixed, inter = APPENDS[shape]
    _say("append", shape, dtype)
    rng, c, table, x = filled(APPENDS[shape])
    x = torch.from_numpy(x).to(HALF[dtype])
    n, pages = sum(n_new), c.shape[0]
    tab, axis = T.table(max(ctx) + 1, rot, rng), T.axes(rot, n_axes, mixed)
    pos = own_places(ctx, n_new) if n_axes == 1 else places(rng, n_axes, n, max(ctx) + 1)
    rope = nk.Rope(sel, dev(tab, np.float32), axis if n_axes > 1 else None, interleaved=inter)
    cache, seqs, xd = upload(nk, sel, c), sequences(nk, n_new, ctx, table), x.cuda()
    before = cache.k.clone()
    q, k, v = xd[:, :heads], xd[:, heads:heads + hk], xd[:, heads + hk:]
    pd = dev(pos, np.int32).view(torch.uint32) if n_axes > 1 or shape % 2 else None
    out = cache.append(seqs, rope, k, v, q if heads else None, pd)
    sel.sync_errors()
    if heads:
        _say(check_rotated(out, x[:, :heads], tab, pos, axis, inter))
    else:
        assert out is None
    f = x.double().numpy()
    ref_store(c, table, ctx, n_new, T.rotate(f[:, heads:heads + hk], tab, pos, axis, inter), f[:, heads + hk:])
    same_cache(cache, c, table, ctx)
    spare = np.setdiff1d(np.arange(pages), np.concatenate([table[s, :-(-t // block)] for s, t in enumerate(ctx)]))
    assert torch.equal(cache.k.view(pages, -1)[spare], before.view(pages, -1)[spare])


def test_append_equals_its_parts(nk, sel):
    """Queries as by the rotation alone; keys that do not turn (angle 0) as by the store."""
    shape = APPENDS[4]
    ctx, n_new, heads, hk, dim, block = shape[:6]
    rng, c, table, x = filled(shape)
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    still = np.concatenate([np.ones((1, 32)), np.zeros((1, 32))], 1).repeat(2000, 0).astype(np.float32)
    seqs, a, b = sequences(nk, n_new, ctx, table), upload(nk, sel, c), upload(nk, sel, c)
    a.store(seqs, x[:, heads:heads + hk], x[:, heads + hk:])
    q = b.append(seqs, nk.Rope(sel, dev(still, np.float32)), x[:, heads:heads + hk], x[:, heads + hk:], x[:, :heads])
    assert torch.equal(q, x[:, :heads])
    for s, t in enumerate(ctx):
        for i in range(-(-t // block)):
            assert torch.equal(a.k_scale.view(-1, hk)[table[s, i]], b.k_scale.view(-1, hk)[table[s, i]])
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.v_scale, b.v_scale)
    tab = T.table(2000, 64, rng)
    rope = nk.Rope(sel, dev(tab, np.float32))
    q = b.append(seqs, rope, x[:, heads:heads + hk], x[:, heads + hk:], x[:, :heads])
    assert torch.equal(q, rope.rotate(x[:, :heads], dev(own_places(ctx, n_new), np.int32).view(torch.uint32)))
    # in place, inside the product's rows: keys and values beside it are read as they were
    d = upload(nk, sel, c)
    d.append(seqs, rope, x[:, heads:heads + hk], x[:, heads + hk:], None)
    e = upload(nk, sel, c)
    y = x.clone()
    part = y[:, :heads]
    assert e.append(seqs, rope, y[:, heads:heads + hk], y[:, heads + hk:], part, out=part) is part
    assert torch.equal(part, q) and torch.equal(y[:, heads:], x[:, heads:])
    assert torch.equal(d.k, e.k) and torch.equal(d.v, e.v) and torch.equal(d.k_scale, e.k_scale)
    sel.sync_errors()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_append_keys_beside_a_border(nk, sel, dtype):
    """Keys whose rotation lands on and next to the middle of two 8-bit steps
    and next to the scale's borders, where a key rounded to 32 bits on the way
    would fall on the other side."""
    rng = np.random.default_rng(60)
    n, dim, block = 512, 64, 512
    # a cos with a in {1, ...} and cos next to a middle by one fp32 step, sin tiny
    mid = (R.values(np.arange(8, 120).astype(np.uint8)) + R.values(np.arange(9, 121).astype(np.uint8))) / 2
    m = rng.choice(mid, (n, 32))
    cos = np.where(rng.random((n, 32)) < 0.5, np.nextafter(m.astype(np.float32), np.float32(0)), m.astype(np.float32))
    sin = (rng.choice([-1.0, 0.0, 1.0], (n, 32)) * 2.0 ** rng.integers(-60, -28, (n, 32))).astype(np.float32)
    tab = np.concatenate([cos, sin], 1).astype(np.float32)
    x = np.ones((n, 3, dim))
    x[:, 1, 32:] = rng.choice([0.5, -1.0, 2.0], (n, 32))
    x[::7, 1, :] *= 448.0 / 240
    x = torch.from_numpy(x).to(HALF[dtype])
    ctx = [n]
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, 1, dim, block, rng)
    cache = upload(nk, sel, c)
    xd = x.cuda()
    cache.append(sequences(nk, [n], ctx, table), nk.Rope(sel, dev(tab, np.float32)), xd[:, 1:2], xd[:, 2:], xd[:, :1])
    f = x.double().numpy()
    ref_store(c, table, ctx, [n], T.rotate(f[:, 1:2], tab, np.arange(n)[None], [0] * 32, False), f[:, 2:])
    same_cache(cache, c, table, ctx)


def test_append_not_finite_and_past_the_table(nk, sel):
    """What is not finite is NaN in the cache and does not raise the scale;
    positions past the table are reported."""
    shape = ([70, 40], [40, 3], 4, 2, 64, 16, 32, 1, False, False)
    ctx, n_new, heads, hk, dim, block = shape[:6]
    rng, c, table, x = filled(shape)
    x = torch.from_numpy(x).to(torch.float16)
    x[3, heads, 5], x[9, heads + 1, 40], x[11, heads, 20], x[12, heads + hk, 7] = [float(v) for v in ("inf", "nan", "-inf", "inf")]
    tab = T.table(60, 32, rng)                             # places 60 .. 69 have no row
    cache, seqs, xd = upload(nk, sel, c), sequences(nk, n_new, ctx, table), x.cuda()
    q = cache.append(seqs, nk.Rope(sel, dev(tab, np.float32)), xd[:, heads:heads + hk], xd[:, heads + hk:], xd[:, :heads])
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    sel.sync_errors()
    pos = own_places(ctx, n_new)
    check_rotated(q, x[:, :heads], tab, pos, [0] * 16, False)
    assert torch.isnan(q[30:40, :, :32]).all() and not torch.isnan(q[:30]).any() and not torch.isnan(q[..., 32:]).any()
    f = x.double().numpy()
    with np.errstate(all="ignore"):
        ref_store(c, table, ctx, n_new, T.rotate(f[:, heads:heads + hk], tab, pos, [0] * 16, False), f[:, heads + hk:])
    same_cache(cache, c, table, ctx)


@pytest.mark.parametrize("n_new", [1, 40])
def test_append_invalid_sequences(nk, sel, n_new):
    """Bad pages, lengths and offsets: reported, what counts as without them,
    rows that do not and rows past the last sequence as they were."""
    ctx, new = [100, 200, 300], [n_new] * 3
    shape = (ctx, new, 4, 2, 64, 16, 64, 1, False, False)
    rng, c, table, x = filled(shape)
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    rope = nk.Rope(sel, dev(T.table(400, 64, rng), np.float32))
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    good = upload(nk, sel, c)
    want = good.append(sequences(nk, new, ctx, table), rope, k, v, q)
    sel.sync_errors()

    def run(**kw):
        d = dict(n_new=new, ctx=ctx, table=table)
        d.update(kw)
        cache = upload(nk, sel, c)
        out = torch.full((3 * n_new + 2, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        wide = torch.cat([x, x[:2]])
        n = 3 * n_new + (2 if d.pop("wide", False) else 0)
        cache.append(sequences(nk, d["n_new"], d["ctx"], d["table"], n_tok=n, max_tok=d.get("max_tok"), off=d.get("off")), rope,
                     wide[:, 4:6], wide[:, 6:], wide[:, :4], out=out)
        return cache, out

    lo, hi = n_new, 2 * n_new
    long = [100, table.shape[1] * 16 + 1, 300]             # more tokens than the table holds
    few = [100, n_new - 1, 300]                            # more rows than tokens
    for c2 in (long, few):
        cache, out = run(ctx=c2)
        with pytest.raises(nk.NetKVError, match="block cache"):
            sel.sync_errors()
        assert (out[lo:hi] == 5).all() and torch.equal(out[:lo], want[:lo]) and torch.equal(out[hi:3 * n_new], want[hi:])
        assert (out[3 * n_new:] == 5).all()
        pg = lambda y, s: y.view(c.shape[0], -1)[table[s, :-(-ctx[s] // 16)]]
        for s in (0, 2):
            assert torch.equal(pg(cache.k, s), pg(good.k, s)) and torch.equal(pg(cache.v, s), pg(good.v, s))
        same = upload(nk, sel, c)
        assert torch.equal(pg(cache.k, 1), pg(same.k, 1))
    bad = table.copy()
    bad[1, 199 // 16] = c.shape[0]                         # one past the cache
    cache, out = run(table=bad)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    assert torch.equal(out[:3 * n_new], want)
    cache, out = run(wide=True)                            # rows past the last sequence
    sel.sync_errors()
    assert torch.equal(out[:3 * n_new], want) and (out[3 * n_new:] == 5).all()
    # the second sequence begins among the first one's rows
    cache, out = run(off=[0, 2 * n_new, n_new, 3 * n_new], max_tok=2 * n_new)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()


def test_append_many_sequences(nk, sel):
    """More sequences than a workgroup looks at at a time, some with no rows or no tokens."""
    rng = np.random.default_rng(70)
    n_new = [int(v) for v in rng.integers(0, 3, 1500)]
    ctx = [int(max(a, v)) for a, v in zip(n_new, rng.integers(0, 40, 1500))]
    shape = (ctx, n_new, 4, 2, 64, 16, 64, 1, False, False)
    rng, c, table, x = filled(shape)
    x = torch.from_numpy(x).to(torch.bfloat16)
    tab = T.table(40, 64, rng)
    cache, xd = upload(nk, sel, c), x.cuda()
    q = cache.append(sequences(nk, n_new, ctx, table), nk.Rope(sel, dev(tab, np.float32)), xd[:, 4:6], xd[:, 6:], xd[:, :4])
    sel.sync_errors()
    pos = own_places(ctx, n_new)
    check_rotated(q, x[:, :4], tab, pos, [0] * 32, False)
    f = x.double().numpy()
    ref_store(c, table, ctx, n_new, T.rotate(f[:, 4:6], tab, pos, [0] * 32, False), f[:, 6:])
    same_cache(cache, c, table, ctx)


def test_append_captured_and_on_another_stream(nk, sel):
    """Tokens appended one after the other by a replayed graph, between eager
    attention and synchronizations, equal the same appended eagerly; and on a
    stream of its own after work that takes a while."""
    ctx0 = [30, 64, 5]
    shape = ([40, 70, 20], [1, 1, 1], 8, 2, 64, 16, 64, 1, False, True)
    rng, c, table, _ = filled(shape)
    rope = nk.Rope(sel, dev(T.table(100, 64, rng), np.float32), interleaved=True)
    steps = torch.from_numpy(rng.standard_normal((6, 3, 12, 64))).to(torch.bfloat16).cuda()
    outs = []
    off, tb = dev([0, 1, 2, 3], np.int64).view(torch.uint64), dev(table, np.int32).view(torch.uint32)
    for captured in (False, True):
        cache = upload(nk, sel, c)
        lens = dev(ctx0, np.int32).view(torch.uint32)
        seqs = nk.Sequences(off, lens, tb, 3, 1)
        x = steps[0].clone()
        q = torch.empty((3, 8, 64), dtype=torch.bfloat16, device="cuda")
        run = lambda: cache.append(seqs, rope, x[:, 8:10], x[:, 10:], x[:, :8], out=q)
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run()
        got = []
        for i in range(6):
            x.copy_(steps[i])
            lens.view(torch.int32).add_(1)
            torch.cuda.synchronize()
            g.replay() if captured else run()
            got.append(torch.cat([q.float().flatten(), cache.attend(seqs, q).float().flatten()]))
            torch.cuda.synchronize()
        outs.append((torch.stack(got), cache.k.clone(), cache.v.clone(), cache.k_scale.clone()))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    seqs = sequences(nk, [1, 1, 1], [31, 65, 6], table)
    a, b = upload(nk, sel, c), upload(nk, sel, c)
    want = a.append(seqs, rope, steps[1][:, 8:10], steps[1][:, 10:], steps[1][:, :8])
    with torch.cuda.stream(s):
        x = torch.zeros_like(steps[1])
        torch.cuda._sleep(2000000)
        x.copy_(steps[1])
        got = b.append(seqs, rope, x[:, 8:10], x[:, 10:], x[:, :8])
    s.synchronize()
    assert torch.equal(want, got) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    sel.sync_errors()


def test_append_then_attend(nk, sel):
    """A sequence appended as a prompt and then token by token is attended to as
    the definition's cache is."""
    ctx = [0, 0]
    rng = np.random.default_rng(80)
    table, pages = R.tables(rng, [90, 50], 16)
    c = R.Cache(pages, 2, 128, 16, rng)
    cache = upload(nk, sel, c)
    tab = T.table(90, 128, rng)
    rope = nk.Rope(sel, dev(tab, np.float32))
    for n_new in ([70, 33], [1, 1], [3, 1], [1, 2]):
        ctx = [a + b for a, b in zip(ctx, n_new)]
        x = torch.from_numpy(rng.standard_normal((sum(n_new), 12, 128))).to(torch.bfloat16)
        xd, seqs = x.cuda(), sequences(nk, n_new, ctx, table)
        q = cache.append(seqs, rope, xd[:, 8:10], xd[:, 10:], xd[:, :8])
        f = x.double().numpy()
        ref_store(c, table, ctx, n_new, T.rotate(f[:, 8:10], tab, own_places(ctx, n_new), [0] * 64, False), f[:, 10:])
        check_attend(c, table, ctx, n_new, q.cpu(), cache.attend(seqs, q))
    same_cache(cache, c, table, ctx)
    sel.sync_errors()


def test_append_empty_and_refusals(nk, sel):
    rng = np.random.default_rng(81)
    c = R.Cache(3, 2, 64, 16, rng)
    cache = upload(nk, sel, c)
    rope = nk.Rope(sel, dev(T.table(20, 64, rng), np.float32))
    kv = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    idle = sequences(nk, [0, 0], [5, 0], np.zeros((2, 1)))
    before = cache.k.clone()
    assert cache.append(idle, rope, kv, kv, torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")).shape == (0, 4, 64)
    seqs = sequences(nk, [2], [2], np.zeros((1, 1)))
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    with pytest.raises(nk.NetKVError, match="overlap q"):
        cache.append(seqs, rope, k, v, q, out=x[:, 1:5])
    with pytest.raises(nk.NetKVError, match="overlap k or v"):
        cache.append(seqs, rope, k, v, q.clone(), out=x[:, 1:5])
    with pytest.raises(nk.NetKVError, match="overlap k or v"):
        cache.append(seqs, rope, k, v, q.clone(), out=x[:, 4:])
    with pytest.raises(nk.NetKVError, match="rot_dim"):
        cache.append(seqs, nk.Rope(sel, torch.zeros((4, 80), device="cuda")), k, v, q)
    with pytest.raises(TypeError, match="dtype"):
        cache.append(seqs, rope, k, v, q.half())
    with pytest.raises(ValueError, match="gradient"):
        cache.append(seqs, rope, k.clone().requires_grad_(), v, q)
    with pytest.raises(ValueError, match="pos"):
        cache.append(seqs, rope, k, v, q, torch.zeros((1, 1), dtype=torch.int32, device="cuda").view(torch.uint32))
    with pytest.raises(ValueError):
        cache.append(seqs, rope, k[:, :1], v, q)
    assert torch.equal(before, cache.k)
    sel.sync_errors()


def test_append_offsets_past_32_bits(nk, sel):
    """Pages beyond 4 GiB of the cache, and table rows beyond 2^31 bytes."""
    block, hk, dim = 16, 8, 128
    n_pages = (1 << 32) // (block * hk * dim) + 3
    cache = nk.BlockCache.empty(sel, n_pages, hk, dim, block)
    rng = np.random.default_rng(82)
    rows = (1 << 31) // (dim * 4) + 5
    tab = torch.zeros((rows, dim), device="cuda")
    last = T.table(4, dim, rng)
    tab[-4:] = dev(last, np.float32)
    rope = nk.Rope(sel, tab)
    table = np.array([[n_pages - 1]])
    x = torch.from_numpy(rng.standard_normal((4, 3 * hk, dim))).to(torch.bfloat16)
    xd = x.cuda()
    seqs = sequences(nk, [4], [4], table)
    q = cache.append(seqs, rope, xd[:, hk:2 * hk], xd[:, 2 * hk:], xd[:, :hk], dev(np.arange(rows - 4, rows), np.int32).view(torch.uint32))
    sel.sync_errors()
    pos = np.arange(4)[None]
    check_rotated(q, x[:, :hk], last, pos, [0] * 64, False)
    k, v = cache.read(seqs)
    want = T.rotate(x[:, hk:2 * hk].double().numpy(), last, pos, [0] * 64, False)
    s = np.array([R.scale_for(np.abs(want[:, h]).max()) for h in range(hk)])
    assert np.array_equal(k.double().cpu().numpy(), R.values(R.nearest(want / s[:, None])) * s[:, None])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n_new", [1, 30, 500])
def test_pages_begun_with_any_scale(nk, sel, n_new, dtype):
    """A page that another program began with a larger scale which is no power of
    two keeps it: new keys and values are over that scale, by store and append."""
    rng = np.random.default_rng(83)
    ctx, block = [700], 512
    table, pages = R.tables(rng, ctx, block)
    for how in ("store", "append"):
        c = R.Cache(pages, 2, 64, block, rng)
        for i in range(2):
            c.put(table[0, i], max(0, min(block, ctx[0] - n_new - i * block)))
        c.ks, c.vs = ((x * 1.37).astype(np.float32).astype(np.float64) for x in (c.ks, c.vs))
        x = torch.from_numpy(rng.standard_normal((n_new, 4, 64)) * 0.2).to(HALF[dtype])
        cache, seqs, xd = upload(nk, sel, c), sequences(nk, [n_new], ctx, table), x.cuda()
        f = x.double().numpy()
        k = f[:, :2]
        if how == "append":
            tab = T.table(700, 64, rng)
            cache.append(seqs, nk.Rope(sel, dev(tab, np.float32)), xd[:, :2], xd[:, 2:])
            k = T.rotate(k, tab, own_places(ctx, [n_new]), [0] * 32, False)
        else:
            cache.store(seqs, xd[:, :2], xd[:, 2:])
        sel.sync_errors()
        ref_store(c, table, ctx, [n_new], k, f[:, 2:])
        got = R.Cache(pages, 2, 64, block, rng)
        got.from_device(cache.k.cpu().numpy(), cache.v.cpu().numpy())
        assert np.array_equal(cache.k_scale.cpu().numpy().reshape(pages, 2), c.ks.astype(np.float32))
        assert np.array_equal(cache.v_scale.cpu().numpy().reshape(pages, 2), c.vs.astype(np.float32))
        for a, b, s in ((got.k, c.k, c.ks), (got.v, c.v, c.vs)):
            for i in range(2):
                n = min(block, ctx[0] - i * block)
                pg = table[0, i]
                va, vb = R.values(a[pg, :, :n]), R.values(b[pg, :, :n])
                # x / s is computed as x (1 / s), 2^-23 off: next to the middle of two steps either is right
                step = np.maximum(np.abs(vb), 2.0 ** -6) * 2.0 ** -3
                assert (np.abs(va - vb) <= step).all() and (va != vb).mean() < 1e-3


def test_positions_wider_than_the_call(nk, sel):
    """Positions of more rows and axes than a call has, and an axis named where
    there is one, are the same positions."""
    rng = np.random.default_rng(93)
    shape = ([60, 9], [41, 9], 4, 2, 64, 32, 64, 2, False, False)
    rng, c, table, x = filled(shape)
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    tab = dev(T.table(100, 64, rng), np.float32)
    pos = places(rng, 2, 50, 100)
    wide = np.full((3, 77), 1 << 20)
    wide[:2, :50] = pos
    two = nk.Rope(sel, tab, T.axes(64, 2, False))
    a = two.rotate(x[:, :4], u32(pos.astype(np.uint32)))
    assert torch.equal(a, two.rotate(x[:, :4], u32(wide.astype(np.uint32))))
    seqs, caches = sequences(nk, shape[1], shape[0], table), [upload(nk, sel, c) for _ in range(2)]
    for cache, p in zip(caches, (pos, wide)):
        assert torch.equal(cache.append(seqs, two, x[:, 4:6], x[:, 6:], x[:, :4], u32(p.astype(np.uint32))), a)
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].k_scale, caches[1].k_scale)
    named, one = nk.Rope(sel, tab, [0] * 32), nk.Rope(sel, tab)
    assert torch.equal(named.rotate(x, u32(pos[0].astype(np.uint32))), one.rotate(x, u32(wide[:1].astype(np.uint32))))
    sel.sync_errors()


@pytest.mark.parametrize("n_seq,hk", [(7, 2), (701, 2), (200, 64)])
def test_append_rows_of_two_sequences(nk, sel, n_seq, hk):
    """Rows that an earlier sequence names are that one's: of all sequences that
    begin among them nothing is stored."""
    off = ([0, 20] * n_seq)[:n_seq - 1] + [20, 21]
    rng, c, table, x = filled(([20] * n_seq, [0] * n_seq, 4, hk, 64, 32, 64, 1, False, False))
    x = torch.from_numpy(rng.standard_normal((21, 4 + 2 * hk, 64))).to(torch.bfloat16)
    tab = T.table(20, 64, rng)
    cache, xd = upload(nk, sel, c), x.cuda()
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    out = torch.full((21, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    cache.append(sequences(nk, None, [20] * n_seq, table, n_tok=21, max_tok=20, off=off), nk.Rope(sel, dev(tab, np.float32)), xd[:, 4:4 + hk],
                 xd[:, 4 + hk:], xd[:, :4], out=out)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    pos = np.concatenate([np.arange(20), [19]])[None]
    check_rotated(out, x[:, :4], tab, pos, [0] * 32, False)
    f = x.double().numpy()
    keys = T.rotate(f[:, 4:4 + hk], tab, pos, [0] * 32, False)
    two = table[[0, n_seq - 1]]
    ref_store(c, two, [20, 20], [20, 1], keys, f[:, 4 + hk:])
    same_cache(cache, c, two, [20, 20])
    rest = np.setdiff1d(np.arange(c.shape[0]), two[:, 0])
    for t, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before):
        assert torch.equal(t.view(c.shape[0], -1)[rest], b.view(c.shape[0], -1)[rest])


def test_two_appends_at_once(nk, sel):
    """Two streams append to sequences of one cache, as one call does."""
    shape = ([700, 40, 900, 64], [690, 1, 900, 1], 8, 2, 128, 512, 128, 1, False, False)
    rng, c, table, x = filled(shape)
    ctx, n_new = shape[:2]
    x = torch.from_numpy(x).to(torch.bfloat16).cuda()
    rope = nk.Rope(sel, dev(T.table(1000, 128, rng), np.float32))
    a, b = upload(nk, sel, c), upload(nk, sel, c)
    want = a.append(sequences(nk, n_new, ctx, table), rope, x[:, 8:10], x[:, 10:], x[:, :8])
    parts = [(x[:691], sequences(nk, n_new[:2], ctx[:2], table[:2])), (x[691:], sequences(nk, n_new[2:], ctx[2:], table[2:]))]
    torch.cuda.synchronize()
    got = []
    for y, seqs in parts:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(b.append(seqs, rope, y[:, 8:10], y[:, 10:], y[:, :8]))
    torch.cuda.synchronize()
    assert torch.equal(torch.cat(got), want)
    for t, u in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        assert torch.equal(t, u)
    sel.sync_errors()
