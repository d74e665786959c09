"""Appended keys and rotations at both ends of fp32's range, against plain forms in
64 bits.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R
from tests import rope_ref as T
from tests.test_gpu_append import check_rotated, own_places
from tests.test_gpu_block_cache import HALF, dev, ref_store, same_cache, sequences, upload

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


# ------------------------------------------------------------------ appended keys

# ctx after, new, heads, dim, block, rot, interleaved: workgroups of 256 threads, of
# 512 (many rows a block), of 64 (small blocks, many of them)
SHAPES = [([1, 40], [1, 3], 2, 64, 16, 64, False), ([700, 33], [530, 33], 2, 64, 512, 32, True),
          ([300, 90], [290, 90], 1, 256, 128, 240, False), ([17, 40, 64] * 40, [2, 40, 33] * 40, 5, 64, 16, 48, True)]


def append_and_compare(nk, sel, shape, x, tab, scales=None):
    """Bytes and scales equal the definition's: a key past what the largest scale
    holds is as one that is not finite."""
    ctx, n_new, hk, dim, block, rot, inter = shape
    rng = np.random.default_rng(700)
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, hk, dim, block, rng)
    for s, (t, n) in enumerate(zip(ctx, n_new)):
        for i in range(-(-t // block)):
            c.put(table[s, i], max(0, min(block, t - n - i * block)))
    if scales is not None:
        c.ks[:] = scales
    cache, xd = upload(nk, sel, c), x.cuda()
    cache.append(sequences(nk, n_new, ctx, table), nk.Rope(sel, dev(tab, np.float32), interleaved=inter), xd[:, :hk], xd[:, hk:])
    sel.sync_errors()
    f = x.double().numpy()
    k = T.rotate(f[:, :hk], tab, own_places(ctx, n_new), [0] * (rot // 2), inter)
    k[np.abs(k) > 448 * 2.0 ** 127] = np.inf
    with np.errstate(all="ignore"):
        ref_store(c, table, ctx, n_new, k, f[:, hk:])
    same_cache(cache, c, table, ctx)
    return k


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("scale", [1.0, 1.25, 64.0, 160.0, 400.0, 2.0 ** 100])
def test_append_keys_past_the_largest_fp32(nk, sel, shape, scale):
    """Finite keys of 3.4e38 and more, beside ordinary ones and such that are not
    finite; with a scaled table up to and past 448 * 2^127."""
    ctx, n_new, hk, dim, block, rot, inter = SHAPES[shape]
    rng = np.random.default_rng(710 + shape)
    n = sum(n_new)
    tab = T.table(max(ctx) + 1, rot, rng, scale=scale)
    x = rng.standard_normal((n, 2 * hk, dim))
    far = rng.random((n, hk, dim)) < np.where(rng.random((n, hk, 1)) < 0.5, 0.3, 0.0)
    x[:, :hk][far] = (rng.choice([-1.0, 1.0], (n, hk, dim)) * rng.uniform(1e37, 3.35e38, (n, hk, dim)))[far]
    if n > 4:
        x[4, 0, 3], x[3, hk - 1, 1] = np.inf, np.nan
    k = append_and_compare(nk, sel, SHAPES[shape], torch.from_numpy(x).to(torch.bfloat16), tab)
    wide = np.abs(k[np.isfinite(k)]) > 3.4e38
    _say(shape, scale, "keys past fp32:", int(wide.sum()), "past the largest scale:", int(np.isinf(k).sum()))
    # what the case is for is there (2^100 takes every such key past the largest scale)
    assert n < 100 or ((wide.any() or scale == 2.0 ** 100) and (np.isinf(k).sum() > 100 or scale < 200))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("e", [-118, -122, -124, -126, -130, -136, -142, -152])
def test_append_keys_of_the_smallest_scales(nk, sel, shape, e, dtype):
    """Keys around 2^e, below which a block's scale stays 2^-126: among the
    format's own subnormal steps, 2^-135."""
    ctx, n_new, hk, dim, block, rot, inter = SHAPES[shape]
    rng = np.random.default_rng(720 + shape)
    n = sum(n_new)
    # what does not turn is not scaled by the table: bfloat16's own small values there, none in fp16
    tab = T.table(max(ctx) + 1, rot, rng, scale=2.0 ** -110)
    x = rng.standard_normal((n, 2 * hk, dim))
    x[:, :hk, :rot] *= 2.0 ** max(e + 110, -40 if dtype == "bf16" else -14)
    x[:, :hk, rot:] *= 2.0 ** e if dtype == "bf16" else 0.0
    if e + 110 < -14 and dtype == "fp16":
        tab = T.table(max(ctx) + 1, rot, rng, scale=2.0 ** (e + 14)).astype(np.float32)
    append_and_compare(nk, sel, SHAPES[shape], torch.from_numpy(x).to(HALF[dtype]), tab)


@pytest.mark.parametrize("e", [-126, -125, -124, -123, -122, -121, -118])
def test_append_keys_into_pages_of_small_scales(nk, sel, e):
    """Pages begun with a scale near the smallest keep it: keys of a few of its
    steps, next to the middle of two of them."""
    shape = ([700, 33, 90], [180, 20, 5], 2, 64, 512, 64, False)
    rng = np.random.default_rng(730)
    n = sum(shape[1])
    # a cos with a power of two and cos of steps and halves of them, sin a speck
    m = rng.integers(0, 12, (701, 32)) * 0.5
    cos = (m + rng.choice([-1.0, 0.0, 1.0], m.shape) * 2.0 ** -15) * 2.0 ** (e + 80 - 9)
    tab = np.concatenate([cos, rng.choice([-1.0, 0.0, 1.0], m.shape) * 2.0 ** (e + 80 - 9 - 30)], 1).astype(np.float32)
    x = np.full((n, 4, 64), 2.0 ** -80) * rng.choice([-1.0, 1.0], (n, 4, 64))
    append_and_compare(nk, sel, shape, torch.from_numpy(x).to(torch.bfloat16), tab, scales=2.0 ** e)


# ------------------------------------------------------------------ products past fp32

@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,scale", [("bf16", 1.25), ("bf16", 4.0), ("fp16", 2.0 ** 116), ("fp16", 2.0 ** 126)])
def test_rotate_products_past_fp32(nk, sel, dtype, scale, inter, transpose):
    """Finite elements whose products with a scaled table are past fp32's largest:
    the sum is infinite, or finite where they cancel, and never NaN."""
    rng = np.random.default_rng(740)
    n, big = 600, 3.3e38 if dtype == "bf16" else 65000.0
    # factors of 8 bits, so that elements equal to them cancel to 0
    tab = (torch.from_numpy(T.table(n, 64, rng)).to(torch.bfloat16).double().numpy() * scale).astype(np.float32)
    x = rng.standard_normal((n, 5, 64))
    x[:, 0] = big * rng.choice([-1.0, 1.0], (n, 64))
    x[:, 1] *= np.where(rng.random((n, 64)) < 0.2, big / 5, 1.0)
    first, second = (slice(0, 64, 2), slice(1, 64, 2)) if inter else (slice(0, 32), slice(32, 64))
    c, s = tab[:, :32].astype(np.float64) / scale, tab[:, 32:].astype(np.float64) / scale
    x[:, 2, first], x[:, 2, second] = 0.9 * big * s, 0.9 * big * c          # a cos - b sin nearly cancels
    power = 2.0 ** 127 if dtype == "bf16" else 2.0 ** 15
    x[:, 3, first], x[:, 3, second] = power * c, -power * s                 # b cos + a sin cancels
    x[:, 4, first] = 1.0                                                    # b alone is large
    x[:, 4, second] = big
    x = torch.from_numpy(np.clip(x, -big, big)).to(HALF[dtype])
    rope = nk.Rope(sel, dev(tab, np.float32), interleaved=inter)
    pos = np.arange(n)[None]
    got = rope.rotate(x.cuda(), dev(pos, np.int32).view(torch.uint32), transpose=transpose)
    assert not torch.isnan(got).any()
    _say(check_rotated(got, x, tab, pos, [0] * 32, inter, transpose))
    wide = torch.isinf(got)
    assert wide.any() and not wide.all()
    sel.sync_errors()


@pytest.mark.parametrize("e", [-133, -130, -126, -124, -121, -116, 110, 126])
@pytest.mark.parametrize("n_new", [3, 530])
def test_store_at_both_ends_of_bfloat16(nk, sel, n_new, e):
    rng = np.random.default_rng(750)
    ctx, block = [700], 512
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, 2, 64, block, rng)
    c.ks[:] = c.vs[:] = 2.0 ** max(-126, e - 9)
    for i in range(2):
        c.put(table[0, i], max(0, min(block, ctx[0] - n_new - i * block)))
    x = torch.from_numpy(np.clip(rng.standard_normal((n_new, 4, 64)) * 2.0 ** e, -3.38e38, 3.38e38)).to(torch.bfloat16)
    cache, xd = upload(nk, sel, c), x.cuda()
    cache.store(sequences(nk, [n_new], ctx, table), xd[:, :2], xd[:, 2:])
    sel.sync_errors()
    f = x.double().numpy()
    ref_store(c, table, ctx, [n_new], f[:, :2], f[:, 2:])
    same_cache(cache, c, table, ctx)
