"""The block cache's operators and the eviction at their limits and side by
side: caches past 4 GiB, the longest sequence, two streams, captured prompts,
many segments.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R
from tests.test_gpu_block_cache import HALF, case, check_attend, dev, sequences, upload
from tests.test_gpu_evict import draw, run

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


@pytest.mark.parametrize("n_new", [[1, 2, 1], [70, 66, 1]])
def test_offsets_past_32_bits(nk, sel, n_new):
    """The last pages of a cache of 4.6 GB: stored, attended, weighed and read
    as in a small one."""
    ctx, hk, dim, block = [300, 70, 1030], 4, 128, 512
    c, table, q = case(nk, sel, 31, ctx, n_new, 16, hk, dim, block, "bf16")
    small = upload(nk, sel, c)
    pages = c.shape[0]
    total = (4_600_000_000 // (hk * dim * block))
    big = nk.BlockCache.empty(sel, total, hk, dim, block)
    for a, b in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
        a.view(total, -1)[total - pages:].copy_(b.view(pages, -1))
    near, far = sequences(nk, n_new, ctx, table), sequences(nk, n_new, ctx, table + (total - pages))
    x = torch.randn((sum(n_new), 2 * hk, dim), dtype=torch.bfloat16, device="cuda")
    qd = q.cuda()
    got = []
    for cache, seqs in ((small, near), (big, far)):
        cache.store(seqs, x[:, :hk], x[:, hk:])
        o, w = cache.attend(seqs, qd, weights=True)
        acc = torch.zeros(cache.c.n_pages, dtype=torch.int64, device="cuda")
        cache.weigh(seqs, w, acc.view(torch.uint64))
        got.append((o, w, acc[-pages:], *cache.read(seqs)))
    sel.sync_errors()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.equal(big.k.view(total, -1)[total - pages:], small.k.view(pages, -1))
    assert torch.equal(big.v.view(total, -1)[total - pages:], small.v.view(pages, -1))


@pytest.mark.parametrize("n_new", [1, 33])
def test_longest_sequence(nk, sel, n_new):
    """2^31 - 1024 tokens, all of one page (a page may be in a sequence more
    than once): what one page gives, as every token counts 2^21 - 1 times.
    With 33 rows of 2 heads (a prompt), the first rows see 32 tokens less of
    2^31, which changes nothing that fp32 shows.

    Tolerance: a range of the 512 adds at most 2^31 / 64 / 512 = 2^16 steps one
    after the other, each rounded by 2^-24 of the sum: 2^-8 for the weights'
    sum and as much of the largest value for the values', 2^-11 for a weight's
    rounding, half a step for the output's."""
    block, dim = 1024, 64
    rng = np.random.default_rng(3)
    c = R.Cache(1, 1, dim, block, rng)
    c.put(0, block)
    q = torch.from_numpy(rng.standard_normal((n_new, 2, dim))).to(torch.float16)
    cache = upload(nk, sel, c)
    pages = (1 << 21) - 1
    seqs = sequences(nk, [n_new], [pages * block], np.zeros((1, pages)))
    o = cache.attend(seqs, q.cuda()).double().cpu().numpy()
    sel.sync_errors()
    k, v = c.held(np.zeros(1, np.int64), block, 0, "k"), c.held(np.zeros(1, np.int64), block, 0, "v")
    s = q.double().numpy() @ k.T * dim ** -0.5
    p = np.exp(s - s.max(-1, keepdims=True))
    want = p @ v / p.sum(-1, keepdims=True)
    worst = float(np.abs(o - want).max() / np.abs(v).max())
    _say("longest", n_new, worst)
    assert worst <= 2.0 ** -8 + 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -11
    with pytest.raises(nk.NetKVError, match="max_pages"):
        cache.attend(sequences(nk, [n_new], [1], np.zeros((1, pages + 1))), q.cuda())


def test_one_page_many_times(nk, sel):
    """Several blocks of a sequence in one page, other sequences in it too."""
    ctx, n_new = [500, 130, 64], [1, 70, 3]
    c, table, q = case(nk, sel, 33, ctx, n_new, 8, 2, 128, 64, "fp16")
    for page in range(c.shape[0]):
        c.put(page, 64)
    table[0, :8] = [2, 2, 5, 2, 5, 5, 2, 1]
    table[1, :3] = [2, 2, 5]
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


def test_many_prompts(nk, sel):
    """More sequences than a workgroup plans for itself, prompts among them,
    one invalid."""
    rng = np.random.default_rng(34)
    n_new = [int(x) for x in rng.integers(0, 4, 400)]
    n_new[7], n_new[250], n_new[399] = 90, 33, 129
    ctx = [int(x) + n for x, n in zip(rng.integers(0, 50, 400), n_new)]
    c, table, q = case(nk, sel, 34, ctx, n_new, 8, 2, 64, 16, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    good, w = cache.attend(sequences(nk, n_new, ctx, table), qd, weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, good, w))
    bad = table.copy()
    bad[250, 0] = c.shape[0] + 5
    o, w2 = cache.attend(sequences(nk, n_new, ctx, bad), qd, weights=True)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    lo = sum(n_new[:250])
    hi = lo + n_new[250]
    assert torch.isnan(o[lo:hi]).all() and torch.equal(o[:lo], good[:lo]) and torch.equal(o[hi:], good[hi:])
    keep = [i for i in range(400) if i != 250]
    assert torch.equal(w2[keep], w[keep])


def test_calls_at_once(nk, sel):
    """Prompts, single tokens, stores into other pages and an eviction on four
    streams at a time, each as alone."""
    pc, dc = ([700, 500], [300, 500]), ([5000, 900, 40], [1, 1, 1])
    p_host, p_table, p_q = case(nk, sel, 35, pc[0], pc[1], 16, 2, 128, 64, "bf16")
    d_host, d_table, d_q = case(nk, sel, 36, dc[0], dc[1], 16, 2, 128, 512, "fp16")
    pcache, dcache = upload(nk, sel, p_host), upload(nk, sel, d_host)
    pseq, dseq = sequences(nk, pc[1], pc[0], p_table), sequences(nk, dc[1], dc[0], d_table)
    x = torch.randn((800, 4, 128), dtype=torch.bfloat16, device="cuda")
    spare = nk.BlockCache.empty(sel, p_host.shape[0], 2, 128, 64)
    off = dev([0, 20000, 20100, 90000], np.int64).view(torch.uint64)
    resident = dict(hash_off=off, hashes=torch.arange(90000, device="cuda").view(torch.uint64))
    weight = torch.randint(0, 1 << 40, (90000,), device="cuda").view(torch.uint64)
    keep = dev([9000, 50, 20000], np.int32).view(torch.uint32)
    pq, dq = p_q.cuda(), d_q.cuda()

    def store():
        spare.store(pseq, x[:, :2], x[:, 2:])
        return spare.read(pseq)

    def evict():
        r = sel.evict(resident, weight, keep, 10, 29050)
        return r["hash_off"], r["hashes"], r["pos"]

    jobs = [lambda: pcache.attend(pseq, pq, weights=True), lambda: dcache.attend(dseq, dq, weights=True), store, evict]
    alone = [j() for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = []
        for s, j in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(j())
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            for u, v in zip(a, b):
                assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))
    sel.sync_errors()


def test_prompts_and_stores_captured(nk, sel):
    """Store, attention with weights and their sum in a graph, replayed between
    eager calls on the same arrays, rows and lengths changed in place."""
    ctx, n_new = [400, 90], [100, 90]
    c, table, q = case(nk, sel, 37, ctx, n_new, 8, 2, 128, 64, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    lens = dev(ctx, np.int32).view(torch.uint32)
    seqs = nk.Sequences(dev([0, 100, 190], np.int64).view(torch.uint64), lens, dev(table, np.int32).view(torch.uint32), 190, 100)
    x = torch.randn((190, 4, 128), dtype=torch.bfloat16, device="cuda")
    acc = torch.zeros(c.shape[0], dtype=torch.int64, device="cuda")
    start = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]

    def step():
        cache.store(seqs, x[:, :2], x[:, 2:])
        o, w = cache.attend(seqs, qd, weights=True)
        cache.weigh(seqs, w, acc.view(torch.uint64))
        return o, w

    def reset():
        for t, s in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), start):
            t.copy_(s)
        acc.zero_()

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        lens.view(torch.int32).copy_(dev([400 - 3 * i, 90], np.int32))
        x.copy_(torch.randn_like(x) * (1 + i))
        reset()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, acc, cache.k, cache.v)]
        reset()
        o, w = step()
        for a, b in zip(got, (o, w, acc, cache.k, cache.v)):
            assert torch.equal(a, b)
    sel.sync_errors()


@pytest.mark.parametrize("n_seg", [1023, 1024, 1025, 2049, 4096, 4097, 9000])
def test_evict_many_segments_of_all_sizes(nk, sel, n_seg):
    """Around the numbers of segments where the plan and the groups change:
    tiny, small and long segments mixed."""
    rng = np.random.default_rng(n_seg)
    n = rng.integers(0, 300, n_seg)
    n[rng.integers(0, n_seg, 9)] = [64, 65, 256, 257, 4096, 4097, 9000, 20000, 0]
    n[-1], n[0] = 5000, 4097
    for kind in ("spread", "few"):
        w = draw(rng, int(n.sum()), kind)
        run(nk, sel, n, w, [int(x * f) for x, f in zip(n, rng.random(n_seg))], int(rng.integers(0, 9)))


def test_evict_bad_offsets_of_many_segments(nk, sel):
    off = np.arange(0, 3 * 3001, 3).astype(np.uint64)
    w = torch.arange(9000, device="cuda").view(torch.uint64)
    keep = dev(np.ones(3000), np.int32).view(torch.uint32)
    for at, to in ((1, 10), (1500, 0), (3000, 9001), (1024, 1 << 40)):
        bad = off.copy()
        bad[at] = to
        cache = dict(hash_off=nk.to_device(bad, sel.device), hashes=w)
        r = sel.evict(cache, w, keep, n_keep=3000)
        with pytest.raises(nk.NetKVError, match="eviction"):
            sel.sync_errors()
        assert not nk.to_numpy(r["hash_off"]).any()


@pytest.mark.parametrize("kind", ["half", "all", "dense", "steps"])
def test_evict_weights_of_every_width(nk, sel, kind):
    """Weights over all 64 bits (their top bit differs), and more than a
    wavefront's in one bin, at sizes of every form."""
    rng = np.random.default_rng(len(kind))
    n = [1, 2, 63, 64, 65, 200, 256, 257, 1000, 4096, 4097, 30000, 100000]
    m = sum(n)
    if kind == "half":
        w = rng.integers(0, 2, m).astype(np.uint64) << np.uint64(63)
    elif kind == "all":
        w = rng.integers(0, 1 << 63, m).astype(np.uint64) * np.uint64(2) + rng.integers(0, 2, m).astype(np.uint64)
    elif kind == "dense":
        w = np.uint64(1 << 40) + rng.integers(0, 1 << 34, m).astype(np.uint64)
    else:
        w = np.uint64(1) << rng.integers(0, 64, m).astype(np.uint64)
    for f in (0.0, 0.3, 0.97, 1.0):
        run(nk, sel, n, w, [max(1, int(f * x)) for x in n], 2 if f == 0.3 else 0)


@pytest.mark.parametrize("block", [64, 256, 1024])
def test_prompt_weights_both_ways(nk, sel, block):
    """A prompt's block weights from its rows' sums (at most 256 blocks a
    sequence) and from the second pass (more), whole and split, with rows that
    see nothing."""
    ctx, n_new = [9000, 600, 3, 64, 129], [40, 600, 70, 64, 1]
    c, table, q = case(nk, sel, 38, ctx, n_new, 6, 2, 64, block, "fp16")
    cache, qd = upload(nk, sel, c), q.cuda()
    wide = np.concatenate([table, np.full((5, 257), 1 << 30)], 1)     # never read
    for t in (table, wide):
        o, w = cache.attend(sequences(nk, n_new, ctx, t), qd, weights=True)
        sel.sync_errors()
        _say(check_attend(c, t, ctx, n_new, q, o, w))
        o2, w2 = cache.attend(sequences(nk, n_new, ctx, t), qd, weights=True)
        assert torch.equal(o, o2) and torch.equal(w, w2)


@pytest.mark.parametrize("block", [16, 64, 512])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompt_nan_in_what_a_row_does_not_see(nk, sel, dim, block):
    """As for few rows: a NaN key or value reaches the rows that see its token
    and no others (360 rows a head)."""
    ctx, n_new = [100], 90
    c, table, q = case(nk, sel, 40, ctx, [n_new], 8, 2, dim, block, "bf16")
    tok, kt = 100 - n_new // 2, 100 - n_new // 4
    c.v[table[0, tok // block], 1, tok % block, 5] = 0xFF
    c.k[table[0, kt // block], 0, kt % block, 9] = 0x7F
    o, w = upload(nk, sel, c).attend(sequences(nk, [n_new], ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    check_attend(c, table, ctx, [n_new], q, o)
    nan = torch.isnan(o.float())
    first = tok - (100 - n_new)                            # the row whose own token it is
    assert not nan[:first, 4:].any() and nan[first:, 4:, 5].all() and nan[:, 4:].sum() == (n_new - first) * 4
    first = kt - (100 - n_new)
    assert not nan[:first, :4].any() and nan[first:, :4].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [16, 128])
def test_prompt_large_scores_and_unequal_scales(nk, sel, block, dtype):
    ctx, n_new = [400, 130], [80, 1]
    c, table, q = case(nk, sel, 41, ctx, n_new, 8, 2, 128, block, dtype, qstd=60.0)
    c.vs = c.vs * 2.0 ** c.rng.integers(-28, 28, c.vs.shape)
    if dtype == "fp16":
        c.vs = np.clip(c.vs, 2.0 ** -12, 2.0 ** 5)
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


@pytest.mark.parametrize("block", [16, 64])
def test_prompt_rows_that_see_nothing(nk, sel, block):
    ctx, n_new = [2, 0, 1], [70, 66, 1]
    c, table, q = case(nk, sel, 42, ctx, n_new, 12, 2, 128, block, "bf16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    check_attend(c, table, ctx, n_new, q, o, w)
    assert not o[:68].any() and not o[70:136].any()


@pytest.mark.parametrize("block", [16, 64])
def test_prompt_invalid_sequences(nk, sel, block):
    ctx, n_new = [100, 200, 300], [80] * 3
    c, table, q = case(nk, sel, 43, ctx, n_new, 12, 2, 64, block, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    good, gw = cache.attend(sequences(nk, n_new, ctx, table), qd, weights=True)
    sel.sync_errors()
    bad = table.copy()
    bad[1, 1] = c.shape[0]
    long = [100, table.shape[1] * block + 1, 300]
    for lens, tab in ((ctx, bad), (long, table)):
        o, w = cache.attend(sequences(nk, n_new, lens, tab), qd, weights=True)
        with pytest.raises(nk.NetKVError, match="block cache"):
            sel.sync_errors()
        assert torch.isnan(o[80:160]).all() and torch.equal(o[:80], good[:80]) and torch.equal(o[160:], good[160:])
        assert torch.isnan(w[1, :2]).all() and torch.equal(w[[0, 2]], gw[[0, 2]])


@pytest.mark.parametrize("dim,rows", [(64, 240), (64, 241), (128, 160), (128, 161), (256, 32), (256, 33)])
def test_rows_at_the_forms_border(nk, sel, dim, rows):
    """The most rows that the form for few takes, and one more."""
    ctx, n_new = [rows + 150, 40, 700], [rows, 3, 1]
    c, table, q = case(nk, sel, 44, ctx, n_new, 2, 2, dim, 64, "fp16")
    o, w = upload(nk, sel, c).attend(sequences(nk, n_new, ctx, table), q.cuda(), weights=True)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


@pytest.mark.parametrize("dim,block,heads,hk,ctx,n_new", [
    (128, 64, 16, 1, [66, 130], [4, 4]), (64, 16, 24, 2, [70, 65], [5, 3]), (128, 512, 16, 2, [700, 515], [64, 40]),
    (256, 64, 8, 2, [129, 66], [4, 8]), (64, 16, 8, 2, [400, 100], [90, 66])])
def test_weights_do_not_read_what_was_not_written(nk, sel, dim, block, heads, hk, ctx, n_new):
    """A workspace full of large numbers: row tiles that end at different
    steps give the weights of the tokens they see."""
    c, table, q = case(nk, sel, 45, ctx, n_new, heads, hk, dim, block, "bf16")
    cache, seqs, qd = upload(nk, sel, c), sequences(nk, n_new, ctx, table), q.cuda()
    work = torch.full((nk.netkv_kv_attend_workspace(sel.h, cache.c, seqs, heads, True),), 0x7E, dtype=torch.uint8, device="cuda")
    o, w = torch.empty_like(qd), torch.empty(table.shape, dtype=torch.float32, device="cuda")
    nk.netkv_kv_attend(sel.h, cache.c, seqs, qd, dim ** -0.5, o, w, work, sel.device)
    sel.sync_errors()
    _say(check_attend(c, table, ctx, n_new, q, o, w))


@pytest.mark.parametrize("block,dim", [(16, 128), (32, 128), (16, 256), (32, 64)])
def test_prompt_weights_of_small_blocks_both_ways(nk, sel, block, dim):
    """Blocks of less than a step: the last ones of a table, groups past the
    last token, two sequences and a split one."""
    ctx, n_new = [256 * block, 600, 3, 64, 129 + block], [400, 600, 70, 64, 100]
    c, table, q = case(nk, sel, 46, ctx, n_new, 4, 2, dim, block, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    wide = np.concatenate([table, np.full((5, 3), 1 << 30)], 1)       # never read
    for t in (table, wide):
        seqs = sequences(nk, n_new, ctx, t)
        work = torch.full((nk.netkv_kv_attend_workspace(sel.h, cache.c, seqs, 4, True),), 0x7E, dtype=torch.uint8, device="cuda")
        o, w = torch.empty_like(qd), torch.empty(t.shape, dtype=torch.float32, device="cuda")
        nk.netkv_kv_attend(sel.h, cache.c, seqs, qd, dim ** -0.5, o, w, work, sel.device)
        sel.sync_errors()
        _say(check_attend(c, t, ctx, n_new, q, o, w))
        assert torch.equal(o, cache.attend(seqs, qd))
