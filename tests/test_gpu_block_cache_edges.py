"""The block cache's operators on calls at the edge of what include/netkv.h
allows: sequences that name the same rows, outputs over the
queries, dominant tokens, tensors that require a gradient.  Needs an MI355X and the built
library."""
import ctypes

import numpy as np
import pytest

from tests import blockcache_ref as R
from tests.test_gpu_block_cache import case, check_attend, dev, ref_store, same_cache, sequences, upload

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


# ------------------------------------------------------------------ rows of two sequences

def counts(off, n_tok, max_tok):
    """Which sequences count, and the rows that are NaN after an attention."""
    before, ok, nan = 0, [], np.zeros(n_tok, bool)
    for b, e in zip(off[:-1], off[1:]):
        rows = b <= e <= n_tok
        ok.append(bool(rows and e - b <= max_tok and b >= before))
        if rows and not ok[-1]:
            nan[max(b, before):e] = True
        if rows:
            before = max(before, e)
    return ok, nan


OVERLAPS = [
    # offsets, max_tok, heads, kv heads, dim, block, tokens of every sequence
    ([0, 128, 0, 128, 0, 128, 0, 128, 170], 128, 64, 8, 128, 512, 2048),   # 63 slots if all of them counted, of 44
    ([0, 20, 0, 20, 0, 20, 21], 20, 64, 8, 128, 512, 512),
    ([0, 1, 0, 1, 0, 1, 0, 1, 2], 1, 16, 2, 64, 16, 700),
    ([3, 9, 1, 5, 40, 30, 33, 33, 44], 12, 4, 2, 256, 64, 130),
    ([0, 4, 1 << 40, 4, 8], 4, 8, 2, 64, 32, 100),
]


@pytest.mark.parametrize("at", range(len(OVERLAPS)))
def test_attend_rows_of_two_sequences(nk, sel, at):
    """A sequence that begins among rows of an earlier one is invalid: NaN
    where no other names the row, its block weights NaN; the others as without
    it, and nothing past the workspace."""
    off, max_tok, heads, hk, dim, block, held = OVERLAPS[at]
    _say("overlap", at)
    n_seq, n_tok = len(off) - 1, max(x for x in off if x < 1 << 30)
    ok, nan = counts(off, n_tok, max_tok)
    assert not all(ok) and any(ok)
    ctx = [held - 3 * s for s in range(n_seq)]
    c, table, q = case(nk, sel, 50 + at, ctx, [n_tok] + [0] * (n_seq - 1), heads, hk, dim, block, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    seqs = sequences(nk, None, ctx, table, n_tok=n_tok, max_tok=max_tok, off=np.array(off, np.int64))
    for weights in (True, False):
        size = nk.netkv_kv_attend_workspace(sel.h, cache.c, seqs, heads, weights)
        work = torch.full((size + 4096,), 0x7E, dtype=torch.uint8, device="cuda")
        out = torch.full_like(qd, 5.0)
        w = torch.full(table.shape, 7.0, device="cuda") if weights else None
        nk.netkv_kv_attend(sel.h, cache.c, seqs, qd, dim ** -0.5, out, w, work[:size], sel.device)
        with pytest.raises(nk.NetKVError, match="block cache"):
            sel.sync_errors()
        assert (work[size:] == 0x7E).all()
        for s in range(n_seq):
            if ok[s]:
                b, e = off[s], off[s + 1]
                check_attend(c, table[s:s + 1], ctx[s:s + 1], [e - b], q[b:e], out[b:e], w[s:s + 1] if weights else None)
            elif weights:
                assert torch.isnan(w[s]).all()
        named = nan.copy()
        for s in range(n_seq):
            if ok[s]:
                named[off[s]:off[s + 1]] = True
        assert torch.isnan(out[torch.from_numpy(nan).cuda()]).all()
        assert (out[torch.from_numpy(~named).cuda()] == 5).all()


def _fallen(n_seq, at, to):
    off = np.arange(n_seq + 1, dtype=np.int64)
    for a, t in zip(at, to):
        off[a] = t
    return off


FALLS = [(600, [300], [290]), (600, [256], [3]), (600, [10, 400], [0, 255]), (1500, [1024, 1300], [1000, 5]),
         (300, [299], [1 << 33]), (2000, [0, 1999], [1 << 50, 1])]


@pytest.mark.parametrize("at", range(len(FALLS)))
def test_many_sequences_with_offsets_that_fall(nk, sel, at):
    """More sequences than a workgroup looks through at a time: attention,
    store and read leave out the same ones."""
    n, where, to = FALLS[at]
    _say("falls", at)
    off, max_tok = _fallen(n, where, to), 20
    ok, nan = counts(off.tolist(), n, max_tok)
    assert not all(ok)
    rng = np.random.default_rng(60 + at)
    hk, heads, dim, block = 2, 4, 64, 16
    ctx = [int(x) for x in rng.integers(20, 40, n)]
    c, table, q = case(nk, sel, 60 + at, ctx, [n] + [0] * (n - 1), heads, hk, dim, block, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    seqs = sequences(nk, None, ctx, table, n_tok=n, max_tok=max_tok, off=off)
    out = torch.full_like(qd, 5.0)
    _, w = cache.attend(seqs, qd, out=out, weights=True)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    good = [s for s in range(n) if ok[s]]
    rows = np.concatenate([np.arange(off[s], off[s + 1]) for s in good]).astype(np.int64)
    new = [int(off[s + 1] - off[s]) for s in good]
    check_attend(c, table[good], [ctx[s] for s in good], new, q[rows], out[torch.from_numpy(rows).cuda()], w[good])
    assert torch.isnan(w[[s for s in range(n) if not ok[s]]]).all()
    assert torch.isnan(out[torch.from_numpy(nan).cuda()]).all()
    left = ~nan
    left[rows] = False
    assert (out[torch.from_numpy(left).cuda()] == 5).all()
    # store and read
    x = torch.from_numpy(rng.standard_normal((n, 2 * hk, dim))).to(torch.bfloat16)
    xd = x.cuda()
    cache.store(seqs, xd[:, :hk], xd[:, hk:])
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    f = x[rows].double().numpy()
    ref_store(c, table[good], [ctx[s] for s in good], new, f[:, :hk], f[:, hk:])
    same_cache(cache, c, table, ctx)                       # the others' pages as they were
    k, v = (torch.full((n, hk, dim), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nk.netkv_kv_read(sel.h, cache.c, seqs, k, v, sel.device)
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    for s in good:
        b, e = int(off[s]), int(off[s + 1])
        for h in range(hk):
            for got, which in ((k, "k"), (v, "v")):
                assert np.array_equal(got[b:e, h].double().cpu().numpy(), c.held(table[s], ctx[s], h, which)[ctx[s] - (e - b):])
    rest = np.ones(n, bool)
    rest[rows] = False
    assert (k[torch.from_numpy(rest).cuda()] == 9).all() and (v[torch.from_numpy(rest).cuda()] == 9).all()


@pytest.mark.parametrize("n_new", [60, 200])
def test_store_blocks_of_rows_named_twice(nk, sel, n_new):
    """The rows that two sequences name are stored for the first; a later
    sequence with rows of its own is stored whole."""
    hk, dim, block = 2, 64, 16
    rng = np.random.default_rng(70)
    off = [0, n_new, 0, n_new, 0, n_new, 0, n_new, 2 * n_new]
    ctx = [n_new + 5 * s for s in range(8)]
    ok, _ = counts(off, 2 * n_new, n_new)
    table, pages = R.tables(rng, ctx, block)
    c = R.Cache(pages, hk, dim, block, rng)
    for s, t in enumerate(ctx):
        for i in range(-(-t // block)):
            c.put(table[s, i], min(block, t - i * block))
    cache = upload(nk, sel, c)
    x = torch.from_numpy(rng.standard_normal((2 * n_new, 2 * hk, dim))).to(torch.float16)
    xd = x.cuda()
    seqs = sequences(nk, None, ctx, table, n_tok=2 * n_new, max_tok=n_new, off=off)
    cache.store(seqs, xd[:, :hk], xd[:, hk:])
    with pytest.raises(nk.NetKVError, match="block cache"):
        sel.sync_errors()
    good = [s for s in range(8) if ok[s]]
    assert good == [0, 7]
    f = x.double().numpy()
    ref_store(c, table[good], [ctx[s] for s in good], [n_new, n_new], f[:, :hk], f[:, hk:])
    same_cache(cache, c, table, ctx)


# ------------------------------------------------------------------ outputs over the queries

@pytest.mark.parametrize("ctx,n_new,dim", [([700, 33], [1, 1], 128), ([9000, 40], [3, 4], 64), ([9000, 600], [40, 600], 64),
                                           ([300, 200], [30, 70], 256)])
def test_attend_in_place(nk, sel, ctx, n_new, dim):
    """out may be q itself without weights, and lie beside it in wider rows."""
    c, table, q = case(nk, sel, 80, ctx, n_new, 8, 2, dim, 64, "bf16")
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    qd = q.cuda()
    want = cache.attend(seqs, qd)
    x = qd.clone()
    assert cache.attend(seqs, x, out=x) is x and torch.equal(x, want)
    wide = torch.cat([qd, torch.zeros_like(qd), qd], 1)
    cache.attend(seqs, wide[:, 16:], out=wide[:, 8:16], weights=True)
    assert torch.equal(wide[:, 8:16], want) and torch.equal(wide[:, :8], qd) and torch.equal(wide[:, 16:], qd)
    sel.sync_errors()


@pytest.mark.parametrize("blocks", [3, 300])
def test_attend_refuses_outputs_over_queries(nk, sel, blocks):
    """With weights, where a prompt's second pass would read them, and any
    other overlap."""
    ctx, n_new = [170], [120]
    c, table, q = case(nk, sel, 81, ctx, n_new, 8, 2, 128, 64, "bf16")
    table = np.concatenate([table, np.zeros((1, blocks - 3), np.int64)], 1)
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    wide = torch.cat([q, q], 1).cuda()
    a = wide[:, :8]
    for out, weights in ((a, True), (wide[:, 4:12], False), (wide[:, 4:12], True)):
        with pytest.raises(nk.NetKVError, match="overlap"):
            cache.attend(seqs, a, out=out, weights=weights)
    flat = torch.zeros(122 * 1024, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(nk.NetKVError, match="overlap"):
        cache.attend(seqs, flat[:120 * 1024].view(120, 8, 128), out=flat[1024:121 * 1024].view(120, 8, 128))
    o, w = cache.attend(seqs, a, weights=True)
    sel.sync_errors()
    check_attend(c, table, ctx, n_new, q, o, w)


# ------------------------------------------------------------------ dominant tokens

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("dim,n_new,ctx,block", [(128, 1, 32768, 512), (64, 7, 5000, 16), (256, 2, 9000, 64),
                                                 (128, 40, 32768, 512), (64, 70, 5000, 16), (256, 20, 3000, 64)])
def test_attend_dominant_token(nk, sel, dim, n_new, ctx, block, where, dtype):
    """One token far above many equal ones whose values alone are not zero:
    the output is what those keep of the weight.

    Relative limit: a weight e^-S of the largest is rounded by half of the
    larger of 2^-10 of itself and 2^-30 of the largest, so relatively by
    max(2^-11, 2^-31 e^S); the others' values are 1, so all of them may be off
    to the same side.  Scores are exact (ones and zeros, one product with the
    scale) up to S 2^-23 by that product and S log2(e) 2^-23 by the exponential's
    argument, twice; the exponential and sums in fp32, at most 2^9 one after
    the other, 2^-15 in all; and the output's own half step."""
    heads, hk = 16, 2
    rng = np.random.default_rng(90)
    table, pages = R.tables(rng, [ctx], block)
    c = R.Cache(pages, hk, dim, block, rng)
    c.ks[:], c.vs[:] = 1.0, 1.0
    c.k[:], c.v[:] = 0, 0x38                               # 0 and 1.0
    tok = dict(first=0, middle=ctx // 2 + 5, last=ctx - n_new)[where]
    c.k[table[0, tok // block], :, tok % block] = 0x38
    c.v[table[0, tok // block], :, tok % block] = 0
    cache, seqs = upload(nk, sel, c), sequences(nk, [n_new], [ctx], table)
    q = torch.ones((n_new, heads, dim), dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device="cuda")
    for S in (0.0, 9.0, 14.0, 17.5, 19.0):
        o = cache.attend(seqs, q, S / dim).double().cpu().numpy()
        s = dim * float(np.float32(S / dim))
        for t in range(n_new):
            others = ctx - n_new + t
            want = others / (others + np.exp(s))
            rel = max(2.0 ** -11, 2.0 ** -31 * np.exp(s)) + s * 2.0 ** -21 + 2.0 ** -15 + torch.finfo(q.dtype).eps / 2
            assert (np.abs(o[t] - want) <= rel * want).all(), (S, t, o[t].min() / want, o[t].max() / want)
    sel.sync_errors()


@pytest.mark.parametrize("n_new", [1, 90])
@pytest.mark.parametrize("e", [-126, 119])
def test_attend_smallest_and_largest_scales(nk, sel, n_new, e):
    """Values of the smallest and of very large scales (448 * 2^119 is the
    format's largest scale's), in bf16, whole and split."""
    ctx, new = [200, 3000], [n_new, 1]
    c, table, q = case(nk, sel, 91, ctx, new, 8, 2, 128, 64, "bf16")
    c.vs[:] = 2.0 ** e
    c.v[:] = np.where((c.v & 127) < 0x20, 0x40, c.v)       # no value below 2^-3: none of the outputs is subnormal
    o = upload(nk, sel, c).attend(sequences(nk, new, ctx, table), q.cuda())
    sel.sync_errors()
    _say(check_attend(c, table, ctx, new, q, o))


@pytest.mark.parametrize("n_new", [1, 90])
def test_attend_scales_of_zero(nk, sel, n_new):
    """Blocks of zeros whose scale says so."""
    ctx, new = [200, 3000], [n_new, 1]
    c, table, q = case(nk, sel, 95, ctx, new, 8, 2, 128, 64, "bf16")
    c.vs[:, 0] = 0.0
    c.vs[table[0, 1], 1] = 0.0
    o = upload(nk, sel, c).attend(sequences(nk, new, ctx, table), q.cuda())
    sel.sync_errors()
    check_attend(c, table, ctx, new, q, o)
    assert not o[:, :4].any() and (o[:, 4:] != 0).any(2).all()


@pytest.mark.parametrize("n_new", [1, 90])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_attend_scores_that_are_all_infinite(nk, sel, n_new, sign):
    """An infinite query over keys of one sign has scores of one infinity: the
    row and its block weights are no numbers, as with any other query that is
    not finite."""
    ctx, new, heads, hk = [70, 3000, 2], [n_new, 1, 4], 8, 2
    c, table, q = case(nk, sel, 92, ctx, new, heads, hk, 128, 64, "fp16")
    c.k[..., 3] = np.clip(c.k[..., 3] & 127, 1, 0x7E)               # positive
    inf = np.zeros((sum(new), heads), bool)
    for row, head in ((n_new // 2, 1), (n_new, 6), (n_new + 4, 0)):
        q[row, head, 3] = sign * float("inf")
        inf[row, head] = True
    cache, seqs = upload(nk, sel, c), sequences(nk, new, ctx, table)
    o, w = cache.attend(seqs, q.cuda(), weights=True)
    sel.sync_errors()
    nan = torch.isnan(o.float()).cpu().numpy()
    assert nan[inf].all() and not nan[~inf].any()
    seen = np.zeros(table.shape, bool)
    seen[0, :-(-(70 - n_new + n_new // 2 + 1) // 64)] = seen[1, :-(-3000 // 64)] = seen[2, :1] = True
    assert np.array_equal(torch.isnan(w).cpu().numpy(), seen)
    # rows that see nothing are still 0
    assert not o[n_new + 1:n_new + 3].any()


# ------------------------------------------------------------------ weigh

def test_weigh_reads_only_what_it_says(nk, sel):
    """ctx_len, pages, n_seq and max_pages: offsets may be NULL, the bounds of
    the rows anything."""
    ctx, table = [40, 5], np.array([[1, 0, 2], [3, 0, 0]])
    seqs = sequences(nk, [0, 0], ctx, table)
    w = torch.tensor([[0.5, 0.25, 2.0], [1.0, 9.0, 9.0]], device="cuda")
    got = [torch.zeros(4, dtype=torch.int64, device="cuda") for _ in range(2)]
    nk.netkv_kv_weigh(sel.h, seqs, 16, w, got[0].view(torch.uint64), sel.device)
    bare = nk.netkv_kv_seqs_t.from_buffer_copy(seqs.c)
    bare.tok_off, bare.n_tok, bare.max_tok = None, 1 << 40, 1 << 50
    lib = nk.load_library()
    assert lib.netkv_kv_weigh(sel.h, ctypes.byref(bare), 16, w.data_ptr(), 4, got[1].data_ptr(), nk._stream(sel.device)) == 0
    with pytest.raises(nk.NetKVError, match="EINVAL.*seqs must not be NULL"):
        nk._check(sel.h, lib.netkv_kv_weigh(sel.h, None, 16, w.data_ptr(), 4, got[1].data_ptr(), nk._stream(sel.device)))
    sel.sync_errors()
    assert torch.equal(*got) and (got[0] / 2 ** 24).tolist() == [0.25, 0.5, 2.0, 1.0]


@pytest.mark.parametrize("off", [[7, 6, 5, 4], [0, 600, 500, 900], [0, 1 << 60, 1 << 61, 1 << 62], [900, 0, 0, 0]])
def test_evict_bad_offsets_without_a_count(nk, sel, off):
    """Reported by the call, whatever their sizes add up to."""
    cache = dict(hash_off=dev(off, np.int64).view(torch.uint64), hashes=torch.arange(900, device="cuda").view(torch.uint64))
    weight = torch.arange(900, device="cuda").view(torch.uint64)
    r = sel.evict(cache, weight, torch.full((3,), -1, dtype=torch.int32, device="cuda").view(torch.uint32))
    with pytest.raises(nk.NetKVError, match="eviction"):
        sel.sync_errors()
    assert not r["hash_off"].view(torch.int64).any()


# ------------------------------------------------------------------ gradients

def test_tensors_that_require_a_gradient(nk, sel):
    """Refused where a gradient would be lost; as ever without one."""
    ctx, n_new = [30, 50], [1, 2]
    c, table, q = case(nk, sel, 93, ctx, n_new, 8, 2, 128, 16, "bf16")
    cache, seqs = upload(nk, sel, c), sequences(nk, n_new, ctx, table)
    qd = q.cuda()
    want = cache.attend(seqs, qd)
    x = qd.clone().requires_grad_()
    with pytest.raises(ValueError, match="q requires a gradient"):
        cache.attend(seqs, x)
    with pytest.raises(ValueError, match="q requires a gradient"):
        cache.attend(seqs, x * 1)
    assert torch.equal(cache.attend(seqs, x.detach()), want)
    with torch.no_grad():
        assert torch.equal(cache.attend(seqs, x), want)
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="v requires a gradient"):
        cache.store(seqs, k, k.clone().requires_grad_())
    sel.sync_errors()


def test_stream_both_ways(nk, sel, monkeypatch):
    s = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), s):
        with torch.cuda.stream(stream):
            got = nk._stream(sel.device)
            with monkeypatch.context() as m:
                m.setattr(nk, "_raw_stream", None)
                assert nk._stream(sel.device) == got == stream.cuda_stream


# ------------------------------------------------------------------ capacities

@pytest.mark.parametrize("n_tok,max_tok,n_heads,fits", [
    (200000, 200000, 8192, True), (300000, 300000, 8192, False),          # 512 threads: 2^23 workgroups
    (32764, 2, 8192, True), (32766, 2, 8192, False)])                     # 256 threads: 2^24
def test_grids_that_no_launch_takes(nk, sel, n_tok, max_tok, n_heads, fits):
    """Refused as documented, from the host's values alone."""
    kv = nk.netkv_kv_t(n_pages=1, block_tokens=16, n_kv_heads=1024, head_dim=64, k=256, v=256, k_scale=256, v_scale=256)
    seqs = sequences(nk, None, [1], np.zeros((1, 1)), n_tok=n_tok, max_tok=max_tok, off=[0, 1])
    if fits:
        assert nk.netkv_kv_attend_workspace(sel.h, kv, seqs, n_heads, False) > 0
    else:
        with pytest.raises(nk.NetKVError, match="ECAPACITY"):
            nk.netkv_kv_attend_workspace(sel.h, kv, seqs, n_heads, False)


@pytest.mark.parametrize("n_seq,n_tok,max_tok,max_pages,block,heads,hk,dim", [
    (256, 256, 1, 8192, 16, 64, 8, 128), (256, 1792, 7, 8192, 16, 64, 8, 128), (512, 15360, 30, 8192, 16, 64, 8, 64),
    (64, 64, 1, 32, 512, 64, 8, 128), (16, 131072, 16384, 256, 512, 64, 8, 128), (2, 2048, 1024, 64, 512, 64, 8, 128)])
def test_workspace_is_bounded(nk, sel, n_seq, n_tok, max_tok, max_pages, block, heads, hk, dim):
    """One long sequence among many does not make the others' sums as wide:
    2^32 bytes of them, parts of split rows (2 x 512 workgroups' slots of 256
    rows of 128 dimensions and their sums), the work list, a number a row and
    head, and one a head's unit."""
    kv = nk.netkv_kv_t(n_pages=1, block_tokens=block, n_kv_heads=hk, head_dim=dim, k=256, v=256, k_scale=256, v_scale=256)
    seqs = sequences(nk, None, np.ones(n_seq), np.zeros((n_seq, max_pages)), n_tok=n_tok, max_tok=max_tok,
                     off=np.arange(n_seq + 1))
    tiles = n_tok * heads // hk // 16 + n_seq
    without = nk.netkv_kv_attend_workspace(sel.h, kv, seqs, heads, False)
    assert without <= (1024 + hk) * 256 * (4 * 128 + 16) + 48 * (tiles + 1024) + 4096
    units = n_seq * hk * (max_pages * block // min(block, 64) + 4)
    _say(without, nk.netkv_kv_attend_workspace(sel.h, kv, seqs, heads, True) - without)
    assert nk.netkv_kv_attend_workspace(sel.h, kv, seqs, heads, True) - without <= (1 << 32) + 4 * (n_tok * heads + n_seq + units) + 4096


@pytest.mark.parametrize("dim,block,heads,hk,ctx,n_new,pages", [
    (64, 16, 60, 1, [700, 4, 65, 0], [4, 4, 1, 0], 1200000),      # 240 rows a sequence, of few
    (128, 64, 128, 2, [3000, 64, 1], [2, 1, 1], 1600000), (256, 32, 64, 2, [100, 3, 70], [1, 1, 1], 5200000),
    (64, 512, 8, 2, [900, 600, 3], [600, 100, 5], 250)])
def test_weights_without_kept_sums(nk, sel, dim, block, heads, hk, ctx, n_new, pages):
    """Few rows over tables too wide for every unit's sum, and a prompt whose
    rows' sums would be too many: the second pass over the keys gives the same
    weights."""
    c, table, q = case(nk, sel, 94, ctx, n_new, heads, hk, dim, block, "bf16")
    cache, qd = upload(nk, sel, c), q.cuda()
    wide = np.concatenate([table, np.full((len(ctx), pages - table.shape[1]), 1 << 30)], 1)     # never read
    # a bound of rows that makes the prompt's sums too many; the rows that there are stay the same
    n_tok = 1200000 if max(n_new) > 100 else sum(n_new)
    if n_tok > sum(n_new):
        qd = torch.cat([qd, torch.zeros((n_tok - sum(n_new), heads, dim), dtype=qd.dtype, device="cuda")])
    seqs = sequences(nk, n_new, ctx, wide, n_tok=n_tok)
    size = nk.netkv_kv_attend_workspace(sel.h, cache.c, seqs, heads, True)
    assert size < 1 << 30
    work = torch.full((size,), 0x7E, dtype=torch.uint8, device="cuda")
    o, w = torch.empty_like(qd), torch.empty(wide.shape, dtype=torch.float32, device="cuda")
    nk.netkv_kv_attend(sel.h, cache.c, seqs, qd, dim ** -0.5, o, w, work, sel.device)
    sel.sync_errors()
    assert not w[:, table.shape[1]:].any()
    _say(check_attend(c, table, ctx, n_new, q, o, w[:, :table.shape[1]]))
    assert torch.equal(o[:sum(n_new)], cache.attend(sequences(nk, n_new, ctx, table), qd)[:sum(n_new)])
