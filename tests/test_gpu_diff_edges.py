"""Differential attention's rounding of small weights, and its workspace's bound.
Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests import blockcache_ref as R
from tests.test_gpu_block_cache import dev, sequences, upload

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


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("dim,n_new,ctx,block", [
    (64, 1, 32768, 512), (64, 7, 5000, 16), (64, 2, 600, 64), (128, 2, 9000, 64), (128, 1, 400, 32), (128, 9, 3000, 16),
    (64, 70, 5000, 16), (64, 60, 32768, 512), (64, 200, 500, 64), (128, 40, 32768, 512), (128, 40, 5000, 16), (128, 90, 300, 64)])
def test_a_dominant_token_leaves_the_others(nk, sel, dim, n_new, ctx, block, where, dtype):
    """One token far above many equal ones whose values alone are not zero: the
    output is what those keep of the weight, of the first map alone and of the
    second one nearly alone (lambda -8); few rows and prompts, split and whole.

    Relative limit: a weight e^-S of the largest is rounded by half of the
    larger of 2^-10 of itself and 2^-30 of the largest, so relatively by
    max(2^-11, 2^-31 e^S); the others' values are 1, so all of them may be off
    to the same side.  Scores are exact (ones and zeros, one product with the
    scale) up to S 2^-23 by that product and S log2(e) 2^-23 by the exponential's
    argument, twice; the exponential and sums in fp32, at most 2^9 one after
    the other, 2^-15 in all; the maps' sum, both of one sign here, 2^-23 twice; and
    the output's own half step."""
    heads, hk = 16, 4
    rng = np.random.default_rng(95)
    table, pages = R.tables(rng, [ctx], block)
    c = R.Cache(pages, hk, dim, block, rng)
    c.ks[:], c.vs[:] = 1.0, 1.0
    c.k[:], c.v[:] = 0, 0x38                               # 0 and 1.0
    tok = dict(first=0, middle=ctx // 2 + 5, last=ctx - n_new)[where]
    c.k[table[0, tok // block], :, tok % block] = 0x38
    c.v[table[0, tok // block], :, tok % block] = 0
    cache, seqs = upload(nk, sel, c), sequences(nk, [n_new], [ctx], table)
    q = torch.ones((n_new, heads, dim), dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device="cuda")
    lam = np.tile([0.0, -8.0], heads // 4)
    q[:, 2::4] *= 0.5                                      # the first map of the pairs of -8: half of S
    lam_d = dev(lam, np.float32)
    _say(dim, n_new, ctx, block, where, dtype)
    for S in (0.0, 9.0, 14.0, 17.5, 19.0):
        o = cache.attend_diff(seqs, q, lam_d, scale=S / dim).double().cpu().numpy()
        s = dim * float(np.float32(S / dim))
        for t in range(n_new):
            seen = ctx - n_new + t + 1
            others = seen - (tok < seen)
            assert others < seen
            keep = lambda s: others / (others + np.exp(s))
            rel = lambda s: max(2.0 ** -11, 2.0 ** -31 * np.exp(s)) + s * 2.0 ** -21 + 2.0 ** -15
            for j, l in enumerate(lam):
                first = s / 2 if l else s
                want = keep(first) - l * keep(s)
                lim = rel(first) * keep(first) + abs(l) * rel(s) * keep(s) + (2.0 ** -22 + torch.finfo(q.dtype).eps / 2) * want
                assert (np.abs(o[t, j] - want) <= lim).all(), (S, t, j, o[t, j].min() / want, o[t, j].max() / want)
    sel.sync_errors()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_new", [1, 30, 300])
@pytest.mark.parametrize("hk", [2, 6, 10, 62, 126, 190, 200, 342, 344, 400, 510, 514, 600, 682, 684, 800, 1022, 1024])
def test_workspace_is_bounded_for_any_number_of_heads(nk, sel, hk, n_new, dim):
    """Also where the pairs do not divide the card's workgroups."""
    for n_seq, block, max_pages, g in ((2, 64, 2048, 1), (64, 512, 256, 4), (300, 16, 8192, 1)):
        kv = nk.netkv_kv_t(n_pages=1, block_tokens=block, n_kv_heads=hk, head_dim=dim, k=256, v=256, k_scale=256, v_scale=256)
        seqs = sequences(nk, None, [1] * n_seq, np.zeros((n_seq, max_pages)), n_tok=n_seq * n_new, max_tok=n_new,
                         off=[0] * (n_seq + 1))
        tiles = n_seq * -(-n_new * g // 16)
        assert nk.netkv_kv_attend_diff_workspace(sel.h, kv, seqs, hk * g) <= 300e6 + 48 * tiles, (n_seq, block, g)
