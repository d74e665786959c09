"""Differential attention's workspace.  Needs an MI355X and the built library."""
import numpy as np
import pytest

from tests.test_gpu_block_cache import sequences

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
