"""A rotation's table that requires a gradient.  Needs an MI355X and the built
library."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


def test_a_table_that_requires_a_gradient(nk, sel):
    """Refused where a gradient would be lost; as ever without one."""
    tab = torch.randn((9, 64), device="cuda")
    x = torch.randn((4, 3, 64), device="cuda").bfloat16()
    pos = torch.arange(4, dtype=torch.int32, device="cuda").view(torch.uint32)
    want = nk.Rope(sel, tab).rotate(x, pos)
    learnt = tab.clone().requires_grad_()
    with pytest.raises(ValueError, match="table requires a gradient"):
        nk.Rope(sel, learnt)
    with pytest.raises(ValueError, match="table requires a gradient"):
        nk.Rope(sel, learnt * 1)
    assert torch.equal(nk.Rope(sel, learnt.detach()).rotate(x, pos), want)
    with torch.no_grad():
        assert torch.equal(nk.Rope(sel, learnt).rotate(x, pos), want)
    sel.sync_errors()
