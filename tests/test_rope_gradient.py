"""A rotation's table that requires a gradient, without a GPU."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")


def test_table_that_requires_a_gradient():
    from paper_2606_03910_amd import netkv as nk
    sel = SimpleNamespace(h=None, device=torch.device("cuda:0"))
    learnt = torch.zeros((4, 64), requires_grad=True)
    for table in (learnt, learnt * 2):
        with pytest.raises(ValueError, match="table requires a gradient"):
            nk.Rope(sel, table)
    with torch.no_grad(), pytest.raises(TypeError, match="table"):      # as a table without one: not on the device
        nk.Rope(sel, learnt)
