"""What the block cache's tests stand on, and the binding's refusals that need
no GPU: e4m3 against torch's, the scale's definition, attention against a loop."""
import math

import numpy as np
import pytest

from tests import blockcache_ref as R

torch = pytest.importorskip("torch")


def test_values_of_all_bytes():
    b = np.arange(256).astype(np.uint8)
    want = torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy()
    got = R.values(b)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_nearest_is_nearest_even():
    """Every value, every middle between two (to the even one), and what lies
    just beside a middle."""
    v = R.values(np.arange(127).astype(np.uint8))          # 0 .. 448, ascending
    assert np.array_equal(R.nearest(v), np.arange(127)) and np.array_equal(R.nearest(-v), np.arange(127) + 128)
    mid = (v[1:] + v[:-1]) / 2
    lo = np.arange(126)
    assert np.array_equal(R.nearest(mid), lo + lo % 2)
    assert np.array_equal(R.nearest(np.nextafter(mid, 0)), lo) and np.array_equal(R.nearest(np.nextafter(mid, 448)), lo + 1)
    assert np.array_equal(R.nearest(np.array([np.nan, np.inf, -np.inf])) & 127, [127] * 3)


@pytest.mark.parametrize("amax", [0.0, 1e-45, 2.0 ** -126, 448 * 2.0 ** -126, 1.0, 448.0, 448.1, 449.0, 512.0, 65504.0, 3.38e38])
def test_scale_is_the_smallest_power_of_two(amax):
    s = R.scale_for(amax)
    assert math.frexp(s)[0] == 0.5 and s >= 2.0 ** -126 and amax <= 448 * s
    assert s == 2.0 ** -126 or amax > 448 * s / 2


def test_attend_by_hand():
    """One row over three tokens in two blocks, by a loop."""
    rng = np.random.default_rng(0)
    c = R.Cache(3, 1, 64, 16, rng)
    c.put(2, 16)
    c.put(0, 1)
    q = rng.standard_normal((2, 1, 64))
    o, w, _, _ = R.attend(c, np.array([[2, 0]]), [17], [2], q, 1, 0.125)
    for t, seen in ((0, 16), (1, 17)):
        k = [R.values(c.k[2, 0, i]) * c.ks[2, 0] if i < 16 else R.values(c.k[0, 0, 0]) * c.ks[0, 0] for i in range(seen)]
        v = [R.values(c.v[2, 0, i]) * c.vs[2, 0] if i < 16 else R.values(c.v[0, 0, 0]) * c.vs[0, 0] for i in range(seen)]
        e = [math.exp(0.125 * float(q[t, 0] @ x)) for x in k]
        want = sum(a * x for a, x in zip(e, v)) / sum(e)
        assert np.allclose(o[t, 0], want, rtol=1e-12, atol=0)
    assert abs(w.sum() - 2) < 1e-12


def test_evict_by_hand():
    off, w, h = [0, 5, 5, 8], np.array([3, 9, 9, 1, 0, 7, 7, 7], np.uint64), np.arange(10, 18).astype(np.uint64)
    o, pos, hs = R.evict(off, w, h, [3, 1, 2], 1)
    assert o.tolist() == [0, 3, 3, 5] and pos.tolist() == [1, 2, 4, 0, 2] and hs.tolist() == [11, 12, 14, 15, 17]


def test_stream_without_the_short_way(monkeypatch):
    """A torch without the name that is not public still gives its stream."""
    from types import SimpleNamespace

    from paper_2606_03910_amd import netkv as nk
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev: SimpleNamespace(cuda_stream=40 + dev.index))
    monkeypatch.setattr(nk, "_raw_stream", None)
    assert nk._stream(torch.device("cuda:2")) == 42
    monkeypatch.setattr(nk, "_raw_stream", lambda i: 70 + i)
    assert nk._stream(torch.device("cuda:2")) == 72


def test_binding_refuses_a_gradient():
    """It would be lost without a word."""
    from paper_2606_03910_amd import netkv as nk
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16, requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        nk._no_gradient(q, "q")
    with torch.no_grad():
        nk._no_gradient(q, "q")
    nk._no_gradient(q.detach(), "q")


def test_binding_refuses_without_a_gpu():
    from paper_2606_03910_amd import netkv as nk
    off, ctx = torch.zeros(2, dtype=torch.int64).view(torch.uint64), torch.zeros(1, dtype=torch.int32).view(torch.uint32)
    with pytest.raises(TypeError, match="tok_off"):
        nk.Sequences(off, ctx, torch.zeros((1, 3), dtype=torch.int32).view(torch.uint32), 1, 1)
    with pytest.raises(ValueError, match="pages"):
        nk.Sequences(off, ctx, torch.zeros((2, 3), dtype=torch.int32).view(torch.uint32), 1, 1)
    with pytest.raises(ValueError, match="n_tok"):
        nk.Sequences(off, ctx, torch.zeros((1, 3), dtype=torch.int32).view(torch.uint32), -1, 1)
