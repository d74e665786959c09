"""Rotary positions without a GPU: the plain form by hand, how a call's work is
laid out (compiled for the host), what is refused."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from tests import rope_ref as T

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SOURCE = r"""
#include "ropeplan.h"
using namespace ropeplan;
extern "C" void unit(uint32_t u, uint32_t pairs, int interleaved, uint32_t dim, uint32_t *out) {
    const Unit x = unit_of(u, pairs, interleaved, dim);
    out[0] = x.lo; out[1] = x.hi; out[2] = x.turns; out[3] = x.both;
}
extern "C" uint32_t units(uint32_t pairs, uint32_t dim, int in_place) { return units_of(pairs, dim, in_place); }
extern "C" const char *error(const netkv_rope_t *r, uint32_t dim, const uint32_t *pos, uint64_t stride, uint64_t rows, int need) {
    return rope_error(r, dim, pos, stride, rows, need);
}
extern "C" void chunks(uint32_t n_seq, uint64_t n_tok, uint64_t max_tok, const uint64_t *off, const uint32_t *ctx, uint32_t chunk, uint64_t *out) {
    blockplan::Kv a{};
    a.n_seq = n_seq; a.max_pages = 1 << 20; a.btl = 4; a.n_tok = n_tok;
    a.max_tok = (uint32_t)(max_tok < n_tok ? max_tok : n_tok); a.off = off; a.ctx = ctx;
    uint32_t before = 0;
    for (uint32_t s = 0; s < n_seq; ++s) {
        blockplan::Head h = blockplan::seq_head(a, s);
        if (h.row0 < before) h.n = h.ctx = 0;
        const uint32_t e = blockplan::rows_end(a, s);
        if (e > before) before = e;
        out[0] += row_chunks(h, chunk);
    }
    out[1] = row_groups(a, chunk);
}
extern "C" int overlap(uint64_t p, uint64_t ps, uint64_t pw, uint64_t q, uint64_t qs, uint64_t qw, uint64_t n) {
    return blockplan::rows_overlap((void *)(uintptr_t)p, ps, pw, (void *)(uintptr_t)q, qs, qw, n);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("rope")
    (d / "rope.cpp").write_text(_SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2606_03910_amd", "csrc"), "-I", os.path.join(ROOT, "include"), "-o",
                           str(d / "rope.so"), str(d / "rope.cpp")])
    x = ctypes.CDLL(str(d / "rope.so"))
    x.error.restype = ctypes.c_char_p
    return x


def test_rotate_by_hand():
    rng = np.random.default_rng(0)
    tab = T.table(9, 16, rng)
    x = rng.standard_normal((2, 1, 24))
    y = T.rotate(x, tab, [[3, 8], [0, 5]], T.axes(16, 2, True), False)
    for r, pos in ((0, (3, 0)), (1, (8, 5))):
        for i in range(8):
            c, s = float(tab[pos[i % 2], i]), float(tab[pos[i % 2], 8 + i])
            z = complex(x[r, 0, i], x[r, 0, 8 + i]) * complex(c, s)
            assert abs(z - complex(y[r, 0, i], y[r, 0, 8 + i])) < 1e-14
    assert np.array_equal(y[..., 16:], x[..., 16:])
    z = T.rotate(x, tab, [[3, 8]], [0] * 8, True)
    assert abs(z[1, 0, 5] - (x[1, 0, 5] * float(tab[8, 2]) + x[1, 0, 4] * float(tab[8, 10]))) < 1e-14


def test_transpose_is_the_gradient():
    """<rotate(x), g> = <x, transposed(g)>, and differences of it."""
    rng = np.random.default_rng(1)
    tab = T.table(9, 32, rng, scale=1.7)
    x, g = rng.standard_normal((2, 3, 2, 40))
    pos, ax = rng.integers(0, 9, (3, 3)), T.axes(32, 3, False)
    for inter in (False, True):
        y, d = T.rotate(x, tab, pos, ax, inter), T.rotate(g, tab, pos, ax, inter, transpose=True)
        assert abs((y * g).sum() - (x * d).sum()) < 1e-12
        e = np.zeros_like(x)
        e[1, 1, 7] = 1e-3
        diff = ((T.rotate(x + e, tab, pos, ax, inter) - T.rotate(x - e, tab, pos, ax, inter)) * g).sum() / 2e-3
        assert abs(diff - d[1, 1, 7]) < 1e-10


@pytest.mark.parametrize("in_place", [False, True])
def test_units_cover_a_head_once(lib, in_place):
    out = (ctypes.c_uint32 * 4)()
    for dim in range(16, 1025, 8):
        for rot in range(16, min(dim, 256) + 1, 16):
            for inter in (0, 1):
                seen = np.zeros(dim, int)
                for u in range(lib.units(rot // 2, dim, int(in_place))):
                    lib.unit(u, rot // 2, inter, dim, out)
                    lo, hi, turns, both = list(out)
                    assert both or not turns
                    assert turns == (u < rot // 16)
                    if turns and inter:
                        assert (lo, hi) == (16 * u, 16 * u + 8)
                    elif turns:
                        assert (lo, hi) == (8 * u, 8 * u + rot // 2)
                    for p in (lo, hi)[:1 + both]:
                        assert p % 8 == 0 and p + 8 <= dim
                        seen[p:p + 8] += 1
                assert (seen[:rot] == 1).all() and (seen[rot:] == (0 if in_place else 1)).all()


@pytest.mark.parametrize("seed", range(10))
def test_row_chunks_within_their_workgroups(lib, seed):
    rng = np.random.default_rng(seed)
    for _ in range(200):
        n_seq, n_tok = int(rng.integers(1, 40)), int(rng.integers(0, 3000))
        off = rng.integers(0, n_tok + 2, n_seq + 1) if rng.integers(0, 2) else np.sort(rng.integers(0, n_tok + 1, n_seq + 1))
        off = off.astype(np.uint64)
        ctx = rng.integers(0, 4000, n_seq).astype(np.uint32)
        out = np.zeros(2, np.uint64)
        lib.chunks(ctypes.c_uint32(n_seq), ctypes.c_uint64(n_tok), ctypes.c_uint64(int(rng.choice([n_tok, n_tok // 3]))),
                   ctypes.c_void_p(off.ctypes.data), ctypes.c_void_p(ctx.ctypes.data), ctypes.c_uint32(int(rng.choice([1, 16]))),
                   ctypes.c_void_p(out.ctypes.data))
        assert out[0] <= out[1]


def test_overlap_of_rows_of_unlike_widths(lib):
    """Against the elements themselves, for rows of one stride; the whole
    ranges for others."""
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(4000):
        n, stride = int(rng.integers(0, 6)), int(rng.integers(12, 36))
        pw, qw = (int(x) for x in rng.integers(1, 12, 2))
        qs = stride if rng.integers(0, 4) else stride + int(rng.integers(1, 9))
        p, q = (int(x) for x in rng.integers(0, 160, 2))
        rows = [{a + i * s + e for i in range(n) for e in range(w)} for a, s, w in ((p, stride, pw), (q, qs, qw))]
        if stride == qs:
            want = bool(rows[0] & rows[1])
        else:
            want = n > 0 and max(p, q) <= min(max(rows[0]), max(rows[1]))
        got = bool(lib.overlap(*(ctypes.c_uint64(x) for x in (2 * p, stride, pw, 2 * q, qs, qw, n))))
        assert got == want, (p, stride, pw, q, qs, qw, n)
        seen[got] += 1
    assert min(seen) > 500


def test_refusals_on_the_host(lib):
    from paper_2606_03910_amd import netkv as nk
    axes = (ctypes.c_uint8 * 64)(*([0, 1, 2, 1] * 16))

    def why(dim=128, pos=16, stride=10, rows=10, need=1, **kw):
        f = dict(rot_dim=128, n_pos=5, n_axes=1, interleaved=0, table=256, axis=None)
        f.update(kw)
        r = lib.error(ctypes.byref(nk.netkv_rope_t(**f)), ctypes.c_uint32(dim), ctypes.c_void_p(pos), ctypes.c_uint64(stride),
                      ctypes.c_uint64(rows), ctypes.c_int(need))
        return r.decode() if r else None

    at = ctypes.addressof(axes)
    assert why() is None and why(n_axes=3, axis=at) is None and why(pos=None, need=0) is None and why(pos=None, rows=0) is None
    for bad in (dict(rot_dim=0), dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=144), dict(rot_dim=272, dim=1024)):
        assert "rot_dim" in why(**bad), bad
    assert "n_axes" in why(n_axes=0) and "n_axes" in why(n_axes=5, axis=at)
    assert "axis" in why(n_axes=2) and "below n_axes" in why(n_axes=2, axis=at)
    assert "interleaved" in why(interleaved=2) and "n_pos" in why(n_pos=0)
    assert "table" in why(table=None) and "table" in why(table=264)
    assert "pos" in why(pos=None) and "pos_stride" in why(n_axes=3, axis=at, stride=9)
    assert lib.error(None, 128, None, 0, 0, 0) == b"rope must not be NULL"


def test_binding_refuses_without_a_gpu():
    from types import SimpleNamespace

    from paper_2606_03910_amd import netkv as nk
    sel = SimpleNamespace(h=None, device=torch.device("cuda:0"))
    with pytest.raises(TypeError, match="table"):
        nk.Rope(sel, torch.zeros((4, 128)))
    assert nk._positions(None, nk.netkv_rope_t(n_axes=1), 3, sel.device) == (None, 0)
    with pytest.raises(TypeError, match="pos"):
        nk._positions(torch.zeros(3, dtype=torch.int32), nk.netkv_rope_t(n_axes=1), 3, sel.device)


def test_differential_attention_by_hand():
    """Against a loop over tokens, with the norm."""
    from tests import blockcache_ref as R
    from tests import diff_ref as F
    rng = np.random.default_rng(3)
    c = R.Cache(3, 2, 64, 16, rng)
    c.put(2, 16)
    c.put(0, 2)
    q, lam, norm = rng.standard_normal((2, 4, 64)), np.array([0.4, -0.2]), rng.standard_normal(128)
    for nm in (None, norm):
        o, tol = F.attend(c, np.array([[2, 0]]), [18], [2], q, 0.125, lam, nm, 1e-3, 0.7)
        for t, seen in ((0, 17), (1, 18)):
            for j in range(2):
                d = np.zeros(128)
                for m, f in ((0, 1.0), (1, -lam[j])):
                    e, acc = [], np.zeros(128)
                    for i in range(seen):
                        pg, sl = ((2, i) if i < 16 else (0, i - 16))
                        k = R.values(c.k[pg, m, sl]) * c.ks[pg, m]
                        v = np.concatenate([R.values(c.v[pg, h, sl]) * c.vs[pg, h] for h in range(2)])
                        e.append(np.exp(0.125 * (q[t, 2 * j + m] @ k)))
                        acc += e[-1] * v
                    d += f * acc / sum(e)
                if nm is not None:
                    d = d / np.sqrt((d * d).mean() + 1e-3) * nm
                assert np.allclose(o[t, j], 0.7 * d, rtol=1e-11, atol=1e-13) and (tol[t, j] > 0).all()
