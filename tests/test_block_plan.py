"""The split of a block cache call, compiled for the host: what the kernels
list for any offsets stays within what the host lays out.  CPU only."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Items, slots and joins of a call (with `look`, sequences that begin among
# rows of an earlier one left out, as the kernels do) and their capacities.
_SOURCE = r"""
#include "blockplan.h"
using namespace blockplan;
extern "C" void plan(uint32_t n_seq, uint32_t max_pages, uint32_t btl, uint64_t n_tok, uint64_t max_tok, const uint64_t *off,
                     const uint32_t *ctx, uint32_t G, uint32_t tile_rows, uint32_t target, uint32_t fine, uint32_t least,
                     uint32_t round, int look, uint64_t *out) {
    Kv a{};
    a.n_seq = n_seq; a.max_pages = max_pages; a.btl = btl; a.n_tok = n_tok;
    a.max_tok = (uint32_t)(max_tok < n_tok ? max_tok : n_tok); a.off = off; a.ctx = ctx;
    Split y{G, tile_rows, target, fine, least, round};
    unsigned long long work = 0;
    uint64_t rows = 0;
    for (int pass = 0; pass < 2; ++pass) {
        const uint32_t C = pass ? range_steps(y, work) : 0;
        uint32_t before = 0;
        for (uint32_t s = 0; s < n_seq; ++s) {
            Head h = seq_head(a, s);
            if (look && h.row0 < before) h.n = h.ctx = 0;
            const uint32_t e = rows_end(a, s);
            if (e > before) before = e;
            const uint32_t rt = tiles_of(h, y), kt = steps_of(h);
            if (!pass) { work += (unsigned long long)rt * kt; rows += h.n; continue; }
            const uint32_t p = parts_of(kt, C);
            out[0] += (uint64_t)rt * p;
            if (p > 1) { out[1] += (uint64_t)rt * p; out[2] += rt; }
        }
    }
    const Caps c = caps_of(a, y);
    out[3] = c.items; out[4] = c.slots; out[5] = c.joins; out[6] = rows;
    uint32_t before = 0;
    for (uint32_t s = 0; s < n_seq; ++s) {
        Head h = seq_head(a, s);
        if (look && h.row0 < before) h.n = h.ctx = 0;
        const uint32_t e = rows_end(a, s);
        if (e > before) before = e;
        out[7] += stored_blocks(a, h);
        out[8] += read_steps(h);
    }
    out[9] = store_groups(a); out[10] = read_groups(a);
}
extern "C" int fits(uint64_t groups, uint32_t threads) { return grid_fits(groups, threads); }
extern "C" int overlap(uint64_t p, uint64_t ps, uint64_t q, uint64_t qs, uint64_t width, uint64_t n) {
    return rows_overlap((void *)(uintptr_t)p, ps, (void *)(uintptr_t)q, qs, width, n);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(_SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2606_03910_amd", "csrc"), "-o", str(d / "plan.so"), str(d / "plan.cpp")])
    return ctypes.CDLL(str(d / "plan.so"))


@pytest.fixture(scope="module")
def plan(lib):
    def run(off, ctx, n_tok, max_tok, max_pages, btl, G, tile_rows, target, fine, least, rnd, look=True):
        off, ctx, out = np.asarray(off, np.uint64), np.asarray(ctx, np.uint32), np.zeros(11, np.uint64)
        lib.plan(ctypes.c_uint32(len(ctx)), ctypes.c_uint32(max_pages), ctypes.c_uint32(btl), ctypes.c_uint64(n_tok),
                 ctypes.c_uint64(max_tok), ctypes.c_void_p(off.ctypes.data), ctypes.c_void_p(ctx.ctypes.data),
                 *(ctypes.c_uint32(x) for x in (G, tile_rows, target, fine, least, rnd)), ctypes.c_int(look),
                 ctypes.c_void_p(out.ctypes.data))
        return [int(x) for x in out]

    return run


def within(r):
    return r[0] <= r[3] and r[1] <= r[4] and r[2] <= r[5] and r[7] <= r[9] and r[8] <= r[10]


@pytest.mark.parametrize("off,ctx,args", [
    # rows named four times over; 8 KV heads, blocks of 512 tokens
    ([0, 128, 0, 128, 0, 128, 0, 128], [2048] * 7, (128, 128, 4, 9, 8, 256, 64, 64, 8, 8)),
    ([0, 20, 0, 20, 0, 20], [512] * 5, (20, 20, 1, 9, 8, 32, 64, 128, 4, 4)),
])
def test_rows_of_two_sequences_count_once(plan, off, ctx, args):
    """Sequences that each are right by themselves but name the same rows
    would pass the slots if they all counted."""
    n_tok = args[0]
    every, once = plan(off, ctx, *args, look=False), plan(off, ctx, *args)
    assert every[1] > every[4] and every[6] > n_tok
    assert within(once) and once[6] == n_tok


@pytest.mark.parametrize("seed", range(40))
def test_capacities_hold_for_any_offsets(plan, seed):
    rng = np.random.default_rng(seed)
    for _ in range(250):
        n_seq = int(rng.integers(1, 40))
        n_tok = int(rng.integers(0, 3000))
        kind = rng.integers(0, 4)
        if kind == 0:
            off = np.sort(rng.integers(0, n_tok + 1, n_seq + 1))
        elif kind == 1:
            off = rng.integers(0, n_tok + 2, n_seq + 1)
        elif kind == 2:
            off = np.where(np.arange(n_seq + 1) % 2, n_tok, 0)
        else:
            off = np.sort(rng.integers(0, n_tok + 1, n_seq + 1))
            off[rng.integers(0, n_seq + 1, 3)] = rng.integers(0, 1 << 40, 3)
        btl = int(rng.integers(4, 11))
        max_pages = int(rng.integers(1, 1 + (1 << 17 >> btl)))
        ctx = np.minimum(np.exp(rng.uniform(0, 12, n_seq)), (max_pages << btl) + 1).astype(np.uint32)
        max_tok = int(rng.choice([n_tok, n_tok // 2, 1 + n_tok // 7]))
        hk, prompt = int(rng.choice([1, 2, 5, 8, 32, 700])), bool(rng.integers(0, 2))
        target = -(-512 // hk)
        fine = target if prompt else int(rng.choice([target, -(-1024 // hk)]))
        rnd = max(1, (1 << btl) // 64) if prompt else 4
        r = plan(off, ctx, n_tok, max_tok, max_pages, btl, int(rng.choice([1, 3, 8, 64])),
                 int(rng.choice([128, 256]) if prompt else rng.choice([16, 32])), target, fine, 8 if prompt else 4, rnd)
        assert within(r) and r[6] <= n_tok, (seed, off, r)


def test_overlap_of_rows(lib):
    """Against the elements themselves, for rows of one stride; the whole
    ranges for others."""
    rng = np.random.default_rng(0)
    seen = [0, 0]
    for _ in range(4000):
        width, n = int(rng.integers(1, 12)), int(rng.integers(0, 6))
        ps = width + int(rng.integers(0, 25))
        qs = ps if rng.integers(0, 4) else width + int(rng.integers(0, 25))
        p, q = (int(x) for x in rng.integers(0, 160, 2))
        rows = [{a + i * s + e for i in range(n) for e in range(width)} for a, s in ((p, ps), (q, qs))]
        if ps == qs:
            want = bool(rows[0] & rows[1])
        else:
            want = n > 0 and max(p, q) <= min(max(rows[0]), max(rows[1]))
        got = bool(lib.overlap(*(ctypes.c_uint64(x) for x in (2 * p, ps, 2 * q, qs, width, n))))
        assert got == want, (p, ps, q, qs, width, n)
        seen[got] += 1
    assert min(seen) > 500


def test_grids_of_less_than_2_32_threads(lib):
    for threads in (256, 512, 1024):
        most = (1 << 32) // threads - 1                    # 2^32 threads are one workgroup more
        assert lib.fits(ctypes.c_uint64(most), ctypes.c_uint32(threads))
        assert not lib.fits(ctypes.c_uint64(most + 1), ctypes.c_uint32(threads))
        assert not lib.fits(ctypes.c_uint64(1 << 40), ctypes.c_uint32(threads))
