"""The split of a differential attention of few rows, compiled for the host:
ranges cover each tile once, and what the kernels list for any offsets stays
within what the host lays out.  CPU only."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SOURCE = r"""
#include "pairplan.h"
using namespace blockplan;
using namespace pairplan;
extern "C" uint32_t len(uint32_t steps, uint32_t C) { return even_steps(steps, C); }
extern "C" uint32_t parts(uint32_t steps, uint32_t C) { return even_parts(steps, C); }
extern "C" uint32_t narrow(void) { return kNarrow; }
extern "C" int same_steps(uint32_t target, uint32_t fine, uint64_t work) {
    const Split y{1, 16, target, fine, 4, 2};
    return narrow_steps(y, (uint32_t)work) == range_steps(y, work);
}
extern "C" void plan(uint32_t n_seq, uint32_t max_pages, uint32_t btl, uint64_t n_tok, uint64_t max_tok, const uint64_t *off,
                     const uint32_t *ctx, uint32_t G, uint32_t tile_rows, uint32_t target, uint32_t fine, uint32_t least, uint64_t *out) {
    Kv a{};
    a.n_seq = n_seq; a.max_pages = max_pages; a.btl = btl; a.n_tok = n_tok;
    a.max_tok = (uint32_t)(max_tok < n_tok ? max_tok : n_tok); a.off = off; a.ctx = ctx;
    Split y{G, tile_rows, target, fine, least, 2};
    unsigned long long work = 0;
    for (int pass = 0; pass < 2; ++pass) {
        const uint32_t C = pass ? range_steps(y, work) : 0;
        uint32_t before = 0;
        for (uint32_t s = 0; s < n_seq; ++s) {
            Head h = seq_head(a, s);
            if (h.row0 < before) h.n = h.ctx = 0;
            const uint32_t e = rows_end(a, s);
            if (e > before) before = e;
            const uint32_t rt = tiles_of(h, y), kt = steps_of(h);
            if (!pass) { work += (unsigned long long)rt * kt; continue; }
            const uint32_t p = even_parts(kt, C);
            out[0] += (uint64_t)rt * p;
            if (p > 1) { out[1] += (uint64_t)rt * p; out[2] += rt; }
        }
    }
    const Caps c = caps_of(a, y);
    out[3] = c.items; out[4] = c.slots; out[5] = c.joins;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("pairs")
    (d / "pairs.cpp").write_text(_SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                           os.path.join(ROOT, "paper_2606_03910_amd", "csrc"), "-o", str(d / "pairs.so"), str(d / "pairs.cpp")])
    return ctypes.CDLL(str(d / "pairs.so"))


def test_even_ranges_cover_a_tile_once(lib):
    for C in (4, 6, 8, 40, 42, 256):
        for steps in list(range(0, 600)) + [4095, 4096, 4097, 1 << 25]:
            n, p = lib.len(steps, C), lib.parts(steps, C)
            if steps <= C:
                assert p == 1
            else:
                assert n % 2 == 0 and n <= C and p >= 2 and (p - 1) * n < steps <= p * n
                assert p <= -(-steps // C)


def test_ranges_by_32_bits(lib):
    """As by 64, up to the most that the kernels sum so: a sum that wrapped
    would name more ranges than the host makes room for."""
    rng = np.random.default_rng(0)
    most = 64 * ((1 << lib.narrow()) - 1)
    works = [0, 1, 3, 39, 40, 41, most, most - 1, most - 383] + [int(x) for x in np.exp2(rng.uniform(0, np.log2(most), 3000))]
    for work in works:
        for target, fine in ((1, 1), (1, 2), (7, 7), (320, 320), (384, 1024)):
            assert lib.same_steps(target, fine, ctypes.c_uint64(work)), (work, target, fine)


@pytest.mark.parametrize("seed", range(20))
def test_capacities_hold_for_any_offsets(lib, seed):
    rng = np.random.default_rng(seed)
    for _ in range(250):
        n_seq, n_tok = int(rng.integers(1, 40)), int(rng.integers(0, 3000))
        kind = rng.integers(0, 3)
        off = (np.sort(rng.integers(0, n_tok + 1, n_seq + 1)) if kind == 0 else rng.integers(0, n_tok + 2, n_seq + 1) if kind == 1
               else np.where(np.arange(n_seq + 1) % 2, n_tok, 0)).astype(np.uint64)
        btl = int(rng.integers(4, 11))
        max_pages = int(rng.integers(1, 1 + (1 << 18 >> btl)))
        ctx = np.minimum(np.exp(rng.uniform(0, 13, n_seq)), (max_pages << btl) + 1).astype(np.uint32)
        pairs = int(rng.choice([1, 2, 3, 4, 8, 16, 512]))
        slots = -(-512 // pairs)
        tile_rows = int(rng.choice([16, 32, 128]))
        target = slots if tile_rows == 128 else max(1, int(rng.choice([slots // 2, 5 * slots // 8, 3 * slots // 4])))
        fine = target if tile_rows == 128 else int(rng.choice([target, 2 * slots]))
        out = np.zeros(6, np.uint64)
        lib.plan(*(ctypes.c_uint32(v) for v in (n_seq, max_pages, btl)), ctypes.c_uint64(n_tok),
                 ctypes.c_uint64(int(rng.choice([n_tok, 1 + n_tok // 7]))), ctypes.c_void_p(off.ctypes.data),
                 ctypes.c_void_p(ctx.ctypes.data), ctypes.c_uint32(int(rng.choice([1, 3, 8, 64]))),
                 ctypes.c_uint32(tile_rows), ctypes.c_uint32(target), ctypes.c_uint32(fine), ctypes.c_uint32(8 if tile_rows == 128 else int(rng.choice([4, 7, 12]))),
                 ctypes.c_void_p(out.ctypes.data))
        assert out[0] <= out[3] and out[1] <= out[4] and out[2] <= out[5], (seed, out)
