// How a call of the block cache's operators is split: which sequences count,
// how long the ranges of an attention are, and what its workspace has to hold.
// Plain arithmetic, the same for the kernels and for the host, and compiled
// for the host alone by its test.
#pragma once

#include <cstdint>

#ifdef __HIPCC__
#define NETKV_BOTH __host__ __device__
#else
#define NETKV_BOTH
#endif

namespace blockplan {

constexpr int kWaves = 4;
constexpr uint32_t kStep = 64;        // tokens a wavefront takes at a time

struct Kv {
    uint8_t *k, *v;
    float *ks, *vs;
    uint32_t n_pages, hk, btl;        // 2^btl tokens a block
    uint32_t n_seq, max_pages, max_tok;
    const uint64_t *off;
    const uint32_t *ctx, *pages;
    uint64_t n_tok;
    uint32_t *err;
};

struct Head {
    uint64_t row0;       // first row of the token arrays
    uint32_t n, ctx;     // rows, tokens held (rows included)
    bool rows_ok, ok;
};

// A sequence by itself.  It counts only if, besides, its rows begin at or past
// `rows_before`: then no row is two sequences', the rows of all that count are
// at most n_tok, and the capacities below hold whatever the offsets say.
// Offsets that never fall need no such look.
NETKV_BOTH inline Head seq_head(const Kv &a, uint32_t s) {
    const uint64_t b = a.off[s], e = a.off[s + 1];
    Head h;
    h.row0 = b;
    h.ctx = a.ctx[s];
    h.rows_ok = b <= e && e <= a.n_tok;
    h.ok = h.rows_ok && e - b <= a.max_tok && (uint64_t)h.ctx <= ((uint64_t)a.max_pages << a.btl);
    h.n = h.ok ? (uint32_t)(e - b) : 0u;
    if (!h.ok) h.ctx = 0;
    return h;
}

// What a sequence adds to the largest end of rows that is `rows_before` for
// those after it (n_tok is at most 2^31).
NETKV_BOTH inline uint32_t rows_end(const Kv &a, uint32_t s) {
    const uint64_t e = a.off[s + 1];
    return a.off[s] <= e && e <= a.n_tok ? (uint32_t)e : 0u;
}

struct Split {
    uint32_t G, tile_rows;
    uint32_t target, fine;            // ranges a head, with kEnough steps at most and with more
    uint32_t least, round;            // ranges of at least `least` steps, multiples of `round`
};

NETKV_BOTH inline uint32_t tiles_of(const Head &h, const Split &a) {
    return (uint32_t)(((uint64_t)h.n * a.G + a.tile_rows - 1) / a.tile_rows);
}

NETKV_BOTH inline uint32_t steps_of(const Head &h) { return (h.ctx + kStep - 1) / kStep; }

// Steps of a range: what spreads `work` steps over `target` ranges, or from
// kEnough steps on, where beginning a range costs little, over `fine`.
constexpr uint32_t kEnough = 40;
NETKV_BOTH inline uint32_t range_steps(const Split &a, unsigned long long work) {
    unsigned long long len = (work + a.target - 1) / a.target;
    const unsigned long long fine = (work + a.fine - 1) / a.fine;
    if (len > kEnough) len = fine > kEnough ? fine : kEnough;
    if (len < a.least) len = a.least;
    len = (len + a.round - 1) / a.round * a.round;
    return len > 0x7FFFFFFFull ? 0x7FFFFFFFu : (uint32_t)len;
}

// Ranges that a row tile of `steps` steps is split into.
NETKV_BOTH inline uint32_t parts_of(uint32_t steps, uint32_t C) { return steps > C ? (steps + C - 1) / C : 1u; }

// How many items, slots and joins a call can have, from the host's bounds.
// With W = sum tiles steps, a range is at least W / fine steps, so the full
// ranges (all but a tile's last) are at most `fine`; the last ones are the
// tiles.  A split tile has a full range at least: at most `fine` of them, and
// 2 fine slots.
struct Caps {
    uint64_t items, slots, joins;
};

NETKV_BOTH inline Caps caps_of(const Kv &a, const Split &s) {
    const uint64_t tiles = a.n_tok * s.G / s.tile_rows + a.n_seq;
    // no more ranges a tile than there are of the shortest length
    const uint64_t steps = (((uint64_t)a.max_pages << a.btl) + kStep - 1) / kStep, parts = (steps + s.least - 1) / s.least;
    Caps c;
    c.items = s.fine + tiles < tiles * parts ? s.fine + tiles : tiles * parts;
    c.slots = c.items < 2 * (uint64_t)s.fine ? c.items : 2 * (uint64_t)s.fine;
    c.joins = tiles < s.fine ? tiles : s.fine;
    return c;
}

// What a call with block weights may keep of its rows for them: a sum for each
// row and block (prompts) or row and unit (few rows).  Both are as wide as the
// call's longest table, whatever the sequences hold; beyond kMostKept (1.5 % of
// the memory) a second pass over the keys takes their place, which needs a
// number for each row and each head's unit only.  256 sequences, one of 131,072
// tokens and the others of 1,000, 16-token blocks, 56 rows a head: 653 us with
// 3.75 GiB of sums, 891 with the second pass.
constexpr uint64_t kMostKept = 4ull << 30;
inline uint64_t row_sum_bytes(const Kv &a, uint32_t G) { return 4ull * a.n_tok * G * a.hk * a.max_pages; }
inline uint64_t unit_bytes(const Kv &a, uint32_t n_units, uint32_t unit_rows) {
    return 4ull * a.n_seq * a.hk * n_units * unit_rows;
}

// Workgroups a head of a store, one a block that the rows touch (n rows of a
// sequence touch at most n / block + 2, and at most n), and of a read, one for
// up to kStep tokens.
NETKV_BOTH inline uint32_t stored_blocks(const Kv &a, const Head &h) {
    return h.n && h.n <= h.ctx ? ((h.ctx - 1) >> a.btl) - ((h.ctx - h.n) >> a.btl) + 1 : 0u;
}
NETKV_BOTH inline uint32_t read_steps(const Head &h) {
    return h.n && h.n <= h.ctx ? (h.ctx - 1) / kStep - (h.ctx - h.n) / kStep + 1 : 0u;
}
inline uint64_t store_groups(const Kv &a) {
    const uint64_t n = (a.n_tok >> a.btl) + 2ull * a.n_seq;
    return n < a.n_tok ? n : a.n_tok;
}
inline uint64_t read_groups(const Kv &a) {
    const uint64_t n = a.n_tok / kStep + 2ull * a.n_seq;
    return n < a.n_tok ? n : a.n_tok;
}

// A launch has less than 2^32 threads along a grid's axis.
inline bool grid_fits(uint64_t groups, uint32_t threads) { return groups <= 0xFFFFFFFFull / threads; }

// Whether two arrays of n rows of `width` 16-bit elements share one.  With
// unlike strides: whether the memory from their first to their last does.
inline bool rows_overlap(const void *p, uint64_t p_stride, const void *q, uint64_t q_stride, uint64_t width, uint64_t n) {
    if (!n || !width) return false;
    const uint64_t a = (uint64_t)(uintptr_t)p / 2, b = (uint64_t)(uintptr_t)q / 2;
    if (a + (n - 1) * p_stride + width <= b || b + (n - 1) * q_stride + width <= a) return false;
    if (p_stride != q_stride || n == 1) return true;
    const uint64_t d = a < b ? b - a : a - b, rows = d / p_stride, rest = d % p_stride;
    return (rest < width && rows < n) || (p_stride - rest < width && rows + 1 < n);
}

}  // namespace blockplan
