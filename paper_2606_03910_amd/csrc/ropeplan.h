// How a rotation's work is laid out, and what a call may ask for: plain
// arithmetic, the same for the kernels and for the host, and compiled for the
// host alone by its test.
#pragma once

#include "blockplan.h"
#include "netkv.h"

namespace ropeplan {

constexpr uint32_t kMaxPairs = 128;

// Why a rotation of heads of `head_dim` elements cannot be; null if it can.
inline const char *rope_error(const netkv_rope_t *r, uint32_t head_dim, const uint32_t *pos, uint64_t pos_stride, uint64_t rows, bool need_pos) {
    if (!r) return "rope must not be NULL";
    if (r->rot_dim < 16 || r->rot_dim % 16 || r->rot_dim > 2 * kMaxPairs || r->rot_dim > head_dim)
        return "rot_dim must be a multiple of 16 from 16 to 256 and at most head_dim";
    if (r->n_axes < 1 || r->n_axes > 4) return "n_axes must be in [1, 4]";
    if (r->n_axes > 1 && !r->axis) return "axis must not be NULL with several axes";
    if (r->interleaved > 1) return "interleaved must be 0 or 1";
    if (r->n_pos < 1) return "n_pos must be >= 1";
    if (!r->table || (uintptr_t)r->table & 15) return "table must be 16-byte aligned and not NULL";
    if (need_pos && rows && !pos) return "pos must not be NULL";
    if (pos && r->n_axes > 1 && pos_stride < rows) return "pos_stride must be at least the rows";
    for (uint32_t i = 0; r->axis && i < r->rot_dim / 2; ++i)
        if (r->axis[i] >= r->n_axes) return "an axis must be below n_axes";
    return nullptr;
}

// A head is taken in units of two pieces of eight elements: those of eight
// pairs, then what does not turn (whose last unit may have one piece).
struct Unit {
    uint32_t lo, hi;                  // first elements
    bool turns, both;
};
NETKV_BOTH inline Unit unit_of(uint32_t u, uint32_t pairs, bool interleaved, uint32_t dim) {
    Unit x;
    x.turns = u < pairs / 8;
    if (!x.turns)
        x.lo = 2 * pairs + 16 * (u - pairs / 8);
    else
        x.lo = interleaved ? 16 * u : 8 * u;
    x.hi = x.turns && !interleaved ? x.lo + pairs : x.lo + 8;
    x.both = x.hi < dim;
    return x;
}
inline uint32_t units_of(uint32_t pairs, uint32_t dim, bool in_place) { return pairs / 8 + (in_place ? 0 : (dim - 2 * pairs + 15) / 16); }

// Heads that a thread takes with one look at its angles, their loads at once.  1,
// 2, 4, 8, us: 16,384 rows of 32 heads of 128 elements 62, 48, 48, 52, 10,007 of 16
// heads of 80 20, 16, 15, 18, 64 rows of 64 heads 10, 10, 10, 13.
constexpr uint32_t kHeadsEach = 4;

// Workgroups for a call's query rows, `chunk` at most each, all of one sequence.
NETKV_BOTH inline uint32_t row_chunks(const blockplan::Head &h, uint32_t chunk) { return h.n <= h.ctx ? (h.n + chunk - 1) / chunk : 0u; }
inline uint64_t row_groups(const blockplan::Kv &a, uint32_t chunk) {
    const uint64_t n = a.n_tok / chunk + a.n_seq;
    return n < a.n_tok ? n : a.n_tok;
}

}  // namespace ropeplan
