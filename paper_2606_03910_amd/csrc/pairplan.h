// How a differential attention of few rows is split: plain arithmetic, the same
// for the kernels and for the host, and compiled for the host alone by its test.
#pragma once

#include "blockplan.h"

namespace pairplan {

// Ranges of a row tile of `steps` steps where C is the most (range_steps):
// all of one length, a multiple of two, so that no tile leaves a short rest
// behind, which as a workgroup of its own takes nearly as long to begin and end.
NETKV_BOTH inline uint32_t even_steps(uint32_t steps, uint32_t C) {
    const uint32_t p = blockplan::parts_of(steps, C), len = (steps + p - 1) / p;
    return len + (len & 1);
}
NETKV_BOTH inline uint32_t even_parts(uint32_t steps, uint32_t C) {
    return steps > C ? (steps + even_steps(steps, C) - 1) / even_steps(steps, C) : 1u;
}

// range_steps, to a multiple of two, in 32 bits: for the sum of 64 numbers below
// 2^kNarrow each.
constexpr uint32_t kNarrow = 25;
NETKV_BOTH inline uint32_t narrow_steps(const blockplan::Split &a, uint32_t work) {
    uint32_t len = (work + a.target - 1) / a.target;
    if (len > blockplan::kEnough) {
        len = (work + a.fine - 1) / a.fine;
        len = len > blockplan::kEnough ? len : blockplan::kEnough;
    }
    len = len > a.least ? len : a.least;
    return len + (len & 1);
}

}  // namespace pairplan
