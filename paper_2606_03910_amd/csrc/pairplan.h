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

}  // namespace pairplan
