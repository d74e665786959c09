// Eviction from the resident sets by accumulated attention weight, for
// MI355X (gfx950): every segment (a decode instance's resident blocks, or a
// sequence's) keeps its `keep` heaviest entries, ties to the lowest index, in
// their order.
//
// The threshold of a segment, its keep-th largest weight, is found digit by
// digit from counts (weights are 64-bit integers, so a digit's counts say
// exactly which digit the threshold has), never by sorting:
//   plan_kernel      -- offsets of the kept entries; the long segments' chunks.
//   small_kernel     -- a segment of up to 4,096 entries in one workgroup's
//                       registers, one read of everything.
//   long segments, in chunks of 16,384 entries:
//   count_kernel     -- counts by power of two and 5 bits below it.
//   gather_kernel    -- the weights that share the threshold's count.
//   threshold_kernel -- the threshold among them; where each chunk's kept go.
//   write_kernel     -- the kept entries.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "netkv.h"
#include "netkv_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPlanThreads = 1024;
constexpr uint32_t kEach = 16;                     // entries a thread of small_kernel keeps
constexpr uint32_t kSmall = kThreads * kEach;      // longest segment of small_kernel
constexpr uint32_t kChunk = 16384;
constexpr uint32_t kBins = 2048;

struct Seg {
    uint64_t first;      // entry
    uint32_t n, keep;
};

struct Chunk {
    uint32_t seg, large, first, n;   // segment, its place among the long ones, first entry within it, entries
};

struct LongSeg {
    uint32_t seg, chunk0, chunks, pad;
    uint64_t prefix;                 // a weight stays if (w >> shift) > prefix, or
    uint32_t shift, need;            // equal to it and among the first `need` of those
};

struct EvictArgs {
    uint32_t n_seg, newest;
    const uint64_t *off, *weight, *hashes;
    const uint32_t *keep;
    uint64_t n, n_out;
    uint64_t *out_off, *out_hashes;
    uint32_t *out_pos;
    uint32_t *err;
    // workspace
    uint32_t *counts;                // [0] chunks, [1] long segments, [2] whether the offsets are good
    Chunk *chunks;
    LongSeg *longs;
    uint32_t *hist;                  // [long][kBins]
    uint2 *chunk_counts;             // above the bin, within it; then the kept before, the ties before
    uint64_t *cand;                  // [n]: each chunk's weights within the bin, from its first entry
    uint32_t chunk_cap, long_cap;
};

__device__ inline Seg seg_at(const EvictArgs &a, uint32_t s, bool good) {
    Seg g;
    g.first = a.off[s];
    g.n = good ? (uint32_t)(a.off[s + 1] - g.first) : 0u;
    g.keep = min(a.keep[s], g.n);
    return g;
}
__device__ inline Seg seg_at(const EvictArgs &a, uint32_t s) { return seg_at(a, s, a.counts[2] != 0); }

// The weight that counts: the last `newest` of those that may stay (and no
// more than those) come before everything.
__device__ inline uint64_t key_of(const EvictArgs &a, const Seg &g, uint32_t i, uint64_t w) {
    return i >= g.n - min(a.newest, g.keep) ? ~0ull : w == ~0ull ? ~0ull - 1 : w;
}

// Monotone: below 32 the weight itself, else its power of two and 5 bits.
__device__ inline uint32_t bin_of(uint64_t w) {
    if (w < 32) return (uint32_t)w;
    const uint32_t e = 63 - __clzll((long long)w);
    return ((e - 4) << 5) | ((uint32_t)(w >> (e - 5)) & 31u);
}

__device__ inline void put(const EvictArgs &a, const Seg &g, uint64_t at, uint32_t i) {
    if (at >= a.n_out) return;
    if (a.out_pos) a.out_pos[at] = i;
    if (a.out_hashes) a.out_hashes[at] = a.hashes[g.first + i];
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(EvictArgs a) {
    __shared__ uint64_t sums[kPlanThreads / 64][3];
    __shared__ uint32_t bad;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < a.n_seg; s += kPlanThreads)
        if (a.off[s] > a.off[s + 1] || a.off[s + 1] > a.n) bad = 1;
    __syncthreads();
    const bool good = !bad;   // else every segment counts as empty
    uint64_t at[3] = {0, 0, 0};   // kept, chunks, long segments so far
    for (uint32_t s0 = 0; s0 < a.n_seg; s0 += kPlanThreads) {
        const uint32_t s = s0 + threadIdx.x;
        Seg g{0, 0, 0};
        if (s < a.n_seg) g = seg_at(a, s, good);
        const bool big = g.n > kSmall;
        const uint32_t nc = big ? (g.n + kChunk - 1) / kChunk : 0u;
        uint64_t x[3] = {g.keep, nc, big ? 1u : 0u}, in[3];
        for (int i = 0; i < 3; ++i) {
            uint64_t y = x[i];
            for (int d = 1; d < 64; d <<= 1) {
                const uint64_t z = __shfl_up((unsigned long long)y, d, 64);
                if (lane >= d) y += z;
            }
            in[i] = y;
            if (lane == 63) sums[w][i] = y;
        }
        __syncthreads();
        uint64_t tot[3];
        for (int i = 0; i < 3; ++i) {
            uint64_t before = 0, all = 0;
            for (int v = 0; v < kPlanThreads / 64; ++v) {
                if (v < w) before += sums[v][i];
                all += sums[v][i];
            }
            x[i] = at[i] + before + in[i] - x[i];
            tot[i] = all;
        }
        if (s < a.n_seg) {
            a.out_off[s] = x[0];
            if (big && x[2] < a.long_cap && x[1] + nc <= a.chunk_cap) {
                a.longs[x[2]] = LongSeg{s, (uint32_t)x[1], nc, 0, 0, 0, 0};
                for (uint32_t i = 0; i < nc; ++i)
                    a.chunks[x[1] + i] = Chunk{s, (uint32_t)x[2], i * kChunk, min(kChunk, g.n - i * kChunk)};
            }
        }
        for (int i = 0; i < 3; ++i) at[i] += tot[i];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.out_off[a.n_seg] = at[0];
        if (!good || at[0] > a.n_out) atomicOr(a.err, kErrEntryBit);
        a.counts[0] = (uint32_t)min(at[1], (uint64_t)a.chunk_cap);
        a.counts[1] = (uint32_t)min(at[2], (uint64_t)a.long_cap);
        a.counts[2] = good;
    }
}

// The bin of the `rest`-th from the top, and what is left of `rest` in it.
// `hist` holds 64 * PER counts; one wavefront, every lane gets the answer.
template <int PER, typename F>
__device__ inline void find_bin(F hist, uint32_t &rest, uint32_t &bin, uint32_t &in_bin) {
    const int lane = threadIdx.x & 63;
    uint32_t mine = 0;
    for (int i = 0; i < PER; ++i) mine += hist(lane * PER + i);
    uint32_t above = mine;   // counts of this lane's bins and the higher lanes'
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t z = __shfl_down(above, d, 64);
        if (lane + d < 64) above += z;
    }
    const uint64_t has = __ballot(above >= rest);   // lane 0 .. the lane of the bin
    const int l = 63 - __clzll((long long)has);
    uint32_t left = rest - (above - mine), b = 0, c = 0;
    if (lane == l)
        for (int i = PER - 1; i >= 0; --i) {
            c = hist(lane * PER + i);
            b = lane * PER + i;
            if (left <= c) break;
            left -= c;
        }
    rest = __shfl(left, l, 64);
    bin = __shfl(b, l, 64);
    in_bin = __shfl(c, l, 64);
}

__global__ __launch_bounds__(kThreads) void small_kernel(EvictArgs a) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[3];
    __shared__ uint64_t differ[kWaves];
    __shared__ uint32_t cg[kEach * kWaves], ce[kEach * kWaves];
    const Seg g = seg_at(a, blockIdx.x);
    if (g.n > kSmall || g.keep == 0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t out = a.out_off[blockIdx.x];
    if (g.keep == g.n) {
        for (uint32_t i = threadIdx.x; i < g.n; i += kThreads) put(a, g, out + i, i);
        return;
    }
    uint64_t k[kEach];
    const uint64_t one = key_of(a, g, 0, a.weight[g.first]);
    uint64_t d = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kThreads + threadIdx.x;
        k[i] = e < g.n ? key_of(a, g, e, a.weight[g.first + e]) : one;
        d |= k[i] ^ one;
    }
    for (int i = 32; i; i >>= 1) d |= (uint64_t)__shfl_xor((unsigned long long)d, i, 64);
    if (lane == 0) differ[w] = d;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) d |= differ[i];
    // bits above `shift` of the threshold are `prefix`
    uint32_t shift = d ? 64 - __clzll((long long)d) : 0u, need = g.keep;
    uint64_t prefix = shift < 64 ? one >> shift : 0ull;
    while (shift) {
        const uint32_t by = min(shift, 8u);
        hist[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t e = i * kThreads + threadIdx.x;
            if (e < g.n && (shift < 64 ? k[i] >> shift : 0ull) == prefix)
                atomicAdd(&hist[(uint32_t)(k[i] >> (shift - by)) & ((1u << by) - 1)], 1u);
        }
        __syncthreads();
        if (w == 0) {
            uint32_t rest = need, bin, c;
            find_bin<4>([&](uint32_t i) { return hist[i]; }, rest, bin, c);
            if (lane == 0) {
                found[0] = bin;
                found[1] = rest;
                found[2] = c;
            }
        }
        __syncthreads();
        shift -= by;
        prefix = (prefix << by) | found[0];
        need = found[1];
        if (need == found[2]) break;   // all of them stay
    }
    uint64_t mg[kEach], me[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kThreads + threadIdx.x;
        const uint64_t p = shift < 64 ? k[i] >> shift : 0ull;
        mg[i] = __ballot(e < g.n && p > prefix);
        me[i] = __ballot(e < g.n && p == prefix);
        if (lane == 0) {
            cg[i * kWaves + w] = __popcll(mg[i]);
            ce[i * kWaves + w] = __popcll(me[i]);
        }
    }
    __syncthreads();
    if (w == 0) {   // kEach * kWaves = 64 counts, one a lane
        uint32_t x = cg[lane], y = ce[lane];
        const uint32_t x0 = x, y0 = y;
        for (int i = 1; i < 64; i <<= 1) {
            const uint32_t p = __shfl_up(x, i, 64), q = __shfl_up(y, i, 64);
            if (lane >= i) {
                x += p;
                y += q;
            }
        }
        cg[lane] = x - x0;
        ce[lane] = y - y0;
    }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t ng = cg[i * kWaves + w] + __popcll(mg[i] & below), ne = ce[i * kWaves + w] + __popcll(me[i] & below);
        const bool stays = (mg[i] >> lane & 1) || ((me[i] >> lane & 1) && ne < need);
        if (stays) put(a, g, out + ng + min(ne, need), i * kThreads + threadIdx.x);
    }
}

__global__ __launch_bounds__(kThreads) void clear_kernel(EvictArgs a) {
    const uint64_t n = (uint64_t)a.counts[1] * kBins;
    for (uint64_t i = blockIdx.x * (uint64_t)kThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kThreads) a.hist[i] = 0;
}

__global__ __launch_bounds__(kThreads) void count_kernel(EvictArgs a) {
    __shared__ uint32_t hist[kBins];
    if (blockIdx.x >= a.counts[0]) return;
    const Chunk c = a.chunks[blockIdx.x];
    const Seg g = seg_at(a, c.seg);
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    const uint64_t *wt = a.weight + g.first;
    for (uint32_t i = threadIdx.x; i < c.n; i += kThreads) {
        const uint32_t e = c.first + i;
        atomicAdd(&hist[bin_of(key_of(a, g, e, wt[e]))], 1u);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads)
        if (hist[i]) atomicAdd(&a.hist[(uint64_t)c.large * kBins + i], hist[i]);
}

__global__ __launch_bounds__(kThreads) void gather_kernel(EvictArgs a) {
    __shared__ uint32_t found[2], n_in[kWaves], above;
    if (blockIdx.x >= a.counts[0]) return;
    const Chunk c = a.chunks[blockIdx.x];
    const Seg g = seg_at(a, c.seg);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (g.keep == 0) return;
    if (threadIdx.x == 0) above = 0;
    if (w == 0) {
        const uint32_t *h = a.hist + (uint64_t)c.large * kBins;
        uint32_t rest = g.keep, bin, in;
        find_bin<kBins / 64>([&](uint32_t i) { return h[i]; }, rest, bin, in);
        if (lane == 0) {
            found[0] = bin;
            found[1] = rest;
        }
    }
    __syncthreads();
    const uint32_t bin = found[0];
    const uint64_t *wt = a.weight + g.first;
    uint64_t *cand = a.cand + g.first + c.first;
    uint32_t at = 0, up = 0;
    for (uint32_t i0 = 0; i0 < c.n; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x, e = c.first + i;
        const uint64_t k = i < c.n ? key_of(a, g, e, wt[e]) : 0ull;
        const uint32_t b = i < c.n ? bin_of(k) : 0u;
        const bool in = i < c.n && b == bin;
        up += i < c.n && b > bin;
        const uint64_t m = __ballot(in);
        if (lane == 0) n_in[w] = __popcll(m);
        __syncthreads();
        uint32_t before = at, all = 0;
        for (int v = 0; v < kWaves; ++v) {
            if (v < w) before += n_in[v];
            all += n_in[v];
        }
        if (in) cand[before + __popcll(m & ((1ull << lane) - 1))] = k;
        at += all;
        __syncthreads();
    }
    for (int d = 32; d; d >>= 1) up += __shfl_xor(up, d, 64);
    if (lane == 0) atomicAdd(&above, up);
    __syncthreads();
    if (threadIdx.x == 0) {
        a.chunk_counts[blockIdx.x] = make_uint2(above, at);
        if (c.first == 0) {
            // the bin's weights share what is above `shift`
            LongSeg &l = a.longs[c.large];
            const uint32_t sh = bin < 32 ? 0u : (bin >> 5) - 1;
            l.shift = sh;
            l.prefix = bin < 32 ? bin : 32u | (bin & 31u);
            l.need = found[1];
        }
    }
}

__global__ __launch_bounds__(kThreads) void threshold_kernel(EvictArgs a) {
    __shared__ uint32_t hist[256], found[3], carry[2], cw[kWaves][2];
    if (blockIdx.x >= a.counts[1]) return;
    const LongSeg l = a.longs[blockIdx.x];
    const Seg g = seg_at(a, l.seg);
    if (g.keep == 0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t *cand = a.cand + g.first;
    uint32_t shift = l.shift, need = l.need;
    uint64_t prefix = l.prefix;
    uint32_t all = 0;
    for (uint32_t c = threadIdx.x; c < l.chunks; c += kThreads) all += a.chunk_counts[l.chunk0 + c].y;
    for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d, 64);
    if (lane == 0) cw[w][0] = all;
    __syncthreads();
    all = 0;
    for (int v = 0; v < kWaves; ++v) all += cw[v][0];
    while (shift && need != all) {
        const uint32_t by = min(shift, 8u);
        hist[threadIdx.x] = 0;
        __syncthreads();
        // a wavefront a chunk
        for (uint32_t c = w; c < l.chunks; c += kWaves) {
            const uint32_t m = a.chunk_counts[l.chunk0 + c].y;
            for (uint32_t i = lane; i < m; i += 64) {
                const uint64_t k = cand[(uint64_t)c * kChunk + i];
                if (k >> shift == prefix) atomicAdd(&hist[(uint32_t)(k >> (shift - by)) & ((1u << by) - 1)], 1u);
            }
        }
        __syncthreads();
        if (w == 0) {
            uint32_t rest = need, bin, in;
            find_bin<4>([&](uint32_t i) { return hist[i]; }, rest, bin, in);
            if (lane == 0) {
                found[0] = bin;
                found[1] = rest;
                found[2] = in;
            }
        }
        __syncthreads();
        shift -= by;
        prefix = (prefix << by) | found[0];
        need = found[1];
        all = found[2];
        __syncthreads();
    }
    // where each chunk's kept entries and ties begin
    if (threadIdx.x == 0) carry[0] = carry[1] = 0;
    __syncthreads();
    for (uint32_t c0 = 0; c0 < l.chunks; c0 += kWaves) {
        const uint32_t c = c0 + w;
        uint32_t ng = 0, ne = 0;
        if (c < l.chunks) {
            const uint2 n = a.chunk_counts[l.chunk0 + c];
            for (uint32_t i = lane; i < n.y; i += 64) {
                const uint64_t p = cand[(uint64_t)c * kChunk + i] >> shift;
                ng += p > prefix;
                ne += p == prefix;
            }
            for (int d = 32; d; d >>= 1) {
                ng += __shfl_xor(ng, d, 64);
                ne += __shfl_xor(ne, d, 64);
            }
            ng += n.x;
        }
        if (lane == 0) {
            cw[w][0] = ng;
            cw[w][1] = ne;
        }
        __syncthreads();
        uint32_t bg = carry[0], be = carry[1];
        for (int v = 0; v < w; ++v) {
            bg += cw[v][0];
            be += cw[v][1];
        }
        __syncthreads();
        if (lane == 0 && c < l.chunks) a.chunk_counts[l.chunk0 + c] = make_uint2(bg, be);
        if (threadIdx.x == 0)
            for (int v = 0; v < kWaves; ++v) {
                carry[0] += cw[v][0];
                carry[1] += cw[v][1];
            }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.longs[blockIdx.x].shift = shift;
        a.longs[blockIdx.x].prefix = prefix;
        a.longs[blockIdx.x].need = need;
    }
}

__global__ __launch_bounds__(kThreads) void write_kernel(EvictArgs a) {
    __shared__ uint32_t cw[kWaves][2];
    if (blockIdx.x >= a.counts[0]) return;
    const Chunk c = a.chunks[blockIdx.x];
    const LongSeg l = a.longs[c.large];
    const Seg g = seg_at(a, c.seg);
    if (g.keep == 0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t out = a.out_off[c.seg], below = (1ull << lane) - 1;
    const uint64_t *wt = a.weight + g.first;
    const uint2 start = a.chunk_counts[blockIdx.x];
    uint32_t ng = start.x, ne = start.y;
    for (uint32_t i0 = 0; i0 < c.n; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x, e = c.first + i;
        const uint64_t p = i < c.n ? key_of(a, g, e, wt[e]) >> l.shift : 0ull;
        const bool up = i < c.n && p > l.prefix, tie = i < c.n && p == l.prefix;
        const uint64_t mg = __ballot(up), me = __ballot(tie);
        if (lane == 0) {
            cw[w][0] = __popcll(mg);
            cw[w][1] = __popcll(me);
        }
        __syncthreads();
        uint32_t bg = ng, be = ne;
        for (int v = 0; v < kWaves; ++v) {
            if (v < w) {
                bg += cw[v][0];
                be += cw[v][1];
            }
            ng += cw[v][0];
            ne += cw[v][1];
        }
        bg += __popcll(mg & below);
        be += __popcll(me & below);
        if (up || (tie && be < l.need)) put(a, g, out + bg + min(be, l.need), e);
        __syncthreads();
    }
}

constexpr uint64_t align256(uint64_t x) { return (x + 255) & ~255ull; }

struct Layout {
    uint32_t chunk_cap, long_cap;
    uint64_t counts, chunks, longs, hist, chunk_counts, cand, total;
};

Layout make_layout(uint64_t n) {
    Layout y{};
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t p = at;
        at += align256(bytes);
        return p;
    };
    y.counts = take(12);
    if (n > kSmall) {
        y.long_cap = (uint32_t)(n / (kSmall + 1));
        y.chunk_cap = (uint32_t)(n / kChunk) + y.long_cap;
        y.chunks = take(sizeof(Chunk) * (uint64_t)y.chunk_cap);
        y.longs = take(sizeof(LongSeg) * (uint64_t)y.long_cap);
        y.hist = take(4ull * kBins * y.long_cap);
        y.chunk_counts = take(8ull * y.chunk_cap);
        y.cand = take(8 * n);
    }
    y.total = at;
    return y;
}

}  // namespace

extern "C" netkv_status netkv_cache_evict_workspace(netkv_handle h, uint64_t n_entries, uint64_t *bytes) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (!bytes) return netkv_internal_fail(h, NETKV_EINVAL, "bytes must not be NULL");
    if (n_entries >= (1ull << 31)) return netkv_internal_fail(h, NETKV_ECAPACITY, "2^31 or more entries");
    *bytes = make_layout(n_entries).total;
    return NETKV_OK;
}

extern "C" netkv_status netkv_cache_evict(netkv_handle h, uint32_t n_seg, const uint64_t *hash_off, uint64_t n_entries,
                                          const uint64_t *weight, const uint64_t *hashes, const uint32_t *keep,
                                          uint32_t newest, uint64_t n_out, uint64_t *out_off, uint32_t *out_pos,
                                          uint64_t *out_hashes, void *work, uint64_t work_bytes, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (n_entries >= (1ull << 31)) return netkv_internal_fail(h, NETKV_ECAPACITY, "2^31 or more entries");
    if (!out_off) return netkv_internal_fail(h, NETKV_EINVAL, "out_off must not be NULL");
    if (n_seg > 0x7FFFFFu) return netkv_internal_fail(h, NETKV_ECAPACITY, "more than 2^23 - 1 segments");
    if (n_seg && (!hash_off || !keep)) return netkv_internal_fail(h, NETKV_EINVAL, "hash_off and keep must not be NULL");
    if (n_entries && !weight) return netkv_internal_fail(h, NETKV_EINVAL, "weight is NULL");
    if (n_out && !out_pos && !out_hashes) return netkv_internal_fail(h, NETKV_EINVAL, "out_pos and out_hashes are both NULL");
    if (n_entries && out_hashes && !hashes) return netkv_internal_fail(h, NETKV_EINVAL, "hashes is NULL");
    const Layout y = make_layout(n_entries);
    if (!work || ((uintptr_t)work & 255) || work_bytes < y.total)
        return netkv_internal_fail(h, NETKV_EINVAL, "work must be 256-byte aligned and of at least netkv_cache_evict_workspace's bytes");
    const int dev = netkv_internal_device(h);
    int prev = -1;
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    if (prev != dev) (void)hipSetDevice(dev);
    hipStream_t s = (hipStream_t)stream;
    uint8_t *ws = (uint8_t *)work;
    EvictArgs a{};
    a.n_seg = n_seg;
    a.newest = newest;
    a.off = hash_off;
    a.weight = weight;
    a.hashes = hashes;
    a.keep = keep;
    a.n = n_entries;
    a.n_out = n_out;
    a.out_off = out_off;
    a.out_hashes = out_hashes;
    a.out_pos = out_pos;
    a.err = netkv_internal_errword(h);
    a.counts = (uint32_t *)(ws + y.counts);
    a.chunks = (Chunk *)(ws + y.chunks);
    a.longs = (LongSeg *)(ws + y.longs);
    a.hist = (uint32_t *)(ws + y.hist);
    a.chunk_counts = (uint2 *)(ws + y.chunk_counts);
    a.cand = (uint64_t *)(ws + y.cand);
    a.chunk_cap = y.chunk_cap;
    a.long_cap = y.long_cap;
    plan_kernel<<<1, kPlanThreads, 0, s>>>(a);
    if (n_seg && n_entries) {
        small_kernel<<<n_seg, kThreads, 0, s>>>(a);
        if (y.long_cap) {
            const uint32_t clear = y.long_cap < 2048 ? y.long_cap : 2048;
            clear_kernel<<<clear, kThreads, 0, s>>>(a);
            count_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
            gather_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
            threshold_kernel<<<y.long_cap, kThreads, 0, s>>>(a);
            write_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
        }
    }
    const hipError_t e = hipGetLastError();
    if (prev >= 0 && prev != dev) (void)hipSetDevice(prev);
    if (e != hipSuccess) return netkv_internal_fail(h, NETKV_EDEVICE, "eviction launch failed");
    return NETKV_OK;
}
