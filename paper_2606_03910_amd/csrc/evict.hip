// Eviction from the resident sets by accumulated attention weight, for
// MI355X (gfx950): every segment (a decode instance's resident blocks, or a
// sequence's) keeps its `keep` heaviest entries, ties to the lowest index, in
// their order.
//
// The threshold of a segment, its keep-th largest weight, is found from counts,
// never by sorting: first by power of two and the 5 bits below it (2,048 bins
// that cover 64 bits; accumulated attention spreads over powers of two, so the
// threshold's bin holds few), then, among the weights of that bin, by 8 bits
// at a time until 64 are left, which one wavefront compares with each other.
//   sums_kernel, running_kernel, plan_kernel -- offsets of the kept, the long
//                       segments' places; up to 1,024 segments by the first workgroup of
//   small_kernel     -- segments of up to 4,096 entries in one workgroup's
//                       registers, one read of everything.
//   Long segments, in chunks of a workgroup and parts of a wavefront:
//   count_kernel     -- counts, and each entry's bin in 16 bits: the two
//                       passes that follow read those in place of the weights.
//   gather_kernel    -- the weights of the threshold's bin.
//   threshold_kernel -- the threshold; where each part's kept entries go.
//   write_kernel     -- the kept entries.
//
// 768 segments of 65,536 entries, half of them kept, have to read 805 MB (all
// weights, and with half of the hashes every line of them) and write 302 MB:
// 221 us at 5 TB/s (181 if the kept hashes could be read alone).  The call takes
// 359 us, its kernels under the profiler 9, 129, 36, 12 and 178 in the order
// above.  One segment of 65,536 takes 30 us and 48 of 4,096 32 us, launches and
// the latency of their chains of loads.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "netkv.h"
#include "netkv_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kEach = 16;                     // entries a thread of small_kernel keeps
constexpr uint32_t kSmall = kThreads * kEach;      // longest segment of small_kernel
constexpr uint32_t kTiny = 256;                     // longest segment of one wavefront
constexpr uint32_t kBins = 2048;
constexpr uint32_t kBatch = 8;                     // loads a lane has in flight
constexpr uint32_t kGather = 4;                    // and of eight bins each
constexpr uint32_t kListed = 1024;                 // segments that every workgroup looks through itself
constexpr uint32_t kTile = 1024;                   // segments a workgroup of plan_kernel places
constexpr uint32_t kMaxSeg = 0x7FFFFFu;

struct Seg {
    uint64_t first;      // entry
    uint32_t n, keep;
};

struct Long {
    uint64_t first, out;             // first entry, where its kept entries begin
    uint32_t n, keep, chunk0, bin;   // the threshold's bin
    uint64_t prefix;                 // a weight of the bin stays if (w >> shift) > prefix, or
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
    Long *longs;
    uint32_t *hist;                  // [long][kBins]
    uint2 *parts;                    // [chunk][kWaves]: above the bin, within it; then the kept before, the ties before
    ulonglong2 *bits;                // [chunk][kWaves]: those that all of a part's weights of the bin have; that any has
    uint16_t *bins;                  // [n], a long segment's from a multiple of 8 (bins_of)
    uint64_t *cand;                  // [n]: each part's weights within the bin, from its first entry
    uint32_t chunk, chunk_cap, long_cap, clear;
};

__device__ inline Seg seg_at(const EvictArgs &a, uint32_t s, bool good) {
    Seg g;
    g.first = a.off[s];
    g.n = good ? (uint32_t)(a.off[s + 1] - g.first) : 0u;
    g.keep = min(a.keep[s], g.n);
    return g;
}
__device__ inline bool bad_at(const EvictArgs &a, uint32_t s) { return a.off[s] > a.off[s + 1] || a.off[s + 1] > a.n; }
__device__ inline uint32_t chunks_of(const EvictArgs &a, const Seg &g) { return g.n > kSmall ? (g.n + a.chunk - 1) / a.chunk : 0u; }

// The weight that counts: the last `newest` of those that may stay (and no
// more than those) come before everything.
__device__ inline uint64_t key_of(const EvictArgs &a, uint32_t n, uint32_t keep, uint32_t i, uint64_t w) {
    return i >= n - min(a.newest, keep) ? ~0ull : w == ~0ull ? ~0ull - 1 : w;
}

__device__ inline uint16_t *bins_of(const EvictArgs &a, const Long &l, uint32_t at) {
    return a.bins + ((l.first + 8ull * at) & ~7ull);
}

// Monotone: below 32 the weight itself, else its power of two and 5 bits.
__device__ inline uint32_t bin_of(uint64_t w) {
    if (w < 32) return (uint32_t)w;
    const uint32_t e = 63 - __clzll((long long)w);
    return ((e - 4) << 5) | ((uint32_t)(w >> (e - 5)) & 31u);
}

// One count a lane.  Lanes of the first one's bin are counted together: many
// entries of no weight would otherwise wait for each other.
__device__ inline void count_one(uint32_t *hist, uint32_t bin, bool is) {
    const uint64_t m = __ballot(is);
    if (!m) return;
    const uint32_t lead = __builtin_amdgcn_readlane(bin, __builtin_ctzll(m));
    const uint64_t same = __ballot(is && bin == lead);
    if (is && bin != lead) atomicAdd(&hist[bin], 1u);
    if ((threadIdx.x & 63) == 0) atomicAdd(&hist[lead], (uint32_t)__popcll(same));
}

__device__ inline void put(const EvictArgs &a, uint64_t at, uint32_t i, uint64_t hash) {
    if (at >= a.n_out) return;
    if (a.out_pos) a.out_pos[at] = i;
    if (a.out_hashes) a.out_hashes[at] = hash;
}

// Places the segments of one tile, as many as the workgroup has threads, after
// at = {kept entries, chunks, long segments}, which it moves on.
template <int THREADS>
__device__ inline void place(const EvictArgs &a, uint32_t s0, bool good, uint64_t at[3]) {
    __shared__ uint64_t sums[THREADS / 64][3];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t s = s0 + threadIdx.x;
    Seg g{0, 0, 0};
    if (s < a.n_seg) g = seg_at(a, s, good);
    const uint32_t nc = chunks_of(a, g);
    uint64_t x[3] = {g.keep, nc, nc ? 1u : 0u}, in[3];
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
    for (int i = 0; i < 3; ++i) {
        uint64_t before = 0, all = 0;
        for (int v = 0; v < THREADS / 64; ++v) {
            if (v < w) before += sums[v][i];
            all += sums[v][i];
        }
        x[i] = at[i] + before + in[i] - x[i];
        at[i] += all;
    }
    __syncthreads();
    if (s < a.n_seg) {
        a.out_off[s] = x[0];
        if (nc && x[2] < a.long_cap && x[1] + nc <= a.chunk_cap)
            a.longs[x[2]] = Long{g.first, x[0], g.n, g.keep, (uint32_t)x[1], 0, 0, 0, 0};
    }
}

__device__ inline void placed(const EvictArgs &a, bool good, const uint64_t at[3]) {
    a.out_off[a.n_seg] = at[0];
    if (!good || at[0] > a.n_out) atomicOr(a.err, kErrEntryBit);
    a.counts[0] = (uint32_t)min(at[1], (uint64_t)a.chunk_cap);
    a.counts[1] = (uint32_t)min(at[2], (uint64_t)a.long_cap);
    a.counts[2] = good;
}

// More than kListed segments: each tile's sums, their running sums, each
// tile's places (100,000 segments: 6 us for the last; one workgroup for all of
// it took 940).  A tile's sums lie in the first two of its own offsets until
// those are written: the kept entries (top bit: bad offsets), and the chunks
// with the long segments above them.
__global__ __launch_bounds__(kTile) void sums_kernel(EvictArgs a) {
    __shared__ unsigned long long sum[2];
    if (threadIdx.x < 2) sum[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t s = blockIdx.x * kTile + threadIdx.x;
    const bool in = s < a.n_seg, bad = in && bad_at(a, s);
    Seg g{0, 0, 0};
    if (in) g = seg_at(a, s, !bad);
    const uint32_t nc = chunks_of(a, g);
    if (g.keep) atomicAdd(&sum[0], (unsigned long long)g.keep);
    if (nc) atomicAdd(&sum[1], nc | 1ull << 32);
    const bool any_bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        a.out_off[(uint64_t)blockIdx.x * kTile] = any_bad ? 1ull << 63 : sum[0];
        a.out_off[(uint64_t)blockIdx.x * kTile + 1] = sum[1];
    }
}

__global__ __launch_bounds__(kTile) void running_kernel(EvictArgs a, uint32_t tiles) {
    __shared__ uint64_t sums[kTile / 64][2];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    bool bad = false;
    uint64_t at[2] = {0, 0};
    for (uint32_t t0 = 0; t0 < tiles; t0 += kTile) {
        const uint32_t t = t0 + threadIdx.x;
        uint64_t x[2] = {0, 0}, in[2];
        for (int i = 0; i < 2; ++i) {
            if (t < tiles) x[i] = a.out_off[(uint64_t)t * kTile + i];
            if (x[i] >> 63) {
                bad = true;
                x[i] = 0;
            }
            uint64_t y = x[i];
            for (int d = 1; d < 64; d <<= 1) {
                const uint64_t z = __shfl_up((unsigned long long)y, d, 64);
                if (lane >= d) y += z;
            }
            in[i] = y;
            if (lane == 63) sums[w][i] = y;
        }
        __syncthreads();
        for (int i = 0; i < 2; ++i) {
            uint64_t before = at[i];
            for (int v = 0; v < kTile / 64; ++v) {
                if (v < w) before += sums[v][i];
                at[i] += sums[v][i];
            }
            if (t < tiles) a.out_off[(uint64_t)t * kTile + i] = before + in[i] - x[i];
        }
        __syncthreads();
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) a.counts[2] = !bad;
}

__global__ __launch_bounds__(kTile) void plan_kernel(EvictArgs a) {
    const bool good = a.counts[2] != 0;   // else every segment counts as empty
    const uint64_t x = a.out_off[(uint64_t)blockIdx.x * kTile], y = a.out_off[(uint64_t)blockIdx.x * kTile + 1];
    uint64_t at[3] = {good ? x : 0, good ? (uint32_t)y : 0, good ? y >> 32 : 0};
    __syncthreads();   // every thread has read the sums
    place<kTile>(a, blockIdx.x * kTile, good, at);
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) placed(a, good, at);
}

// The bin of the `rest`-th from the top among 2,048 counts of which each of
// 256 threads holds eight, what is left of `rest` in it, and its count:
// in out[0..2], for every thread.
__device__ inline void find_top(const uint32_t (&h)[8], uint32_t rest, uint32_t *out) {
    __shared__ uint32_t sums[kWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t mine = 0;
    for (int i = 0; i < 8; ++i) mine += h[i];
    uint32_t above = mine;   // this thread's bins and the higher threads'
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t z = __shfl_down(above, d, 64);
        if (lane + d < 64) above += z;
    }
    if (lane == 0) sums[w] = above;
    __syncthreads();
    for (int v = w + 1; v < kWaves; ++v) above += sums[v];
    if (above >= rest && above - mine < rest) {
        uint32_t left = rest - (above - mine);
        bool is = false;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            if (!is && left <= h[i]) {
                is = true;
                out[0] = threadIdx.x * 8 + i;
                out[1] = left;
                out[2] = h[i];
            }
            if (!is) left -= h[i];
        }
    }
    __syncthreads();
}

// The digit of the `rest`-th from the top among 256 counts; one wavefront.
__device__ inline void find_digit(const uint32_t *hist, uint32_t rest, uint32_t *out) {
    const int lane = threadIdx.x & 63;
    const uint4 h = *(const uint4 *)(hist + 4 * lane);
    const uint32_t c[4] = {h.x, h.y, h.z, h.w}, mine = h.x + h.y + h.z + h.w;
    uint32_t above = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t z = __shfl_down(above, d, 64);
        if (lane + d < 64) above += z;
    }
    if (above >= rest && above - mine < rest) {
        uint32_t left = rest - (above - mine);
        bool is = false;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            if (!is && left <= c[i]) {
                is = true;
                out[0] = 4 * lane + i;
                out[1] = left;
                out[2] = c[i];
            }
            if (!is) left -= c[i];
        }
    }
}

// The `rest`-th largest of n <= 64 weights, how many of its equals are among
// the first `rest`; one wavefront.
__device__ inline void rank64(const unsigned long long *list, uint32_t n, uint32_t rest, uint64_t *value, uint32_t *need) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t v = lane < n ? list[lane] : 0ull;
    uint32_t above = 0, equal = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t x = list[i];
        above += x > v;
        equal += x == v;
    }
    if (lane < n && above < rest && rest <= above + equal) {   // the equals write the same
        *value = v;
        *need = rest - above;
    }
}

// A segment of at most kTiny entries by one wavefront: the threshold bit by
// bit, from counts of ballots.  100,000 of up to 200 entries take 220 us under
// the profiler (190 without it; a workgroup each, as for larger ones, 616), 40
// of memory: bound by the vector units, 820 instructions a segment, which at 4
// cycles each are 134 us, and shifts and comparisons of 64 bits take more.
__device__ inline void tiny_segment(const EvictArgs &a, const Seg &g, uint64_t out) {
    constexpr uint32_t kMine = kTiny / 64;
    const uint32_t lane = threadIdx.x & 63;
    uint64_t k[kMine], every = ~0ull, some = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) k[i] = i * 64 + lane < g.n ? a.weight[g.first + i * 64 + lane] : 0ull;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t e = i * 64 + lane;
        if (e >= g.n) continue;
        k[i] = key_of(a, g.n, g.keep, e, k[i]);
        every &= k[i];
        some |= k[i];
    }
    for (int d = 32; d; d >>= 1) {
        every &= (uint64_t)__shfl_xor((unsigned long long)every, d, 64);
        some |= (uint64_t)__shfl_xor((unsigned long long)some, d, 64);
    }
    // every key agrees above `shift`, which may be 64: then by two shifts, and
    // 63 does as well where all stay
    uint32_t shift = every == some ? 0u : 64 - __clzll((long long)(every ^ some)), need = g.keep, among = g.n;
    uint64_t prefix = shift ? some >> (shift - 1) >> 1 : some;
    if (need == among) shift = min(shift, 63u);
    while (shift && need != among) {
        --shift;
        const uint64_t up = prefix << 1 | 1;
        uint32_t c = 0, both = 0;
#pragma unroll
        for (uint32_t i = 0; i < kMine; ++i) {
            const bool in = i * 64 + lane < g.n;
            c += __popcll(__ballot(in && k[i] >> shift == up));
            both += __popcll(__ballot(in && k[i] >> shift == (up ^ 1)));
        }
        const bool one = c >= need;
        prefix = one ? up : up ^ 1;
        among = one ? c : both;
        need = one ? need : need - c;
    }
    uint32_t ng = 0, ne = 0;
    uint32_t at[kMine];
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const bool in = i * 64 + lane < g.n;
        const uint64_t mg = __ballot(in && k[i] >> shift > prefix), me = __ballot(in && k[i] >> shift == prefix);
        const uint32_t e = ne + __popcll(me & below);
        const bool stays = (mg >> lane & 1) || ((me >> lane & 1) && e < need);
        at[i] = stays ? ng + __popcll(mg & below) + min(e, need) : ~0u;
        k[i] = stays && a.out_hashes ? a.hashes[g.first + i * 64 + lane] : 0ull;
        ng += __popcll(mg);
        ne += __popcll(me);
    }
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i)
        if (at[i] != ~0u) put(a, out + at[i], i * 64 + lane, k[i]);
}

struct SmallShared {
    __align__(16) uint32_t hist[kBins];
    uint32_t found[3], n_list, n_need;
    uint64_t value;
    unsigned long long list[64];
    uint32_t cg[kEach * kWaves], ce[kEach * kWaves];
};

// A segment of at most kSmall entries by the workgroup: 48 of 4,096 take 15 us,
// bound by five loads and ten barriers one after the other.
__device__ inline void small_segment(const EvictArgs &a, const Seg &g, uint64_t out, SmallShared &sh) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t k[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kThreads + threadIdx.x;
        k[i] = e < g.n ? a.weight[g.first + e] : 0ull;
    }
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads) sh.hist[i] = 0;
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    uint32_t b[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        b[i] = 0;
        if (i * kThreads >= g.n) continue;
        const uint32_t e = i * kThreads + threadIdx.x;
        if (e < g.n) k[i] = key_of(a, g.n, g.keep, e, k[i]);
        b[i] = bin_of(k[i]);
        count_one(sh.hist, b[i], e < g.n);
    }
    __syncthreads();
    {
        uint32_t h[8];
        for (int i = 0; i < 8; ++i) h[i] = sh.hist[threadIdx.x * 8 + i];
        find_top(h, g.keep, sh.found);
    }
    const uint32_t bin = sh.found[0];
    uint32_t need = sh.found[1], among = sh.found[2];
    // the bin's weights share what is above `shift`
    uint32_t shift = bin < 32 ? 0u : (bin >> 5) - 1;
    uint64_t prefix = bin < 32 ? bin : 32u | (bin & 31u);
    while (shift && need != among && among > 64) {
        const uint32_t by = min(shift, 8u);
        __syncthreads();
        sh.hist[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i)
            count_one(sh.hist, (uint32_t)(k[i] >> (shift - by)) & ((1u << by) - 1),
                      i * kThreads + threadIdx.x < g.n && k[i] >> shift == prefix);
        __syncthreads();
        if (w == 0) find_digit(sh.hist, need, sh.found);
        __syncthreads();
        shift -= by;
        prefix = (prefix << by) | sh.found[0];
        need = sh.found[1];
        among = sh.found[2];
    }
    if (shift && need != among) {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i)
            if (i * kThreads + threadIdx.x < g.n && k[i] >> shift == prefix) sh.list[atomicAdd(&sh.n_list, 1u)] = k[i];
        __syncthreads();
        if (w == 0) rank64(sh.list, among, need, &sh.value, &sh.n_need);
        __syncthreads();
        shift = 0;
        prefix = sh.value;
        need = sh.n_need;
    }
    uint64_t mg[kEach], me[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const bool in = i * kThreads + threadIdx.x < g.n;
        const uint64_t p = k[i] >> shift;
        mg[i] = __ballot(in && p > prefix);
        me[i] = __ballot(in && p == prefix);
        if (lane == 0) {
            sh.cg[i * kWaves + w] = __popcll(mg[i]);
            sh.ce[i * kWaves + w] = __popcll(me[i]);
        }
    }
    __syncthreads();
    if (w == 0) {   // kEach * kWaves = 64 counts, one a lane
        uint32_t x = sh.cg[lane], y = sh.ce[lane];
        const uint32_t x0 = x, y0 = y;
        for (int i = 1; i < 64; i <<= 1) {
            const uint32_t p = __shfl_up(x, i, 64), q = __shfl_up(y, i, 64);
            if (lane >= i) {
                x += p;
                y += q;
            }
        }
        sh.cg[lane] = x - x0;
        sh.ce[lane] = y - y0;
    }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {   // the kept entries' places, then all of their hashes at once
        const uint32_t ng = sh.cg[i * kWaves + w] + __popcll(mg[i] & below), ne = sh.ce[i * kWaves + w] + __popcll(me[i] & below);
        const bool stays = (mg[i] >> lane & 1) || ((me[i] >> lane & 1) && ne < need);
        b[i] = stays ? ng + min(ne, need) : ~0u;
        k[i] = stays && a.out_hashes ? a.hashes[g.first + i * kThreads + threadIdx.x] : 0ull;
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
        if (b[i] != ~0u) put(a, out + b[i], i * kThreads + threadIdx.x, k[i]);
}

// The first workgroup places up to kListed segments, the next a.clear ones
// clear the long segments' counts, the others have `group` segments each (up to
// kWaves where those still fill the card): the tiny ones a wavefront each, the
// others one after the other.
template <bool LISTED>
__global__ __launch_bounds__(kThreads, 4) void small_kernel(EvictArgs a, uint32_t group) {
    __shared__ SmallShared sh;
    __shared__ unsigned long long before;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if (blockIdx.x >= 1 && blockIdx.x <= a.clear) {
        const uint64_t n = (uint64_t)(LISTED ? min(a.long_cap, a.n_seg) : a.counts[1]) * (kBins / 4);
        for (uint64_t i = (blockIdx.x - 1) * (uint64_t)kThreads + threadIdx.x; i < n; i += (uint64_t)a.clear * kThreads)
            ((uint4 *)a.hist)[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    if constexpr (LISTED) {
        if (threadIdx.x == 0) before = 0;
        bool bad = false;
        for (uint32_t i = threadIdx.x; i < a.n_seg; i += kThreads) bad |= bad_at(a, i);
        const bool good = !__syncthreads_or(bad);
        if (blockIdx.x == 0) {
            uint64_t at[3] = {0, 0, 0};
            for (uint32_t s0 = 0; s0 < a.n_seg; s0 += kThreads) place<kThreads>(a, s0, good, at);
            if (threadIdx.x == 0) placed(a, good, at);
            return;
        }
        const uint32_t s = blockIdx.x - a.clear - 1;
        const Seg g = seg_at(a, s, good);
        if (g.n > kSmall || g.keep == 0) return;
        unsigned long long sum = 0;
        for (uint32_t i = threadIdx.x; i < s; i += kThreads) sum += seg_at(a, i, true).keep;
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
        if (lane == 0) atomicAdd(&before, sum);
        __syncthreads();
        if (g.n > kTiny)
            small_segment(a, g, before, sh);
        else if (w == 0)
            tiny_segment(a, g, before);
    } else {
        if (blockIdx.x == 0) return;
        const bool good = a.counts[2] != 0;
        const uint32_t s0 = (blockIdx.x - a.clear - 1) * group;
        if (w < group && s0 + w < a.n_seg) {
            const Seg g = seg_at(a, s0 + w, good);
            if (g.n <= kTiny && g.keep) tiny_segment(a, g, a.out_off[s0 + w]);
        }
        for (uint32_t s = s0; s < min(s0 + group, a.n_seg); ++s) {
            const Seg g = seg_at(a, s, good);
            if (g.n <= kTiny || g.n > kSmall || g.keep == 0) continue;
            __syncthreads();
            small_segment(a, g, a.out_off[s], sh);
        }
    }
}

// The long segment that chunk c belongs to, by the whole workgroup.
__device__ inline uint32_t find_long(const EvictArgs &a, uint32_t c) {
    uint32_t lo = 0, hi = a.counts[1];
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + kThreads - 1) / kThreads, i = lo + threadIdx.x * step;
        const uint32_t in = __syncthreads_count(i < hi && a.longs[i].chunk0 <= c);
        lo += (in - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// Bound by the weights' bytes: 402 MB in and 101 MB of bins out take 129 us,
// 3.9 TB/s.  Weights and hashes are read once, past the cache, which keeps the
// bins (145 us through it).
__global__ __launch_bounds__(kThreads) void count_kernel(EvictArgs a) {
    __shared__ uint32_t hist[kBins];
    if (blockIdx.x >= a.counts[0]) return;
    const uint32_t at = find_long(a, blockIdx.x);
    const Long &l = a.longs[at];
    const uint32_t first = (blockIdx.x - l.chunk0) * a.chunk, end = min(l.n, first + a.chunk), n = l.n, keep = l.keep;
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    const uint64_t *wt = a.weight + l.first;
    uint16_t *bins = bins_of(a, l, at);
    for (uint32_t i0 = first; i0 < end; i0 += kThreads * kBatch) {
        uint64_t k[kBatch];
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = i0 + j * kThreads + threadIdx.x;
            k[j] = i < end ? __builtin_nontemporal_load(wt + i) : 0ull;
        }
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = i0 + j * kThreads + threadIdx.x, b = bin_of(key_of(a, n, keep, i, k[j]));
            if (i < end) bins[i] = (uint16_t)b;
            count_one(hist, b, i < end);
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads)
        if (hist[i]) atomicAdd(&a.hist[(uint64_t)at * kBins + i], hist[i]);
}

// 101 MB of bins in 36 us, and the few weights of one bin.
__global__ __launch_bounds__(kThreads, 6) void gather_kernel(EvictArgs a) {
    __shared__ uint32_t found[3];
    if (blockIdx.x >= a.counts[0]) return;
    const uint32_t at = find_long(a, blockIdx.x);
    Long &l = a.longs[at];
    if (l.keep == 0) return;
    {
        const uint4 *p = (const uint4 *)(a.hist + (uint64_t)at * kBins) + 2 * threadIdx.x;
        const uint4 x = p[0], y = p[1];
        const uint32_t h[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        find_top(h, l.keep, found);
    }
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t bin = found[0], n = l.n, keep = l.keep;
    const uint64_t *wt = a.weight + l.first;
    const uint16_t *bins = bins_of(a, l, at);
    const uint32_t part = a.chunk / kWaves, first = (blockIdx.x - l.chunk0) * a.chunk + w * part, end = min(n, first + part);
    uint64_t *cand = a.cand + l.first + first;
    uint32_t above = 0, in = 0;
    uint64_t every = ~0ull, some = 0;
    // eight entries a lane: the order of a part's weights does not matter.  The
    // last eight bins may lie past the segment's, not past the array.
    for (uint32_t i0 = first + 8 * lane; i0 - 8 * lane < end; i0 += 512 * kGather) {
        uint4 x[kGather];
#pragma unroll
        for (uint32_t j = 0; j < kGather; ++j) {
            x[j] = make_uint4(0, 0, 0, 0);
            if (i0 + 512 * j < end) x[j] = *(const uint4 *)(bins + i0 + 512 * j);
        }
        uint32_t is = 0;   // the lane's entries of the bin
#pragma unroll
        for (uint32_t j = 0; j < kGather; ++j) {
            const uint32_t y[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) {
                const uint32_t b = q & 1 ? y[q / 2] >> 16 : y[q / 2] & 0xFFFFu;
                const bool in = i0 + 512 * j + q < end;
                above += in && b > bin;
                is |= in && b == bin ? 1u << (8 * j + q) : 0u;
            }
        }
        const uint32_t mine = __popc(is);
        uint32_t to = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t z = __shfl_up(to, d, 64);
            if (lane >= d) to += z;
        }
        const uint32_t all = __shfl(to, 63, 64);
        to += in - mine;
        if (bin < 32) {
            // such a bin holds one weight: none is looked at
        } else if (all <= 512) {
            for (; is; is &= is - 1) {
                const uint32_t q = __builtin_ctz(is), i = i0 + 512 * (q / 8) + q % 8;
                const uint64_t k = key_of(a, n, keep, i, wt[i]);
                cand[to++] = k;
                every &= k;
                some |= k;
            }
        } else {
            // a lane's entries are lines apart: where every fourth is of the bin the
            // lanes take them side by side (768 segments of 65,536 weights within 3 %
            // of each other 233 us against 328, within 0.3 % 219 against 658)
            uint32_t next = in;
            for (uint32_t q = 0; q < 8 * kGather; ++q) {
                const uint32_t i = i0 - 8 * lane + 64 * q + lane;
                const bool own = i < end && bins[i] == bin;
                const uint64_t m = __ballot(own);
                if (own) {
                    const uint64_t k = key_of(a, n, keep, i, wt[i]);
                    cand[next + __popcll(m & ((1ull << lane) - 1))] = k;
                    every &= k;
                    some |= k;
                }
                next += __popcll(m);
            }
        }
        in += all;
    }
    for (int d = 32; d; d >>= 1) {
        above += __shfl_xor(above, d, 64);
        every &= (uint64_t)__shfl_xor((unsigned long long)every, d, 64);
        some |= (uint64_t)__shfl_xor((unsigned long long)some, d, 64);
    }
    if (lane == 0) {
        a.parts[(uint64_t)blockIdx.x * kWaves + w] = make_uint2(above, in);
        if (bin < 32 && in) every = some = bin;
        a.bits[(uint64_t)blockIdx.x * kWaves + w] = make_ulonglong2(every, some);
    }
    if (threadIdx.x == 0 && blockIdx.x == l.chunk0) {
        l.bin = bin;
        l.need = found[1];
    }
}

// A workgroup a long segment, latency: 768 of them take 12 us (26 with 1,024
// threads each, three rounds in place of one).
__global__ __launch_bounds__(kThreads) void threshold_kernel(EvictArgs a) {
    __shared__ __align__(16) uint32_t hist[256];
    __shared__ uint32_t found[3], cw[kWaves][2], n_list, n_need;
    __shared__ uint64_t value, bw[kWaves][2];
    __shared__ unsigned long long list[64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t part = a.chunk / kWaves;
    for (uint32_t at = blockIdx.x; at < a.counts[1]; at += gridDim.x) {
        Long &l = a.longs[at];
        if (l.keep == 0) continue;
        uint2 *parts = a.parts + (uint64_t)l.chunk0 * kWaves;
        const uint32_t n_part = (l.n + part - 1) / part;
        const uint64_t *cand = a.cand + l.first;
        uint32_t need = l.need, among = 0;
        uint64_t every = ~0ull, some = 0;
        for (uint32_t c = threadIdx.x; c < n_part; c += kThreads) {
            const ulonglong2 b = a.bits[(uint64_t)l.chunk0 * kWaves + c];
            among += parts[c].y;
            every &= b.x;
            some |= b.y;
        }
        for (int d = 32; d; d >>= 1) {
            among += __shfl_xor(among, d, 64);
            every &= (uint64_t)__shfl_xor((unsigned long long)every, d, 64);
            some |= (uint64_t)__shfl_xor((unsigned long long)some, d, 64);
        }
        __syncthreads();
        if (lane == 0) {
            cw[w][0] = among;
            bw[w][0] = every;
            bw[w][1] = some;
        }
        if (threadIdx.x == 0) n_list = 0;
        __syncthreads();
        among = 0;
        for (int v = 0; v < kWaves; ++v) {
            among += cw[v][0];
            every &= bw[v][0];
            some |= bw[v][1];
        }
        // every weight of the bin agrees above `shift`; nothing to look at where all are one
        const uint64_t differ = every ^ some;
        uint32_t shift = differ ? 64 - __clzll((long long)differ) : 0u;   // below 64: the bin fixes the top bits
        uint64_t prefix = some >> shift;
        // as many lanes a part as parts have weights on average, at most a wavefront
        const uint32_t lg = among > n_part ? min(32 - __clz((among - 1) / n_part), 6) : 0;
        const uint32_t c_own = threadIdx.x >> lg, c_step = kThreads >> lg, i_own = threadIdx.x & ((1u << lg) - 1);
        auto each = [&](auto f) {
            for (uint32_t c = c_own; c < n_part; c += c_step) {
                const uint32_t m = parts[c].y;
                for (uint32_t i = i_own; i < m; i += 1u << lg) f(cand[(uint64_t)c * part + i]);
            }
        };
        while (shift && need != among && among > 64) {
            const uint32_t by = min(shift, 8u);
            hist[threadIdx.x] = 0;
            __syncthreads();
            each([&](uint64_t k) {
                if (k >> shift == prefix) atomicAdd(&hist[(uint32_t)(k >> (shift - by)) & ((1u << by) - 1)], 1u);
            });
            __syncthreads();
            if (w == 0) find_digit(hist, need, found);
            __syncthreads();
            shift -= by;
            prefix = (prefix << by) | found[0];
            need = found[1];
            among = found[2];
        }
        if (shift && need != among) {
            each([&](uint64_t k) {
                if (k >> shift == prefix) list[atomicAdd(&n_list, 1u)] = k;
            });
            __syncthreads();
            if (w == 0) rank64(list, among, need, &value, &n_need);
            __syncthreads();
            shift = 0;
            prefix = value;
            need = n_need;
        }
        // where each part's kept entries and ties begin
        uint32_t bg = 0, be = 0;
        for (uint32_t c0 = 0; c0 < n_part; c0 += c_step) {
            const uint32_t c = c0 + c_own;
            uint32_t ng = 0, ne = 0;
            if (c < n_part) {
                const uint2 p = parts[c];
                if (differ) {
                    for (uint32_t i = i_own; i < p.y; i += 1u << lg) {
                        const uint64_t k = cand[(uint64_t)c * part + i] >> shift;
                        ng += k > prefix;
                        ne += k == prefix;
                    }
                } else if (i_own == 0) {
                    ne = p.y;
                }
                if (i_own == 0) ng += p.x;
            }
            uint32_t ig = ng, ie = ne;   // the parts' lanes lie next to each other: one running sum
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t x = __shfl_up(ig, d, 64), y = __shfl_up(ie, d, 64);
                if (lane >= d) {
                    ig += x;
                    ie += y;
                }
            }
            __syncthreads();
            if (lane == 63) {
                cw[w][0] = ig;
                cw[w][1] = ie;
            }
            __syncthreads();
            uint32_t g0 = bg, e0 = be;
            for (int v = 0; v < kWaves; ++v) {
                if (v < w) {
                    g0 += cw[v][0];
                    e0 += cw[v][1];
                }
                bg += cw[v][0];
                be += cw[v][1];
            }
            if (i_own == 0 && c < n_part) parts[c] = make_uint2(g0 + ig - ng, e0 + ie - ne);
        }
        if (threadIdx.x == 0) {
            l.shift = shift;
            l.prefix = prefix;
            l.need = need;
        }
    }
}

// Bound by memory: bins, all lines of the hashes and the outputs, 805 MB, take
// 178 us, 4.5 TB/s.
__global__ __launch_bounds__(kThreads) void write_kernel(EvictArgs a) {
    if (blockIdx.x >= a.counts[0]) return;
    const uint32_t at = find_long(a, blockIdx.x);
    const Long &l = a.longs[at];
    if (l.keep == 0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint64_t below = (1ull << lane) - 1, prefix = l.prefix, out = l.out;
    const uint64_t *wt = a.weight + l.first, *hashes = a.hashes + l.first;
    const uint16_t *bins = bins_of(a, l, at);
    const uint32_t n = l.n, keep = l.keep, bin = l.bin, shift = l.shift, need = l.need;
    const uint32_t part = a.chunk / kWaves, first = (blockIdx.x - l.chunk0) * a.chunk + w * part, end = min(n, first + part);
    const uint2 start = a.parts[(uint64_t)blockIdx.x * kWaves + w];
    uint32_t ng = start.x, ne = start.y;
    uint32_t next[kBatch];   // bins
    auto ahead = [&](uint32_t i0) {
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = i0 + j * 64 + lane;
            next[j] = i < end ? bins[i] : 0u;
        }
    };
    ahead(first);
    for (uint32_t i0 = first; i0 < end; i0 += 64 * kBatch) {
        uint32_t b[kBatch];
        uint64_t x[kBatch];
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) b[j] = next[j];
        ahead(i0 + 64 * kBatch);
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = i0 + j * 64 + lane;
            bool up = i < end && b[j] > bin, tie = i < end && b[j] == bin;
            if (tie && bin >= 32) {
                const uint64_t p = key_of(a, n, keep, i, wt[i]) >> shift;
                up = p > prefix;
                tie = p == prefix;
            }
            const uint64_t mg = __ballot(up), me = __ballot(tie);
            const uint32_t e = ne + __popcll(me & below);
            const bool stays = up || (tie && e < need);
            b[j] = stays ? ng + __popcll(mg & below) + min(e, need) : ~0u;
            x[j] = stays && a.out_hashes ? __builtin_nontemporal_load(hashes + i) : 0ull;
            ng += __popcll(mg);
            ne += __popcll(me);
        }
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j)
            if (b[j] != ~0u) put(a, out + b[j], i0 + j * 64 + lane, x[j]);
    }
}

constexpr uint64_t align256(uint64_t x) { return (x + 255) & ~255ull; }

struct Layout {
    uint32_t chunk, chunk_cap, long_cap;
    uint64_t counts, longs, hist, parts, bits, bins, cand, total;
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
        // chunks of 16,384 entries, of less where those would not fill the card:
        // 2,048 against 16,384, us: 768 segments of 65,536 entries 513, 362; one 30, 67
        y.chunk = kThreads * kBatch;
        while (y.chunk < 16384 && n / y.chunk > 1024) y.chunk *= 2;
        y.long_cap = (uint32_t)(n / (kSmall + 1));
        y.chunk_cap = (uint32_t)(n / y.chunk) + y.long_cap;
        y.longs = take(sizeof(Long) * (uint64_t)y.long_cap);
        y.hist = take(4ull * kBins * y.long_cap);
        y.parts = take(8ull * kWaves * y.chunk_cap);
        y.bits = take(16ull * kWaves * y.chunk_cap);
        y.bins = take(2 * (n + 8ull * y.long_cap + 8));
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
    if (n_seg > kMaxSeg) return netkv_internal_fail(h, NETKV_ECAPACITY, "more than 2^23 - 1 segments");
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
    a.longs = (Long *)(ws + y.longs);
    a.hist = (uint32_t *)(ws + y.hist);
    a.parts = (uint2 *)(ws + y.parts);
    a.bits = (ulonglong2 *)(ws + y.bits);
    a.bins = (uint16_t *)(ws + y.bins);
    a.cand = (uint64_t *)(ws + y.cand);
    a.chunk = y.chunk ? y.chunk : 1;
    a.chunk_cap = y.chunk_cap;
    a.long_cap = y.long_cap;
    a.clear = y.long_cap < 256 ? y.long_cap : 256;
    if (n_seg <= kListed) {
        small_kernel<true><<<1 + a.clear + n_seg, kThreads, 0, s>>>(a, 1);
    } else {
        const uint32_t tiles = (n_seg + kTile - 1) / kTile;
        sums_kernel<<<tiles, kTile, 0, s>>>(a);
        running_kernel<<<1, kTile, 0, s>>>(a, tiles);
        plan_kernel<<<tiles, kTile, 0, s>>>(a);
        // 1 against 4, us: 2,000 segments of up to 3,000 entries 23, 37; 100,000 of
        // up to 200 281, 192
        const uint32_t group = n_seg <= 4 * kListed ? 1 : kWaves;
        small_kernel<false><<<1 + a.clear + (n_seg + group - 1) / group, kThreads, 0, s>>>(a, group);
    }
    if (n_seg && y.long_cap) {
        count_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
        gather_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
        threshold_kernel<<<y.long_cap < 1024 ? y.long_cap : 1024, kThreads, 0, s>>>(a);
        write_kernel<<<y.chunk_cap, kThreads, 0, s>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (prev >= 0 && prev != dev) (void)hipSetDevice(prev);
    if (e != hipSuccess) return netkv_internal_fail(h, NETKV_EDEVICE, "eviction launch failed");
    return NETKV_OK;
}
