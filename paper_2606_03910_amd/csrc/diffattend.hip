// Differential attention over the block cache on MI355X (gfx950): the
// difference of two softmax maps over one head's values, of twice the keys'
// dimension.
//
//   pair_kernel         -- up to 16 rows over a token range.
//   pair_prompt_kernel  -- the same of up to 128 or 64 rows.
//   pair_join_kernel    -- joins the ranges of the rows that were split.
//
// KV heads 2 p and 2 p + 1 of the cache are a pair: each has its own keys, and
// their values side by side are the pair's values v of 2 D elements.  A row is
// a token's query pair j (heads 2 j and 2 j + 1) on KV pair p = j / G:
//     out = softmax(s q_2j k_2p) v - lambda_j softmax(s q_2j+1 k_2p+1) v,
// normalised on demand by the root of its mean square.  Each map has a running
// maximum and sum of its own, as attend_kernel keeps them; what they cannot
// share is only known at the end, so each has its own sums over the values
// too.  A product of 2 D with the difference of the maps would need every
// score's sum first, and so all scores twice: 6 D operations a head and token
// either way.
//
// The two value heads of a page have scales of their own.  The weights are
// multiplied by the larger one S, as attend_kernel does with its one; the other
// head's values are widened times r = its scale / S in fp16, exact for the
// powers of two that the cache's own calls write down to 2^-15 (of smaller
// ones what is below 2^-25 S is lost), and rounded to 11 bits for others.

#include <hip/hip_runtime.h>

#include "blockdev.h"
#include "pairplan.h"

namespace {

using namespace blockdev;
using namespace pairplan;
using blockdev::weights_of;

struct PairArgs : PlanArgs {
    uint32_t pairs;                  // KV pairs
    uint32_t tile_log;               // log2 of tile_rows
    uint64_t q_stride;
    const void *q;
    void *out;
    float c0;                        // |scale| * log2(e)
    uint32_t q_sign;
    const float *lambda;             // [query pair]
    const float *norm;               // [2 D], or null
    float root_eps, gain;
    float *part;                     // [slot][pair][map][tile_rows][2 D]
    f32x4 *part_ml;                  // [slot][pair][map][tile_rows] m, l, y
    uint32_t by_size;                // pair_kernel's longest ranges first
};

// 1 / sqrt(mean of o^2 + eps) of a row as a product of two factors: with its
// largest element or sqrt(eps) brought near 1 the squares neither overflow nor
// vanish.
struct Rms {
    float t, f;
    __device__ explicit Rms(float most, float root_eps) {
        const float s = fmaxf(most, root_eps);
        const uint32_t e = min(max(__float_as_uint(s) >> 23, 1u), 253u);
        t = __uint_as_float((254u - e) << 23);
        f = 1.0f;
    }
    __device__ float square(float o) const { return o * t * (o * t); }
    __device__ void close(float sum, float inv_n, float root_eps) {
        const float e = root_eps * t;
        f = 1.0f / sqrtf(fmaf(e, e, sum * inv_n));
    }
    __device__ float operator()(float o) const { return o * t * f; }
};

// Four elements of a row at column `col` to the output, by kCols lanes side by
// side that hold it all: o1 and o2 are the two maps' products.
template <int VD, typename T>
__device__ inline void finish(const PairArgs &a, f32x4 o1, f32x4 o2, uint32_t j, T *out, uint32_t col) {
    constexpr uint32_t kCols = VD / 4;
    const float lam = a.lambda[j];
    f32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(-lam, o2[i], o1[i]);
    if (a.norm) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(o[i]));
        for (uint32_t d = kCols / 2; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
        Rms rms(most, a.root_eps);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += rms.square(o[i]);
        for (uint32_t d = kCols / 2; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
        rms.close(sum, 1.0f / VD, a.root_eps);
        const f32x4 w = *(const f32x4 *)(a.norm + 4 * col);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = rms(o[i]) * w[i];
    }
    T z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = (T)(o[i] * a.gain);
    *(u32x2 *)(out + 4 * col) = *(u32x2 *)z;
}

// What a step's values are multiplied by: S, and each half's r.
struct ValScale {
    float s, r[2];
};
__device__ inline ValScale val_scale(float x, float y) {
    ValScale v;
    v.s = fmaxf(x, y);
    v.r[0] = v.r[1] = 1.0f;
    if (x != y) {                              // NaN too, which s then stays
        v.r[0] = v.s > 0.0f ? x / v.s : 1.0f;
        v.r[1] = v.s > 0.0f ? y / v.s : 1.0f;
        if (!(x == x && y == y)) v.s = NAN;
    }
    return v;
}

__device__ inline f16x8 times(f16x8 x, float r) {
    const _Float16 h = (_Float16)r;
    return x * f16x8{h, h, h, h, h, h, h, h};
}

// Inclusive sums over the wavefront.
__device__ inline uint32_t wave_sums(uint32_t x) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);   // from 1, 2, 4, 8 lanes before, within 16
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);   // lane 15 to 16 .. 31, 47 to 48 .. 63
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);   // lane 31 to 32 .. 63
    return x;
}

// The largest of the wavefront.
__device__ inline uint32_t wave_most(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// The work list as a wavefront has it in its registers, as Shares: each lane
// takes up to four sequences in a row (n_seq <= kListed), and a row tile's
// ranges are of one length; a sequence's last tiles, which see most, come
// first.  By sums across lanes in place of LDS shuffles and by 32-bit divisions,
// against Shares: six prompts of up to 2,777 tokens of which every workgroup takes
// 17 steps (D = 64, 16 KV heads) 439 us and 448, the first tiles first 447.
// BY_SIZE: a call's longest ranges first, by quarters of the longest's length.
template <bool BY_SIZE>
struct PairShares {
    static constexpr int kSizes = BY_SIZE ? 4 : 1;
    uint32_t rt[4], len[4], parts[4], per, most;
    uint32_t items[kSizes], slots, joins, own_items[kSizes], own_slots, own_joins;   // sums up to this lane, and its own
    bool bad;

    __device__ explicit PairShares(const PairArgs &a) {
        const uint32_t lane = threadIdx.x & 63;
        per = (a.kv.n_seq + 63) / 64;
        bool rows_ok = true;
        uint32_t kt[4];
        bad = false;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            rt[j] = kt[j] = 0;
            const uint32_t s = lane * per + j;
            if (j >= per || s >= a.kv.n_seq) continue;
            const Head h = seq_head(a.kv, s);
            rt[j] = (h.n * a.G + a.tile_rows - 1) >> a.tile_log;   // below 2^32 (make_pair_layout)
            kt[j] = steps_of(h);
            bad |= !h.ok;
            rows_ok &= h.rows_ok;
        }
        if (__builtin_expect(__any(!rows_ok), 0)) {
            // without those that begin among rows of an earlier one
            const Shares sh(a);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                rt[j] = sh.rt[j];
                kt[j] = sh.kt[j];
            }
        }
        // the call's steps; their sum by halves of 32 bits
        uint64_t work = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) work += (uint64_t)rt[j] * kt[j];
        uint32_t C;
        if (!__any(work >> kNarrow)) {
            C = narrow_steps(a, (uint32_t)__builtin_amdgcn_readlane((int)wave_sums((uint32_t)work), 63));
        } else {
            for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d, 64);
            C = range_steps(a, work);
        }
        own_slots = own_joins = most = 0;
#pragma unroll
        for (int z = 0; z < kSizes; ++z) own_items[z] = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            len[j] = parts[j] = 1;
            if (j >= per) continue;
            len[j] = even_steps(kt[j], C);
            parts[j] = even_parts(kt[j], C);
            if (!BY_SIZE) own_items[0] += rt[j] * parts[j];
            own_slots += parts[j] > 1 ? rt[j] * parts[j] : 0u;
            own_joins += parts[j] > 1 ? rt[j] : 0u;
            most = max(most, len[j]);
        }
        if (BY_SIZE) {
            most = wave_most(most);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
                for (int z = 0; z < kSizes; ++z) own_items[z] += j < per && size(j) == z ? rt[j] * parts[j] : 0u;
        }
#pragma unroll
        for (int z = 0; z < kSizes; ++z) items[z] = wave_sums(own_items[z]);
        slots = wave_sums(own_slots);
        joins = wave_sums(own_joins);
    }

    // By how much of the longest range's length: more than 3/4, 1/2, 1/4, less.
    __device__ int size(uint32_t j) const {
        int z = 0;
#pragma unroll
        for (int k = 1; k < kSizes; ++k) z += len[j] <= most * k / kSizes ? 1 : 0;
        return z;
    }

    // Item or join i; false if there are not so many.
    __device__ bool item(const PairArgs &a, uint32_t i, Item &it) const {
        uint32_t sum = items[0], own = own_items[0];
        int which = 0;
#pragma unroll
        for (int z = 1; z < kSizes; ++z) {
            const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)items[z - 1], 63);
            const bool past = which == z - 1 && i >= all;
            const uint32_t x = items[z], y = own_items[z];
            i -= past ? all : 0u;
            which = past ? z : which;
            sum = past ? x : sum;
            own = past ? y : own;
        }
        const uint64_t past = __ballot(sum > i);
        if (!past) return false;
        const int l = __ffsll((unsigned long long)past) - 1;
        uint32_t at = sum - own, slot = slots - own_slots, seq = 0, p = 1, n = 1, rest = 0, tiles = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t y = rt[j] * parts[j], x = size(j) == which ? y : 0u;
            if (i >= at && i < at + x) {
                seq = (threadIdx.x & 63) * per + j;
                p = parts[j];
                n = len[j];
                tiles = rt[j];
                rest = i - at;
                break;
            }
            at += x;
            slot += parts[j] > 1 ? y : 0u;
        }
        auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
        p = of(p);
        n = of(n);
        rest = of(rest);
        it.seq = of(seq);
        it.tile = of(tiles) - 1 - rest / p;
        const uint32_t part = rest % p;
        it.k0 = part * n;
        const Head h = seq_head(a.kv, it.seq);
        const uint32_t end = tile_end(h, a.G, it.tile, a.tile_rows);
        it.k1 = p > 1 ? min(end, it.k0 + n) : end;
        it.slot = p > 1 ? of(slot) + it.tile * p + part : kNoSlot;
        return true;
    }
    __device__ uint32_t n_joins() const { return (uint32_t)__builtin_amdgcn_readlane((int)joins, 63); }
    __device__ Join join(uint32_t i) const {
        const int l = __ffsll((unsigned long long)__ballot(joins > i)) - 1;
        uint32_t at = joins - own_joins, slot = slots - own_slots, seq = 0, tile = 0, p = 1;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t q = parts[j], x = q > 1 ? rt[j] : 0u;
            if (i >= at && i < at + x) {
                seq = (threadIdx.x & 63) * per + j;
                tile = i - at;
                p = q;
                slot += tile * q;
                break;
            }
            at += x;
            slot += x * q;
        }
        auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
        return Join{of(seq), of(tile), of(slot), of(p)};
    }
};

// find_item by it.
template <bool BY_SIZE>
__device__ inline bool find_range(const PairArgs &a, uint32_t i, Item &it, Head &hd) {
    if (a.items) return find_item(a, i, it, hd);
    const PairShares<BY_SIZE> sh(a);
    if (blockIdx.x == 0 && __builtin_expect(__any(sh.bad), 0)) fill_bad(a);
    if (!sh.item(a, i, it)) return false;
    auto one = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    it = Item{one(it.seq), one(it.tile), one(it.k0), one(it.k1), one(it.slot), {0, 0, 0}};
    hd = seq_head(a.kv, it.seq);
    hd.row0 = (uint64_t)one((uint32_t)(hd.row0 >> 32)) << 32 | one((uint32_t)hd.row0);
    hd.n = one(hd.n);
    hd.ctx = one(hd.ctx);
    return true;
}

// weights_of (blockdev.h) of 8 scores.
__device__ __forceinline__ float weights_of(const f32x4 (&st)[2], float sc, float by, f16x8 (&pf)[1]) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = exp2_of(fmaf(st[t][i], sc, by));
            sum += p[i];
        }
        const f16x2 u = __builtin_convertvector((f32x2{p[0], p[1]}), f16x2), v = __builtin_convertvector((f32x2{p[2], p[3]}), f16x2);
        pf[0][4 * t] = u[0];
        pf[0][4 * t + 1] = u[1];
        pf[0][4 * t + 2] = v[0];
        pf[0][4 * t + 3] = v[1];
    }
    asm volatile("" : "+v"(pf[0]), "+v"(sum));
    return sum;
}

// As attend_kernel, each wavefront for one map: the first and third take the
// first map, the others the second, two steps of the range at a time.  The two
// that work on one step read its values once from memory and once from the
// caches.  Joined through LDS.  (At 128 dimensions 39 to 43 registers are kept in
// private memory: four from before the steps to behind them, the others while a NaN
// value that only some rows see is looked for; none within an ordinary step.)  Both maps in one wavefront would read them once,
// but with twice the sums in registers, one wavefront a SIMD: 64 sequences of up to
// 16,384 tokens 174 us, 8 of 131,071 378, 200 of up to 1,000 80 and not 51.  Bound by
// memory: 8 sequences of 131,071 tokens, 8 KV heads of 128 dimensions (2.1 GB) 367
// us with the join, 5.8 TB/s; 64 of up to 16,384 (0.68 GB) 165, 4.1 TB/s, by the ends
// of unequal ranges.  One row after 700 tokens takes 14 us, its chain of loads:
// lengths, pages, keys, and through LDS.
template <int D, int NT, bool HALF, bool SMALL>
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(PairArgs a) {
    typedef typename Elem<HALF>::T T;
    typedef typename Elem<HALF>::T8 T8;
    constexpr int VD = 2 * D, kDT = VD / 16, kHalf = D / 16;
    constexpr int kPitch = VD + 4;
    __shared__ float lds[kWaves * 16 * kPitch];
    __shared__ float lds_ml[kWaves][16 * NT][3];

    const uint32_t hk = a.kv.hk;
    const uint32_t p = blockIdx.x % a.pairs, item = blockIdx.x / a.pairs;
    Item it;
    Head hd;
    if (!(a.by_size ? find_range<true>(a, item, it, hd) : find_range<false>(a, item, it, hd))) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // known to be uniform
    const uint32_t map = w & 1, first = it.k0 + (w >> 1);
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t n_rows = hd.n * a.G;
    const uint32_t row0 = it.tile * a.tile_rows;
    const uint32_t bt = 1u << a.kv.btl, tile = min(bt, kStep);
    const uint64_t hb = head_bytes(a.kv, D);
    const uint32_t *pages = a.kv.pages + (uint64_t)it.seq * a.kv.max_pages;
    const uint32_t last_block = hd.ctx ? (hd.ctx - 1) >> a.kv.btl : 0u;

    T8 qf[NT][D / 32];
    uint32_t lim[NT];
    // tokens that every row sees, and steps that any row sees
    const uint32_t row_last = min(row0 + a.tile_rows, n_rows) - 1;
    const int64_t see_all = (int64_t)hd.ctx - hd.n + row0 / a.G + 1;
    const int64_t see_any = (int64_t)hd.ctx - hd.n + row_last / a.G + 1;
    const uint32_t all_lim = see_all > 0 ? (uint32_t)min(see_all, (int64_t)hd.ctx) : 0u;
    const uint32_t end = min(it.k1, see_any > 0 ? (uint32_t)((see_any + kStep - 1) / kStep) : 0u);

    f32x4 acc[NT][kDT];
    float m[NT], l[NT], y[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = y[n] = -INFINITY;
        l[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < kDT; ++d) acc[n][d] = f32x4{0, 0, 0, 0};
    }

    // pages, scales and addresses are scalar where a step lies in one block
    auto page_at = [&](uint32_t kt, uint32_t group) {
        const uint32_t b = min((kt * kStep + (SMALL ? 16 * group : 0u)) >> a.kv.btl, last_block);
        return SMALL ? pages[b] : scalar(pages)[b];
    };
    const uint64_t page_bytes = hk * hb;
    const uint32_t key_in_page = (((SMALL ? (16 * (c >> 2)) & (tile - 1) : 16 * (c >> 2)) + (c & 3)) * D + 16 * g);
    const uint32_t val_in_page = SMALL ? c * tile + ((16 * g) & (tile - 1)) : c * kStep + 16 * g;
    const uint32_t val_piece = SMALL ? 16 * tile : 16 * kStep;
    const uint8_t *keys = a.kv.k + (2 * p + map) * hb, *vals = a.kv.v + 2 * p * hb;
    auto in_cache = [&](const uint8_t *x, uint32_t kt, uint32_t page) {
        return x + (page < a.kv.n_pages ? page : 0u) * page_bytes + (uint64_t)((kt * kStep) & (bt - 1)) * D;
    };

    // The next step's keys are asked for as soon as this one's have been
    // multiplied, its values likewise; pages a step earlier.
    constexpr uint32_t kOn = kWaves / 2;
    KeyRegs<D> kf;
    ValRegs<VD> vf;
    f32x4 st[NT][4];
    f16x8 pf[NT][2];
    float sc_next = 0.0f, va_next = 0.0f, vb_next = 0.0f, sc = 0.0f;
    ValScale vs;
    uint64_t nan_sums = 0;                             // sums of this lane that a NaN value belongs to
    static_assert(4 * NT * kDT <= 64, "a bit a sum");
    uint32_t pk = 0, pv = 0;
    auto load_keys = [&](uint32_t kt, uint32_t page) {
        const uint8_t *x = in_cache(keys, kt, page);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) kf.f[t][i] = *(const u32x4 *)(x + key_in_page + 4 * t * D + 64 * i);
    };
    auto load_vals = [&](uint32_t kt, uint32_t page) {
        const uint8_t *x = in_cache(vals, kt, page);
#pragma unroll
        for (int d = 0; d < kDT; ++d) vf.f[d] = *(const u32x4 *)(x + (d / kHalf) * hb + val_in_page + (d % kHalf) * val_piece);
    };
    auto load_scales = [&]() {
        const bool bad = pv >= a.kv.n_pages;
        if (bad) report(a.kv);
        const uint64_t si = (uint64_t)(bad ? 0u : pv) * hk + 2 * p;
        sc_next = SMALL ? a.kv.ks[si + map] : scalar(a.kv.ks)[si + map];
        va_next = SMALL ? a.kv.vs[si] : scalar(a.kv.vs)[si];
        vb_next = SMALL ? a.kv.vs[si + 1] : scalar(a.kv.vs)[si + 1];
        if (bad) sc_next = va_next = vb_next = NAN;
    };
    auto find_pages = [&](uint32_t kt) {
        pk = page_at(kt, c >> 2);
        pv = SMALL ? page_at(kt, g) : pk;
    };
    auto scores = [&](uint32_t kt) {
        vs = val_scale(va_next, vb_next);
        const float x = sc_next * a.c0;
        sc = x == 0.0f ? 1.0e-30f : x;                 // not 0, which would turn a masked score's -inf into NaN
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < 4; ++t) st[n][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const T8 lo = widen<HALF>(kf.f[t][i][0], kf.f[t][i][1]);
                const T8 hi = widen<HALF>(kf.f[t][i][2], kf.f[t][i][3]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    st[n][t] = product(lo, qf[n][2 * i], st[n][t]);
                    st[n][t] = product(hi, qf[n][2 * i + 1], st[n][t]);
                }
            }
        if (kt + kOn < end) {
            load_keys(kt + kOn, pk);
            load_scales();
        }
    };
    auto values = [&](uint32_t kt) {
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            const f16x8 lo = times(widen_f16(vf.f[d][0], vf.f[d][1]), vs.r[d / kHalf]);
            const f16x8 hi = times(widen_f16(vf.f[d][2], vf.f[d][3]), vs.r[d / kHalf]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                acc[n][d] = product(lo, pf[n][0], acc[n][d]);
                acc[n][d] = product(hi, pf[n][1], acc[n][d]);
            }
        }
        if (kt + kOn < end) {
            load_vals(kt + kOn, pv);
            find_pages(kt + 2 * kOn);
        }
    };
    // as attend_kernel's
    auto softmax = [&]() {
        const float vlog = log2_of(vs.s);
        float up[NT], sum[NT];
        bool fits = true;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float by = vlog - y[n];
            up[n] = -by - m[n];
            sum[n] = weights_of(st[n], sc, by, pf[n]);
            fits &= sum[n] <= kMaxSum && fabsf(up[n]) < 64.0f;
        }
        if (!__all(fits)) return false;
#pragma unroll
        for (int n = 0; n < NT; ++n) l[n] += sum[n] * exp2_of(up[n]);
        return true;
    };
    auto softmax_any = [&](uint32_t kt) {
        const float vlog = log2_of(vs.s);
        const uint32_t tok0 = kt * kStep + 16 * g;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int left = (int)lim[n] - (int)tok0;
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[n][t][i] = left > 4 * t + i ? st[n][t][i] : -INFINITY;
                    mx = fmaxf(mx, st[n][t][i]);
                }
            mx = mx == -INFINITY ? -INFINITY : mx * sc;
            const float mn = fmaxf(m[n], row_max(mx)), yn = fmaxf(y[n], row_max(mx + vlog) - kLift);
            l[n] *= m[n] == -INFINITY ? 1.0f : exp2_of(m[n] - mn);   // nothing so far: 0, or NaN
            const float al = y[n] == -INFINITY ? 1.0f : exp2_of(y[n] - yn);
            m[n] = mn;
            y[n] = yn;
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][d][i] *= al;
            // the weights and their sum from one pass where fp32 holds both
            const float by = yn == -INFINITY ? -INFINITY : vlog - yn, up = -by - mn;
            if (__all(fabsf(up) < 64.0f)) {
                l[n] += weights_of(st[n], sc, by, pf[n]) * exp2_of(up);
            } else {
                l[n] += weights_of(st[n], sc, mn == -INFINITY ? 0.0f : -mn, pf[n]);
                weights_of(st[n], sc, by, pf[n]);
            }
        }
        if (kt * kStep + kStep <= all_lim) return;
        // Tokens that not every row sees: bytes of slots that hold none may be
        // anything, and a NaN that some rows see and others do not is left out of
        // the product and found by one of the masks (see attend_kernel).
        const int have = (int)min(16u, hd.ctx > tok0 ? hd.ctx - tok0 : 0u);
        u32x4 keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = have - 4 * i;
            keep[i] = b >= 4 ? 0xFFFFFFFFu : b <= 0 ? 0u : (1u << (8 * b)) - 1u;
        }
        bool nan = false;
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            vf.f[d] &= keep;
#pragma unroll
            for (int i = 0; i < 4; ++i) nan |= nan_bytes(vf.f[d][i]) != 0;
        }
        if (!__any(nan)) return;
        uint64_t found = 0;                            // four bits at a time, from the top
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            u32x4 z;
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = nan_bytes(vf.f[d][i]);
            const u32x4 one = z * 0x38u;               // 1.0 per NaN
            vf.f[d] &= ~(z * 0xFFu);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int left = (int)lim[n] - (int)tok0;
                f16x8 see[2];
#pragma unroll
                for (int j = 0; j < 16; ++j) see[j >> 3][j & 7] = left > j ? (_Float16)1.0f : (_Float16)0.0f;
                f32x4 hit = {0, 0, 0, 0};
                hit = product(widen_f16(one[0], one[1]), see[0], hit);
                hit = product(widen_f16(one[2], one[3]), see[1], hit);
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) bits |= hit[i] > 0.0f ? 1u << i : 0u;
                found = found >> 4 | (uint64_t)bits << 60;
            }
        }
        nan_sums |= found;
    };
    if (first < end) {
        find_pages(first);
        load_keys(first, pk);
        load_scales();
        load_vals(first, pv);
        find_pages(first + kOn);
    }
    // the queries, behind the first step's loads
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t r = row0 + n * 16 + c;
        const bool valid = r < n_rows;
        const uint32_t t = valid ? r / a.G : 0u, j = p * a.G + (valid ? r % a.G : 0u);
        const int64_t seen = (int64_t)hd.ctx - hd.n + t + 1;
        lim[n] = !valid ? hd.ctx : seen > 0 ? (uint32_t)seen : 0u;
        const T *q = (const T *)a.q + (hd.row0 + t) * a.q_stride + (uint64_t)(2 * j + map) * D + 16 * g;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4 x = {0, 0, 0, 0};
            if (valid) x = *(const u32x4 *)(q + (i / 2) * 64 + (i % 2) * 8);
            qf[n][i] = __builtin_bit_cast(T8, x ^ a.q_sign);
        }
    }
    // the ordinary steps have a loop of their own (see prompt_kernel)
    for (uint32_t kt = first; kt < end; kt += kOn) {
        bool done;
        do {
            scores(kt);
            done = kt * kStep + kStep <= all_lim;
            if (done) done = softmax();
            if (!done) break;
            values(kt);
            kt += kOn;
        } while (kt < end);
        if (done) break;
        softmax_any(kt);
        values(kt);
    }
    if (nan_sums)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (nan_sums >> (64 - 4 * NT * kDT + 4 * (d * NT + n) + i) & 1) acc[n][d][i] = NAN;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] = row_sum(l[n]);
        if (g == 0) {
            lds_ml[w][n * 16 + c][0] = m[n];
            lds_ml[w][n * 16 + c][1] = l[n];
            lds_ml[w][n * 16 + c][2] = y[n];
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDT; ++d) *(f32x4 *)&lds[(w * 16 + c) * kPitch + d * 16 + 4 * g] = acc[n][d];
        __syncthreads();
        for (uint32_t e = threadIdx.x; e < 16 * VD / 4; e += kThreads) {
            const uint32_t row = e / (VD / 4), d4 = e % (VD / 4) * 4, r = row0 + n * 16 + row;
            if (r >= n_rows) continue;                 // a row's lanes go together
            f32x4 o[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float *a0 = lds_ml[q][n * 16 + row], *a1 = lds_ml[q + 2][n * 16 + row];
                const float M = fmaxf(a0[0], a1[0]), Y = fmaxf(a0[2], a1[2]);
                const float L = joined(a0[0], M) * a0[1] + joined(a1[0], M) * a1[1];
                const float f0 = joined(a0[2], Y), f1 = joined(a1[2], Y);
                const f32x4 x0 = *(const f32x4 *)&lds[(q * 16 + row) * kPitch + d4], x1 = *(const f32x4 *)&lds[((q + 2) * 16 + row) * kPitch + d4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[q][i] = x0[i] * f0 + x1[i] * f1;
                if (it.slot != kNoSlot) {
                    const uint64_t at = (((uint64_t)it.slot * a.pairs + p) * 2 + q) * a.tile_rows + n * 16 + row;
                    if (d4 == 0) a.part_ml[at] = f32x4{M, L, Y, 0.0f};
                    *(f32x4 *)(a.part + at * VD + d4) = o[q];
                } else {
                    const Over over(Y, M, L, hd.ctx + r / a.G >= hd.n);   // both below 2^31
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[q][i] = over(o[q][i]);
                }
            }
            if (it.slot != kNoSlot) continue;
            const uint32_t j = p * a.G + r % a.G;
            finish<VD>(a, o[0], o[1], j, (T *)a.out + (hd.row0 + r / a.G) * a.out_stride + (uint64_t)j * VD, d4 / 4);
        }
    }
}

// The same for prompts, as prompt_kernel: every step's keys and values are
// widened into LDS once, and two groups of four wavefronts go through the
// tokens half a step apart.  The first group has the first map, the second one
// the other, of the same 64 NT rows, so each reads its own keys and both the
// pair's values.  Slot 2 k is the first group's products of step k (O of the
// step before, S of this one) and the second one's softmax of step k - 1, slot
// 2 k + 1 the reverse.  The first group widens both maps' keys k + 1 with its
// softmax k (slot 2 k + 1: its own keys k - 1, in the same buffer, were last
// read in slot 2 k - 2, the second group's in slot 2 k - 1), the second one
// values k + 1 with its own (slot 2 k + 2: values k - 1 were last read in slot
// 2 k + 1, values k + 1 are first read in slot 2 k + 4).  At the end the second
// map's rows go to the first group through LDS.
// Two chunks of 1,024 rows after 31,744 tokens, 64 and 8 heads of 128 dimensions (3.2
// TFLOP) 3,240 us with all launches, 990 TFLOP/s, 81 % of a large matrix product's
// rate; six prompts of up to 2,777, 64 and 16 heads of 64 (233 GFLOP) 443 us, 525 TFLOP/s:
// a tile has 17 steps, of which the first and the masked one take nearly twice the
// others' 2 us, and 9 us beside them.  The chunks are bound by the chains in a slot,
// which two wavefronts a SIMD do not cover: of its 1,880 cycles the matrix unit
// works for 770 and vector instructions for 630.  The prompts, in blocks of 16 tokens,
// by both units in turn, as there the groups are in step: of a step's 4,800 cycles
// two wavefronts' products take 1,540 and their vector instructions 2,900.  Counted
// over the chunks (prompts) the matrix unit is busy 41 (25) % of the time, vector
// instructions 44 (53), LDS 31 (17), and a wavefront waits for the other group or for
// data for 40 (37) % of its own.
// Measured and not kept: loads straight into LDS (chunks 3.8 ms: what they wait
// for is not the memory), more priority for the products (no change), and the
// widening in loops of its own behind them (registers do not suffice).
template <int D, int NT, int STEP, bool HALF, bool SMALL>
__global__ __launch_bounds__(kPromptThreads, 2) void pair_prompt_kernel(PairArgs a) {
    typedef typename Elem<HALF>::T T;
    typedef typename Elem<HALF>::T8 T8;
    constexpr int VD = 2 * D, kDT = VD / 16;
    constexpr int kAhead = D == 128 ? 4 : 6;          // fragments read ahead of their products
    constexpr int kT = STEP / 16, kU = STEP / 32;     // products with the keys, fragments of a tile of values a step
    constexpr uint32_t kGroup = STEP / 4;             // tokens of a lane
    constexpr bool kApart = !SMALL;                   // the groups half a step apart
    constexpr int kShare = kT * D / 128;              // 16-byte pieces of keys or values a lane stages
    constexpr int kKeys = kT * D / 32, kVals = kU * kDT;   // fragments of one map's keys, of the values
    __shared__ u32x4 lds[2 * (2 * kKeys + kVals)][64];
    __shared__ uint8_t lds_bits[2][kVals][64];        // which of a fragment lane's 8 values were NaN
    __shared__ uint64_t lds_sums[NT][kPromptThreads];   // sums of a lane that a NaN value belongs to, a bit each
    __shared__ uint32_t lds_nan[2];
    static_assert(4 * kDT <= 2 * (2 * kKeys + kVals), "a map's 64 rows fit");

    const uint32_t hk = a.kv.hk;
    const uint32_t p = blockIdx.x % a.pairs, item = blockIdx.x / a.pairs;
    Item it;
    Head hd;
    if (!find_range<false>(a, item, it, hd)) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // known to be uniform
    const bool second = w >= 4;
    const uint32_t map = second;
    auto lds_k = [&](int b, uint32_t q, int f) -> u32x4 * { return lds[(2 * b + q) * kKeys + f]; };
    auto lds_v = [&](int b, int f) -> u32x4 * { return lds[4 * kKeys + b * kVals + f]; };
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t n_rows = hd.n * a.G;
    const uint32_t row0 = it.tile * a.tile_rows + (w & 3) * 16 * NT;
    const uint32_t bt = 1u << a.kv.btl, tile = min(bt, kStep), in_step = min(bt, (uint32_t)STEP);
    const uint64_t hb = head_bytes(a.kv, D);
    const uint32_t *pages = a.kv.pages + (uint64_t)it.seq * a.kv.max_pages;
    const uint32_t last_block = hd.ctx ? (hd.ctx - 1) >> a.kv.btl : 0u;

    T8 qf[NT][D / 32];
    // tokens that a row sees (all for one that is none); not kept, only some steps need it
    auto lim_of = [&](int n) {
        const uint32_t r = row0 + n * 16 + c;
        const int64_t seen = (int64_t)hd.ctx - hd.n + r / a.G + 1;
        return r >= n_rows ? hd.ctx : seen > 0 ? (uint32_t)seen : 0u;
    };
    // tokens that every row of this wavefront sees, and of the tile (see prompt_kernel)
    const int64_t see_all = (int64_t)hd.ctx - hd.n + row0 / a.G + 1;
    const uint32_t all_lim = see_all > 0 ? (uint32_t)min(see_all, (int64_t)hd.ctx) : 0u;
    const int64_t see_tile = (int64_t)hd.ctx - hd.n + it.tile * a.tile_rows / a.G + 1;
    const uint32_t tile_lim = see_tile > 0 ? (uint32_t)min(see_tile, (int64_t)hd.ctx) : 0u;

    // the range's steps, those that no row sees left out
    const int64_t see_any = (int64_t)hd.ctx - hd.n + (min((it.tile + 1) * a.tile_rows, n_rows) - 1) / a.G + 1;
    const uint32_t k0 = it.k0 * (kStep / STEP), k1 = min(it.k1 * (kStep / STEP), see_any > 0 ? (uint32_t)((see_any + STEP - 1) / STEP) : 0u);

    f32x4 acc[NT][kDT], st[NT][kT];
    f16x8 pf[NT][kU];
    float m[NT], l[NT], y[NT];
    static_assert(4 * kDT <= 64, "a bit a sum");
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = y[n] = -INFINITY;
        l[n] = 0.0f;
        lds_sums[n][threadIdx.x] = 0;
#pragma unroll
        for (int u = 0; u < kU; ++u) pf[n][u] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int d = 0; d < kDT; ++d) acc[n][d] = f32x4{0, 0, 0, 0};
    }

    // this lane's pieces: 16 dimensions of key row c of a product, and values: 16
    // tokens of a dimension, the lane's own 16, or of 32-token steps those of two
    // groups of lanes
    u32x4 px[kShare];
    float sc_at[2], vs_at[2], rv_at[2];                // scales of this step and the next; r of the half that this wavefront widens
    const uint32_t half = second ? (w - 4) >> 1 : 0u;
    const uint32_t v_dim = STEP == 64 ? c : lane >> 1, v_group = STEP == 64 ? g : lane & 1;
    const uint32_t own_group = SMALL ? second ? v_group : kGroup * (c >> 2) / 16 : 0u;   // whose page this lane's pieces are in
    const uint32_t group = kGroup * g / 16;            // and its scores' tokens
    auto page_at = [&](uint32_t kt, uint32_t group) {
        const uint32_t block = min((kt * STEP + (SMALL ? 16 * group : 0u)) >> a.kv.btl, last_block);
        return SMALL ? pages[block] : scalar(pages)[block];
    };
    const uint8_t *own = (second ? a.kv.v : a.kv.k) + (2 * p + half) * hb;
    const uint64_t page_bytes = hk * hb;
    constexpr int kTiles = STEP == 64 ? 1 : 2;         // value tiles a piece
    // pieces i: keys, of product t D / 64 of one map, then of the other (64-token
    // steps), or of one map (32); values, kTiles tiles in a row
    const uint32_t t_own = STEP == 64 ? w & 3 : w & 1, q_own = STEP == 64 ? 0u : (w & 3) >> 1;
    const uint32_t in_page = second ? v_dim * tile + ((16 * v_group) & (in_step - 1)) + (w & 1) * kShare * kTiles * 16 * tile
                                    : (((kGroup * (c >> 2)) & (in_step - 1)) + (c & 3) + 4 * t_own) * D + 16 * g;
    const uint64_t piece = second ? kTiles * 16 * tile : 64;
    const uint64_t jump = second ? (uint64_t)(D / 64) * piece : hb;   // from piece D / 64 on
    if (!second) own += q_own * hb;
    const float *ks = a.kv.ks + 2 * p + map, *vs = a.kv.vs + 2 * p;
    // The scales of the scores' page pv, and for r those of the pieces' page pr:
    // asked for first, looked at later.
    struct Scales {
        float k, va, vb, wa, wb;
    };
    auto ask = [&](uint32_t pv, uint32_t pr, Scales &x) {
        const uint64_t si = (uint64_t)(pv < a.kv.n_pages ? pv : 0u) * hk;
        x.k = SMALL ? ks[si] : scalar(ks)[si];
        x.va = SMALL ? vs[si] : scalar(vs)[si];
        x.vb = SMALL ? vs[si + 1] : scalar(vs)[si + 1];
        if constexpr (SMALL && STEP == 32) {
            const uint64_t so = (uint64_t)(pr < a.kv.n_pages ? pr : 0u) * hk;
            x.wa = vs[so];
            x.wb = vs[so + 1];
        }
    };
    auto look = [&](uint32_t pv, const Scales &x, float &sc, float &vsc, float &rv) {
        const ValScale v = val_scale(x.va, x.vb);
        sc = x.k;
        vsc = v.s;
        rv = half ? v.r[1] : v.r[0];
        if constexpr (SMALL && STEP == 32) {
            const ValScale o = val_scale(x.wa, x.wb);
            rv = half ? o.r[1] : o.r[0];
        }
        if (pv >= a.kv.n_pages) {
            report(a.kv);
            sc = vsc = NAN;
        }
        if constexpr (!SMALL) {                        // the same for all lanes: in scalar registers
            auto one = [](float &x) { x = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x))); };
            one(sc);
            one(vsc);
            one(rv);
        }
    };
    auto fetch = [&](uint32_t kt, uint32_t po) {
        const uint32_t t0 = (kt * STEP) & (bt - 1);
        const uint8_t *x = own + (po < a.kv.n_pages ? po : 0u) * page_bytes + (second ? (uint64_t)(t0 & ~(tile - 1)) * D + (t0 & (tile - 1)) : (uint64_t)t0 * D);
#pragma unroll
        for (int i = 0; i < kShare; ++i) px[i] = *(const u32x4 *)(x + in_page + (i / (D / 64)) * jump + (i % (D / 64)) * piece);
    };
    auto stage = [&](uint32_t kt, float rv) {
        const int b = kt & 1;
        if (!second) {
#pragma unroll
            for (int i = 0; i < kShare; ++i) {
                const int f = t_own * (D / 32) + 2 * (i % (D / 64));
                lds_k(b, q_own + i / (D / 64), f)[lane] = __builtin_bit_cast(u32x4, widen<HALF>(px[i][0], px[i][1]));
                lds_k(b, q_own + i / (D / 64), f + 1)[lane] = __builtin_bit_cast(u32x4, widen<HALF>(px[i][2], px[i][3]));
            }
            return;
        }
        // where a piece's 16 tokens go: two fragments of a tile at the lane's own
        // place, or one at two lanes' places
        auto place = [&](int i, int h) {
            const uint32_t d = ((w - 4) * kShare + i) * kTiles + (STEP == 64 ? 0u : v_dim >> 4);
            return STEP == 64 ? (2 * d + h) * 64 + lane : d * 64 + (2 * v_group + h) * 16 + (v_dim & 15);
        };
        if (kt * STEP + STEP > tile_lim) {
            // bytes of slots that hold no token are cleared, a NaN is taken out
            // and noted
            const uint32_t tok0 = kt * STEP + 16 * v_group;
            const int have = (int)min(16u, hd.ctx > tok0 ? hd.ctx - tok0 : 0u);
            bool nan = false;
#pragma unroll
            for (int i = 0; i < kShare; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = have - 4 * j;
                    px[i][j] &= n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
                    nan |= nan_bytes(px[i][j]) != 0;
                }
            if (__any(nan)) {
                uint8_t *bits_at = &lds_bits[b][0][0];
#pragma unroll
                for (int i = 0; i < kShare; ++i) {
                    uint32_t bits = 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t z = nan_bytes(px[i][q]);
                        px[i][q] &= ~(z * 0xFFu);
                        bits |= ((z | z >> 7 | z >> 14 | z >> 21) & 15u) << (4 * q);
                    }
                    bits_at[place(i, 0)] = (uint8_t)bits;
                    bits_at[place(i, 1)] = (uint8_t)(bits >> 8);
                }
                if (lane == 0) atomicOr(&lds_nan[b], 1u << (w - 4));
            } else if (lane == 0) {
                atomicAnd(&lds_nan[b], ~(1u << (w - 4)));
            }
        }
        const bool scaled = !__all(rv == 1.0f);
        u32x4 *to = lds_v(b, 0);
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            f16x8 lo = widen_f16(px[i][0], px[i][1]), hi = widen_f16(px[i][2], px[i][3]);
            if (scaled) {
                lo = times(lo, rv);
                hi = times(hi, rv);
            }
            to[place(i, 0)] = __builtin_bit_cast(u32x4, lo);
            to[place(i, 1)] = __builtin_bit_cast(u32x4, hi);
        }
    };
    // LDS alone is handed over: loads from memory stay in flight
    auto meet = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    // a product's sums are four fragments apart: each waits for none
    auto scores = [&](uint32_t kt) {
        const int b = kt & 1;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < kT; ++t) st[n][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < kT; t += 2)
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const T8 kf = __builtin_bit_cast(T8, lds_k(b, map, (t + q) * (D / 32) + i)[lane]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) st[n][t + q] = product(kf, qf[n][i], st[n][t + q]);
                }
    };
    auto values = [&](uint32_t kt) {
        const int b = kt & 1;
#pragma unroll
        for (int d = 0; d < kDT; d += 2)
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f16x8 vf = __builtin_bit_cast(f16x8, lds_v(b, kU * (d + q) + u)[lane]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][d + q] = product(vf, pf[n][u], acc[n][d + q]);
                }
    };
    // `reads` fragments in all, each for NT products: kAhead on their way
    auto interleave = [&](auto reads) {
        constexpr int kReads = decltype(reads)::value;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < kReads - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, NT, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead * NT, 0);
    };
    // not 0, which would turn a masked score's -inf into NaN
    auto scale_of = [&]() {
        const float x = sc_at[0] * a.c0;
        return x == 0.0f ? 1.0e-30f : x;
    };
    // as prompt_kernel's
    auto softmax = [&]() {
        const float sc = scale_of(), vlog = log2_of(vs_at[0]);
        float up[NT], sum[NT];                         // up: log2 of a weight over its P
        bool fits = true;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float by = vlog - y[n];
            up[n] = -by - m[n];
            sum[n] = weights_of(st[n], sc, by, pf[n]);
            fits &= sum[n] <= kMaxSum && fabsf(up[n]) < 64.0f;
        }
        if (!__all(fits)) return false;
#pragma unroll
        for (int n = 0; n < NT; ++n) l[n] += sum[n] * exp2_of(up[n]);
        return true;
    };
    auto softmax_any = [&](uint32_t kt) {
        const float sc = scale_of(), vlog = log2_of(vs_at[0]);
        const uint32_t tok0 = kt * STEP + kGroup * g;
        if (kt * STEP + STEP > tile_lim) {
            const uint32_t noted = lds_nan[kt & 1];
            if (noted)
#pragma unroll 1
                for (int d = 0; d < kDT; ++d) {
                    if (!(noted >> (d / (kDT / 4)) & 1)) continue;
                    f32x4 hit[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) hit[n] = f32x4{0, 0, 0, 0};
#pragma unroll 1
                    for (int u = 0; u < kU; ++u) {
                        const uint32_t bits = lds_bits[kt & 1][kU * d + u][lane];
                        f16x8 one;
#pragma unroll
                        for (int j = 0; j < 8; ++j) one[j] = bits >> j & 1 ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const int left = (int)lim_of(n) - (int)tok0 - 8 * u;
                            f16x8 see;
#pragma unroll
                            for (int j = 0; j < 8; ++j) see[j] = left > j ? (_Float16)1.0f : (_Float16)0.0f;
                            hit[n] = product(one, see, hit[n]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) lds_sums[n][threadIdx.x] |= (uint64_t)(hit[n][i] > 0.0f) << (4 * d + i);
                }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int left = (int)lim_of(n) - (int)tok0;
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < kT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[n][t][i] = left > 4 * t + i ? st[n][t][i] : -INFINITY;
                    mx = fmaxf(mx, st[n][t][i]);
                }
            mx = mx == -INFINITY ? -INFINITY : mx * sc;
            const float mn = fmaxf(m[n], row_max(mx)), yn = fmaxf(y[n], row_max(mx + vlog) - kLift);
            l[n] *= m[n] == -INFINITY ? 1.0f : exp2_of(m[n] - mn);   // nothing so far: 0, or NaN
            const float al = y[n] == -INFINITY ? 1.0f : exp2_of(y[n] - yn);
            m[n] = mn;
            y[n] = yn;
#pragma unroll
                for (int d = 0; d < kDT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][d][i] *= al;
            // the weights and their sum from one pass where fp32 holds both
            const float by = yn == -INFINITY ? -INFINITY : vlog - yn, up = -by - mn;
            if (__all(fabsf(up) < 64.0f)) {
                l[n] += weights_of(st[n], sc, by, pf[n]) * exp2_of(up);
            } else {
                l[n] += weights_of(st[n], sc, mn == -INFINITY ? 0.0f : -mn, pf[n]);
                weights_of(st[n], sc, by, pf[n]);
            }
        }
    };

    // pages of the step after next and the one after it
    uint32_t po = 0, pv = 0, po_on = 0, pv_on = 0;
    Scales on;                                        // scales of the step after next
    float sc_on = 0.0f, vs_on = 0.0f, rv_on = 1.0f;
    auto load_queries = [&]() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t r = row0 + n * 16 + c;
            const bool valid = r < n_rows;
            const uint32_t t = valid ? r / a.G : 0u, j = p * a.G + (valid ? r % a.G : 0u);
            const T *q = (const T *)a.q + (hd.row0 + t) * a.q_stride + (uint64_t)(2 * j + map) * D + 16 * g;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                u32x4 x = {0, 0, 0, 0};
                if (valid) x = *(const u32x4 *)(q + (i / 2) * 64 + (i % 2) * 8);
                qf[n][i] = __builtin_bit_cast(T8, x);
            }
        }
    };
    if (threadIdx.x < 2) lds_nan[threadIdx.x] = 0;
    // the first step's products with "the step before" are of zeros
    for (uint32_t i = threadIdx.x; i < kVals * 64; i += kPromptThreads) lds_v(~k0 & 1, 0)[i] = u32x4{0, 0, 0, 0};
    meet();
    sc_at[0] = vs_at[0] = sc_at[1] = vs_at[1] = 0.0f;
    rv_at[0] = rv_at[1] = 1.0f;
    if (k0 < k1) {
        // one wait for the pages, one for what they hold
        const uint32_t o0 = page_at(k0, own_group), s0 = SMALL ? page_at(k0, group) : o0;
        const uint32_t o1 = page_at(k0 + 1, own_group), s1 = SMALL ? page_at(k0 + 1, group) : o1;
        po = page_at(k0 + 2, own_group);
        pv = SMALL ? page_at(k0 + 2, group) : po;
        Scales x0, x1;
        ask(s0, o0, x0);
        fetch(k0, o0);
        ask(s1, o1, x1);
        load_queries();
        look(s0, x0, sc_at[0], vs_at[0], rv_at[0]);
        stage(k0, rv_at[0]);
        fetch(k0 + 1, o1);
        look(s1, x1, sc_at[1], vs_at[1], rv_at[1]);
    }
    meet();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) qf[n][i] = __builtin_bit_cast(T8, __builtin_bit_cast(u32x4, qf[n][i]) ^ a.q_sign);
    if (kApart && second) meet();
    // Small loads for later steps go out before the softmax, which hides them
    // (page_at stays within the sequence's blocks past its end).
    auto look_ahead = [&](uint32_t kt) {
        ask(pv, po, on);
        if constexpr (!SMALL) look(pv, on, sc_on, vs_on, rv_on);
        po_on = page_at(kt + 3, own_group);
        pv_on = SMALL ? page_at(kt + 3, group) : po_on;
    };
    auto pass_on = [&](uint32_t kt) {
        if (kt + 1 < k1) {
            stage(kt + 1, rv_at[1]);
            fetch(kt + 2, po);
        }
        sc_at[0] = sc_at[1];
        vs_at[0] = vs_at[1];
        if constexpr (SMALL) look(pv, on, sc_on, vs_on, rv_on);
        sc_at[1] = sc_on;
        vs_at[1] = vs_on;
        rv_at[1] = rv_on;
        po = po_on;
        pv = pv_on;
        meet();
    };
    // the ordinary steps have a loop of their own (see prompt_kernel)
    for (uint32_t kt = k0; kt < k1; ++kt) {
        bool done;
        do {
            values(kt - 1);
            scores(kt);
            interleave(std::integral_constant<int, kVals + kKeys>());
            meet();
            done = kt * STEP + STEP <= all_lim && kt > k0;   // the first step sets the maxima
            if (kt * STEP + STEP > tile_lim) done = done && __builtin_amdgcn_readfirstlane(lds_nan[kt & 1]) == 0;
            look_ahead(kt);
            if (done) done = softmax();
            if (!done) break;
            pass_on(kt);
            ++kt;
        } while (kt < k1);
        if (done) break;
        softmax_any(kt);
        pass_on(kt);
    }
    if (kApart && !second) meet();
    if (k0 < k1) values(k1 - 1);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] = row_sum(l[n]);
        const uint64_t nan_sums = lds_sums[n][threadIdx.x];
        if (nan_sums)
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (nan_sums >> (4 * d + i) & 1) acc[n][d][i] = NAN;
    }
    if (it.slot != kNoSlot) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t tr = (w & 3) * 16 * NT + n * 16 + c;
            if (row0 + n * 16 + c >= n_rows) continue;
            const uint64_t at = (((uint64_t)it.slot * a.pairs + p) * 2 + map) * a.tile_rows + tr;
            if (g == 0) a.part_ml[at] = f32x4{m[n], l[n], y[n], 0.0f};
#pragma unroll
            for (int d = 0; d < kDT; ++d) *(f32x4 *)(a.part + at * VD + d * 16 + 4 * g) = acc[n][d];
        }
        return;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const Over over(y[n], m[n], l[n], lim_of(n) > 0);
#pragma unroll
        for (int d = 0; d < kDT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][d][i] = over(acc[n][d][i]);
    }
    f32x4(*other)[64] = (f32x4(*)[64]) & lds[(w & 3) * kDT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        __syncthreads();                              // the last values, or the rows before these, have been read
        if (second)
#pragma unroll
            for (int d = 0; d < kDT; ++d) other[d][lane] = acc[n][d];
        __syncthreads();
        if (second) continue;
        const uint32_t r = row0 + n * 16 + c;
        const bool valid = r < n_rows;
        const uint32_t j = p * a.G + (valid ? r % a.G : 0u);
        const float lam = a.lambda[j];
        float most = 0.0f;
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            const f32x4 x = other[d][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[n][d][i] = fmaf(-lam, x[i], acc[n][d][i]);
                most = fmaxf(most, fabsf(acc[n][d][i]));
            }
        }
        if (a.norm) {
            Rms rms(row_max(most), a.root_eps);
            float sum = 0.0f;
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += rms.square(acc[n][d][i]);
            rms.close(row_sum(sum), 1.0f / VD, a.root_eps);
#pragma unroll
            for (int d = 0; d < kDT; ++d) {
                const f32x4 wn = *(const f32x4 *)(a.norm + d * 16 + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][d][i] = rms(acc[n][d][i]) * wn[i];
            }
        }
        if (!valid) continue;
        T *out = (T *)a.out + (hd.row0 + r / a.G) * a.out_stride + (uint64_t)j * VD + 4 * g;
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            T o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = (T)(acc[n][d][i] * a.gain);
            *(u32x2 *)(out + d * 16) = *(u32x2 *)o;
        }
    }
}

// Joins the ranges of one row, each map as join_row does, by WAVES wavefronts:
// 7 to 9 us for what up to 512 workgroups left, latency.
template <int VD, bool HALF, int WAVES>
__device__ inline void join_pair(const PairArgs &a, const Join &j, uint32_t p, uint32_t tr, f32x4 *lo, float *factor, float (*red)[kWaves]) {
    typedef typename Elem<HALF>::T T;
    constexpr uint32_t kLanes = 64 * WAVES, kCols = VD / 4, kGroups = kLanes / kCols;
    auto meet = [&]() {
        if constexpr (WAVES > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    const uint32_t rows = a.tile_rows;
    const uint32_t me = threadIdx.x % kLanes, lane = threadIdx.x & 63, w = me >> 6;
    const uint32_t col = me % kCols, grp = me / kCols;
    const Head hd = seq_head(a.kv, j.seq);
    const uint32_t r = j.tile * rows + tr;
    if (r >= hd.n * a.G) return;
    const uint64_t by = (uint64_t)a.pairs * 2 * rows, at = ((uint64_t)j.slot * a.pairs + p) * 2 * rows + tr;
    float M[2] = {-INFINITY, -INFINITY}, Y[2] = {-INFINITY, -INFINITY};
    for (uint32_t i = me; i < j.n; i += kLanes)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const f32x4 ml = a.part_ml[at + i * by + q * rows];
            M[q] = fmaxf(M[q], ml[0]);
            Y[q] = fmaxf(Y[q], ml[2]);
        }
#pragma unroll
    for (int q = 0; q < 2; ++q)
        for (int d = 32; d; d >>= 1) {
            M[q] = fmaxf(M[q], __shfl_xor(M[q], d, 64));
            Y[q] = fmaxf(Y[q], __shfl_xor(Y[q], d, 64));
        }
    if constexpr (WAVES > 1) {
        if (lane == 0)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                red[q][w] = M[q];
                red[2 + q][w] = Y[q];
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 2; ++q)
            for (int v = 0; v < WAVES; ++v) {
                M[q] = fmaxf(M[q], red[q][v]);
                Y[q] = fmaxf(Y[q], red[2 + q][v]);
            }
    }
    float L[2] = {0.0f, 0.0f};
    f32x4 o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    for (uint32_t i0 = 0; i0 < j.n; i0 += kLanes) {
        const uint32_t i = i0 + me;
        if (i < j.n)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x4 ml = a.part_ml[at + i * by + q * rows];
                factor[q * kThreads + me] = joined(ml[2], Y[q]);
                L[q] += joined(ml[0], M[q]) * ml[1];
            }
        meet();
        const uint32_t n = min(j.n - i0, kLanes);
        const float *x0 = a.part + (at + i0 * by) * VD + col * 4;
#pragma unroll 4
        for (uint32_t g = grp; g < n; g += kGroups)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x4 x = *(const f32x4 *)(x0 + (g * by + q * rows) * VD);
                const float f = factor[q * kThreads + g];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[q][e] += f * x[e];
            }
        meet();
    }
    f32x4 both[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        for (int d = 32; d; d >>= 1) L[q] += __shfl_xor(L[q], d, 64);
        if (WAVES > 1 && lane == 0) red[4 + q][w] = L[q];
        lo[q * kThreads + grp * kCols + col] = o[q];
    }
    meet();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if constexpr (WAVES > 1) {
            L[q] = 0.0f;
            for (int v = 0; v < WAVES; ++v) L[q] += red[4 + q][v];
        }
        o[q] = f32x4{0, 0, 0, 0};
        for (uint32_t i = 0; i < kGroups; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[q][e] += lo[q * kThreads + i * kCols + col][e];
        const Over over(Y[q], M[q], L[q], hd.ctx + r / a.G >= hd.n);   // both below 2^31
#pragma unroll
        for (int e = 0; e < 4; ++e) both[q][e] = over(o[q][e]);
    }
    meet();
    if (grp) return;
    const uint32_t jq = p * a.G + r % a.G;
    finish<VD>(a, both[0], both[1], jq, (T *)a.out + (hd.row0 + r / a.G) * a.out_stride + (uint64_t)jq * VD, col);
}

// As join_kernel: a workgroup a row as long as there are no more rows than
// workgroups, else a wavefront a row.
template <int VD, bool HALF>
__global__ __launch_bounds__(kThreads) void pair_join_kernel(PairArgs a, uint32_t rows) {
    __shared__ f32x4 lo[2 * kThreads];
    __shared__ float factor[2 * kThreads], red[6][kWaves];
    const uint32_t w = threadIdx.x >> 6;
    auto all = [&](uint32_t n_joins, auto join) {
        const uint32_t n = n_joins * a.pairs * rows;   // at most 2,048 joins and pairs, 128 rows
        auto row = [&](uint32_t task, auto waves, uint32_t at) {
            const uint32_t jp = task / rows;
            join_pair<VD, HALF, decltype(waves)::value>(a, join(jp / a.pairs), jp % a.pairs, task % rows, lo + at, factor + at, red);
        };
        if (n <= gridDim.x) {
            if (blockIdx.x < n) row(blockIdx.x, std::integral_constant<int, kWaves>(), 0);
        } else {
            for (uint32_t task = blockIdx.x * kWaves + w; task < n; task += gridDim.x * kWaves) row(task, std::integral_constant<int, 1>(), 64 * w);
        }
    };
    if (a.joins) {
        all(a.head->n_joins, [&](uint32_t i) { return a.joins[i]; });
    } else {
        const PairShares<false> sh(a);
        all(sh.n_joins(), [&](uint32_t i) { return sh.join(i); });
    }
}

// ------------------------------------------------------------------ host

struct PairLayout : Split {
    uint32_t pairs;
    bool rows;             // pair_prompt_kernel
    bool by_size;          // longest ranges first
    int NT;                // row tiles of pair_kernel
    uint32_t item_cap, slot_cap, join_cap, tile_most;
    uint64_t head, items, joins, ml, part, total;
};

netkv_status make_pair_layout(netkv_handle h, const Kv &a, uint32_t D, uint32_t heads, PairLayout &y) {
    if (D != 64 && D != 128) return invalid(h, "head_dim must be 64 or 128");
    if (a.hk % 2) return invalid(h, "n_kv_heads must be even");
    if (heads < 1 || heads % a.hk) return invalid(h, "n_heads must be a multiple of n_kv_heads");
    y.pairs = a.hk / 2;
    y.G = heads / a.hk;
    if (y.G > 64) return invalid(h, "n_heads / n_kv_heads must be <= 64");
    const uint64_t most = (uint64_t)a.max_tok * y.G;   // rows of the longest sequence's pair
    if (most > 0xFFFFFFFFull - 1024) return invalid(h, "max_tok * n_heads / n_kv_heads must be < 2^32 - 1024");
    // Rows from which pair_prompt_kernel pays.  64 sequences of 8,192 tokens, 64 and
    // 8 heads, pair_kernel against it, us: 64 dimensions, 96 rows 322, 360, 128 rows
    // 376, 377, 192 rows 530, 597, 256 rows 671, 582; 128 dimensions, 32 rows 358, 464,
    // 48 rows 415, 500, 64 rows 524, 496, 96 rows 733, 500.
    y.rows = most > (D == 64 ? 192u : 48u);
    y.NT = D == 128 || most <= 16 ? 1 : 2;
    y.tile_rows = !y.rows ? 16u * y.NT : 128u;
    y.tile_most = (uint32_t)(most < y.tile_rows ? most : y.tile_rows);
    // Ranges a pair, of the card's 512 workgroup slots.  Prompts: no more than those in
    // all, which bounds the workspace (1,024 slots of 128 rows) and leaves none for
    // a second turn; us, rounded up to more and so: 128 dimensions, 300 rows after
    // 16,084 tokens of 20 pairs 302, 252, 128 after 3,968 of 200 pairs 288, 266, 256 after
    // 32,512 of 3 pairs 477, 479, 64 dimensions, the first 185, 155.
    // Few rows, 128 dimensions: one workgroup a CU streams as fast as two, whose
    // second reads of the values miss the caches more often, so few tiles (long
    // sequences) get 256 ranges in all; where unequal tiles leave some short 320,
    // us, 256, 320, 512: 8 sequences of 131,071 tokens and 4 pairs 368, 510, 411, one
    // of 131,072 54, 73, 59, 64 of up to 16,384 195, 169, 190, 16 of up to 30,000
    // and 16 pairs 400, 321, 360, 37 of up to 3,000 33, 33, 42, 200 of up to 1,000
    // 48, 54, 56.  64 dimensions: 384, or with more than kEnough steps each 1,024;
    // us, 256, 384, 512 and 1,024: 64 of up to 16,384 and 8 pairs 197, 170, 159, 37 of
    // up to 5,003 and 3 pairs 30, 27, 31.
    const uint64_t slots = (512u + y.pairs - 1) / y.pairs, tiles = (uint64_t)a.n_seq * ((most + y.tile_rows - 1) / y.tile_rows);
    uint64_t ranges = y.pairs < 512 ? 512u / y.pairs : 1u;
    if (!y.rows) ranges = D == 64 ? 3 * slots / 4 : tiles <= slots / 8 || tiles > slots ? slots / 2 : 5 * slots / 8;
    y.target = (uint32_t)(ranges ? ranges : 1);
    y.fine = y.rows || D == 128 ? y.target : (uint32_t)(2 * slots);
    // Where no sequence is longer than this nothing is split and no join started: us,
    // one of 300 tokens (5 steps) 14.8, split by 4 17.2, of 700 at 64 dimensions 13.7,
    // 16.5; of 700 at 128 19.8, 18.1.
    const uint64_t steps_most = (((uint64_t)a.max_pages << a.btl) + kStep - 1) / kStep;
    const uint32_t whole = D == 64 ? 12 : 7;
    y.least = y.rows ? 8 : steps_most <= whole ? whole : 4;
    // Longest ranges first where a range can have more than 32 steps: us, in the
    // sequences' order and so, 8 KV heads of 128 dimensions, 200 of up to 16,384 tokens
    // 497, 406, 120 of up to 8,000 208, 162, 16 of up to 30,000 62, 54, 64 of up to 16,384
    // 170, 164; 8 of 131,071 367, 370.  Shorter ones gain less than finding the order
    // takes: 37 of up to 5,003 and 6 KV heads of 64 25.4, 27.
    y.by_size = !y.rows && tiles > 1 && tiles * steps_most > 32 * ranges;
    y.round = 2;
    const Caps caps = caps_of(a, y);
    if (!grid_fits(caps.items * y.pairs, y.rows ? kPromptThreads : kThreads)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many query rows for one call");
    y.item_cap = (uint32_t)caps.items;
    y.slot_cap = (uint32_t)caps.slots;
    y.join_cap = (uint32_t)caps.joins;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t p = at;
        at += align256(bytes);
        return p;
    };
    y.head = take(sizeof(PlanHead));
    y.items = take(sizeof(Item) * y.item_cap);
    y.joins = take(sizeof(Join) * y.join_cap);
    const uint64_t parts = 2ull * y.slot_cap * y.pairs * y.tile_rows;
    y.ml = take(16 * parts);
    y.part = take(4 * parts * 2 * D);
    y.total = at;
    return NETKV_OK;
}

template <int D, bool HALF>
void launch_pairs(const PairLayout &y, const PairArgs &a, hipStream_t s) {
    const dim3 grid(y.item_cap * y.pairs);
    const bool small = a.kv.btl < 6;
    if (y.rows)
        small ? pair_prompt_kernel<D, 2, D == 64 ? 64 : 32, HALF, true><<<grid, kPromptThreads, 0, s>>>(a)
              : pair_prompt_kernel<D, 2, D == 64 ? 64 : 32, HALF, false><<<grid, kPromptThreads, 0, s>>>(a);
    else if (D == 128 || y.NT == 1)
        small ? pair_kernel<D, 1, HALF, true><<<grid, kThreads, 0, s>>>(a) : pair_kernel<D, 1, HALF, false><<<grid, kThreads, 0, s>>>(a);
    else if constexpr (D == 64)
        small ? pair_kernel<D, 2, HALF, true><<<grid, kThreads, 0, s>>>(a) : pair_kernel<D, 2, HALF, false><<<grid, kThreads, 0, s>>>(a);
    // nothing is split where no sequence can be longer than the shortest range
    const uint64_t steps_most = (((uint64_t)a.kv.max_pages << a.kv.btl) + kStep - 1) / kStep;
    const uint64_t joins_most = (uint64_t)y.join_cap * y.pairs * y.tile_most, quarter = (joins_most + 3) / 4;
    // as launch_attend's
    const uint64_t groups = joins_most < 512 ? joins_most : quarter < 512 ? 512 : quarter < 1024 ? quarter : 1024;
    if (steps_most > a.least && groups) pair_join_kernel<2 * D, HALF><<<(uint32_t)groups, kThreads, 0, s>>>(a, y.tile_most);
}

}  // namespace

extern "C" netkv_status netkv_kv_attend_diff_workspace(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs,
                                                       uint32_t n_heads, uint64_t *bytes) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (!bytes) return invalid(h, "bytes must not be NULL");
    Kv a{};
    netkv_status st = make_kv(h, kv, seqs, a);
    if (st != NETKV_OK) return st;
    PairLayout y{};
    if ((st = make_pair_layout(h, a, kv->head_dim, n_heads, y)) != NETKV_OK) return st;
    *bytes = y.total;
    return NETKV_OK;
}

extern "C" netkv_status netkv_kv_attend_diff(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs, const void *q,
                                             int dtype, uint32_t n_heads, uint64_t q_stride, float scale, const float *lambda,
                                             const float *norm, float eps, float gain, void *out, uint64_t out_stride,
                                             void *work, uint64_t work_bytes, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    Kv a{};
    netkv_status st = make_kv(h, kv, seqs, a);
    if (st != NETKV_OK) return st;
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    PairLayout y{};
    if ((st = make_pair_layout(h, a, kv->head_dim, n_heads, y)) != NETKV_OK) return st;
    if (!std::isfinite(scale) || !std::isfinite(gain)) return invalid(h, "scale and gain must be finite");
    if (!lambda || (uintptr_t)lambda & 3) return invalid(h, "lambda must not be NULL");
    if (norm && !aligned16(norm)) return invalid(h, "norm must be 16-byte aligned");
    if (norm && !(std::isfinite(eps) && eps > 0.0f)) return invalid(h, "eps must be finite and > 0");
    const uint64_t width = (uint64_t)n_heads * kv->head_dim;
    if ((st = check_rows(h, q, q_stride, width, a.n_tok, "q must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, out, out_stride, width, a.n_tok, "out must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    // a row is read by the one workgroup that writes it, or before a join does
    if (rows_overlap(q, q_stride, out, out_stride, width, a.n_tok) && (q != out || q_stride != out_stride))
        return invalid(h, "out must not overlap q (it may be q itself)");
    if (a.n_seq == 0) return NETKV_OK;
    if (!work || ((uintptr_t)work & 255) || work_bytes < y.total) return invalid(h, "work must be 256-byte aligned and of at least netkv_kv_attend_diff_workspace's bytes");
    DeviceScope scope(netkv_internal_device(h));
    hipStream_t s = (hipStream_t)stream;
    uint8_t *ws = (uint8_t *)work;
    const bool half = dtype == NETKV_FP16;
    PairArgs t{};
    t.kv = a;
    (Split &)t = y;
    t.bad_out = (uint16_t *)out;
    t.out_stride = out_stride;
    t.row_elems = (uint32_t)width;
    t.nan16 = half ? 0x7E00u : 0x7FC0u;
    if (a.n_seq > kListed) {
        t.head = (PlanHead *)(ws + y.head);
        t.items = (Item *)(ws + y.items);
        t.joins = (Join *)(ws + y.joins);
        launch_plan(t, s);
    }
    t.pairs = y.pairs;
    t.by_size = y.by_size;
    t.tile_log = y.rows ? 7 : y.NT == 2 ? 5 : 4;
    t.q_stride = q_stride;
    t.q = q;
    t.out = out;
    t.c0 = std::fabs(scale) * kLog2e;
    t.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    t.lambda = lambda;
    t.norm = norm;
    t.root_eps = norm ? std::sqrt(eps) : 0.0f;
    t.gain = gain;
    t.part = (float *)(ws + y.part);
    t.part_ml = (f32x4 *)(ws + y.ml);
    if (kv->head_dim == 64)
        half ? launch_pairs<64, true>(y, t, s) : launch_pairs<64, false>(y, t, s);
    else
        half ? launch_pairs<128, true>(y, t, s) : launch_pairs<128, false>(y, t, s);
    return launched(h, "differential attention launch failed");
}
