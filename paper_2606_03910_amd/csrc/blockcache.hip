// The decode instance's block cache for MI355X (gfx950): keys and values of
// resident blocks in 8 bits, and the operators on them.
//
//   store_kernel    -- new keys and values quantised into their blocks (store_block).
//   read_kernel     -- tokens given back in 16 bits.
//   plan_kernel     -- a call's work list: (sequence, row tile, token range).
//   attend_kernel   -- attention of up to 32 rows over a token range.
//   prompt_kernel   -- the same of up to 256 rows.
//   join_kernel     -- joins the ranges of the rows that were split.
//   unit_kernel, row_kernel, column_kernel, block_kernel -- block weights.
//   weigh_kernel    -- block weights summed over pages in fixed point.
//
// A block ("page") holds block_tokens tokens of every head.  An element is
// e4m3 (1 sign, 4 exponent, 3 mantissa bits; largest 448; no infinity); a
// (page, head) has one scale for its keys and one for its values.  Keys lie
// token by token, values dimension by dimension within tiles of
// min(block_tokens, 64) tokens: the product with the keys contracts over
// dimensions and the one with the values over tokens, and each operand's
// lane then reads 16 bytes in a row.

#include <hip/hip_runtime.h>

#include "blockdev.h"
#include "blockstore.h"

namespace {

using namespace blockdev;

// One workgroup.  Ranges are as long as spreads the call's steps over
// `target` of them, so a batch of unequal sequences fills the card evenly; a
// sequence no longer than one range is not split and writes its rows itself.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
    __shared__ uint32_t wsum[kPlanThreads / 64][3];
    __shared__ uint32_t base[kPlanThreads + 1][3], geo[kPlanThreads][2];
    __shared__ uint32_t ends[kPlanThreads / 64];
    __shared__ unsigned long long work;
    if (threadIdx.x == 0) work = 0;
    bool rows_ok = true;
    for (uint32_t s = threadIdx.x; s < a.kv.n_seq; s += kPlanThreads) rows_ok &= seq_head(a.kv, s).rows_ok;
    const bool falls = __syncthreads_or(!rows_ok);
    // this thread's sequence; without rows if it begins among an earlier one's
    uint32_t named = 0;
    bool early = false;
    auto head_of = [&](uint32_t s) {
        Head h{};
        if (s < a.kv.n_seq) h = seq_head(a.kv, s);
        if (falls) {
            early = h.row0 < rows_before(s < a.kv.n_seq ? rows_end(a.kv, s) : 0u, named, ends);
            if (early) h.n = h.ctx = 0;
        }
        return h;
    };
    unsigned long long mine = 0;
    for (uint32_t s0 = 0; s0 < a.kv.n_seq; s0 += kPlanThreads) {
        const Head h = head_of(s0 + threadIdx.x);
        mine += (unsigned long long)tiles_of(h, a) * steps_of(h);
    }
    atomicAdd(&work, mine);
    __syncthreads();
    const uint32_t C = range_steps(a, work);
    uint32_t at[3] = {0, 0, 0};   // items, slots, joins so far
    named = 0;
    for (uint32_t s0 = 0; s0 < a.kv.n_seq; s0 += kPlanThreads) {
        const uint32_t s = s0 + threadIdx.x;
        uint32_t x[3] = {0, 0, 0}, rt = 0, sp = 1;
        const Head h = head_of(s);
        if (s < a.kv.n_seq) {
            if (a.left_out) a.left_out[s] = early;
            rt = tiles_of(h, a);
            sp = parts_of(steps_of(h), C);
            x[0] = rt * sp;
            x[1] = sp > 1 ? x[0] : 0u;
            x[2] = sp > 1 ? rt : 0u;
        }
        geo[threadIdx.x][0] = rt;
        geo[threadIdx.x][1] = sp;
        uint32_t tot[3];
        scan3(x, tot, wsum);
        for (int i = 0; i < 3; ++i) base[threadIdx.x][i] = x[i];
        if (threadIdx.x == 0) base[kPlanThreads][0] = tot[0];
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < tot[0]; i += kPlanThreads) {
            uint32_t lo = 0, hi = kPlanThreads;   // the last sequence that starts at or before i and has items
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (base[mid][0] <= i) lo = mid; else hi = mid;
            }
            const uint32_t j = i - base[lo][0], n = geo[lo][0], p = geo[lo][1];
            const Item it = item_of(a, s0 + lo, seq_head(a.kv, s0 + lo), C, p, n - 1 - j / p, j % p, at[1] + base[lo][1]);
            a.items[at[0] + i] = it;   // within caps_of, as its joins are
            if (p > 1 && j % p == 0) a.joins[at[2] + base[lo][2] + it.tile] = Join{it.seq, it.tile, it.slot, p};
        }
        for (int i = 0; i < 3; ++i) at[i] += tot[i];
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.head = PlanHead{at[0], at[2], at[1], 0};
    fill_bad(a);
}

}  // namespace

void blockdev::launch_plan(const PlanArgs &a, hipStream_t s) { plan_kernel<<<1, kPlanThreads, 0, s>>>(a); }

namespace {

// ------------------------------------------------------------------ attention

struct AttendArgs : PlanArgs {
    uint32_t Hq;
    uint64_t q_stride;               // elements between tokens, as out_stride
    const void *q;
    void *out;
    float c0;                        // |scale| * log2(e)
    uint32_t q_sign;                 // flips the queries' signs where scale < 0
    float *part;                     // [slot][head][tile_rows][D]
    f32x4 *part_ml;                  // [slot][head][tile_rows] m, l, y
    float *lse;                      // [row][query head] log2 of the row's sum (inf if it sees no token), or null
    float *units;                    // [seq][head][unit][unit_rows] log2 of the unit's sum, or null
    uint32_t n_units, unit_rows;
    float *sums;                     // [head][block][row] log2 of the block's sum for each row of the call, or null
    uint64_t sum_rows;               // rows of a head
};

// Attention of one row tile over steps [k0, k1), the maximum and sum of its
// softmax kept as they run: with x = q.k scale log2(e), m the maximum of x so
// far and l = sum 2^(x - m); with s a block's value scale and v its e4m3
// values, y the maximum of x + log2(s) so far less kLift and O = sum 2^(x - y)
// s v.  The row is O 2^(y - m) / l.
//
// A wavefront multiplies 16-row tiles of S^T = K Q^T and O^T = V^T P^T, so
// that a lane of S^T (a query row, 16 tokens in a row) holds the very P^T
// operand of the second product: the token that key row r of product t means
// is 16 (r / 4) + 4 t + r % 4, and nothing moves between lanes.  P = 2^(x - y) s
// is rounded to fp16 for both types of query, since e4m3 is exact in it: 11
// bits for what is within 2^-20 of the largest, a step of 2^-30 of that below
// (kLift; y is the maximum with s in it, so that a block of small values that a
// row attends to keeps them).  l takes the weights before that rounding.  A
// maximum is raised, and O rescaled, only when 16 weights' sum passes kMaxSum.
//
// The four wavefronts take the same rows and every fourth step each, joined
// through LDS.  Long calls are bound by the cache's bytes: 8 sequences of
// 131,071 tokens and 8 heads of 128 dimensions (2.15 GB) take 361 us, 6.0 TB/s,
// 64 of up to 16,384 with block weights (0.61 GB) 136 us, 4.5 TB/s.  Short ones
// by latency: one of 700 tokens takes 8 us, a wavefront one step of its 11.  A
// step's loads go out as the registers of the one before come free, two
// workgroups a CU.  With a static partition into equal pieces of all steps,
// which needs no ranges of its own, the whole call of the 64 sequences took 166
// us, with ranges as they were then 150 (147 now).
template <int D, int NT, bool HALF, bool UNITS, bool SMALL>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_kernel(AttendArgs a) {
    typedef typename Elem<HALF>::T T;
    typedef typename Elem<HALF>::T8 T8;
    constexpr int kDT = D / 16;
    constexpr int kPitch = D + 4;
    __shared__ float lds[kWaves * 16 * kPitch];
    __shared__ float lds_ml[kWaves][16 * NT][3];

    const uint32_t hk = a.kv.hk;
    const uint32_t h = blockIdx.x % hk, item = blockIdx.x / hk;
    Item it;
    Head hd;
    if (!find_item(a, item, it, hd)) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // known to be uniform
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t n_rows = hd.n * a.G;
    const uint32_t row0 = it.tile * a.tile_rows;
    const uint32_t bt = 1u << a.kv.btl, tile = min(bt, kStep);
    const uint64_t hb = head_bytes(a.kv, D);
    const uint32_t *pages = a.kv.pages + (uint64_t)it.seq * a.kv.max_pages;
    const uint32_t last_block = hd.ctx ? (hd.ctx - 1) >> a.kv.btl : 0u;

    // queries: 16 dimensions a lane, as the keys
    T8 qf[NT][D / 32];
    uint32_t lim[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t r = row0 + n * 16 + c;
        const bool valid = r < n_rows;
        const uint32_t t = valid ? r / a.G : 0u, qh = h * a.G + (valid ? r % a.G : 0u);
        const int64_t seen = (int64_t)hd.ctx - hd.n + t + 1;
        lim[n] = !valid ? hd.ctx : seen > 0 ? (uint32_t)seen : 0u;
        const T *q = (const T *)a.q + (hd.row0 + t) * a.q_stride + (uint64_t)qh * D + 16 * g;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4 x = {0, 0, 0, 0};
            if (valid) x = *(const u32x4 *)(q + (i / 2) * 64 + (i % 2) * 8);
            qf[n][i] = __builtin_bit_cast(T8, x ^ a.q_sign);
        }
    }
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
    auto in_cache = [&](const uint8_t *x, uint32_t kt, uint32_t page) {
        return x + h * hb + (page < a.kv.n_pages ? page : 0u) * page_bytes + (uint64_t)((kt * kStep) & (bt - 1)) * D;
    };
    auto load_keys = [&](KeyRegs<D> &x, uint32_t kt, uint32_t page) {
        const uint8_t *p = in_cache(a.kv.k, kt, page);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < D / 64; ++i) x.f[t][i] = *(const u32x4 *)(p + key_in_page + 4 * t * D + 64 * i);
    };
    auto load_vals = [&](ValRegs<D> &x, uint32_t kt, uint32_t page) {
        const uint8_t *p = in_cache(a.kv.v, kt, page);
#pragma unroll
        for (int d = 0; d < kDT; ++d) x.f[d] = *(const u32x4 *)(p + val_in_page + d * val_piece);
    };

    // The next step's keys are asked for as soon as this one's have been
    // multiplied, its values likewise; pages a step earlier.
    KeyRegs<D> kf;
    ValRegs<D> vf;
    f32x4 st[NT][4];
    f16x8 pf[NT][2];
    float sc_next = 0.0f, vs_next = 0.0f, sc = 0.0f, vsl = 0.0f;
    uint64_t nan_sums = 0;                             // sums of this lane that a NaN value belongs to
    static_assert(4 * NT * kDT <= 64, "a bit a sum");
    uint32_t pk = 0, pv = 0;
    auto load_scales = [&]() {
        const bool bad = pv >= a.kv.n_pages;
        if (bad) report(a.kv);
        const uint64_t si = (uint64_t)(bad ? 0u : pv) * hk + h;
        sc_next = SMALL ? a.kv.ks[si] : scalar(a.kv.ks)[si];
        vs_next = SMALL ? a.kv.vs[si] : scalar(a.kv.vs)[si];
        if (bad) sc_next = vs_next = NAN;
    };
    auto find_pages = [&](uint32_t kt) {
        pk = page_at(kt, c >> 2);
        pv = SMALL ? page_at(kt, g) : pk;
    };
    auto scores = [&](uint32_t kt) {
        const float x = sc_next * a.c0;
        sc = x == 0.0f ? 1.0e-30f : x;                 // not 0, which would turn a masked score's -inf into NaN
        vsl = vs_next;
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
        if (kt + kWaves < end) {
            load_keys(kf, kt + kWaves, pk);
            load_scales();
        }
    };
    auto values = [&](uint32_t kt) {
#pragma unroll
        for (int d = 0; d < kDT; ++d) {
            const f16x8 lo = widen_f16(vf.f[d][0], vf.f[d][1]);
            const f16x8 hi = widen_f16(vf.f[d][2], vf.f[d][3]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                acc[n][d] = product(lo, pf[n][0], acc[n][d]);
                acc[n][d] = product(hi, pf[n][1], acc[n][d]);
            }
        }
        if (kt + kWaves < end) {
            load_vals(vf, kt + kWaves, pv);
            find_pages(kt + 2 * kWaves);
        }
    };
    // log2 of the unit's sum, of which this lane has 2^base sum: 64 tokens are
    // the row's four lanes, 32 two of them, 16 one
    auto keep_unit = [&](uint32_t kt, int n, float sum, float base) {
        if constexpr (UNITS) {
            if (tile >= 32) sum = pair16_sum(sum);
            if (tile >= 64) sum += __shfl_xor(sum, 32, 64);
            const uint32_t u = kt * (kStep / tile) + 16 * g / tile;
            if (((16 * g) & (tile - 1)) == 0 && u < a.n_units && row0 + n * 16 + c < n_rows)
                a.units[(((uint64_t)it.seq * hk + h) * a.n_units + u) * a.unit_rows + row0 + n * 16 + c] = base + log2_of(sum);
        }
    };
    // P in units of 2^y with y as it is, its sum in l's units of 2^m at once;
    // false (and l as it was) where that will not do: a weight passes 2^y by
    // too much (the first step, a larger score), scales are further apart than
    // fp32 takes in one, NaN
    auto softmax = [&](uint32_t kt) {
        const float vlog = log2_of(vsl);
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
        for (int n = 0; n < NT; ++n) {
            l[n] += sum[n] * exp2_of(up[n]);
            // lanes of one row may have pages of their own, so one base for all: m
            keep_unit(kt, n, sum[n] * exp2_of(up[n]), m[n]);
        }
        return true;
    };
    // any step: masks, NaN values, maxima raised
    auto softmax_any = [&](uint32_t kt) {
        const float vlog = log2_of(vsl);
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
            const float mm = mn == -INFINITY ? 0.0f : mn;
            const float total = weights_of(st[n], sc, -mm, pf[n]);
            l[n] += total;
            keep_unit(kt, n, total, mm);
            weights_of(st[n], sc, yn == -INFINITY ? -INFINITY : vlog - yn, pf[n]);
        }
        if (kt * kStep + kStep <= all_lim) return;
        // Tokens that not every row sees: bytes of slots that hold none may be
        // anything.  A NaN among values that some rows see and others do not
        // would come to all of them by a product with P = 0: the rows that see
        // one are found by a product of the masks, and it is left out.
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
        uint64_t found = 0;                            // four bits at a time, from the top (no constant for each sum)
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
    if (it.k0 + w < end) {
        find_pages(it.k0 + w);
        load_keys(kf, it.k0 + w, pk);
        load_scales();
        load_vals(vf, it.k0 + w, pv);
        find_pages(it.k0 + w + kWaves);
    }
    // the ordinary steps have a loop of their own (see prompt_kernel)
    for (uint32_t kt = it.k0 + w; kt < end; kt += kWaves) {
        bool done;
        do {
            scores(kt);
            done = kt * kStep + kStep <= all_lim;
            if (done) done = softmax(kt);
            if (!done) break;
            values(kt);
            kt += kWaves;
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
    for (int n = 0; n < NT; ++n) l[n] = row_sum(l[n]);

#pragma unroll
    for (int n = 0; n < NT; ++n) {
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
        for (uint32_t e = threadIdx.x; e < 16 * D / 4; e += kThreads) {
            const uint32_t row = e / (D / 4), d4 = e % (D / 4) * 4;
            const uint32_t r = row0 + n * 16 + row;
            if (r >= n_rows) continue;
            float M = -INFINITY, Y = -INFINITY;
            for (int v = 0; v < kWaves; ++v) {
                M = fmaxf(M, lds_ml[v][n * 16 + row][0]);
                Y = fmaxf(Y, lds_ml[v][n * 16 + row][2]);
            }
            float L = 0.0f;
            f32x4 o = {0, 0, 0, 0};
            for (int v = 0; v < kWaves; ++v) {
                const float *ml = lds_ml[v][n * 16 + row];
                L += joined(ml[0], M) * ml[1];
                const float f = joined(ml[2], Y);
                const f32x4 x = *(const f32x4 *)&lds[(v * 16 + row) * kPitch + d4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += x[i] * f;
            }
            if (it.slot != kNoSlot) {
                const uint64_t at = ((uint64_t)it.slot * hk + h) * a.tile_rows + n * 16 + row;
                if (d4 == 0) a.part_ml[at] = f32x4{M, L, Y, 0.0f};
                *(f32x4 *)(a.part + at * D + d4) = o;
            } else {
                const uint64_t t = hd.row0 + r / a.G;
                const uint32_t qh = h * a.G + r % a.G;
                const bool sees = hd.ctx + r / a.G >= hd.n;   // both below 2^31
                const Over over(Y, M, L, sees);
                T z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = (T)over(o[i]);
                *(u32x2 *)((T *)a.out + t * a.out_stride + (uint64_t)qh * D + d4) = *(u32x2 *)z;
                if (a.lse && d4 == 0) a.lse[t * a.Hq + qh] = sees ? M + log2_of(L) : INFINITY;
            }
        }
    }
}

// The same for prompts: eight wavefronts with 16 NT rows each go through the
// tokens together, two on a SIMD.  Every step's keys and values are widened to
// 16 bits once, into LDS in the operands' own order (a fragment is 64 lanes
// times 16 bytes in a row).  The wavefronts are two groups half a step apart,
// with a barrier between the halves: while one multiplies (O of the step
// before, S of this one) the other one does its softmax, so a SIMD's matrix
// and vector units work at once.  Slot 2 k is the first group's products of
// step k and the second one's softmax of step k - 1, slot 2 k + 1 the reverse.
// The first group widens keys k + 1 with its softmax k (slot 2 k + 1: keys
// k - 1, in the same buffer, were last read in slot 2 k - 1), the second one
// values k + 1 with its own (slot 2 k + 2: values k - 1 were last read in slot
// 2 k + 1, values k + 1 are first read in slot 2 k + 4).
//
// SMALL: blocks of less than 64 tokens, so a step's four groups of 16 tokens
// may be in different pages; else pages, scales and addresses are scalar.
//
// Bound by the matrix units and the vector units beside them: two chunks of
// 1,024 rows of 64 heads after 31,744 tokens (128 dimensions, 2.16 TFLOP) take
// 1,990 us, 1.09 PFLOP/s, where a product of 8,192 x 8,192 matrices reaches
// 1.17.  An ordinary step of 256 rows takes 1.9 us, the first and the masked
// ones 5, finding the tile, its first loads and its output 9: six prompts of up
// to 2,777 tokens (0.31 TFLOP, 17 steps a tile) take 514 us under the profiler
// (the whole call without it 463).
//
// SUMS: every row's sum over each block is kept for the blocks' weights (ranges
// are whole blocks).
template <int D, int NT, bool HALF, bool SMALL, bool SUMS>
__global__ __launch_bounds__(kPromptThreads, 2) void prompt_kernel(AttendArgs a) {
    typedef typename Elem<HALF>::T T;
    typedef typename Elem<HALF>::T8 T8;
    constexpr int kDT = D / 16;
    constexpr int kAhead = 6;                         // fragments read ahead of their products
    constexpr int kShare = D / 64;                    // 16-byte pieces of keys or values a lane stages
    __shared__ u32x4 lds_k[2][4 * (D / 32)][64];
    __shared__ u32x4 lds_v[2][2 * kDT][64];
    __shared__ uint8_t lds_bits[2][2 * kDT][64];      // which of a fragment lane's 8 values were NaN
    __shared__ uint32_t lds_nan[2];

    const uint32_t hk = a.kv.hk;
    const uint32_t h = blockIdx.x % hk, item = blockIdx.x / hk;
    Item it;
    Head hd;
    if (!find_item(a, item, it, hd)) return;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // known to be uniform
    const bool second = w >= 4;
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t n_rows = hd.n * a.G;
    const uint32_t row0 = it.tile * a.tile_rows + w * 16 * NT;
    const uint32_t bt = 1u << a.kv.btl, tile = min(bt, kStep);
    const uint64_t hb = head_bytes(a.kv, D);
    const uint32_t *pages = a.kv.pages + (uint64_t)it.seq * a.kv.max_pages;
    const uint32_t last_block = hd.ctx ? (hd.ctx - 1) >> a.kv.btl : 0u;

    T8 qf[NT][D / 32];
    uint32_t lim[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t r = row0 + n * 16 + c;
        const bool valid = r < n_rows;
        const uint32_t t = valid ? r / a.G : 0u, qh = h * a.G + (valid ? r % a.G : 0u);
        const int64_t seen = (int64_t)hd.ctx - hd.n + t + 1;
        lim[n] = !valid ? hd.ctx : seen > 0 ? (uint32_t)seen : 0u;
        const T *q = (const T *)a.q + (hd.row0 + t) * a.q_stride + (uint64_t)qh * D + 16 * g;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4 x = {0, 0, 0, 0};
            if (valid) x = *(const u32x4 *)(q + (i / 2) * 64 + (i % 2) * 8);
            qf[n][i] = __builtin_bit_cast(T8, x ^ a.q_sign);
        }
    }
    // tokens that every row of this wavefront sees.  A wavefront whose rows see
    // no more goes on with the others: they wait for one another anyway, and
    // without a branch around the products their sums stay where they are.
    const int64_t see_all = (int64_t)hd.ctx - hd.n + row0 / a.G + 1;
    const uint32_t all_lim = see_all > 0 ? (uint32_t)min(see_all, (int64_t)hd.ctx) : 0u;
    // tokens that every row of the tile sees
    const int64_t see_tile = (int64_t)hd.ctx - hd.n + it.tile * a.tile_rows / a.G + 1;
    const uint32_t tile_lim = see_tile > 0 ? (uint32_t)min(see_tile, (int64_t)hd.ctx) : 0u;

    f32x4 acc[NT][kDT], st[NT][4];
    f16x8 pf[NT][2];
    float m[NT], l[NT], y[NT], lb[NT];                // lb: the share of l that is the present block's
    uint64_t nan_sums = 0;                            // sums of this lane that a NaN value belongs to
    static_assert(4 * NT * kDT <= 64, "a bit a sum");
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = y[n] = -INFINITY;
        l[n] = lb[n] = 0.0f;
        pf[n][0] = pf[n][1] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int d = 0; d < kDT; ++d) acc[n][d] = f32x4{0, 0, 0, 0};
    }

    // this lane's pieces: 64 dimensions of key row c of a product, or 16
    // tokens of dimension 16 d + c
    u32x4 px[kShare];
    float sc_at[2], vs_at[2];                          // scales of this step and the next
    const uint32_t own_group = SMALL ? second ? g : c >> 2 : 0u;   // whose page this lane's pieces are in
    auto page_at = [&](uint32_t kt, uint32_t group) {
        const uint32_t block = min((kt * kStep + (SMALL ? 16 * group : 0u)) >> a.kv.btl, last_block);
        return SMALL ? pages[block] : scalar(pages)[block];
    };
    const uint8_t *own = (second ? a.kv.v : a.kv.k) + h * hb;
    const uint64_t page_bytes = hk * hb;
    const uint32_t in_page = second ? c * tile + ((16 * g) & (tile - 1)) + (w - 4) * kShare * 16 * tile
                                    : ((16 * (c >> 2)) & (tile - 1)) * D + ((c & 3) + 4 * w) * D + 16 * g;
    const uint32_t piece = second ? 16 * tile : 64;
    const float *ks = a.kv.ks + h, *vs = a.kv.vs + h;
    auto scales_of = [&](uint32_t pv, float &sc, float &vsc) {
        const bool bad = pv >= a.kv.n_pages;
        if (bad) report(a.kv);
        const uint64_t si = (uint64_t)(bad ? 0u : pv) * hk;
        sc = SMALL ? ks[si] : scalar(ks)[si];
        vsc = SMALL ? vs[si] : scalar(vs)[si];
        if (bad) sc = vsc = NAN;
    };
    auto fetch = [&](uint32_t kt, uint32_t po) {
        const uint8_t *p = own + (po < a.kv.n_pages ? po : 0u) * page_bytes + (uint64_t)((kt * kStep) & (bt - 1)) * D;
#pragma unroll
        for (int i = 0; i < kShare; ++i) px[i] = *(const u32x4 *)(p + in_page + i * piece);
    };
    auto stage = [&](uint32_t kt) {
        const int b = kt & 1;
        if (!second) {
#pragma unroll
            for (int i = 0; i < kShare; ++i) {
                const uint32_t j = w * kShare + i;
                lds_k[b][2 * j][lane] = __builtin_bit_cast(u32x4, widen<HALF>(px[i][0], px[i][1]));
                lds_k[b][2 * j + 1][lane] = __builtin_bit_cast(u32x4, widen<HALF>(px[i][2], px[i][3]));
            }
            return;
        }
        if (kt * kStep + kStep > tile_lim) {
            // bytes of slots that hold no token are cleared, a NaN is taken out
            // and noted
            const uint32_t tok0 = kt * kStep + 16 * g;
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
#pragma unroll
                for (int i = 0; i < kShare; ++i) {
                    const uint32_t j = (w - 4) * kShare + i;
                    uint32_t bits = 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t y = nan_bytes(px[i][q]);
                        px[i][q] &= ~(y * 0xFFu);
                        bits |= ((y | y >> 7 | y >> 14 | y >> 21) & 15u) << (4 * q);
                    }
                    lds_bits[b][2 * j][lane] = (uint8_t)bits;
                    lds_bits[b][2 * j + 1][lane] = (uint8_t)(bits >> 8);
                }
                if (lane == 0) atomicOr(&lds_nan[b], 1u << (w - 4));
            } else if (lane == 0) {
                atomicAnd(&lds_nan[b], ~(1u << (w - 4)));
            }
        }
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            const uint32_t j = (w - 4) * kShare + i;
            lds_v[b][2 * j][lane] = __builtin_bit_cast(u32x4, widen_f16(px[i][0], px[i][1]));
            lds_v[b][2 * j + 1][lane] = __builtin_bit_cast(u32x4, widen_f16(px[i][2], px[i][3]));
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
            for (int t = 0; t < 4; ++t) st[n][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < 4; t += 2)
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const T8 kf = __builtin_bit_cast(T8, lds_k[b][(t + q) * (D / 32) + i][lane]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) st[n][t + q] = product(kf, qf[n][i], st[n][t + q]);
                }
    };
    auto values = [&](uint32_t kt) {
        const int b = kt & 1;
#pragma unroll
        for (int d = 0; d < kDT; d += 2)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f16x8 vf = __builtin_bit_cast(f16x8, lds_v[b][2 * (d + q) + u][lane]);
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
    // P in units of 2^y with y as it is, its sum in l's units of 2^m at once;
    // false (and l as it was) where that will not do: a weight passes 2^y by
    // too much (the first step, a larger score), scales are further apart than
    // fp32 takes in one, NaN
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
        for (int n = 0; n < NT; ++n) {
            const float add = sum[n] * exp2_of(up[n]);
            l[n] += add;
            if constexpr (SUMS) lb[n] += add;
        }
        return true;
    };
    // any step: masks, NaN values among those that not every row sees, maxima
    // raised
    auto softmax_any = [&](uint32_t kt) {
        const float sc = scale_of(), vlog = log2_of(vs_at[0]);
        const uint32_t tok0 = kt * kStep + 16 * g;
        if (kt * kStep + kStep > tile_lim) {
            const uint32_t noted = lds_nan[kt & 1];
            // as in attend_kernel: the rows that see a NaN value are found by
            // a product of the masks
            if (noted)
#pragma unroll 1
                for (int d = 0; d < kDT; ++d) {
                    if (!(noted >> (d / kShare) & 1)) continue;
                    f32x4 hit[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) hit[n] = f32x4{0, 0, 0, 0};
#pragma unroll 1
                    for (int u = 0; u < 2; ++u) {
                        const uint32_t bits = lds_bits[kt & 1][2 * d + u][lane];
                        f16x8 one;
#pragma unroll
                        for (int j = 0; j < 8; ++j) one[j] = bits >> j & 1 ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const int left = (int)lim[n] - (int)tok0 - 8 * u;
                            f16x8 see;
#pragma unroll
                            for (int j = 0; j < 8; ++j) see[j] = left > j ? (_Float16)1.0f : (_Float16)0.0f;
                            hit[n] = product(one, see, hit[n]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) nan_sums |= (uint64_t)(hit[n][i] > 0.0f) << (4 * (n * kDT + d) + i);
                }
        }
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
            const float ml = m[n] == -INFINITY ? 1.0f : exp2_of(m[n] - mn);   // nothing so far: 0, or NaN
            l[n] *= ml;
            if constexpr (SUMS) lb[n] *= ml;
            const float al = y[n] == -INFINITY ? 1.0f : exp2_of(y[n] - yn);
            m[n] = mn;
            y[n] = yn;
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][d][i] *= al;
            const float add = weights_of(st[n], sc, mn == -INFINITY ? 0.0f : -mn, pf[n]);
            l[n] += add;
            if constexpr (SUMS) lb[n] += add;
            weights_of(st[n], sc, yn == -INFINITY ? -INFINITY : vlog - yn, pf[n]);
        }
    };

    // a lane has the sum of its own 16 tokens
    const uint32_t per = SMALL ? 1u : bt / kStep;
    auto keep_sums = [&](uint32_t kt) {
        if constexpr (SUMS) {
            if (((kt + 1) & (per - 1)) != 0 && kt + 1 < it.k1) return;
            const uint32_t block = (kt * kStep + (SMALL ? 16 * g : 0u)) >> a.kv.btl;
            const bool keeps = SMALL ? ((16 * g) & (bt - 1)) == 0 && block < a.kv.max_pages : g == 0;
            float *to = a.sums + ((uint64_t)h * a.kv.max_pages + block) * a.sum_rows + hd.row0 * a.G + row0 + c;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float sum = !SMALL ? row_sum(lb[n]) : bt == 32 ? pair16_sum(lb[n]) : lb[n];
                if (keeps && row0 + n * 16 + c < n_rows) to[n * 16] = m[n] + log2_of(sum);
                lb[n] = 0.0f;
            }
        }
    };
    // pages of the step after next and the one after it
    uint32_t po = 0, pv = 0, po_on = 0, pv_on = 0;
    float sc_on = 0.0f, vs_on = 0.0f;                 // scales of the step after next
    if (threadIdx.x < 2) lds_nan[threadIdx.x] = 0;
    // the first step's products with "the step before" are of zeros
    for (uint32_t i = threadIdx.x; i < 2 * kDT * 64; i += kPromptThreads) (&lds_v[~it.k0 & 1][0][0])[i] = u32x4{0, 0, 0, 0};
    meet();
    sc_at[0] = vs_at[0] = sc_at[1] = vs_at[1] = 0.0f;
    if (it.k0 < it.k1) {
        fetch(it.k0, page_at(it.k0, own_group));
        scales_of(page_at(it.k0, g), sc_at[0], vs_at[0]);
        stage(it.k0);
        fetch(it.k0 + 1, page_at(it.k0 + 1, own_group));
        scales_of(page_at(it.k0 + 1, g), sc_at[1], vs_at[1]);
        po = page_at(it.k0 + 2, own_group);
        pv = SMALL ? page_at(it.k0 + 2, g) : po;
    }
    meet();
    if (second) meet();
    // Small loads for later steps go out before the softmax, which hides them
    // (page_at stays within the sequence's blocks past its end).
    auto look_ahead = [&](uint32_t kt) {
        scales_of(pv, sc_on, vs_on);
        po_on = page_at(kt + 3, own_group);
        pv_on = SMALL ? page_at(kt + 3, g) : po_on;
    };
    auto pass_on = [&](uint32_t kt) {
        if (kt + 1 < it.k1) {
            stage(kt + 1);
            fetch(kt + 2, po);
        }
        sc_at[0] = sc_at[1];
        vs_at[0] = vs_at[1];
        sc_at[1] = sc_on;
        vs_at[1] = vs_on;
        po = po_on;
        pv = pv_on;
        meet();
    };
    // The ordinary steps have a loop of their own: with the other ones as a
    // branch in it the compiler keeps the sums in two places and moves them
    // back and forth in every step.
    for (uint32_t kt = it.k0; kt < it.k1; ++kt) {
        bool done;
        do {
            values(kt - 1);
            scores(kt);
            interleave(std::integral_constant<int, D / 4>());
            meet();
            done = kt * kStep + kStep <= all_lim && kt > it.k0;   // the first step sets the maxima
            if (kt * kStep + kStep > tile_lim) done = done && __builtin_amdgcn_readfirstlane(lds_nan[kt & 1]) == 0;
            look_ahead(kt);
            if (done) done = softmax();
            if (!done) break;
            keep_sums(kt);
            pass_on(kt);
            ++kt;
        } while (kt < it.k1);
        if (done) break;
        softmax_any(kt);
        keep_sums(kt);
        pass_on(kt);
    }
    if (!second) meet();
    if (it.k0 < it.k1) values(it.k1 - 1);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] = row_sum(l[n]);
        if (nan_sums)
#pragma unroll
            for (int d = 0; d < kDT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (nan_sums >> (4 * (n * kDT + d) + i) & 1) acc[n][d][i] = NAN;
        const uint32_t tr = w * 16 * NT + n * 16 + c, r = row0 + n * 16 + c;
        if (r >= n_rows) continue;
        if (it.slot != kNoSlot) {
            const uint64_t at = ((uint64_t)it.slot * hk + h) * a.tile_rows + tr;
            if (g == 0) a.part_ml[at] = f32x4{m[n], l[n], y[n], 0.0f};
#pragma unroll
            for (int d = 0; d < kDT; ++d) *(f32x4 *)(a.part + at * D + d * 16 + 4 * g) = acc[n][d];
        } else {
            const uint64_t t = hd.row0 + r / a.G;
            const uint32_t qh = h * a.G + r % a.G;
            const Over over(y[n], m[n], l[n], lim[n] > 0);
            T *out = (T *)a.out + t * a.out_stride + (uint64_t)qh * D + 4 * g;
#pragma unroll
            for (int d = 0; d < kDT; ++d) {
                T o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (T)over(acc[n][d][i]);
                *(u32x2 *)(out + d * 16) = *(u32x2 *)o;
            }
            if (a.lse && g == 0) a.lse[t * a.Hq + qh] = lim[n] > 0 ? m[n] + log2_of(l[n]) : INFINITY;
        }
    }
}

// Joins the ranges of one row: with M and Y the largest of their maxima,
// O = sum 2^(y - Y) O_i, l = sum 2^(m - M) l_i, by WAVES wavefronts: their
// lanes first take a range each for the factors, then the row's columns by
// four times a share of the ranges (loads that wait for nothing).
template <int D, bool HALF, int WAVES>
__device__ inline void join_row(const AttendArgs &a, const Join &j, uint32_t h, uint32_t tr, f32x4 *lo, float *factor, float (*red)[kWaves]) {
    typedef typename Elem<HALF>::T T;
    constexpr uint32_t kLanes = 64 * WAVES, kCols = D / 4, kGroups = kLanes / kCols;
    auto meet = [&]() {
        if constexpr (WAVES > 1) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    const uint32_t hk = a.kv.hk, rows = a.tile_rows;
    const uint32_t me = threadIdx.x % kLanes, lane = threadIdx.x & 63, w = me >> 6;
    const uint32_t col = me % kCols, grp = me / kCols;
    const Head hd = seq_head(a.kv, j.seq);
    const uint32_t r = j.tile * rows + tr;
    if (r >= hd.n * a.G) return;
    const uint64_t at = ((uint64_t)j.slot * hk + h) * rows + tr, by = (uint64_t)hk * rows;
    float M = -INFINITY, Y = -INFINITY;
    for (uint32_t i = me; i < j.n; i += kLanes) {
        const f32x4 ml = a.part_ml[at + i * by];
        M = fmaxf(M, ml[0]);
        Y = fmaxf(Y, ml[2]);
    }
    for (int d = 32; d; d >>= 1) {
        M = fmaxf(M, __shfl_xor(M, d, 64));
        Y = fmaxf(Y, __shfl_xor(Y, d, 64));
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) {
            red[0][w] = M;
            red[1][w] = Y;
        }
        __syncthreads();
        for (int v = 0; v < WAVES; ++v) {
            M = fmaxf(M, red[0][v]);
            Y = fmaxf(Y, red[1][v]);
        }
    }
    float L = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (uint32_t i0 = 0; i0 < j.n; i0 += kLanes) {
        const uint32_t i = i0 + me;
        if (i < j.n) {
            const f32x4 ml = a.part_ml[at + i * by];
            factor[me] = joined(ml[2], Y);
            L += joined(ml[0], M) * ml[1];
        }
        meet();
        const uint32_t n = min(j.n - i0, kLanes);
        const float *p = a.part + (at + i0 * by) * D + col * 4;
#pragma unroll 4
        for (uint32_t q = grp; q < n; q += kGroups) {
            const f32x4 x = *(const f32x4 *)(p + q * by * D);
            const float f = factor[q];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += f * x[e];
        }
        meet();
    }
    for (int d = 32; d; d >>= 1) L += __shfl_xor(L, d, 64);
    if (WAVES > 1 && lane == 0) red[2][w] = L;
    lo[grp * kCols + col] = o;
    meet();
    if (grp == 0) {
        if constexpr (WAVES > 1) {
            L = 0.0f;
            for (int v = 0; v < WAVES; ++v) L += red[2][v];
        }
        o = f32x4{0, 0, 0, 0};
        for (uint32_t i = 0; i < kGroups; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += lo[i * kCols + col][e];
        const uint64_t t = hd.row0 + r / a.G;
        const uint32_t qh = h * a.G + r % a.G;
        const bool sees = hd.ctx + r / a.G >= hd.n;   // both below 2^31
        const Over over(Y, M, L, sees);
        T z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (T)over(o[e]);
        *(u32x2 *)((T *)a.out + t * a.out_stride + (uint64_t)qh * D + col * 4) = *(u32x2 *)z;
        if (a.lse && col == 0) a.lse[t * a.Hq + qh] = sees ? M + log2_of(L) : INFINITY;
    }
    meet();
}

// A workgroup a row as long as there are no more rows than workgroups, else a
// wavefront a row: latency, 5 us for the 64 rows of one sequence's heads, 9 us
// for the 4,096 of 64 sequences.
template <int D, bool HALF>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs a, uint32_t rows) {
    __shared__ f32x4 lo[kThreads];
    __shared__ float factor[kThreads], red[3][kWaves];
    const uint32_t hk = a.kv.hk, w = threadIdx.x >> 6;
    auto all = [&](uint32_t n_joins, auto join) {
        const uint32_t n = n_joins * hk * rows;   // at most 2,048 joins and heads, 256 rows
        auto row = [&](uint32_t task, auto waves, uint32_t at) {
            const uint32_t jh = task / rows;
            join_row<D, HALF, decltype(waves)::value>(a, join(jh / hk), jh % hk, task % rows, lo + at, factor + at, red);
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
        const Shares sh(a);
        all(sh.n_joins(), [&](uint32_t i) { return sh.join(i); });
    }
}

// ------------------------------------------------------------------ block weights

// A sequence as the attention saw it.
__device__ inline Head weight_head(const AttendArgs &a, uint32_t s) {
    Head h = seq_head(a.kv, s);
    if (a.left_out[s]) {
        h.ok = false;
        h.n = h.ctx = 0;
    }
    return h;
}

// Weights are sums of many equal shares, so they are added in 64 bits (fp32
// one after the other loses 2^-24 of the sum each time: 2e-6 after 14,000 rows).
struct WeightArgs {
    float *w;            // [seq][max_pages]
    float *cols;         // [seq][head][unit], or null
    uint32_t tile;       // tokens of a unit of cols
};

// Block weights of a call of few rows: a wavefront a block, lanes over (head,
// row); every unit's sum was kept as its log2, so
// w = sum over rows and units of 2^(unit - lse).  64 sequences of up to 32
// blocks, 64 heads: 5 us (one load at a time: 7; 16 rows each: 23 against 63).
__global__ __launch_bounds__(kThreads) void unit_kernel(AttendArgs a, WeightArgs wa) {
    const uint32_t s = blockIdx.y, b = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= a.kv.max_pages) return;
    const Head hd = weight_head(a, s);
    const uint32_t bt = 1u << a.kv.btl, tile = min(bt, kStep), per = bt / tile;
    const uint32_t have = (hd.ctx + tile - 1) / tile;   // units that hold tokens
    const uint32_t u0 = b * per, u1 = min(u0 + per, have);
    double sum = 0.0;
    if (u0 < u1)
        for (uint32_t i = lane; i < hd.n * a.Hq; i += 64) {
            const uint32_t h = i / (hd.n * a.G), row = i % (hd.n * a.G);
            const float lse = a.lse[(hd.row0 + row / a.G) * a.Hq + h * a.G + row % a.G];
            const float *p = a.units + (((uint64_t)s * a.kv.hk + h) * a.n_units + u0) * a.unit_rows + row;
            // only units that the row sees: its tile may have ended before the others
            const int64_t seen = (int64_t)hd.ctx - hd.n + row / a.G + 1;
            const uint32_t end = seen <= 0 ? 0u : min(u1, (uint32_t)((seen + tile - 1) / tile));
            for (uint32_t u = u0; u < end; u += 8, p += 8ull * a.unit_rows) {   // loads that wait for nothing
                float x[8];
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) x[j] = u + j < end ? p[(uint64_t)j * a.unit_rows] : 0.0f;
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) sum += u + j < end ? exp2_of(x[j] - lse) : 0.0f;
            }
        }
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) wa.w[(uint64_t)s * a.kv.max_pages + b] = hd.ok ? (float)sum : NAN;
}

// Block weights of a call of many rows that kept its rows' sums: a workgroup
// a block and head adds 2^(sum - lse) over the rows that see it: 15 us for
// 131,072 rows and 64 blocks (34 MB).  prompt_kernel takes 3 % longer for it
// with blocks of 512 tokens and 9 to 14 % with smaller ones.
__global__ __launch_bounds__(kThreads) void row_kernel(AttendArgs a, WeightArgs wa) {
    __shared__ double red[kWaves];
    const uint32_t b = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
    const Head hd = weight_head(a, s);
    const uint64_t from = (uint64_t)b << a.kv.btl;
    if (!hd.ok || from >= hd.ctx) return;
    // rows before the block's first token do not see it (and kept nothing)
    const int64_t first = (int64_t)from - ((int64_t)hd.ctx - hd.n);
    const float *p = a.sums + ((uint64_t)h * a.kv.max_pages + b) * a.sum_rows + hd.row0 * a.G;
    double sum = 0.0;
    for (uint32_t r = (first > 0 ? (uint32_t)first * a.G : 0u) + threadIdx.x; r < hd.n * a.G; r += kThreads)
        sum += exp2_of(p[r] - a.lse[(hd.row0 + r / a.G) * a.Hq + h * a.G + r % a.G]);
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) wa.cols[((uint64_t)s * a.kv.hk + h) * a.n_units + b] = (float)((red[0] + red[1]) + (red[2] + red[3]));
}

// The same without such sums: with every row's lse known, the
// scores are formed once more, 256 tokens a workgroup (64 a wavefront, their
// keys in registers) against all rows, and 2^(x - lse) is summed over them (a
// prompt's partial sums of every row would be larger than its cache).  Rows
// come 64 at a time, 16 by each wavefront, through LDS: read by each wavefront
// for itself, every CU of a head's XCD asked its cache for the same lines
// (two chunks of 1,024 rows of 64 heads and 32,768 tokens, 1.08 TFLOP: 1,030 us
// against 1,880).
template <int D, bool HALF>
__global__ __launch_bounds__(kThreads, D == 256 ? 2 : 3) void column_kernel(AttendArgs a, WeightArgs wa) {
    typedef typename Elem<HALF>::T T;
    typedef typename Elem<HALF>::T8 T8;
    __shared__ u32x4 lds_q[2][kWaves][D / 32][64];
    __shared__ float lds_lse[2][16 * kWaves];
    __shared__ int lds_seen[2][16 * kWaves];           // tokens that a row sees
    const uint32_t hk = a.kv.hk;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t h = blockIdx.x % hk, kt0 = blockIdx.x / hk * kWaves, kt = kt0 + w, s = blockIdx.y;
    const Head hd = weight_head(a, s);
    if ((uint64_t)kt0 * kStep >= hd.ctx) return;
    const uint32_t c = lane & 15, g = lane >> 4;
    const uint32_t bt = 1u << a.kv.btl;
    const uint32_t *pages = a.kv.pages + (uint64_t)s * a.kv.max_pages;
    const uint32_t last_block = (hd.ctx - 1) >> a.kv.btl;
    const uint32_t pk = pages[min((kt * kStep + 16 * (c >> 2)) >> a.kv.btl, last_block)];
    const uint32_t pv = pages[min((kt * kStep + 16 * g) >> a.kv.btl, last_block)];
    const bool bad = pv >= a.kv.n_pages;
    const float sc = bad ? NAN : a.kv.ks[(uint64_t)pv * hk + h] * (a.q_sign ? -a.c0 : a.c0);
    const uint32_t tok = ((kt * kStep + 16 * (c >> 2)) & (bt - 1)) + (c & 3);
    const uint8_t *p = a.kv.k + ((uint64_t)(pk < a.kv.n_pages ? pk : 0u) * hk + h) * head_bytes(a.kv, D) + (uint64_t)tok * D + 16 * g;
    T8 kf[4][D / 32];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const u32x4 x = *(const u32x4 *)(p + 4 * t * D + 64 * i);
            kf[t][2 * i] = widen<HALF>(x[0], x[1]);
            kf[t][2 * i + 1] = widen<HALF>(x[2], x[3]);
        }
    const int tok0 = (int)(kt * kStep + 16 * g);
    const uint32_t n_rows = hd.n * a.G;
    // the first row that sees a token of the workgroup's; rows from `full` on
    // see all of this wavefront's
    const int64_t old = (int64_t)hd.ctx - hd.n;
    const uint32_t first = (int64_t)kt0 * kStep > old ? (uint32_t)((int64_t)kt0 * kStep - old) * a.G / 16 * 16 : 0u;
    const int64_t need = (int64_t)kt * kStep + kStep - 1 - old;
    const uint64_t full = (uint64_t)kt * kStep + kStep > hd.ctx ? ~0ull : need > 0 ? (uint64_t)need * a.G : 0ull;
    double total = 0.0;
    T8 qf[D / 32];
    float lse = 0.0f;
    int seen = 0;
    auto fetch = [&](uint32_t r0) {                    // rows r0 + 16 w + c
        const uint32_t r = r0 + 16 * w + c;
        const uint32_t at = min(r, n_rows - 1), t = at / a.G, qh = h * a.G + at % a.G;
        const int64_t sees = old + t + 1;
        seen = r < n_rows && sees > 0 ? (int)sees : 0;
        lse = a.lse[(hd.row0 + t) * a.Hq + qh];
        const T *q = (const T *)a.q + (hd.row0 + t) * a.q_stride + (uint64_t)qh * D + 16 * g;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) qf[i] = *(const T8 *)(q + (i / 2) * 64 + (i % 2) * 8);
    };
    auto stage = [&](int b) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) lds_q[b][w][i][lane] = __builtin_bit_cast(u32x4, qf[i]);
        if (g == 0) {
            lds_lse[b][16 * w + c] = lse;
            lds_seen[b][16 * w + c] = seen;
        }
    };
    if (first < n_rows) {
        fetch(first);
        stage(0);
        __syncthreads();
    }
    int b = 0;
    for (uint32_t r0 = first; r0 < n_rows; r0 += 16 * kWaves, b ^= 1) {
        if (r0 + 16 * kWaves < n_rows) fetch(r0 + 16 * kWaves);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            f32x4 st[4] = {{0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const T8 x = __builtin_bit_cast(T8, lds_q[b][v][i][lane]);
#pragma unroll
                for (int u = 0; u < 4; ++u) st[u] = product(kf[u][i], x, st[u]);
            }
            const float of = lds_lse[b][16 * v + c];
            if (r0 + 16 * v >= full && r0 + 16 * v + 16 <= n_rows) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[u] += exp2_of(fmaf(st[u][i], sc, -of));
            } else {
                const int left = lds_seen[b][16 * v + c] - tok0;   // tokens of this lane's 16 that the row sees
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = exp2_of(fmaf(st[u][i], sc, -of));
                        sum[u] += 4 * u + i < left ? e : 0.0f;
                    }
            }
        }
        total += (double)((sum[0] + sum[1]) + (sum[2] + sum[3]));
        if (r0 + 16 * kWaves < n_rows) stage(b ^ 1);
        __syncthreads();
    }
    // over the rows (16 lanes), then the units' groups of 16 tokens
    const uint32_t tile = min(bt, kStep);
    double x = total;
    for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d, 64);
    if (tile >= 32) x += __shfl_xor(x, 16, 64);
    if (tile >= 64) x += __shfl_xor(x, 32, 64);
    const uint32_t u = kt * (kStep / tile) + 16 * g / tile;
    if (c == 0 && ((16 * g) & (tile - 1)) == 0 && u < a.n_units) wa.cols[((uint64_t)s * hk + h) * a.n_units + u] = (float)x;
}

// The units of a block and the heads, in order: 4 us, a launch's latency.
__global__ __launch_bounds__(kThreads) void block_kernel(AttendArgs a, WeightArgs wa) {
    const uint32_t s = blockIdx.y, b = blockIdx.x * kThreads + threadIdx.x;
    if (b >= a.kv.max_pages) return;
    const Head hd = weight_head(a, s);
    const uint32_t per = (1u << a.kv.btl) / wa.tile, have = (hd.ctx + wa.tile - 1) / wa.tile;
    const uint32_t u0 = b * per, u1 = min(u0 + per, have);
    double sum = 0.0;
    if (hd.n)
        for (uint32_t h = 0; h < a.kv.hk; ++h)
            for (uint32_t u = u0; u < u1; ++u) sum += wa.cols[((uint64_t)s * a.kv.hk + h) * a.n_units + u];
    wa.w[(uint64_t)s * a.kv.max_pages + b] = hd.ok ? (float)sum : NAN;
}

// A page's weight is the sum over the sequences that hold it, in fixed point
// (2^-24 of one row's whole attention) so that their order does not matter.  64
// sequences of 1,024 blocks: 4 us.
__global__ __launch_bounds__(kThreads) void weigh_kernel(Kv a, const float *w, unsigned long long *page_weight) {
    const uint32_t s = blockIdx.y, b = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t held = a.ctx[s];
    if ((uint64_t)held > ((uint64_t)a.max_pages << a.btl)) {
        if (b == 0) report(a);
        return;
    }
    if (b >= (held + (1u << a.btl) - 1) >> a.btl) return;
    const uint32_t page = a.pages[(uint64_t)s * a.max_pages + b];
    const float x = w[(uint64_t)s * a.max_pages + b];
    if (page >= a.n_pages || !(x >= 0.0f && x < 4294967296.0f)) {
        report(a);
        return;
    }
    const unsigned long long q = (unsigned long long)rint((double)x * 16777216.0);
    if (q) atomicAdd(page_weight + page, q);
}

// ------------------------------------------------------------------ store and read

template <int D, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 8 : 1) void store_kernel(MoveArgs a, bool half) {
    if (blockIdx.y == 0 && blockIdx.z == 0) report_bad(a.kv, blockIdx.x, gridDim.x);
    store_block<D, THREADS>(a, half, blockIdx.x, blockIdx.y, blockIdx.z);
}

// One workgroup gives back up to 64 tokens (one tile of positions) of one
// head: keys in rows as they lie, values turned through LDS.  Bound by memory:
// the same prompts (269 MB in, 537 MB out) take 178 us, 4.5 TB/s.
template <int D>
__global__ __launch_bounds__(kThreads) void read_kernel(MoveArgs a, bool half) {
    constexpr uint32_t kPitch = D / 4 + 1;
    __shared__ uint32_t turn[kStep * kPitch];
    const Kv &kv = a.kv;
    const uint32_t task = blockIdx.x, h = blockIdx.y;
    if (h == 0) report_bad(kv, task, gridDim.x);
    uint32_t rest;
    const uint32_t s = locate<kThreads>(kv, task, [&](const Head &h) { return read_steps(h); }, &rest);
    if (s >= kv.n_seq) return;
    const Head hd = seq_head(kv, s);
    const uint32_t start = hd.ctx - hd.n, bt = 1u << kv.btl, tile = min(bt, kStep);
    const uint32_t q0 = (start / kStep + rest) * kStep;
    const uint32_t t0 = max(start, q0), t1 = min(hd.ctx, q0 + kStep);
    const uint32_t *pages = kv.pages + (uint64_t)s * kv.max_pages;
    auto put8 = [&](void *base, uint64_t stride, uint32_t tok, uint32_t d, u32x2 y, float sc) {
        const f16x8 z = widen_f16(y[0], y[1]);
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 p = {(float)z[2 * j] * sc, (float)z[2 * j + 1] * sc};
            o[j] = half ? __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2))
                        : __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        }
        *(u32x4 *)((uint16_t *)base + (hd.row0 + (tok - start)) * stride + (uint64_t)h * D + d) = o;
    };
    for (uint32_t e = threadIdx.x; e < (t1 - t0) * (D / 8); e += kThreads) {
        const uint32_t tok = t0 + e / (D / 8), d = e % (D / 8) * 8;
        const uint32_t page = pages[tok >> kv.btl];
        const bool bad = page >= kv.n_pages;
        if (bad) report(kv);
        const uint64_t at = (uint64_t)(bad ? 0u : page) * kv.hk + h;
        const u32x2 y = *(const u32x2 *)(kv.k + at * head_bytes(kv, D) + (uint64_t)(tok & (bt - 1)) * D + d);
        put8((void *)a.k, a.k_stride, tok, d, y, bad ? NAN : kv.ks[at]);
    }
    // 16 tokens of four dimensions a thread, turned
    for (uint32_t e = threadIdx.x; e < D; e += kThreads) {
        const uint32_t dq = e / 4, tok = q0 + e % 4 * 16;
        if (tok >= t1 || tok + 16 <= t0) continue;
        const uint32_t page = pages[tok >> kv.btl];
        const uint64_t at = (uint64_t)(page < kv.n_pages ? page : 0u) * kv.hk + h;
        const uint32_t slot = tok & (bt - 1);
        const uint8_t *p = kv.v + at * head_bytes(kv, D) + (uint64_t)(slot & ~(tile - 1)) * D + dq * 4 * tile + (slot & (tile - 1));
        u32x4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = *(const u32x4 *)(p + j * tile);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t y[4] = {x[0][j], x[1][j], x[2][j], x[3][j]};
            turn4(y[0], y[1], y[2], y[3]);
#pragma unroll
            for (int q = 0; q < 4; ++q) turn[(tok - q0 + 4 * j + q) * kPitch + dq] = y[q];
        }
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < (t1 - t0) * (D / 8); e += kThreads) {
        const uint32_t tok = t0 + e / (D / 8), d = e % (D / 8) * 8;
        const uint32_t page = pages[tok >> kv.btl];
        const bool bad = page >= kv.n_pages;
        const uint32_t *p = turn + (tok - q0) * kPitch + d / 4;
        put8((void *)a.v, a.v_stride, tok, d, u32x2{p[0], p[1]}, bad ? NAN : kv.vs[(uint64_t)page * kv.hk + h]);
    }
}

// ------------------------------------------------------------------ host

// How a call is split, and its workspace.
struct Layout : Split {
    int NT;
    bool rows;             // prompt_kernel
    bool sums;             // and its rows' sums over the blocks
    bool kept;             // attend_kernel's sums of every unit
    uint32_t item_cap, slot_cap, join_cap, n_units, unit_rows;
    uint64_t head, items, joins, ml, part, lse, left_out, units, cols, sums_at, total;
};

netkv_status make_layout(netkv_handle h, const Kv &a, uint32_t D, uint32_t heads, bool weights, Layout &y) {
    if (heads < 1 || heads % a.hk) return invalid(h, "n_heads must be a multiple of n_kv_heads");
    y.G = heads / a.hk;
    if (y.G > 64) return invalid(h, "n_heads / n_kv_heads must be <= 64");
    const uint64_t most = (uint64_t)a.max_tok * y.G;   // rows of the longest sequence's head
    if (most > 0xFFFFFFFFull - 1024) return invalid(h, "max_tok * n_heads / n_kv_heads must be < 2^32 - 1024");
    // Rows of the longest sequence from which prompt_kernel pays, whose tile
    // takes as long with one row as with all.  The row tiles of attend_kernel
    // lie side by side, and the cache's lines reach them from L2.  64 sequences
    // of 8,192 tokens, attend_kernel against prompt_kernel, us: 64 dimensions,
    // 192 rows 205, 258, 256 rows 268, 265; 128 dimensions, 128 rows 520, 609,
    // 160 rows 626, 673, 192 rows 794, 701; 256 dimensions, 32 rows 81, 84, 64
    // rows 162, 84.  One form for the whole call: beside a chunk of 21 rows (168 a
    // head) 255 such sequences with single tokens take 1,861 us, beside one of 20
    // rows 779, alone 710.
    y.rows = most > (D == 64 ? 240u : D == 128 ? 160u : 32u);
    // 16 rows a tile or 32: 16 rows 79, 85; 32 rows 100, 89; 64 rows 177, 131
    y.NT = most <= 16 || D == 256 ? 1 : 2;
    y.tile_rows = y.rows ? (D == 256 ? 128u : 256u) : 16u * y.NT;
    y.unit_rows = (uint32_t)(most / 4 * 4 + 4);
    // ranges a head: what fills the card's 512 workgroup slots once, or where
    // they stay long enough twice (unequal lengths even out).  512, 1,024, 1,536
    // in all, 128 dimensions, us: 64 ragged sequences of up to 16,384 tokens
    // 146, 136, 137; one of 131,072 51, 56, 60; 200 ragged of up to 700 50, 63, 70.
    y.target = (512u + a.hk - 1) / a.hk;
    y.fine = y.rows || y.NT == 2 || D == 256 ? y.target : (1024u + a.hk - 1) / a.hk;
    const uint32_t bt = 1u << a.btl;
    // The shortest range, steps: one a wavefront (4, 8, 12, 16; single tokens, 64
    // heads of 128 dimensions, the whole call, us: one sequence of 8 steps 14.6,
    // 11.9, 11.7, 11.7, of 16 14.0, 14.7, 15.9, 11.7, of 64 14.3, 14.7, 16.1, 17.2;
    // 64 sequences of 8 steps 22.7, 16.6, 16.5, 16.4, of 16 32.0, 31.0, 31.2, 25.1,
    // of 32 49.7, 50.2, 50.1, 49.2): it pays where a join's 6 us are less than the
    // steps it saves, from some 20 on.  Prompts (4, 8, 16, 32; 64 rows after that
    // many steps): 8 steps 31, 28, 28, 28, 16 37, 37, 41, 41, 64 41, 41, 53, 77.
    y.least = y.rows ? 8 : kWaves;
    // whole blocks for a prompt (its sums), with and without weights the same
    y.round = !y.rows ? kWaves : bt > kStep ? bt / kStep : 1;
    const Caps caps = caps_of(a, y);
    if (!grid_fits(caps.items * a.hk, y.rows ? kPromptThreads : kThreads)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many query rows for one call");
    y.item_cap = (uint32_t)caps.items;
    y.slot_cap = (uint32_t)caps.slots;
    y.join_cap = (uint32_t)caps.joins;
    y.n_units = (uint32_t)(((uint64_t)a.max_pages << a.btl) / (bt < kStep ? bt : kStep)) + (uint32_t)(kStep / 16);
    if (weights && (((uint64_t)a.max_pages << a.btl) / kStep + 1) * a.hk > (1ull << 24))
        return netkv_internal_fail(h, NETKV_ECAPACITY, "too many cache blocks for one call with weights");
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t p = at;
        at += align256(bytes);
        return p;
    };
    y.head = take(sizeof(PlanHead));
    y.items = take(sizeof(Item) * y.item_cap);
    y.joins = take(sizeof(Join) * y.join_cap);
    y.ml = take(16ull * y.slot_cap * a.hk * y.tile_rows);
    y.part = take(4ull * y.slot_cap * a.hk * y.tile_rows * D);
    // A prompt's weights come from every row's sum over each block where a row
    // has at most 256 of them (1 KB; a row's query and output are 512 bytes at
    // 128 dimensions), else from a second pass over the keys, which takes
    // longer but no memory: two chunks of 1,024 rows of 64 heads in 8,192 tokens
    // of 32-token blocks 704 us against 921, in 16,384 of 64-token blocks 1,320
    // against 1,750.  Either form's sums are kept up to kMostKept.
    y.sums = weights && y.rows && a.max_pages <= 256 && row_sum_bytes(a, y.G) <= kMostKept;
    y.kept = weights && !y.rows && unit_bytes(a, y.n_units, y.unit_rows) <= kMostKept;
    if (y.sums) y.n_units = a.max_pages;
    y.lse = y.left_out = y.units = y.cols = y.sums_at = 0;
    if (weights) {
        y.lse = take(4ull * a.n_tok * heads);
        y.left_out = take(4ull * a.n_seq);
        if (y.kept)
            y.units = take(unit_bytes(a, y.n_units, y.unit_rows));
        else
            y.cols = take(4ull * a.n_seq * a.hk * y.n_units);
        if (y.sums) y.sums_at = take(row_sum_bytes(a, y.G));
    }
    y.total = at;
    return NETKV_OK;
}

template <int D, bool HALF>
void launch_attend(const Layout &y, const AttendArgs &a, const WeightArgs &wa, hipStream_t s) {
    const dim3 grid(y.item_cap * a.kv.hk);
#define NETKV_ATTEND(NT, UNITS)                                                             \
    a.kv.btl < 6 ? attend_kernel<D, NT, HALF, UNITS, true><<<grid, kThreads, 0, s>>>(a)     \
                 : attend_kernel<D, NT, HALF, UNITS, false><<<grid, kThreads, 0, s>>>(a)
    if (y.rows) {
        if (y.sums)
            a.kv.btl < 6 ? prompt_kernel<D, D == 256 ? 1 : 2, HALF, true, true><<<grid, kPromptThreads, 0, s>>>(a)
                         : prompt_kernel<D, D == 256 ? 1 : 2, HALF, false, true><<<grid, kPromptThreads, 0, s>>>(a);
        else
            a.kv.btl < 6 ? prompt_kernel<D, D == 256 ? 1 : 2, HALF, true, false><<<grid, kPromptThreads, 0, s>>>(a)
                         : prompt_kernel<D, D == 256 ? 1 : 2, HALF, false, false><<<grid, kPromptThreads, 0, s>>>(a);
    } else if (D == 256 || y.NT == 1) {
        if (y.kept) NETKV_ATTEND(1, true);
        else NETKV_ATTEND(1, false);
    } else if constexpr (D != 256) {
        if (y.kept) NETKV_ATTEND(2, true);
        else NETKV_ATTEND(2, false);
    }
#undef NETKV_ATTEND
    // nothing is split where no sequence can be longer than the shortest range
    const uint64_t steps_most = (((uint64_t)a.kv.max_pages << a.kv.btl) + kStep - 1) / kStep;
    const uint32_t rows = y.unit_rows < y.tile_rows ? y.unit_rows : y.tile_rows;   // that a tile can have
    const uint64_t joins_most = (uint64_t)y.join_cap * a.kv.hk * rows;
    // a workgroup a row up to 512, else a wavefront a row, in at most 1,024
    // workgroups: those without a row find that out first (2,048 against 855 for
    // 37 sequences of 9 rows and 5 heads: 10.8 us, 6.3; against 1,024 for 200
    // sequences of 32 rows and 8 heads: 11.6, 9.3)
    const uint64_t quarter = (joins_most + 3) / 4;
    const uint64_t join_groups = joins_most < 512 ? joins_most : quarter < 512 ? 512 : quarter < 1024 ? quarter : 1024;
    if (steps_most > a.least) join_kernel<D, HALF><<<(uint32_t)join_groups, kThreads, 0, s>>>(a, rows);
    if (!wa.w) return;
    if (!y.kept) {
        const uint32_t steps = (uint32_t)((((uint64_t)a.kv.max_pages << a.kv.btl) + kStep - 1) / kStep);
        if (y.sums)
            row_kernel<<<dim3(a.kv.max_pages, a.kv.hk, a.kv.n_seq), kThreads, 0, s>>>(a, wa);
        else
            column_kernel<D, HALF><<<dim3((steps + kWaves - 1) / kWaves * a.kv.hk, a.kv.n_seq), kThreads, 0, s>>>(a, wa);
        block_kernel<<<dim3((a.kv.max_pages + kThreads - 1) / kThreads, a.kv.n_seq), kThreads, 0, s>>>(a, wa);
    } else {
        unit_kernel<<<dim3((a.kv.max_pages + kWaves - 1) / kWaves, a.kv.n_seq), kThreads, 0, s>>>(a, wa);
    }
}

}  // namespace

extern "C" netkv_status netkv_kv_attend_workspace(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs,
                                                  uint32_t n_heads, int weights, uint64_t *bytes) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (!bytes) return invalid(h, "bytes must not be NULL");
    Kv a{};
    netkv_status st = make_kv(h, kv, seqs, a);
    if (st != NETKV_OK) return st;
    Layout y{};
    st = make_layout(h, a, kv->head_dim, n_heads, weights != 0, y);
    if (st != NETKV_OK) return st;
    *bytes = y.total;
    return NETKV_OK;
}

extern "C" netkv_status netkv_kv_attend(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs, const void *q,
                                        int dtype, uint32_t n_heads, uint64_t q_stride, float scale, void *out,
                                        uint64_t out_stride, float *block_weight, void *work, uint64_t work_bytes,
                                        void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    Kv a{};
    netkv_status st = make_kv(h, kv, seqs, a);
    if (st != NETKV_OK) return st;
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    Layout y{};
    st = make_layout(h, a, kv->head_dim, n_heads, block_weight != nullptr, y);
    if (st != NETKV_OK) return st;
    if (!std::isfinite(scale)) return invalid(h, "scale must be finite");
    const uint64_t width = (uint64_t)n_heads * kv->head_dim;
    if ((st = check_rows(h, q, q_stride, width, a.n_tok, "q must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, out, out_stride, width, a.n_tok, "out must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    // a row is read by the one workgroup that writes it, or before a join does;
    // but the second pass over the keys for block weights reads q again
    if (rows_overlap(q, q_stride, out, out_stride, width, a.n_tok) && (q != out || q_stride != out_stride || block_weight))
        return invalid(h, "out must not overlap q (without block weights it may be q itself)");
    if (a.n_seq == 0) return NETKV_OK;
    if (!work || ((uintptr_t)work & 255) || work_bytes < y.total) return invalid(h, "work must be 256-byte aligned and of at least netkv_kv_attend_workspace's bytes");
    DeviceScope scope(netkv_internal_device(h));
    hipStream_t s = (hipStream_t)stream;
    uint8_t *ws = (uint8_t *)work;
    const bool half = dtype == NETKV_FP16;
    AttendArgs t{};
    t.kv = a;
    (Split &)t = y;
    t.left_out = block_weight ? (uint32_t *)(ws + y.left_out) : nullptr;
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
    t.Hq = n_heads;
    t.q_stride = q_stride;
    t.q = q;
    t.out = out;
    t.c0 = std::fabs(scale) * kLog2e;
    t.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    t.part = (float *)(ws + y.part);
    t.part_ml = (f32x4 *)(ws + y.ml);
    t.lse = block_weight ? (float *)(ws + y.lse) : nullptr;
    t.units = y.kept ? (float *)(ws + y.units) : nullptr;
    t.n_units = y.n_units;
    t.unit_rows = y.unit_rows;
    t.sums = y.sums ? (float *)(ws + y.sums_at) : nullptr;
    t.sum_rows = (uint64_t)a.n_tok * y.G;
    WeightArgs wa{};
    wa.tile = y.sums ? kv->block_tokens : kv->block_tokens < kStep ? kv->block_tokens : kStep;
    wa.w = block_weight;
    wa.cols = block_weight && !y.kept ? (float *)(ws + y.cols) : nullptr;
    switch (kv->head_dim) {
        case 64: half ? launch_attend<64, true>(y, t, wa, s) : launch_attend<64, false>(y, t, wa, s); break;
        case 128: half ? launch_attend<128, true>(y, t, wa, s) : launch_attend<128, false>(y, t, wa, s); break;
        default: half ? launch_attend<256, true>(y, t, wa, s) : launch_attend<256, false>(y, t, wa, s); break;
    }
    return launched(h, "attention launch failed");
}

extern "C" netkv_status netkv_kv_weigh(netkv_handle h, const netkv_kv_seqs_t *q, uint32_t block_tokens, const float *block_weight,
                                       uint32_t n_pages, uint64_t *page_weight, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (!q) return invalid(h, "seqs must not be NULL");
    // neither the cache nor the rows are touched: any address stands for them in the checks
    netkv_kv_seqs_t seqs = *q;
    seqs.n_tok = seqs.max_tok = 0;
    seqs.tok_off = (const uint64_t *)16;
    netkv_kv_t kv{};
    kv.n_pages = n_pages;
    kv.block_tokens = block_tokens;
    kv.n_kv_heads = 1;
    kv.head_dim = 64;
    kv.k = kv.v = (uint8_t *)16;
    kv.k_scale = kv.v_scale = (float *)16;
    Kv a{};
    netkv_status st = make_kv(h, &kv, &seqs, a);
    if (st != NETKV_OK) return st;
    if (a.n_seq == 0) return NETKV_OK;
    if (!block_weight || !page_weight) return invalid(h, "block_weight and page_weight must not be NULL");
    DeviceScope scope(netkv_internal_device(h));
    weigh_kernel<<<dim3((a.max_pages + kThreads - 1) / kThreads, a.n_seq), kThreads, 0, (hipStream_t)stream>>>(
        a, block_weight, (unsigned long long *)page_weight);
    return launched(h, "weight launch failed");
}

namespace {

// One pass over the data where a workgroup's registers hold a block's rows.
// 256 threads against 1,024, us: 64 times 64 rows of 128 dimensions 13, 27;
// single rows 9, 20; prompts in 512-token blocks 267, 226.
uint32_t store_threads(uint32_t rows, uint32_t D) { return rows * D <= 256 * 64 ? 256 : 1024; }

template <int D>
void launch_store(const MoveArgs &a, bool half, uint32_t tasks, uint32_t threads, hipStream_t s) {
    const dim3 grid(tasks, a.kv.hk, 2);
    if (threads == 256)
        store_kernel<D, 256><<<grid, 256, 0, s>>>(a, half);
    else
        store_kernel<D, 1024><<<grid, 1024, 0, s>>>(a, half);
}

}  // namespace

extern "C" netkv_status netkv_kv_store(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs, const void *k,
                                       uint64_t k_stride, const void *v, uint64_t v_stride, int dtype, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    MoveArgs a{};
    netkv_status st = make_kv(h, kv, seqs, a.kv);
    if (st != NETKV_OK) return st;
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    const uint64_t width = (uint64_t)kv->n_kv_heads * kv->head_dim;
    if ((st = check_rows(h, k, k_stride, width, a.kv.n_tok, "k must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, v, v_stride, width, a.kv.n_tok, "v must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if (a.kv.n_seq == 0 || a.kv.n_tok == 0) return NETKV_OK;
    a.k = k;
    a.v = v;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    const uint64_t tasks = store_groups(a.kv);
    const uint32_t threads = store_threads(a.kv.max_tok < kv->block_tokens ? a.kv.max_tok : kv->block_tokens, kv->head_dim);
    if (!grid_fits(tasks, threads)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many blocks for one call");
    DeviceScope scope(netkv_internal_device(h));
    hipStream_t s = (hipStream_t)stream;
    const bool half = dtype == NETKV_FP16;
    switch (kv->head_dim) {
        case 64: launch_store<64>(a, half, (uint32_t)tasks, threads, s); break;
        case 128: launch_store<128>(a, half, (uint32_t)tasks, threads, s); break;
        default: launch_store<256>(a, half, (uint32_t)tasks, threads, s); break;
    }
    return launched(h, "store launch failed");
}

extern "C" netkv_status netkv_kv_read(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs, void *k,
                                      uint64_t k_stride, void *v, uint64_t v_stride, int dtype, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    MoveArgs a{};
    netkv_status st = make_kv(h, kv, seqs, a.kv);
    if (st != NETKV_OK) return st;
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    const uint64_t width = (uint64_t)kv->n_kv_heads * kv->head_dim;
    if ((st = check_rows(h, k, k_stride, width, a.kv.n_tok, "k must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, v, v_stride, width, a.kv.n_tok, "v must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if (a.kv.n_seq == 0 || a.kv.n_tok == 0) return NETKV_OK;
    a.k = k;
    a.v = v;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    const uint64_t tasks = read_groups(a.kv);
    if (!grid_fits(tasks, kThreads)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many tokens for one call");
    DeviceScope scope(netkv_internal_device(h));
    hipStream_t s = (hipStream_t)stream;
    const bool half = dtype == NETKV_FP16;
    const dim3 grid((uint32_t)tasks, kv->n_kv_heads);
    switch (kv->head_dim) {
        case 64: read_kernel<64><<<grid, kThreads, 0, s>>>(a, half); break;
        case 128: read_kernel<128><<<grid, kThreads, 0, s>>>(a, half); break;
        default: read_kernel<256><<<grid, kThreads, 0, s>>>(a, half); break;
    }
    return launched(h, "read launch failed");
}
