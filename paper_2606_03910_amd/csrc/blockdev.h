// What the block cache's kernels share: operands and their types, how a call's
// work is found, the softmax's weights, and the host's checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "blockplan.h"
#include "netkv.h"
#include "netkv_internal.h"

namespace blockdev {

using namespace blockplan;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPromptThreads = 512;
constexpr float kLog2e = 1.44269504088896340736f;
// A weight is held as P = 2^(x - y) s in fp16, with the row's largest 2^kLift
// when y is set: what P loses below fp16's smallest steps is then 2^-(25 +
// kLift) of the largest weight at most, 2^-14 of a row over 131,072 equal
// tokens behind a dominant one (without the lift 2^-8).  From there y stays
// until 16 weights' sum passes kMaxSum, fp16's largest.  A larger lift loses
// less and raises y more often: 5, 6, 7, 8 and 10 take 469, 476, 484, 495 and
// 521 us for six prompts of up to 2,777 tokens whose scores' deviation is up
// to 3, 1,997 to 2,089 us for two chunks of 1,024 rows after 31,744.
constexpr float kLift = 6.0f;
constexpr float kMaxSum = 65504.0f;
constexpr uint32_t kNoSlot = 0xFFFFFFFFu;

__device__ inline void report(const Kv &a) { atomicOr(a.err, kErrBlockBit); }

// rows_before for every thread's sequence, from what each adds to it (rows_end,
// 0 for none); `named` is that of the first thread's, and is moved on to the
// one after the workgroup's last.
__device__ inline uint32_t rows_before(uint32_t end, uint32_t &named, uint32_t *sh) {
    const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x / 64;
    uint32_t most = end;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = __shfl_up(most, d, 64);
        if ((int)lane >= d) most = max(most, v);
    }
    if (lane == 63) sh[w] = most;
    __syncthreads();
    uint32_t before = __shfl_up(most, 1, 64), all = named;
    if (lane == 0) before = 0;
    before = max(before, named);
    for (uint32_t v = 0; v < waves; ++v) {
        if (v < w) before = max(before, sh[v]);
        all = max(all, sh[v]);
    }
    named = all;
    __syncthreads();
    return before;
}

// bytes of one head of one page
__device__ inline uint64_t head_bytes(const Kv &a, int D) { return (uint64_t)D << a.btl; }

template <bool HALF>
struct Elem;
template <>
struct Elem<true> {
    typedef _Float16 T;
    typedef f16x2 T2;
    typedef f16x8 T8;
};
template <>
struct Elem<false> {
    typedef __bf16 T;
    typedef bf16x2 T2;
    typedef bf16x8 T8;
};

// 8 e4m3 bytes to 16 bits, exactly (4 significant bits, exponents -9 to 8)
__device__ inline f16x8 widen_f16(uint32_t a, uint32_t b) {
    const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
    const f16x2 q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
    const f16x2 s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

__device__ inline bf16x8 widen_bf16(uint32_t a, uint32_t b) {
    const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    const bf16x2 q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    const bf16x2 s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

template <bool HALF>
__device__ inline typename Elem<HALF>::T8 widen(uint32_t a, uint32_t b) {
    if constexpr (HALF)
        return widen_f16(a, b);
    else
        return widen_bf16(a, b);
}

__device__ inline f32x4 product(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 product(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// 1 in the lowest bit of each byte that is a NaN
__device__ inline uint32_t nan_bytes(uint32_t x) { return (((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7; }

// over the four lanes of a row (lanes l, l ^ 16, l ^ 32, l ^ 48)
__device__ inline float row_max(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float pair16_sum(float x) {   // lanes l, l ^ 16
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ inline float row_sum(float x) {
    x = pair16_sum(x);
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Memory that no kernel writes while this one runs, at an address that is the
// same for the whole wavefront: loads go through the scalar cache.
template <typename T>
__device__ inline const __attribute__((address_space(4))) T *scalar(const T *p) {
    return (const __attribute__((address_space(4))) T *)p;
}

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float log2_of(float x) { return __builtin_amdgcn_logf(x); }

// ------------------------------------------------------------------ work list

struct Item {
    uint32_t seq, tile, k0, k1;   // row tile, steps [k0, k1)
    uint32_t slot, pad[3];        // partial result, or kNoSlot
};
struct Join {
    uint32_t seq, tile, slot, n;  // ranges slot .. slot + n - 1
};
struct PlanHead {
    uint32_t n_items, n_joins, n_slots, pad;
};

// How a call is split.  With up to kListed sequences every wavefront finds its
// share by itself (Shares); beyond that plan_kernel writes the list.
struct PlanArgs : Split {
    Kv kv;
    PlanHead *head;
    Item *items;                                   // null: not listed
    Join *joins;
    uint32_t *left_out;                            // [seq] 1: begins among rows of an earlier one; null: no weights
    // rows of sequences that cannot be answered
    uint16_t *bad_out;
    uint64_t out_stride;
    uint32_t row_elems, nan16;
};

constexpr uint32_t kListed = 256;

// Starts plan_kernel for a call of more sequences than kListed.
void launch_plan(const PlanArgs &a, hipStream_t s);

constexpr int kPlanThreads = 1024;

// Exclusive scan of three counts over the workgroup; totals in tot.
__device__ inline void scan3(uint32_t (&x)[3], uint32_t (&tot)[3], uint32_t (*wsum)[3]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t in[3];
    for (int i = 0; i < 3; ++i) {
        uint32_t y = x[i];
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t z = __shfl_up(y, d, 64);
            if (lane >= d) y += z;
        }
        in[i] = y;
        if (lane == 63) wsum[w][i] = y;
    }
    __syncthreads();
    for (int i = 0; i < 3; ++i) {
        uint32_t before = 0, all = 0;
        for (int v = 0; v < kPlanThreads / 64; ++v) {
            const uint32_t z = wsum[v][i];
            if (v < w) before += z;
            all += z;
        }
        x[i] = before + in[i] - x[i];
        tot[i] = all;
    }
    __syncthreads();
}

// The last step (exclusive) that a row tile of a sequence sees.
__device__ inline uint32_t tile_end(const Head &h, uint32_t G, uint32_t tile, uint32_t rows) {
    const uint64_t last = min((uint64_t)(tile + 1) * rows, (uint64_t)h.n * G) - 1;
    const int64_t seen = (int64_t)h.ctx - h.n + (int64_t)(last / G) + 1;
    return seen <= 0 ? 0u : (uint32_t)((seen + kStep - 1) / kStep);
}

// Range `part` of `p` of a row tile.
__device__ inline Item item_of(const PlanArgs &a, uint32_t seq, const Head &h, uint32_t C, uint32_t p, uint32_t tile, uint32_t part, uint32_t slot0) {
    const uint32_t end = tile_end(h, a.G, tile, a.tile_rows);
    Item it;
    it.seq = seq;
    it.tile = tile;
    it.k0 = part * C;
    it.k1 = min(end, p > 1 ? (part + 1) * C : end);
    it.slot = p > 1 ? slot0 + tile * p + part : kNoSlot;
    return it;
}

// The rows of sequences that cannot be answered, by one workgroup; those that
// an earlier sequence names as well are left to it.
__device__ inline void fill_bad(const PlanArgs &a) {
    bool bad = false;
    for (uint32_t s = threadIdx.x; s < a.kv.n_seq; s += blockDim.x) bad |= !seq_head(a.kv, s).ok;
    if (!__syncthreads_or(bad)) return;
    uint32_t before = 0;
    for (uint32_t s = 0; s < a.kv.n_seq; ++s) {
        const Head h = seq_head(a.kv, s);
        const uint64_t from = max(h.row0, (uint64_t)before);
        before = max(before, rows_end(a.kv, s));
        if (h.ok && from == h.row0) continue;
        if (threadIdx.x == 0) report(a.kv);
        if (!h.rows_ok || from >= a.kv.off[s + 1]) continue;
        const uint64_t rows = a.kv.off[s + 1] - from;
        for (uint64_t i = threadIdx.x; i < rows * a.row_elems; i += blockDim.x)
            a.bad_out[(from + i / a.row_elems) * a.out_stride + i % a.row_elems] = (uint16_t)a.nan16;
    }
}

// The same list as a wavefront has it in its registers: each lane takes up to
// four sequences in a row (n_seq <= kListed).  The ranges of full length come
// first, then every tile's last one, tiles that see most before others.
struct Shares {
    uint32_t rt[4], kt[4], C, per;
    uint32_t fulls, lasts, slots, joins;      // inclusive sums up to this lane
    uint32_t own_fulls, own_lasts, own_slots, own_joins;
    uint32_t left;                            // a bit for each of the lane's sequences that begin among rows of an earlier one
    bool bad;

    __device__ explicit Shares(const PlanArgs &a) {
        const uint32_t lane = threadIdx.x & 63;
        per = (a.kv.n_seq + 63) / 64;
        bool rows_ok = true;
        left = 0;
        bad = false;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            rt[j] = kt[j] = 0;
            if (j >= per) continue;
            const uint32_t s = lane * per + j;
            if (s < a.kv.n_seq) {
                const Head h = seq_head(a.kv, s);
                rt[j] = tiles_of(h, a);
                kt[j] = steps_of(h);
                bad |= !h.ok;
                rows_ok &= h.rows_ok;
            }
        }
        if (__builtin_expect(__any(!rows_ok), 0)) leave_out(a);
        unsigned long long work = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) work += (unsigned long long)rt[j] * kt[j];
        for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d, 64);
        C = range_steps(a, work);
        own_fulls = own_lasts = own_slots = own_joins = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            if (j >= per) continue;
            const uint32_t p = parts(j);
            own_fulls += rt[j] * (p - 1);
            own_lasts += rt[j];
            own_slots += p > 1 ? rt[j] * p : 0u;
            own_joins += p > 1 ? rt[j] : 0u;
        }
        fulls = own_fulls;
        lasts = own_lasts;
        slots = own_slots;
        joins = own_joins;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(fulls, d, 64), x = __shfl_up(lasts, d, 64), y = __shfl_up(slots, d, 64), z = __shfl_up(joins, d, 64);
            if ((int)lane >= d) {
                fulls += v;
                lasts += x;
                slots += y;
                joins += z;
            }
        }
    }
    __device__ uint32_t parts(uint32_t j) const { return parts_of(kt[j], C); }

    // Sequences that begin among rows of an earlier one.
    __device__ void leave_out(const PlanArgs &a) {
        const uint32_t lane = threadIdx.x & 63;
        uint32_t end = 0;
        for (uint32_t j = 0; j < per; ++j)
            if (lane * per + j < a.kv.n_seq) end = max(end, rows_end(a.kv, lane * per + j));
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(end, d, 64);
            if ((int)lane >= d) end = max(end, v);
        }
        uint32_t before = __shfl_up(end, 1, 64);
        if (lane == 0) before = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t s = lane * per + j;
            if (j >= per || s >= a.kv.n_seq) continue;
            if (a.kv.off[s] < before) {
                rt[j] = kt[j] = 0;
                left |= 1u << j;
            }
            before = max(before, rows_end(a.kv, s));
        }
    }

    // false: there are not so many
    __device__ bool item(const PlanArgs &a, uint32_t i, Item &it) const {
        const uint32_t all_fulls = (uint32_t)__builtin_amdgcn_readlane((int)fulls, 63);
        const bool last = i >= all_fulls;
        if (last) i -= all_fulls;
        const uint64_t past = __ballot((last ? lasts : fulls) > i);
        if (!past) return false;
        const int l = __ffsll((unsigned long long)past) - 1;
        uint32_t at = last ? lasts - own_lasts : fulls - own_fulls, slot = slots - own_slots, seq = 0, n = 0, p = 1, rest = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t q = parts(j), x = rt[j] * (last ? 1u : q - 1);
            if (i >= at && i < at + x) {
                seq = (threadIdx.x & 63) * per + j;
                n = rt[j];
                p = q;
                rest = i - at;
                break;
            }
            at += x;
            slot += q > 1 ? rt[j] * q : 0u;
        }
        auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
        seq = of(seq);
        p = of(p);
        rest = of(rest);
        const uint32_t tile = of(n) - 1 - (last ? rest : rest / (p - 1)), part = last ? p - 1 : rest % (p - 1);
        it = item_of(a, seq, seq_head(a.kv, seq), C, p, tile, part, of(slot));
        return true;
    }
    __device__ uint32_t n_joins() const { return (uint32_t)__builtin_amdgcn_readlane((int)joins, 63); }
    __device__ Join join(uint32_t i) const {
        const int l = __ffsll((unsigned long long)__ballot(joins > i)) - 1;
        uint32_t at = joins - own_joins, slot = slots - own_slots, seq = 0, tile = 0, p = 1;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t q = parts(j), x = q > 1 ? rt[j] : 0u;
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

// This workgroup's share and its sequence; false if there is none.  What every
// lane has the same of goes to scalar registers.
__device__ inline bool find_item(const PlanArgs &a, uint32_t i, Item &it, Head &hd) {
    if (a.items) {
        if (i >= a.head->n_items) return false;
        it = a.items[i];
    } else {
        const Shares sh(a);
        if (blockIdx.x == 0) {
            if (a.left_out)
                for (uint32_t j = 0; j < sh.per; ++j) {
                    const uint32_t s = (threadIdx.x & 63) * sh.per + j;
                    if (s < a.kv.n_seq) a.left_out[s] = sh.left >> j & 1;
                }
            if (__builtin_expect(__any(sh.bad), 0)) fill_bad(a);
        }
        if (!sh.item(a, i, it)) return false;
    }
    auto one = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
    it = Item{one(it.seq), one(it.tile), one(it.k0), one(it.k1), one(it.slot), {0, 0, 0}};
    hd = seq_head(a.kv, it.seq);
    hd.row0 = (uint64_t)one((uint32_t)(hd.row0 >> 32)) << 32 | one((uint32_t)hd.row0);
    hd.n = one(hd.n);
    hd.ctx = one(hd.ctx);
    return true;
}

// 2^(x + by) of 16 scores, as the operand of the product with the values, and
// their sum.  (The empty statement: the weights are rounded here, not where
// they are used, which would keep them in twice the registers.)
__device__ __forceinline__ float weights_of(const f32x4 (&st)[4], float sc, float by, f16x8 (&pf)[2]) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = exp2_of(fmaf(st[t][i], sc, by));
            sum += p[i];
        }
        const f16x2 u = __builtin_convertvector((f32x2{p[0], p[1]}), f16x2);
        const f16x2 v = __builtin_convertvector((f32x2{p[2], p[3]}), f16x2);
        const int j = 4 * (t & 1);
        pf[t >> 1][j] = u[0];
        pf[t >> 1][j + 1] = u[1];
        pf[t >> 1][j + 2] = v[0];
        pf[t >> 1][j + 3] = v[1];
    }
    asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(sum));
    return sum;
}

// O to the row: 2^(y - m) / l in two factors, neither of them subnormal (y - m
// is near log2(s) - kLift, and s may be 2^-126).  A row that sees no token is 0;
// one whose scores are all -inf is no number.
struct Over {
    float a, b;
    __device__ Over(float y, float m, float l, bool sees) {
        const float t = l == 0.0f ? 0.0f : y - m, h = rintf(0.5f * fmaxf(t, -256.0f));   // -inf where every s is 0
        a = l != 0.0f ? exp2_of(h) / l : sees ? NAN : 0.0f;
        b = exp2_of(t - h);
    }
    __device__ float operator()(float o) const { return o * a * b; }
};

// What a part with maximum m counts for beside the maximum of all; a part
// that saw nothing finite holds zeros, or NaN.
__device__ inline float joined(float m, float all) { return m == -INFINITY ? 1.0f : exp2_of(m - all); }

// One step's operands: keys of 64 tokens (lane: key row token, 16 dimensions)
// and values (lane: dimension, 16 tokens).
template <int D>
struct KeyRegs {
    u32x4 f[4][D / 64];
};
template <int D>
struct ValRegs {
    u32x4 f[D / 16];
};

// ------------------------------------------------------------------ host

struct DeviceScope {
    int prev = -1;
    explicit DeviceScope(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev == dev) prev = -1;
        else (void)hipSetDevice(dev);
    }
    ~DeviceScope() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

inline netkv_status invalid(netkv_handle h, const char *msg) { return netkv_internal_fail(h, NETKV_EINVAL, msg); }

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Checks what the host can and fills the kernels' view of it.
inline netkv_status make_kv(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *q, Kv &a) {
    if (!kv || !q) return invalid(h, "kv and seqs must not be NULL");
    uint32_t btl = 0;
    while (btl < 31 && (1u << btl) < kv->block_tokens) ++btl;
    if (kv->block_tokens < 16 || kv->block_tokens > 1024 || (1u << btl) != kv->block_tokens)
        return invalid(h, "block_tokens must be a power of two from 16 to 1024");
    if (kv->head_dim != 64 && kv->head_dim != 128 && kv->head_dim != 256) return invalid(h, "head_dim must be 64, 128 or 256");
    if (kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return invalid(h, "n_kv_heads must be in [1, 1024]");
    if (kv->n_pages < 1 || kv->n_pages > 0x7FFFFFFFu) return invalid(h, "n_pages must be in [1, 2^31)");
    if (!kv->k || !kv->v || !kv->k_scale || !kv->v_scale) return invalid(h, "a cache array is NULL");
    if (!aligned16(kv->k) || !aligned16(kv->v)) return invalid(h, "k and v must be 16-byte aligned");
    if (q->n_seq && (!q->tok_off || !q->ctx_len || !q->pages)) return invalid(h, "a sequence array is NULL");
    if (q->n_seq > 65535) return invalid(h, "n_seq must be <= 65535");
    if (q->n_seq && q->max_pages < 1) return invalid(h, "max_pages must be >= 1");
    if (((uint64_t)q->max_pages << btl) >= (1ull << 31)) return invalid(h, "max_pages * block_tokens must be < 2^31");
    if (q->n_tok > (1ull << 31)) return invalid(h, "n_tok must be <= 2^31");
    a.k = (uint8_t *)kv->k;
    a.v = (uint8_t *)kv->v;
    a.ks = kv->k_scale;
    a.vs = kv->v_scale;
    a.n_pages = kv->n_pages;
    a.hk = kv->n_kv_heads;
    a.btl = btl;
    a.n_seq = q->n_seq;
    a.max_pages = q->max_pages;
    a.max_tok = (uint32_t)(q->max_tok < q->n_tok ? q->max_tok : q->n_tok);
    a.off = q->tok_off;
    a.ctx = q->ctx_len;
    a.pages = q->pages;
    a.n_tok = q->n_tok;
    a.err = netkv_internal_errword(h);
    return NETKV_OK;
}

constexpr uint64_t align256(uint64_t x) { return (x + 255) & ~255ull; }

inline netkv_status launched(netkv_handle h, const char *what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? NETKV_OK : netkv_internal_fail(h, NETKV_EDEVICE, what);
}

inline netkv_status check_rows(netkv_handle h, const void *p, uint64_t stride, uint64_t width, uint64_t n_tok, const char *msg) {
    if (n_tok && (!p || !aligned16(p) || stride % 8 || stride < width)) return invalid(h, msg);
    return NETKV_OK;
}

}  // namespace blockdev
