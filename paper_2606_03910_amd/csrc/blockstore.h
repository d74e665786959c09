// What writes rows into the cache's blocks: which workgroup takes which block,
// the rounding to 8 bits, and the values' way through LDS.
#pragma once

#include "blockdev.h"

namespace blockdev {

// The `task`-th of the sequences' consecutive shares, where count(h) is how
// many sequence h has: found by the whole workgroup of THREADS, 256 sequences at
// a time or as many as it has threads.
// Returns the sequence (n_seq if there is none) and the share in `rest`.  Those
// that count have less than 2^32 (store_groups, read_groups).  Every workgroup
// goes through the sequences before its own, so a call's time grows with their
// square from some thousands on: single tokens of 1,024, 4,096, 16,384 and 65,535
// sequences (8 heads of 128 dimensions) are stored in 66 us, 399 us, 4.3 ms and
// 58 ms and read in 23 us, 164 us, 2.0 ms and 26 ms.
template <int THREADS, typename F>
__device__ inline uint32_t locate(const Kv &a, uint32_t task, F count, uint32_t *rest) {
    constexpr uint32_t kFalls = ~0u;      // a sequence whose rows are not good: every sum after it stays this
    constexpr int kEach = THREADS < kThreads ? THREADS : kThreads, kGroups = kEach / 64;
    __shared__ uint32_t sums[kGroups], found, left, ends[16];
    const int lane = threadIdx.x & 63, w = (threadIdx.x >> 6) & (kGroups - 1);
    const bool in = threadIdx.x < kEach;
    if (threadIdx.x == 0) found = a.n_seq;
    uint32_t before = 0;
    auto look = [&](uint32_t s, uint32_t x) {              // whether that was the last chunk to look at
        uint32_t y = x;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t z = __shfl_up(y, d, 64);
            if (lane >= d) y = __builtin_elementwise_add_sat(y, z);
        }
        if (in && lane == 63) sums[w] = y;
        __syncthreads();
        uint32_t base = before;
        for (int v = 0; v < kGroups; ++v) {
            if (v < w) base = __builtin_elementwise_add_sat(base, sums[v]);
            before = __builtin_elementwise_add_sat(before, sums[v]);
        }
        y = __builtin_elementwise_add_sat(y, base);   // inclusive
        if (in && x && task >= y - x && task < y) {
            found = s;
            left = task - (y - x);
        }
        __syncthreads();
        return found < a.n_seq || task < before;
    };
    uint32_t named = 0;
    for (bool again = false;; again = true) {
        for (uint32_t s0 = 0; s0 < a.n_seq; s0 += kEach) {
            const uint32_t s = s0 + threadIdx.x;
            const bool is = in && s < a.n_seq;
            uint32_t x = 0;
            if (is) {
                const Head h = seq_head(a, s);
                x = h.rows_ok ? count(h) : again ? 0u : kFalls;
            }
            if (__builtin_expect(again, 0)) {
                const uint32_t earlier = rows_before(is ? rows_end(a, s) : 0u, named, ends);
                if (x && a.off[s] < earlier) x = 0;
            }
            if (look(s, x)) break;
        }
        if (__builtin_expect(before != kFalls, 1)) break;
        __syncthreads();
        if (threadIdx.x == 0) found = a.n_seq;
        before = 0;
    }
    __syncthreads();
    *rest = left;
    return found;
}

struct MoveArgs {
    Kv kv;
    const void *k, *v;            // store: the new rows; read: the outputs
    uint64_t k_stride, v_stride;
};

// Reports the sequences that a store or a read leaves out: by the first head's workgroups, `tasks` of them.
__device__ inline void report_bad(const Kv &kv, uint32_t task, uint32_t tasks) {
    for (uint32_t s = task * blockDim.x + threadIdx.x; s < kv.n_seq; s += tasks * blockDim.x) {
        const Head h = seq_head(kv, s);
        if (!h.ok || h.n > h.ctx) report(kv);
    }
}

// The smallest power of two s >= 2^-126 with amax <= 448 s: 448 = 1.75 * 2^8.
__device__ inline float scale_for(float amax) {
    const uint32_t b = __float_as_uint(amax);
    int e = (int)(b >> 23) - 127;
    if (e < -126) return 1.17549435e-38f;
    e += (b & 0x7FFFFFu) <= 0x600000u ? -8 : -7;
    e = e < -126 ? -126 : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

__device__ inline float to_f32(uint32_t bits16, bool half) {
    return half ? (float)__builtin_bit_cast(_Float16, (uint16_t)bits16) : __uint_as_float(bits16 << 16);
}

// Four values to e4m3, nearest even; what is not finite becomes NaN.
__device__ inline uint32_t narrow4(const float *x, float inv) {
    int r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, r, true);
    uint32_t y = (uint32_t)r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(x[i]) < INFINITY)) y = (y & ~(0xFFu << (8 * i))) | (0x7Fu << (8 * i));
    return y;
}

// Four finite 16-bit values over a power of two to e4m3, nearest even.
__device__ inline uint32_t narrow4_finite(uint32_t a, uint32_t b, float scale, bool half) {
    i16x2 r = {0, 0};
    if (half) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2, a), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2, b), scale, true);
    } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, a), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, b), scale, true);
    }
    return __builtin_bit_cast(uint32_t, r);
}

// Four e4m3 bytes under another scale (ratio <= 1, a power of two).
__device__ inline uint32_t rescale4(uint32_t x, float ratio) {
    const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false);
    const f16x2 q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true);
    const float y[4] = {(float)p[0], (float)p[1], (float)q[0], (float)q[1]};
    return narrow4(y, ratio);
}

// Four dwords of four bytes each, turned.
__device__ inline void turn4(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d) {
    const uint32_t t0 = __builtin_amdgcn_perm(b, a, 0x05010400u), t1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t u0 = __builtin_amdgcn_perm(d, c, 0x05010400u), u1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    a = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
    b = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
    c = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
    d = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

// Where the new rows of one block go.
struct Place {
    uint32_t seq, page;
    uint32_t p0, p1;              // slots [p0, p1) are new
    uint32_t token;               // of slot p0 in its sequence
    uint64_t row0;                // its row
};

// The task-th block that the rows touch; false if there is none, or its page
// is not one.
template <int THREADS>
__device__ inline bool find_place(const Kv &kv, uint32_t task, Place &p) {
    uint32_t rest;
    const uint32_t bt = 1u << kv.btl;
    const uint32_t s = locate<THREADS>(kv, task, [&](const Head &h) { return stored_blocks(kv, h); }, &rest);
    if (s >= kv.n_seq) return false;
    const Head hd = seq_head(kv, s);
    const uint32_t start = hd.ctx - hd.n;                     // the first new token
    const uint32_t blk = (start >> kv.btl) + rest;
    p.seq = s;
    p.page = kv.pages[(uint64_t)s * kv.max_pages + blk];
    if (p.page >= kv.n_pages) {
        if (threadIdx.x == 0) report(kv);
        return false;
    }
    p.p0 = max(start, blk << kv.btl) - (blk << kv.btl);
    p.p1 = min(hd.ctx - (blk << kv.btl), bt);
    p.token = (blk << kv.btl) + p.p0;
    p.row0 = hd.row0 + (p.token - start);
    return true;
}

// One workgroup quantises the keys (blockIdx.z = 0) or values of one head
// that a call brings to one block.  The block's scale is the smallest power of
// two that holds them, or the present one if the block was begun with a larger
// one; where it grows, what the block holds is brought under the new scale
// (exact but for values that become subnormal).  What fits the workgroup's
// registers is read once, for the largest value and for the quantisation.
// Values are turned through LDS: written byte by byte from the rows they came
// in, a 512-token block took three times as long.  Bound by memory: 16 prompts
// of up to 16,384 tokens, 8 heads of 128 dimensions (537 MB in, 269 MB out)
// take 228 us, 3.5 TB/s; 64 single tokens 8 us, latency.
template <int D, int THREADS>
__device__ __forceinline__ void store_block(const MoveArgs &a, bool half, uint32_t task, uint32_t h, bool vals) {
    constexpr int kEach = 8;                                  // 16-byte pieces a thread keeps
    constexpr uint32_t kPass = THREADS * kEach * 8 / D;       // tokens that the workgroup keeps
    constexpr uint32_t kPitch = D / 4 + 1;
    __shared__ uint32_t red[THREADS / 64];
    __shared__ uint32_t rows[(kPass + 16) * kPitch];          // quantised values by token
    const Kv &kv = a.kv;
    const uint32_t bt = 1u << kv.btl;
    Place pl;
    if (!find_place<THREADS>(kv, task, pl)) return;
    const uint32_t page = pl.page, p0 = pl.p0, p1 = pl.p1;
    const uint64_t row0 = pl.row0;
    const uint16_t *src = (const uint16_t *)(vals ? a.v : a.k);
    const uint64_t stride = vals ? a.v_stride : a.k_stride;
    const uint64_t at = (uint64_t)page * kv.hk + h;
    uint8_t *dst = (vals ? kv.v : kv.k) + at * head_bytes(kv, D);
    float *scale = (vals ? kv.vs : kv.ks) + at;
    const uint32_t pieces = (p1 - p0) * (D / 8);

    u32x4 x[kEach];
    const uint16_t *own = src + (row0 + threadIdx.x / (D / 8)) * stride + (uint64_t)h * D + threadIdx.x % (D / 8) * 8;
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t e = base + i * THREADS;
            x[i] = u32x4{0, 0, 0, 0};
            if (e + threadIdx.x < pieces) x[i] = *(const u32x4 *)(own + e / (D / 8) * stride);
        }
    };
    // the largest of the values' bits without their signs, which order as the
    // values do; infinities and NaN come last, and make a second look necessary
    const uint32_t not_finite = half ? 0x7C00u : 0x7F80u;
    auto largest = [&](bool all) {
        u16x2 top = {0, 0};
        for (uint32_t base = 0; base < pieces; base += THREADS * kEach) {
            if (all || pieces > THREADS * kEach) load(base);
#pragma unroll
            for (int i = 0; i < kEach; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u16x2 z = __builtin_bit_cast(u16x2, x[i][j] & 0x7FFF7FFFu);
                    if (!all) {
                        z[0] = z[0] < not_finite ? z[0] : (uint16_t)0;
                        z[1] = z[1] < not_finite ? z[1] : (uint16_t)0;
                    }
                    top = __builtin_elementwise_max(top, z);
                }
        }
        uint32_t t = top[0] > top[1] ? top[0] : top[1];
        for (int d = 32; d; d >>= 1) t = max(t, (uint32_t)__shfl_xor(t, d, 64));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = t;
        __syncthreads();
        for (int i = 0; i < THREADS / 64; ++i) t = max(t, red[i]);
        return t;
    };
    uint32_t top = largest(true);
    const bool finite = top < not_finite;
    if (!finite) top = largest(false);
    const float amax = to_f32(top, half);
    float sc = scale_for(amax);
    if (p0) {
        const float was = *scale;
        sc = was > sc ? was : sc;
        if (was != sc) {
            const float ratio = was / sc;
            if (!vals) {
                for (uint32_t i = threadIdx.x; i < p0 * (D / 4); i += THREADS) ((uint32_t *)dst)[i] = rescale4(((uint32_t *)dst)[i], ratio);
            } else {
                // by 4 tokens of a dimension; a group that the new tokens share with old ones by bytes
                const uint32_t tile = min(bt, kStep), quads = (p0 + 3) / 4;
                for (uint32_t i = threadIdx.x; i < quads * D; i += THREADS) {
                    const uint32_t d = i % D, tok = i / D * 4;
                    uint8_t *p = dst + (uint64_t)(tok & ~(tile - 1)) * D + d * tile + (tok & (tile - 1));
                    const uint32_t y = rescale4(*(uint32_t *)p, ratio);
                    if (tok + 4 <= p0)
                        *(uint32_t *)p = y;
                    else
                        for (uint32_t j = 0; tok + j < p0; ++j) p[j] = (uint8_t)(y >> (8 * j));
                }
            }
        }
    }
    __syncthreads();   // every thread has read the old scale
    if (threadIdx.x == 0) *scale = sc;
    const float inv = 1.0f / sc;
    // the narrowing instruction takes a scale's power of two alone
    const bool plain = finite && (__float_as_uint(sc) & 0x7FFFFFu) == 0;
    const uint32_t tile = min(bt, kStep);
    if (pieces > THREADS * kEach) load(0);
    for (uint32_t base = 0;;) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t e = base + i * THREADS + threadIdx.x;
            u32x2 y = {0, 0};
            if (e < pieces) {
                if (plain) {
                    y = u32x2{narrow4_finite(x[i][0], x[i][1], sc, half), narrow4_finite(x[i][2], x[i][3], sc, half)};
                } else {
                    float z[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        z[2 * j] = to_f32(x[i][j] & 0xFFFFu, half);
                        z[2 * j + 1] = to_f32(x[i][j] >> 16, half);
                    }
                    y = u32x2{narrow4(z, inv), narrow4(z + 4, inv)};
                }
            }
            const uint32_t tok = p0 + e / (D / 8), d = e % (D / 8) * 8;
            if (e >= pieces) continue;
            if (!vals) {
                *(u32x2 *)(dst + (uint64_t)tok * D + d) = y;
            } else {
                uint32_t *q = rows + (tok - ((p0 + base / (D / 8)) & ~15u)) * kPitch + d / 4;
                q[0] = y[0];
                q[1] = y[1];
            }
        }
        if (vals) {
            // four dimensions of 16 tokens a thread; groups that the call fills
            // whole are written whole
            __syncthreads();
            const uint32_t t0 = p0 + base / (D / 8), t1 = min(p1, t0 + kPass), g0 = t0 & ~15u;
            for (uint32_t i = threadIdx.x; i < (t1 - g0 + 63) / 64 * D; i += THREADS) {
                // lanes: four groups, then the dimensions
                const uint32_t dq = i / 4 % (D / 4), tg = i % 4 + i / D * 4, tok = g0 + 16 * tg;
                if (tok >= t1) continue;
                const uint32_t *q = rows + 16 * tg * kPitch + dq;
                uint8_t *to = dst + (uint64_t)(tok & ~(tile - 1)) * D + (uint64_t)dq * 4 * tile + (tok & (tile - 1));
                u32x4 o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t x0 = q[(4 * j) * kPitch], x1 = q[(4 * j + 1) * kPitch], x2 = q[(4 * j + 2) * kPitch], x3 = q[(4 * j + 3) * kPitch];
                    turn4(x0, x1, x2, x3);
                    o[0][j] = x0;
                    o[1][j] = x1;
                    o[2][j] = x2;
                    o[3][j] = x3;
                }
                if (tok >= t0 && tok + 16 <= t1) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) *(u32x4 *)(to + j * tile) = o[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e)
                            if (tok + e >= t0 && tok + e < t1) to[j * tile + e] = (uint8_t)(o[j][e >> 2] >> (8 * (e & 3)));
                }
            }
            __syncthreads();
        }
        base += THREADS * kEach;
        if (base >= pieces) break;
        load(base);
    }
}

}  // namespace blockdev
