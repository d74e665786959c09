// Rotary positions on MI355X (gfx950): rows of heads rotated, and a step's
// queries, keys and values taken into the block cache with the rotation on the
// way.
//
//   rotate_kernel  -- rows of heads, each pair turned by its position's angle.
//   append_kernel  -- the sequences' new queries rotated, their keys rotated and
//                     quantised into their blocks, their values quantised.
//
// A pair (a, b) of a head becomes (a cos - b sin, b cos + a sin); the cosines
// and sines come from a table with a row for every position, and a pair's
// position is that of its axis.  The work is in units of 16 elements: eight
// pairs, in two pieces of eight elements, which lie half of the rotated
// elements apart or, interleaved, side by side.

#include <hip/hip_runtime.h>

#include "blockstore.h"
#include "ropeplan.h"

namespace {

using namespace blockdev;
using namespace ropeplan;

// What a rotation is made of, as the kernels see it.
struct Turn {
    const float *table;               // [n_pos][2 pairs]: cosines, sines
    const uint32_t *pos;              // [axis][row]; null: a row's place in its sequence
    uint64_t pos_stride;
    uint32_t n_pos, pairs, n_axes;
    uint32_t interleaved;
    uint32_t sign;                    // flips the sines' signs: the transposed rotation
    uint32_t axes[kMaxPairs / 16];    // two bits a pair
    uint32_t *err;
};

// cos and sin of a unit's eight pairs
struct Angles {
    float c[8], s[8];
};

// Positions past the table make their pairs NaN.
__device__ inline void load_angles(const Turn &t, uint64_t row, uint32_t place, uint32_t u, Angles &a) {
    const uint32_t which = t.axes[u >> 1] >> (16 * (u & 1)) & 0xFFFFu;
    const uint32_t first = which & 3;
    bool bad = false;
    if (which == first * 0x5555u) {
        const uint32_t p = t.pos ? t.pos[first * t.pos_stride + row] : place;
        bad = p >= t.n_pos;
        const float *at = t.table + (uint64_t)(bad ? 0u : p) * 2 * t.pairs + 8 * u;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const f32x4 x = *(const f32x4 *)(at + i), y = *(const f32x4 *)(at + t.pairs + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a.c[i + j] = bad ? NAN : x[j];
                a.s[i + j] = bad ? NAN : y[j];
            }
        }
    } else {
        // each axis's position and row once, then a look into them for each pair
        uint32_t at[4], outside = 0;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            uint32_t p = place;
            if (t.pos) p = t.pos[min(i, t.n_axes - 1) * t.pos_stride + row];
            const bool out = p >= t.n_pos;
            outside |= out ? 1u << i : 0u;
            at[i] = out ? 0u : p;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t k = which >> (2 * i) & 3, p = k & 2 ? (k & 1 ? at[3] : at[2]) : (k & 1 ? at[1] : at[0]);
            const float *x = t.table + (uint64_t)p * 2 * t.pairs + 8 * u + i;
            const bool out = outside >> k & 1;
            a.c[i] = x[0];
            a.s[i] = x[t.pairs];
            if (out) a.c[i] = a.s[i] = NAN;
            bad |= out;
        }
    }
    if (bad) atomicOr(t.err, kErrBlockBit);
#pragma unroll
    for (int i = 0; i < 8; ++i) a.s[i] = __uint_as_float(__float_as_uint(a.s[i]) ^ t.sign);
}

// The 16 elements of a unit's two pieces as eight pairs, and back.
__device__ inline uint32_t half_of(const u32x4 &x, int i) { return x[i / 2] >> (16 * (i & 1)) & 0xFFFFu; }

struct Pairs {
    float a[8], b[8];
};

__device__ inline void to_pairs(const u32x4 &lo, const u32x4 &hi, bool half, bool interleaved, Pairs &p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const u32x4 &x = i < 4 ? lo : hi;
        const uint32_t a = interleaved ? x[i & 3] & 0xFFFFu : half_of(lo, i), b = interleaved ? x[i & 3] >> 16 : half_of(hi, i);
        p.a[i] = to_f32(a, half);
        p.b[i] = to_f32(b, half);
    }
}

__device__ inline uint32_t pack16(float x, float y, bool half) {
    const f32x2 p = {x, y};
    return half ? __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2)) : __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
}

// a c - b s of 16-bit a, b to 1.5 units of fp32's last place, also where the
// products cancel: what the first product loses comes back.  b s is not past
// fp32's largest.
__device__ inline float cross(float a, float c, float b, float s) {
    const float w = b * s, e = fmaf(b, s, -w), t = fmaf(a, c, -w);
    return e == e ? t - e : t;        // w not finite
}

// The same for any b s: where it is, from 64 bits, in which the products are exact.
__device__ inline float cross_any(float a, float c, float b, float s) {
    const float y = cross(a, c, b, s);
    return y == y ? y : (float)fma((double)a, (double)c, -((double)b * (double)s));
}

// A double to fp32, to odd where it is not exact.
__device__ inline float odd_f32(double x) {
    const float f = (float)x;
    uint32_t u = __float_as_uint(f);
    if ((double)f != x) {
        if (fabs((double)f) > fabs(x)) --u;
        u |= 1;
    }
    return __uint_as_float(u);
}

// A double to bfloat16's bits, to odd where it is not exact: what is rounded from
// there to the 4 bits of e4m3 is as if rounded once, and what is compared with
// 448 times a power of two comes out as the double would.
__device__ inline uint32_t to_odd(double x) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t hi = (uint32_t)(bits >> 32), rest = (hi & 0x1FFFu) | (uint32_t)bits;
    uint32_t u = (hi >> 13 & 0x3FFFFu) - (896u << 7);         // exponent and seven bits, by bfloat16's exponents
    if (u - (1u << 7) >= 254u << 7) {                         // 0, or outside its normal numbers
        const uint32_t v = __float_as_uint(odd_f32(x));
        return v >> 16 | (uint32_t)((v & 0xFFFFu) != 0);
    }
    return u | min(rest, 1u) | (hi >> 16 & 0x8000u);
}

// The largest key that a scale holds, 448 * 2^127; past it a key is as one that
// is not finite.
constexpr double kMostKey = 448.0 * 0x1p127;

// The upper half of a key's bits without its sign, to odd; 0 for one that no scale holds.
__device__ inline uint32_t upper_odd(double x) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, fabs(x));
    return fabs(x) <= kMostKey ? (uint32_t)(bits >> 32) | (uint32_t)((uint32_t)bits != 0) : 0u;
}

// scale_for (blockstore.h) of such a one.
__device__ inline float scale_for_upper(uint32_t most) {
    const int e = (int)(most >> 20) - 1023 + ((most & 0xFFFFFu) <= 0xC0000u ? -8 : -7);
    return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

// ------------------------------------------------------------------ rows

struct RowArgs {
    Turn turn;
    const uint16_t *x;
    uint16_t *out;
    uint64_t x_stride, out_stride;
    uint32_t heads, dim;
    uint32_t units;                   // a head's: those that turn, and those copied
    uint32_t half;
};

// A unit's two pieces turned, in their place.
__device__ inline void turn_unit(const Turn &t, bool half, const Angles &g, u32x4 &lo, u32x4 &hi) {
    Pairs e;
    to_pairs(lo, hi, half, t.interleaved, e);
    float y[8], z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        y[j] = cross(e.a[j], g.c[j], e.b[j], g.s[j]);
        z[j] = cross(e.b[j], g.c[j], e.a[j], -g.s[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (t.interleaved) {
            lo[j] = pack16(y[j], z[j], half);
            hi[j] = pack16(y[4 + j], z[4 + j], half);
        } else {
            lo[j] = pack16(y[2 * j], y[2 * j + 1], half);
            hi[j] = pack16(z[2 * j], z[2 * j + 1], half);
        }
    }
}

// The largest of a unit's sines.  Up to 1 no product of it is past fp32's largest.
__device__ inline float most_sine(const Angles &g) {
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x = fmaxf(x, fabsf(g.s[i]));
    return x;
}

// Whether one may be, of the heads that a thread has.
__device__ inline bool past_fp32(const u32x4 (&lo)[kHeadsEach], const u32x4 (&hi)[kHeadsEach], bool half, float sine) {
    u16x2 top = {0, 0};
#pragma unroll
    for (uint32_t i = 0; i < 4 * kHeadsEach; ++i) {
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, lo[i / 4][i % 4] & 0x7FFF7FFFu));
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, hi[i / 4][i % 4] & 0x7FFF7FFFu));
    }
    return !(to_f32(max(top[0], top[1]), half) * sine < INFINITY);
}

// A unit of `heads` heads turned whatever its products, an element after another
// (slower, but in no more registers than turn_unit).
__device__ inline void turn_any(const RowArgs &r, const Angles &g, const Unit &p, const uint16_t *x, uint16_t *out, uint32_t heads) {
#pragma unroll 1
    for (uint32_t j = 0; j < 8 * heads; ++j) {
        const uint32_t k = j & 7, at = j / 8 * r.dim;
        const uint32_t ia = at + p.lo + (r.turn.interleaved ? 2 * k : k), ib = r.turn.interleaved ? ia + 1 : at + p.hi + k;
        float c = g.c[0], s = g.s[0];
#pragma unroll
        for (uint32_t i = 1; i < 8; ++i) {
            c = k == i ? g.c[i] : c;
            s = k == i ? g.s[i] : s;
        }
        const float ea = to_f32(x[ia], r.half), eb = to_f32(x[ib], r.half);
        const uint32_t y = pack16(cross_any(ea, c, eb, s), cross_any(eb, c, ea, -s), r.half);
        out[ia] = (uint16_t)y;
        out[ib] = (uint16_t)(y >> 16);
    }
}

// Rows [row, row + n) of the arrays; a row's position is `place` and on if the
// turn has none of its own.
__device__ inline void rotate_rows(const RowArgs &a, uint64_t row, uint32_t n, uint32_t place) {
    const uint32_t each = (a.heads + kHeadsEach - 1) / kHeadsEach * a.units;
    for (uint32_t i = threadIdx.x; i < n * each; i += blockDim.x) {
        const uint32_t t = i / each, u = i % each % a.units, h0 = i % each / a.units * kHeadsEach;
        const uint32_t last = min(kHeadsEach, a.heads - h0) - 1;
        const Unit p = unit_of(u, a.turn.pairs, a.turn.interleaved, a.dim);
        const uint16_t *x = a.x + (row + t) * a.x_stride + (uint64_t)h0 * a.dim;
        uint16_t *out = a.out + (row + t) * a.out_stride + (uint64_t)h0 * a.dim;
        u32x4 xl[kHeadsEach], xh[kHeadsEach];
#pragma unroll
        for (uint32_t j = 0; j < kHeadsEach; ++j) {
            const uint16_t *from = x + min(j, last) * a.dim;
            xl[j] = *(const u32x4 *)(from + p.lo);
            xh[j] = *(const u32x4 *)(from + (p.both ? p.hi : p.lo));
        }
        Angles g;
        if (p.turns) {
            load_angles(a.turn, row + t, place + t, u, g);
            const float sine = most_sine(g);
            if (__builtin_expect(sine > 1.0f && past_fp32(xl, xh, a.half, sine), 0)) {
                turn_any(a, g, p, x, out, last + 1);
                continue;
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < kHeadsEach; ++j) {
            if (j > last) continue;
            uint16_t *to = out + j * a.dim;
            if (p.turns) turn_unit(a.turn, a.half, g, xl[j], xh[j]);
            *(u32x4 *)(to + p.lo) = xl[j];
            if (p.both) *(u32x4 *)(to + p.hi) = xh[j];
        }
    }
}

// Bound by memory: 16,384 rows of 32 heads of 128 elements of which 64 turn (269 MB)
// 59 us, 4.6 TB/s; 10,007 of 16 heads of 80 on two axes (51 MB) 15.6 us: 834
// workgroups at once, each with one chain of positions, table rows and rows, and
// nearly every wavefront with a unit whose pairs are on both axes.
__global__ __launch_bounds__(kThreads) void rotate_kernel(RowArgs a, uint32_t rows, uint32_t chunk) {
    const uint32_t row = blockIdx.x * chunk;
    rotate_rows(a, row, min(chunk, rows - row), 0);
}

// ------------------------------------------------------------------ append

struct AppendArgs {
    MoveArgs move;
    RowArgs rows;                     // the queries
    uint32_t chunk;                   // of rows that a workgroup rotates
    uint32_t row_tasks, store_tasks;  // workgroups for the queries, for each head's keys and values
};

// One workgroup rotates the keys of one head that a call brings to one block
// and quantises them, as store_block does values.  A rotated key is computed in
// 64 bits, where the products of 16-bit elements and 32-bit cosines are exact,
// and rounded once, to 8 bits: in fp32 one in some hundred thousand would
// come out a step off, and a block's scale by a factor of two.  Between the
// largest value and the rounding it is held in 16 bits, to odd (to_odd), where
// these have two bits more than the block's 8: not past fp32's largest, nor where
// the block's steps (from 2^-9 of its scale) near bfloat16's smallest, 2^-133.
// Such blocks are computed once more from 64 bits.  The products in 64 bits and
// the roundings to odd bound it where calls are large: 131,214 rows of 8 heads of
// 128 dimensions 220 us, of which the memory needs 80.
template <int D, int THREADS, int kEach>
__device__ __forceinline__ void append_keys(const AppendArgs &g, uint32_t task, uint32_t h) {
    constexpr uint32_t kUnits = D / 16;                       // of a token; a thread keeps kEach
    __shared__ uint32_t red[2][THREADS / 64];
    const Kv &kv = g.move.kv;
    const Turn &turn = g.rows.turn;
    Place pl;
    if (!find_place<THREADS>(kv, task, pl)) return;
    const uint64_t at = (uint64_t)pl.page * kv.hk + h;
    uint8_t *dst = kv.k + at * head_bytes(kv, D);
    const uint16_t *src = (const uint16_t *)g.move.k + (uint64_t)h * D;
    const uint32_t units = (pl.p1 - pl.p0) * kUnits, half = g.rows.half;

    u32x4 x[kEach][2];
    auto unit = [&](uint32_t e) { return unit_of(e % kUnits, turn.pairs, turn.interleaved, D); };
    // a unit's eight pairs, turned
    auto turned = [&](uint32_t e, const u32x4 (&x)[2], auto take) {
        const uint32_t t = e / kUnits, u = e % kUnits;
        Angles a;
        Pairs p;
        load_angles(turn, pl.row0 + t, pl.token + t, u, a);
        to_pairs(x[0], x[1], half, turn.interleaved, p);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double c = a.c[j], s = a.s[j], pa = p.a[j], pb = p.b[j];
            take(j, fma(pa, c, -(pb * s)), fma(pb, c, pa * s));
        }
    };
    auto load = [&](uint32_t base) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t e = base + i * THREADS + threadIdx.x;
            x[i][0] = x[i][1] = u32x4{0, 0, 0, 0};
            if (e >= units) continue;
            const uint16_t *p = src + (pl.row0 + e / kUnits) * g.move.k_stride;
            const Unit w = unit(e);
            x[i][0] = *(const u32x4 *)(p + w.lo);
            x[i][1] = *(const u32x4 *)(p + w.hi);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t e = base + i * THREADS + threadIdx.x;
            if (e >= units) continue;
            if (e % kUnits < turn.pairs / 8) {
                uint32_t y[8], z[8];
                turned(e, x[i], [&](int j, double p, double q) {
                    y[j] = to_odd(p);
                    z[j] = to_odd(q);
                });
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[i][0][j] = turn.interleaved ? y[j] | z[j] << 16 : y[2 * j] | y[2 * j + 1] << 16;
                    x[i][1][j] = turn.interleaved ? y[4 + j] | z[4 + j] << 16 : z[2 * j] | z[2 * j + 1] << 16;
                }
            } else if (half) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][q][j] = to_odd(to_f32(x[i][q][j] & 0xFFFFu, true)) | to_odd(to_f32(x[i][q][j] >> 16, true)) << 16;
            }
        }
    };
    // the largest of the values' bits without their signs, and of the finite ones'
    constexpr uint32_t kNotFinite = 0x7F80u;
    u16x2 all = {0, 0}, some = {0, 0};
    for (uint32_t base = 0; base < units; base += THREADS * kEach) {
        load(base);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u16x2 z = __builtin_bit_cast(u16x2, x[i][q][j] & 0x7FFF7FFFu);
                    all = __builtin_elementwise_max(all, z);
                    some = __builtin_elementwise_max(some, u16x2{z[0] < kNotFinite ? z[0] : (uint16_t)0, z[1] < kNotFinite ? z[1] : (uint16_t)0});
                }
    }
    uint32_t top = max(some[0], some[1]), any = max(all[0], all[1]);
    for (int d = 32; d; d >>= 1) {
        top = max(top, (uint32_t)__shfl_xor(top, d, 64));
        any = max(any, (uint32_t)__shfl_xor(any, d, 64));
    }
    if ((threadIdx.x & 63) == 0) {
        red[0][threadIdx.x >> 6] = top;
        red[1][threadIdx.x >> 6] = any;
    }
    __syncthreads();
    for (int i = 0; i < THREADS / 64; ++i) {
        top = max(top, red[0][i]);
        any = max(any, red[1][i]);
    }

    float *scale = kv.ks + at;
    const float was = pl.p0 ? *scale : 0.0f;
    auto or_present = [&](float x) { return was > x ? was : x; };
    float sc = or_present(scale_for(__uint_as_float(top << 16)));
    // the new scale, and what the block holds under it
    auto rescale = [&]() {
        if (pl.p0 && was != sc) {
            const float ratio = was / sc;
            for (uint32_t i = threadIdx.x; i < pl.p0 * (D / 4); i += THREADS) ((uint32_t *)dst)[i] = rescale4(((uint32_t *)dst)[i], ratio);
        }
        __syncthreads();   // every thread has read the old scale
        if (threadIdx.x == 0) *scale = sc;
    };
    // Once more from 64 bits: keys past fp32's largest, which are held as
    // bfloat16's largest; a scale that is no power of two, from another program,
    // over which what is held would be rounded twice; scales under which half of
    // the smallest step is bfloat16's smallest (2^-133 under 2^-123) or less.
    const bool far = top == kNotFinite - 1;
    if (__builtin_expect(far || (top && sc < 0x1p-122f) || (__float_as_uint(sc) & 0x7FFFFFu) != 0, 0)) {
        auto in_64_bits = [&](uint32_t e, const Unit &w, auto take) {
            const uint16_t *from = src + (pl.row0 + e / kUnits) * g.move.k_stride;
            const u32x4 v[2] = {*(const u32x4 *)(from + w.lo), *(const u32x4 *)(from + w.hi)};
            if (w.turns) {
                turned(e, v, [&](int j, double p, double q) {
                    take(turn.interleaved ? 2 * j : j, p);
                    take(turn.interleaved ? 2 * j + 1 : 8 + j, q);
                });
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) take(j, (double)to_f32(half_of(v[j / 8], j % 8), half));
            }
        };
        if (far) {
            uint32_t most = 0;
#pragma unroll 1
            for (uint32_t e = threadIdx.x; e < units; e += THREADS)
                in_64_bits(e, unit(e), [&](int, double x) { most = max(most, upper_odd(x)); });
            for (int d = 32; d; d >>= 1) most = max(most, (uint32_t)__shfl_xor(most, d, 64));
            __syncthreads();   // every thread has read red
            if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = most;
            __syncthreads();
            for (int i = 0; i < THREADS / 64; ++i) most = max(most, red[0][i]);
            sc = or_present(scale_for_upper(most));
        }
        rescale();
#pragma unroll 1
        for (uint32_t e = threadIdx.x; e < units; e += THREADS) {
            const Unit w = unit(e);
            float y[16];
            in_64_bits(e, w, [&](int j, double x) { y[j] = fabs(x) <= kMostKey ? odd_f32(x / (double)sc) : NAN; });
            uint8_t *p = dst + (uint64_t)(pl.p0 + e / kUnits) * D;
            *(u32x2 *)(p + w.lo) = u32x2{narrow4(y, 1.0f), narrow4(y + 4, 1.0f)};
            *(u32x2 *)(p + w.hi) = u32x2{narrow4(y + 8, 1.0f), narrow4(y + 12, 1.0f)};
        }
        return;
    }
    rescale();
    const float inv = 1.0f / sc;
    const bool plain = any < kNotFinite;
    for (uint32_t base = 0; base < units; base += THREADS * kEach) {
        if (units > THREADS * kEach) load(base);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t e = base + i * THREADS + threadIdx.x;
            if (e >= units) continue;
            const Unit w = unit(e);
            uint8_t *p = dst + (uint64_t)(pl.p0 + e / kUnits) * D;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const u32x4 v = x[i][q];
                u32x2 y;
                if (plain) {
                    y = u32x2{narrow4_finite(v[0], v[1], sc, false), narrow4_finite(v[2], v[3], sc, false)};
                } else {
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = to_f32(half_of(v, j), false);
                    y = u32x2{narrow4(f, inv), narrow4(f + 4, inv)};
                }
                *(u32x2 *)(p + (q ? w.hi : w.lo)) = y;
            }
        }
    }
}

// The queries of up to `chunk` rows of one sequence.
template <int THREADS>
__device__ inline void append_queries(const AppendArgs &a, uint32_t task) {
    const Kv &kv = a.move.kv;
    uint32_t rest;
    const uint32_t s = locate<THREADS>(kv, task, [&](const Head &h) { return row_chunks(h, a.chunk); }, &rest);
    if (s >= kv.n_seq) return;
    const Head h = seq_head(kv, s);
    const uint32_t t = rest * a.chunk;
    rotate_rows(a.rows, h.row0 + t, min(a.chunk, h.n - t), h.ctx - h.n + t);
}

// All of a small call: bound by the chain of lengths, pages, rows and the
// largest of them.  64 single tokens of 64 and 8 heads of 128 dimensions 13 us, 10,231 rows
// of 15 and 5 heads of 64 dimensions in blocks of 32 (64 MB) 24 us, 2.7 TB/s.
template <int D, int THREADS>
__global__ __launch_bounds__(THREADS) void append_kernel(AppendArgs a) {
    if (blockIdx.x < a.row_tasks) {
        append_queries<THREADS>(a, blockIdx.x);
        return;
    }
    const uint32_t i = blockIdx.x - a.row_tasks, task = i % a.store_tasks, r = i / a.store_tasks, h = r % a.move.kv.hk;
    const bool vals = r >= a.move.kv.hk;
    if (r == 0) report_bad(a.move.kv, task, a.store_tasks);
    if (vals)
        store_block<D, THREADS>(a.move, a.rows.half, task, h, true);
    else
        append_keys<D, THREADS, 4>(a, task, h);
}

// A large call's queries and keys: the keys' arithmetic beside the queries'
// traffic, so their workgroups alternate.  131,214 rows of 64 and 8 heads of 128
// dimensions, us: queries alone 880 (4.3 GB, 4.9 TB/s), keys alone 220 (0.4 GB),
// together 1,000, 4.7 TB/s.
template <int D>
__global__ __launch_bounds__(512, 4) void append_large_kernel(AppendArgs a) {
    const uint32_t keys = a.store_tasks * a.move.kv.hk, all = a.row_tasks + keys;
    const uint32_t k = (uint32_t)((uint64_t)blockIdx.x * keys / all);
    if ((uint32_t)((uint64_t)(blockIdx.x + 1) * keys / all) == k) {
        append_queries<512>(a, blockIdx.x - k);
        return;
    }
    const uint32_t task = k % a.store_tasks, h = k / a.store_tasks;
    if (h == 0) report_bad(a.move.kv, task, a.store_tasks);
    append_keys<D, 512, 8>(a, task, h);
}

// A large call's values, in a launch of its own with store_kernel's 1,024
// threads: 131,214 rows of 8 heads of 128 dimensions (403 MB) 101 us, 4.0 TB/s.
template <int D>
__global__ __launch_bounds__(1024, 8) void append_values_kernel(AppendArgs a) {
    store_block<D, 1024>(a.move, a.rows.half, blockIdx.x, blockIdx.y, true);
}

// ------------------------------------------------------------------ host

netkv_status make_turn(netkv_handle h, const netkv_rope_t *rope, uint32_t head_dim, const uint32_t *pos, uint64_t pos_stride,
                       uint64_t rows, bool need_pos, Turn &t) {
    if (const char *why = rope_error(rope, head_dim, pos, pos_stride, rows, need_pos)) return invalid(h, why);
    t.table = rope->table;
    t.pos = pos;
    t.pos_stride = pos_stride;
    t.n_pos = rope->n_pos;
    t.pairs = rope->rot_dim / 2;
    t.n_axes = rope->n_axes;
    t.interleaved = rope->interleaved;
    for (uint32_t i = 0; rope->axis && i < t.pairs; ++i) t.axes[i / 16] |= (uint32_t)rope->axis[i] << (2 * (i % 16));
    t.err = netkv_internal_errword(h);
    return NETKV_OK;
}

// Threads of a workgroup that takes a block's rows in one pass (append_keys' and
// store_block's kEach), `groups` of 256 or more; 512 stands for a large call's
// kernels.  256 where the card holds all of them at once, five on each CU: one
// head's tokens are then as soon done by more threads.  Else 64, of which a CU
// holds 20, where they keep a block's rows and find their sequence in four looks
// at most.  us with what is read back, 256, 64: 64 single tokens of 8 heads of 128
// dimensions (1,088 groups) 20.7, 23.4, 256 (4,352) 37, 26, 200 times four 43, 32,
// 5 prompts of up to 5,003 of 5 heads of 64 in blocks of 32 38, 30, 16 of 4,096 of 8
// heads of 128 in blocks of 16 260, 204.
uint32_t append_threads(const Kv &kv, uint32_t D, uint64_t groups) {
    const uint32_t bt = 1u << kv.btl, elems = (kv.max_tok < bt ? kv.max_tok : bt) * D;
    if (elems > 256 * 64) return 512;
    return elems <= 64 * 64 && kv.n_seq <= kThreads && groups > 5 * 256 ? 64u : 256u;
}

template <int D>
void launch_append(const AppendArgs &a, uint32_t threads, hipStream_t s) {
    const uint32_t keys = a.store_tasks * a.move.kv.hk;
    if (threads == 64) {
        append_kernel<D, 64><<<a.row_tasks + 2 * keys, 64, 0, s>>>(a);
    } else if (threads == 256) {
        append_kernel<D, 256><<<a.row_tasks + 2 * keys, 256, 0, s>>>(a);
    } else {
        append_large_kernel<D><<<a.row_tasks + keys, 512, 0, s>>>(a);
        append_values_kernel<D><<<dim3(a.store_tasks, a.move.kv.hk), 1024, 0, s>>>(a);
    }
}

}  // namespace

extern "C" netkv_status netkv_rope_rotate(netkv_handle h, const netkv_rope_t *rope, uint64_t n_rows, const uint32_t *pos,
                                          uint64_t pos_stride, const void *x, uint64_t x_stride, void *out, uint64_t out_stride,
                                          uint32_t n_heads, uint32_t head_dim, int dtype, int transpose, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    if (head_dim < 16 || head_dim % 8 || head_dim > 1024) return invalid(h, "head_dim must be a multiple of 8 from 16 to 1024");
    if (n_heads < 1 || n_heads > 65535) return invalid(h, "n_heads must be in [1, 65535]");
    if (n_rows > (1ull << 31)) return invalid(h, "n_rows must be <= 2^31");
    RowArgs a{};
    netkv_status st = make_turn(h, rope, head_dim, pos, pos_stride, n_rows, true, a.turn);
    if (st != NETKV_OK) return st;
    const uint64_t width = (uint64_t)n_heads * head_dim;
    if ((st = check_rows(h, x, x_stride, width, n_rows, "x must be 16-byte aligned, its stride a multiple of 8 and at least a row's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, out, out_stride, width, n_rows, "out must be 16-byte aligned, its stride a multiple of 8 and at least a row's elements")) != NETKV_OK) return st;
    const bool in_place = x == out && x_stride == out_stride;
    if (!in_place && rows_overlap(x, x_stride, out, out_stride, width, n_rows)) return invalid(h, "out must not overlap x (it may be x itself)");
    if (n_rows == 0) return NETKV_OK;
    a.turn.sign = transpose ? 0x80000000u : 0u;
    a.x = (const uint16_t *)x;
    a.out = (uint16_t *)out;
    a.x_stride = x_stride;
    a.out_stride = out_stride;
    a.heads = n_heads;
    a.dim = head_dim;
    a.half = dtype == NETKV_FP16;
    a.units = units_of(a.turn.pairs, head_dim, in_place);
    const uint64_t each = (uint64_t)((n_heads + kHeadsEach - 1) / kHeadsEach) * a.units;
    const uint32_t chunk = (uint32_t)(each >= kThreads ? 1 : kThreads / each);
    const uint64_t groups = (n_rows + chunk - 1) / chunk;
    if (!grid_fits(groups, kThreads)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many rows for one call");
    DeviceScope scope(netkv_internal_device(h));
    rotate_kernel<<<(uint32_t)groups, kThreads, 0, (hipStream_t)stream>>>(a, (uint32_t)n_rows, chunk);
    return launched(h, "rotation launch failed");
}

extern "C" netkv_status netkv_kv_append(netkv_handle h, const netkv_kv_t *kv, const netkv_kv_seqs_t *seqs, const netkv_rope_t *rope,
                                        const uint32_t *pos, uint64_t pos_stride, const void *q, uint32_t n_heads,
                                        uint64_t q_stride, void *q_out, uint64_t q_out_stride, const void *k, uint64_t k_stride,
                                        const void *v, uint64_t v_stride, int dtype, void *stream) {
    if (!h) return NETKV_EINVAL;
    netkv_internal_clear(h);
    AppendArgs a{};
    Kv &kv_ = a.move.kv;
    netkv_status st = make_kv(h, kv, seqs, kv_);
    if (st != NETKV_OK) return st;
    if (dtype != NETKV_BF16 && dtype != NETKV_FP16) return invalid(h, "dtype must be NETKV_BF16 or NETKV_FP16");
    if ((st = make_turn(h, rope, kv->head_dim, pos, pos_stride, kv_.n_tok, false, a.rows.turn)) != NETKV_OK) return st;
    const uint64_t width = (uint64_t)kv->n_kv_heads * kv->head_dim, q_width = (uint64_t)n_heads * kv->head_dim;
    if ((st = check_rows(h, k, k_stride, width, kv_.n_tok, "k must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    if ((st = check_rows(h, v, v_stride, width, kv_.n_tok, "v must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
    bool in_place = false;
    if (n_heads) {
        if (n_heads > 65535) return invalid(h, "n_heads must be <= 65535");
        if ((st = check_rows(h, q, q_stride, q_width, kv_.n_tok, "q must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
        if ((st = check_rows(h, q_out, q_out_stride, q_width, kv_.n_tok, "q_out must be 16-byte aligned, its stride a multiple of 8 and at least a token's elements")) != NETKV_OK) return st;
        in_place = q == q_out && q_stride == q_out_stride;
        if (!in_place && rows_overlap(q, q_stride, q_out, q_out_stride, q_width, kv_.n_tok)) return invalid(h, "q_out must not overlap q (it may be q itself)");
        if (rows_overlap(k, k_stride, width, q_out, q_out_stride, q_width, kv_.n_tok) || rows_overlap(v, v_stride, width, q_out, q_out_stride, q_width, kv_.n_tok))
            return invalid(h, "q_out must not overlap k or v");
    }
    if (kv_.n_seq == 0 || kv_.n_tok == 0) return NETKV_OK;
    a.move.k = k;
    a.move.v = v;
    a.move.k_stride = k_stride;
    a.move.v_stride = v_stride;
    RowArgs &r = a.rows;
    r.half = dtype == NETKV_FP16;
    const uint64_t tasks = store_groups(kv_);
    const uint32_t threads = append_threads(kv_, kv->head_dim, tasks * kv_.hk * 2 + (n_heads ? kv_.n_tok / 16 : 0));
    uint64_t row_tasks = 0;
    if (n_heads) {
        r.x = (const uint16_t *)q;
        r.out = (uint16_t *)q_out;
        r.x_stride = q_stride;
        r.out_stride = q_out_stride;
        r.heads = n_heads;
        r.dim = kv->head_dim;
        r.units = units_of(r.turn.pairs, kv->head_dim, in_place);
        a.chunk = kv_.max_tok < 16 ? 1 : threads == 64 ? 4 : 16;
        row_tasks = row_groups(kv_, a.chunk);
    }
    const uint64_t groups = row_tasks + tasks * kv_.hk * 2;
    // workgroups of up to 512, or of 1,024 along a head
    if (!grid_fits(groups, 512) || !grid_fits(tasks, 1024)) return netkv_internal_fail(h, NETKV_ECAPACITY, "too many rows for one call");
    a.row_tasks = (uint32_t)row_tasks;
    a.store_tasks = (uint32_t)tasks;
    DeviceScope scope(netkv_internal_device(h));
    hipStream_t s = (hipStream_t)stream;
    switch (kv->head_dim) {
        case 64: launch_append<64>(a, threads, s); break;
        case 128: launch_append<128>(a, threads, s); break;
        default: launch_append<256>(a, threads, s); break;
    }
    return launched(h, "append launch failed");
}
