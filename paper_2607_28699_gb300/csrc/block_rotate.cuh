// Rows of a head's 128 channels, eight lanes a row: their norm and their rotation.
#pragma once

#include "block_common.cuh"

namespace wc {

// Lane i of a row has two chunks of eight channels, a and b.  It works on half of its channels at a time (part 0, 1), four
// pairs: as eight pairs at once the rows waiting in registers would be spilled.  In the half layout a part is four channels of
// either chunk, pair (e, 4 + e), else a chunk, pair (2 e, 2 e + 1).  Eight lanes' chunks lie side by side.
template <bool kHalfLayout>
struct Chunks {
    int i, a, b, rot;
    __device__ __forceinline__ Chunks(int lane, int rotary_dim) : i(lane), rot(rotary_dim) {
        const int nrot = rot >> 4;
        a = kHalfLayout && i >= nrot ? i + nrot : i;
        b = kHalfLayout && i < nrot ? i + nrot : i + 8;
    }
    __device__ __forceinline__ bool rotated(int part) const { return kHalfLayout ? 16 * i < rot : 8 * (part ? b : a) < rot; }
    __device__ __forceinline__ int first_pair(int part) const { return kHalfLayout ? 8 * i + 4 * part : 4 * (part ? b : a); }
};

struct Raw {
    uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const void* row, int a, int b) {
    const uint4* src = static_cast<const uint4*>(row);
    return {load_dep(src + a), load_dep(src + b)};
}

// The compiler forgets what it has unpacked of the row, instead of spilling it: unpacking again is cheaper.
__device__ __forceinline__ void forget(Raw& r) {
    asm("" : "+r"(r.a.x), "+r"(r.a.y), "+r"(r.a.z), "+r"(r.a.w), "+r"(r.b.x), "+r"(r.b.y), "+r"(r.b.z), "+r"(r.b.w));
}

// The channels of a part as fp32.
template <bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void unpack(const Raw& raw, int part, float (&y)[8]) {
    uint32_t w[4];
    if constexpr (kHalfLayout) {
        w[0] = part ? raw.a.z : raw.a.x;
        w[1] = part ? raw.a.w : raw.a.y;
        w[2] = part ? raw.b.z : raw.b.x;
        w[3] = part ? raw.b.w : raw.b.y;
    } else {
        const uint4 x = part ? raw.b : raw.a;
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        y[2 * j] = f.x;
        y[2 * j + 1] = f.y;
    }
}

// Four values as act_type.
template <bool kBf16>
__device__ __forceinline__ uint2 float4_to_act(const float* y) {
    return make_uint2(float2_to_act2<kBf16>(y[0], y[1]), float2_to_act2<kBf16>(y[2], y[3]));
}

// Two words of a part (its first, its last four channels) to their places in the lane's chunks a and b.
template <bool kHalfLayout, typename Word>
__device__ __forceinline__ void place(Word (&a)[2], Word (&b)[2], int part, Word first, Word last) {
    if constexpr (kHalfLayout) a[part] = first, b[part] = last;
    else (part ? b : a)[0] = first, (part ? b : a)[1] = last;
}

// cos and sin of a lane's pairs of a part.
struct Trig {
    float c[4], s[4];
};
// off: the position's first entry of the tables, plus the part's first pair.
__device__ __forceinline__ void load_trig(const float* cos_table, const float* sin_table, size_t off, Trig& t) {
    *reinterpret_cast<float4*>(t.c) = load_dep(reinterpret_cast<const float4*>(cos_table + off));
    *reinterpret_cast<float4*>(t.s) = load_dep(reinterpret_cast<const float4*>(sin_table + off));
}

__device__ __forceinline__ void prefetch_l1(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p) : "memory"); }

// Rotated in place.  Products are rounded one by one: the result does not depend on what the compiler contracts.  They are
// packed where the pairs lie that way, the sums are not: a packed sum of packed products is contracted, whatever its rounding
// is called.
template <bool kHalfLayout>
__device__ __forceinline__ void rotate(const Trig& t, float (&y)[8]) {
    if constexpr (kHalfLayout) {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const float2 a = make_float2(y[e], y[e + 1]), b = make_float2(y[e + 4], y[e + 5]);
            const float2 c = make_float2(t.c[e], t.c[e + 1]), s = make_float2(t.s[e], t.s[e + 1]);
            const float2 ac = __fmul2_rn(a, c), bs = __fmul2_rn(b, s), bc = __fmul2_rn(b, c), as = __fmul2_rn(a, s);
            y[e] = __fsub_rn(ac.x, bs.x);
            y[e + 1] = __fsub_rn(ac.y, bs.y);
            y[e + 4] = __fadd_rn(bc.x, as.x);
            y[e + 5] = __fadd_rn(bc.y, as.y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = y[2 * e], b = y[2 * e + 1];
            y[2 * e] = __fsub_rn(__fmul_rn(a, t.c[e]), __fmul_rn(b, t.s[e]));
            y[2 * e + 1] = __fadd_rn(__fmul_rn(b, t.c[e]), __fmul_rn(a, t.s[e]));
        }
    }
}

// The larger of two magnitudes and a magnitude so far, NaN if any is.
__device__ __forceinline__ float most_of(float most, float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(most), "f"(fabsf(a)), "f"(fabsf(b)));
    return d;
}

// ---- norm ---------------------------------------------------------------------------------------

// A sum as two floats: hi + lo, lo what hi's roundings lost.
struct TwoFloats {
    float hi, lo;
};
// hi of x.hi + y with the rounding's error, exact for any order of magnitudes, added to lo.
__device__ __forceinline__ void add_exactly(TwoFloats& x, float y) {
    const float s = __fadd_rn(x.hi, y), v = __fsub_rn(s, x.hi);
    x.lo = __fadd_rn(x.lo, __fadd_rn(__fsub_rn(x.hi, __fsub_rn(s, v)), __fsub_rn(y, v)));
    x.hi = s;
}

// The sum of a row's squares, in each of its eight lanes.  It is held to about 2^-44, so that the factor below, a page's
// scale and the codes that hang on it do not depend on the order of the sum.  A lane's sums begin with its largest square
// (taken off again): from there on no square is above the sum, so what an addition loses, f^2 - (sum' - sum), is exact in three
// operations and without the square.
template <bool kBf16>
__device__ __forceinline__ TwoFloats sum_of_squares(const Raw& raw) {
    const uint32_t w[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
    uint32_t most = 0;   // without signs the values order like integers
#pragma unroll
    for (int j = 0; j < 8; ++j) most = __vmaxu2(most, w[j] & 0x7FFF7FFFu);
    const float2 two = act2_to_float2<kBf16>(__vmaxu2(most, most >> 16));
    const float first = __fmul_rn(two.x, two.x);
    float2 sum = make_float2(first, first), lost = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        const float2 next = __ffma2_rn(f, f, sum), gained = __fadd2_rn(next, make_float2(-sum.x, -sum.y));
        lost = __fadd2_rn(lost, __ffma2_rn(f, f, make_float2(-gained.x, -gained.y)));
        sum = next;
    }
    TwoFloats s = {sum.x, __fadd_rn(lost.x, lost.y)};
    add_exactly(s, sum.y);
    add_exactly(s, -2.0f * first);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        const float hi = __shfl_xor_sync(0xffffffffu, s.hi, o), lo = __shfl_xor_sync(0xffffffffu, s.lo, o);
        s.lo = __fadd_rn(s.lo, lo);
        add_exactly(s, hi);
    }
    return s;
}

// 1 / sqrt(v), rounded once (but for one in a million): one Newton step on the library's answer, the residual 1 - r^2 v in two
// floats.  For v from 2^-60 to 2^80: what the residual is made of stays above fp32's least numbers.
__device__ __forceinline__ float inverse_root(TwoFloats v) {
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v.hi));
    const float q = __fmul_rn(r, r), q_lo = fmaf(r, r, -q), t = __fmul_rn(q, v.hi), t_lo = fmaf(q, v.hi, -t);
    const float rest = fmaf(-q, v.lo, fmaf(-q_lo, v.hi, __fsub_rn(__fsub_rn(1.0f, t), t_lo)));
    return __fadd_rn(r, __fmul_rn(__fmul_rn(0.5f, r), rest));
}

// The factor of a row (a warp takes four together), 1 / sqrt(mean + eps): NaN for one with infinities or NaN, or with a sum of
// squares past fp32's range (bf16 values from 2^60 on).
template <bool kBf16>
__device__ __forceinline__ float norm_factor(const Raw& raw, float eps) {
    const TwoFloats sum = sum_of_squares<kBf16>(raw);
    TwoFloats v = {sum.hi * (1.0f / kHeadDim), sum.lo * (1.0f / kHeadDim)};
    add_exactly(v, eps);
    return inverse_root(v);
}

// Whether a factor says that mean + eps is so far from 1 that the two floats lost what they are for, or passed the range on the way
// (they hold up to three times the largest square: NaN): wide_factor has those rows'.
__device__ __forceinline__ bool far_factor(float r) { return !(r >= 0x1p-40f && r <= 0x1p30f); }

// The same in 64 bits, for any row.
template <bool kBf16>
__device__ __forceinline__ float wide_factor(const Raw& raw, float eps) {
    const uint32_t w[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        s = fma((double)f.x, (double)f.x, fma((double)f.y, (double)f.y, s));
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return (float)s < INFINITY ? (float)rsqrt(s * (1.0 / kHeadDim) + (double)eps) : NAN;
}

// y = (y r) w, each product rounded; a, b the lane's chunks of the weights.
template <bool kHalfLayout>
__device__ __forceinline__ void scale_part(const float* weight, int a, int b, int part, float r, float (&y)[8]) {
    const float4* w = reinterpret_cast<const float4*>(weight);
    const float4 f = load_dep(w + (kHalfLayout ? 2 * a + part : 2 * (part ? b : a)));
    const float4 g = load_dep(w + (kHalfLayout ? 2 * b + part : 2 * (part ? b : a) + 1));
    const float2 by[4] = {{f.x, f.y}, {f.z, f.w}, {g.x, g.y}, {g.z, g.w}};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 z = __fmul2_rn(__fmul2_rn(make_float2(y[2 * e], y[2 * e + 1]), make_float2(r, r)), by[e]);
        y[2 * e] = z.x;
        y[2 * e + 1] = z.y;
    }
}

// ---- for rows that are stored in 16 bits ---------------------------------------------------------

// The factor of a row as norm_factor's but for rounding, where no code hangs on it: sums of squares in fp32 (8 terms a half of a
// lane, then 4 sums of two: 12 x 2^-24), half of that and 2 x 2^-24 in the root.
template <bool kBf16>
__device__ __forceinline__ float quick_factor(const Raw& raw, float eps) {
    const uint32_t w[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        s = __ffma2_rn(f, f, s);
    }
    float t = s.x + s.y;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    float r;   // of a normal number: eps is
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(t, 1.0f / kHeadDim, eps)));
    return t < INFINITY ? r : NAN;
}

// As rotate, the second product of each sum not rounded; packed where the pairs lie that way.
template <bool kHalfLayout>
__device__ __forceinline__ void quick_rotate(const Trig& t, float (&y)[8]) {
    if constexpr (kHalfLayout) {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const float2 a = make_float2(y[e], y[e + 1]), b = make_float2(y[e + 4], y[e + 5]);
            const float2 c = make_float2(t.c[e], t.c[e + 1]), s = make_float2(t.s[e], t.s[e + 1]), bs = __fmul2_rn(b, s);
            const float2 lo = __ffma2_rn(a, c, make_float2(-bs.x, -bs.y)), hi = __ffma2_rn(a, s, __fmul2_rn(b, c));
            y[e] = lo.x;
            y[e + 1] = lo.y;
            y[e + 4] = hi.x;
            y[e + 5] = hi.y;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = y[2 * e], b = y[2 * e + 1];
            y[2 * e] = fmaf(a, t.c[e], -__fmul_rn(b, t.s[e]));
            y[2 * e + 1] = fmaf(a, t.s[e], __fmul_rn(b, t.c[e]));
        }
    }
}

// A row of a lane, normed (kNormed) and rotated (turn), as 16-bit words of its chunks.  Rows that are not normed are rotated with
// every product rounded, whatever the call.
template <bool kNormed, bool kBf16, bool kOutBf16, bool kHalfLayout>
__device__ __forceinline__ void finished_row(const Raw& raw, const Chunks<kHalfLayout>& at, const float* weight, float r, bool turn, const Trig (&trig)[2],
                                           uint4& a, uint4& b) {
    uint2 wa[2], wb[2];
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        float y[8];
        unpack<kBf16, kHalfLayout>(raw, part, y);
        if constexpr (kNormed) {
            scale_part<kHalfLayout>(weight, at.a, at.b, part, r, y);
            if (turn && at.rotated(part)) quick_rotate<kHalfLayout>(trig[part], y);
        } else {
            if (turn && at.rotated(part)) rotate<kHalfLayout>(trig[part], y);
        }
        place<kHalfLayout>(wa, wb, part, float4_to_act<kOutBf16>(y), float4_to_act<kOutBf16>(y + 4));
    }
    a = make_uint4(wa[0].x, wa[0].y, wa[1].x, wa[1].y);
    b = make_uint4(wb[0].x, wb[0].y, wb[1].x, wb[1].y);
}

}  // namespace wc
