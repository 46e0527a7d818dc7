// Append to the block-scaled cache: rotation, page scales, 8-bit codes; queries rotated beside.
//
// Eight lanes hold a row, sixteen channels each: in the half layout eight pairs' lower and upper channels,
// else sixteen neighbours, so a pair never crosses lanes and every lane's loads are 16 bytes.  A warp takes four
// rows at a time.  Rows are kept as they came and rotated twice, for the page's amax and for the codes: as fp32 they
// take a third of the SM's warps (32k prompt 133 us).
//
// GB300, 28 query / 4 KV heads: a prompt of 32768 tokens 107 us, 5.5 TB/s of the 587 MB that it has to move (0.81 of the
// measured copy rate; the loads' latency at 24 warps an SM), 16 ragged chunks of up to 1023 tokens (40 / 8 heads) 48 us;
// one token 6 us, all of it launch and a chain of five loads (context, block table, scale, angles, row).
#include "block_common.cuh"

namespace wc {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

__device__ __forceinline__ void report(const BlockAppendParams& p, uint32_t bit) {
    if (p.dev_status) atomicOr(p.dev_status, bit);
}

// Sequence b's rows [lo, hi) of the new tokens and its context; false: skipped.
struct Sequence {
    int lo, n, start;   // first row, rows, logical position of the first row
};
template <bool kTell = false>
__device__ __forceinline__ bool sequence(const BlockAppendParams& p, int b, Sequence& s) {
    s.lo = p.cu_new ? load_dep(p.cu_new + b) : b;
    const int hi = p.cu_new ? load_dep(p.cu_new + b + 1) : b + 1;
    const int ctx = load_dep(p.ctx_lens + b);
    if (s.lo < 0 || hi < s.lo || hi > p.n_tok) {
        if (kTell) report(p, WC_DEV_BAD_ROWS);
        return false;
    }
    s.n = hi - s.lo;
    if (s.n > 0 && (ctx < s.n || ctx > (long long)p.max_pages * kPage)) {   // compared, not subtracted: any int32 may come
        if (kTell) report(p, WC_DEV_BAD_CTX);
        return false;
    }
    s.start = ctx - s.n;
    return s.n > 0;
}

// Lane i of a row: its two chunks of eight channels, and whether they are rotated (i < nrot = rotary_dim / 16).
template <bool kHalfLayout>
struct Chunks {
    int a, b;
    bool rotated;
    __device__ __forceinline__ Chunks(int i, int nrot) {
        rotated = i < nrot;
        a = kHalfLayout && rotated ? i : 2 * i;
        b = kHalfLayout && rotated ? i + nrot : 2 * i + 1;
    }
};

struct Raw {
    uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const void* row, int a, int b) {
    const uint4* src = static_cast<const uint4*>(row);
    return {load_dep(src + a), load_dep(src + b)};
}

// cos and sin of a lane's eight pairs.
struct Trig {
    float c[8], s[8];
};
__device__ __forceinline__ void load_trig(const BlockAppendParams& p, long long at, int i, Trig& t) {
    const size_t off = (size_t)at * (p.rotary_dim >> 1) + 8 * i;
    const float4* c = reinterpret_cast<const float4*>(p.cos_table + off);
    const float4* s = reinterpret_cast<const float4*>(p.sin_table + off);
    *reinterpret_cast<float4*>(t.c) = load_dep(c);
    *reinterpret_cast<float4*>(t.c + 4) = load_dep(c + 1);
    *reinterpret_cast<float4*>(t.s) = load_dep(s);
    *reinterpret_cast<float4*>(t.s + 4) = load_dep(s + 1);
}

// A lane's sixteen channels as fp32, rotated.  Products are rounded one by one: the result does not depend on
// what the compiler contracts.
template <bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void rotate(const Raw& raw, bool rotated, const Trig& t, float (&y)[16]) {
    const uint32_t w[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        y[2 * j] = f.x;
        y[2 * j + 1] = f.y;
    }
    if (!rotated) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float& lo = kHalfLayout ? y[e] : y[2 * e];
        float& hi = kHalfLayout ? y[8 + e] : y[2 * e + 1];
        const float a = lo, b = hi;
        lo = __fsub_rn(__fmul_rn(a, t.c[e]), __fmul_rn(b, t.s[e]));
        hi = __fadd_rn(__fmul_rn(b, t.c[e]), __fmul_rn(a, t.s[e]));
    }
}

// The page scale that amax asks for; amax as its bits, which order like the values with
// infinity and NaN above every number.
template <int kCode>
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
    if (amax == 0 || amax >= 0x7F800000u) return amax;   // infinity and NaN stay
    constexpr uint32_t kLeast = (127 - 100) << 23;        // 2^-100
    if constexpr (kCode == WC_CODE_INT8) {
        return max(__float_as_uint(__fmul_rn(__uint_as_float(amax), 1.0f / 127.0f)), kLeast);
    } else {
        // 448 = 1.75 * 2^8: amax = 1.f * 2^e needs 2^(e - 8) while 1.f <= 1.75, else 2^(e - 7)
        const int e = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFFu) > 0x600000u);
        return max((uint32_t)max(e, 0) << 23, kLeast);
    }
}

// rn(y) as four codes; |y| <= 127 (int8: the sum with 1.5 * 2^23 holds the rounded integer in its
// low bits) or <= 448.
template <int kCode>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    if constexpr (kCode == WC_CODE_INT8) {
        constexpr float kMagic = 12582912.0f;
        const uint32_t ia = __float_as_uint(__fadd_rn(a, kMagic)), ib = __float_as_uint(__fadd_rn(b, kMagic));
        const uint32_t ic = __float_as_uint(__fadd_rn(c, kMagic)), id = __float_as_uint(__fadd_rn(d, kMagic));
        return prmt(prmt(ia, ib, 0x0040u), prmt(ic, id, 0x0040u), 0x5410u);
    } else {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
        return (uint32_t)lo | (uint32_t)hi << 16;
    }
}

// One warp: the new rows of one page and KV head, keys (side 0) or values.  A lane holds its channels of every
// fourth row, so the page's amax is one warp reduction and the rows are read once.
template <int kCode, bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void append_page(const BlockAppendParams& p, int task, int head, int side) {
    const int lane = threadIdx.x & 31, sub = lane >> 3, i = lane & 7;
    // page tasks of sequence b: cu[b] / 16 + 2 b on, two more than its whole pages (n rows reach
    // into at most n / 16 + 2)
    int b = task, local = 0;
    if (p.cu_new) {
        auto first = [&](int s) { return (long long)(load_dep(p.cu_new + s) >> 4) + 2LL * s; };
        b = warp_find_last(p.batch, task, first);
        local = task - (int)first(b);
    }
    Sequence s;
    if (!sequence(p, b, s) || local < 0) return;
    const int page = (s.start >> 4) + local;
    const int t0 = max(s.start, page * kPage), t1 = min(s.start + s.n, page * kPage + kPage);   // positions [t0, t1)
    if (t0 >= t1) return;
    const int phys = load_dep(p.block_table + (size_t)b * p.max_pages + page);
    if (phys < 0 || phys >= p.num_pages) {
        if (lane == 0) report(p, WC_DEV_BAD_PAGE);
        return;
    }
    const int keep = local == 0 ? t0 - page * kPage : 0;   // older tokens in the page
    const size_t block = (size_t)phys * p.num_kv_heads + head;
    const uint32_t had = keep ? __float_as_uint(load_dep(p.scale[side] + block)) : 0u;
    const int rot = side == 0 ? p.rotary_dim : 0;

    const Chunks<kHalfLayout> at(i, rot >> 4);
    constexpr int kSteps = kPage / 4;
    Raw raw[kSteps];
    long long position[kSteps];
    bool mine[kSteps];
    const char* rows = static_cast<const char*>(p.x[side]) + 2 * ((size_t)head * kHeadDim);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const int t = page * kPage + 4 * j + sub;
        mine[j] = t >= t0 && t < t1;
        const int row = s.lo + t - s.start;
        raw[j] = {};
        position[j] = t;
        if (mine[j]) {
            raw[j] = load_raw(rows + 2 * ((size_t)row * p.x_stride[side]), at.a, at.b);
            if (p.rotary_dim && p.positions) position[j] = load_dep(p.positions + row);
        }
    }
    // Rows are rotated for their amax and again for their codes: kept as fp32 they would take the registers of a
    // third of the warps.
    auto turned = [&](int j, float (&y)[16]) {
        Trig trig;
        if (at.rotated) load_trig(p, position[j], i, trig);
        rotate<kBf16, kHalfLayout>(raw[j], at.rotated, trig, y);
    };
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        if (p.rotary_dim && mine[j] && (position[j] < 0 || position[j] >= p.num_positions)) {
            report(p, WC_DEV_BAD_POSITION);
            mine[j] = false;
        }
        if (mine[j]) {
            float y[16];
            turned(j, y);
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = max(amax, __float_as_uint(y[e]) & 0x7FFFFFFFu);
        }
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    const uint32_t now = max(scale_bits<kCode>(amax), had);
    const bool finite = now < 0x7F800000u;
    const float scale = __uint_as_float(now), inv = now && finite ? __fdiv_rn(1.0f, scale) : 0.0f;
    uint8_t* codes = p.codes[side] + block * (kPage * kHeadDim);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        if (!mine[j]) continue;
        float v[16];
        turned(j, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = finite ? __fmul_rn(v[e], inv) : 0.0f;
        uint2* dst = reinterpret_cast<uint2*>(codes + (4 * j + sub) * kHeadDim);
        dst[at.a] = make_uint2(encode4<kCode>(v[0], v[1], v[2], v[3]), encode4<kCode>(v[4], v[5], v[6], v[7]));
        dst[at.b] = make_uint2(encode4<kCode>(v[8], v[9], v[10], v[11]), encode4<kCode>(v[12], v[13], v[14], v[15]));
    }
    if (now > had) {
        if (lane == 0) p.scale[side][block] = scale;
        const float ratio = finite ? __fdiv_rn(__uint_as_float(had), scale) : 0.0f;
        for (int r = sub; r < keep; r += 4) {   // older tokens: the page's scale grew
            uint4* old = reinterpret_cast<uint4*>(codes + r * kHeadDim) + i;
            const uint4 c = load_dep(old);
            uint32_t out[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t lo, hi;
                codes4_to_h2<kCode>(word_of(c, k), lo, hi);
                const float2 f = h2_to_float2(lo), g = h2_to_float2(hi);
                out[k] = finite ? encode4<kCode>(__fmul_rn(f.x, ratio), __fmul_rn(f.y, ratio), __fmul_rn(g.x, ratio), __fmul_rn(g.y, ratio)) : 0u;
            }
            *old = make_uint4(out[0], out[1], out[2], out[3]);
        }
    } else if (!keep && lane == 0) {
        p.scale[side][block] = scale;   // a page begun with zeros
    }
}

// One warp: query heads [head0, head0 + p.q_heads) of one token.
template <bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void rotate_queries(const BlockAppendParams& p, int row, int head0) {
    const int lane = threadIdx.x & 31, sub = lane >> 3, i = lane & 7;
    const int rot = p.rotary_dim, end = min(head0 + p.q_heads, p.num_q_heads);
    const Chunks<kHalfLayout> at(i, rot >> 4);
    const char* src = static_cast<const char*>(p.q) + 2 * (size_t)row * p.q_stride;
    char* dst = static_cast<char*>(p.q_out) + 2 * (size_t)row * p.num_q_heads * kHeadDim;
    constexpr int kAhead = 4;   // steps of four heads in flight
    Raw raw[kAhead];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            raw[j] = {};
            if (h0 + 4 * j < end) raw[j] = load_raw(src + 2 * (size_t)(h0 + 4 * j) * kHeadDim, at.a, at.b);
        }
    };
    fetch(head0 + sub);   // the rows do not wait for whose they are
    int b = row;
    if (p.cu_new) b = warp_find_last(p.batch, row, [&](int s) { return (long long)load_dep(p.cu_new + s); });
    Sequence s;
    if (!sequence(p, b, s) || row < s.lo || row >= s.lo + s.n) return;   // reported elsewhere
    long long position = s.start + row - s.lo;
    if (rot && p.positions) position = load_dep(p.positions + row);
    const bool bad = rot && (position < 0 || position >= p.num_positions);
    if (bad && lane == 0) report(p, WC_DEV_BAD_POSITION);
    Trig trig;
    if (at.rotated && !bad) load_trig(p, position, i, trig);
    for (int h0 = head0 + sub; h0 - sub < end; h0 += 4 * kAhead) {
        if (h0 != head0 + sub) fetch(h0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (h0 + 4 * j >= end) continue;
            float y[16];
            if (bad) raw[j] = {};
            rotate<kBf16, kHalfLayout>(raw[j], at.rotated && !bad, trig, y);
            uint4* out = reinterpret_cast<uint4*>(dst + 2 * (size_t)(h0 + 4 * j) * kHeadDim);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = float2_to_act2<kBf16>(y[2 * e], y[2 * e + 1]);
            out[at.a] = make_uint4(w[0], w[1], w[2], w[3]);
            out[at.b] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

template <int kCode, bool kBf16, bool kHalfLayout>
__global__ void __launch_bounds__(kThreads, 3) block_append_kernel(const __grid_constant__ BlockAppendParams p) {
    grid_dep_launch();
    grid_dep_wait();
    const int warp = threadIdx.x >> 5;
    if ((int)blockIdx.x < p.page_ctas) {
        const long long t = (long long)blockIdx.x * kWarps + warp;   // (page task, head, side), side fastest
        const long long per = 2LL * p.num_kv_heads;
        const long long task = t / per;
        if (t == per * p.page_tasks) {   // one warp more reports the sequences that the others skip
            Sequence s;
            for (int b = threadIdx.x & 31; b < p.batch; b += 32) sequence<true>(p, b, s);
        }
        if (task >= p.page_tasks) return;
        const int rest = (int)(t - task * per);
        append_page<kCode, kBf16, kHalfLayout>(p, (int)task, rest >> 1, rest & 1);
    } else {
        const long long t = (long long)(blockIdx.x - p.page_ctas) * kWarps + warp;
        const int per = (p.num_q_heads + p.q_heads - 1) / p.q_heads;
        const long long row = t / per;
        if (row >= p.n_tok) return;
        rotate_queries<kBf16, kHalfLayout>(p, (int)row, (int)(t - row * per) * p.q_heads);
    }
}

}  // namespace

cudaError_t launch_block_append(const BlockAppendParams& params, int code, int act, int rope_layout, cudaStream_t stream) {
    BlockAppendParams p = params;
    const long long pages = p.cu_new ? (long long)p.n_tok / kPage + 2LL * p.batch : p.batch;
    const long long page_ctas = (pages * 2 * p.num_kv_heads + 1 + kWarps - 1) / kWarps;
    // few tokens: eight heads a warp, in parallel; many: 32, behind one read of the angles
    p.q_heads = (long long)p.n_tok * p.num_q_heads >= 16384 ? 32 : 8;
    const long long q_ctas = p.q ? ((long long)p.n_tok * ((p.num_q_heads + p.q_heads - 1) / p.q_heads) + kWarps - 1) / kWarps : 0;
    if (page_ctas + q_ctas > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
    p.page_tasks = (int)pages;
    p.page_ctas = (int)page_ctas;
    auto go = [&](auto kernel) {
        return launch_pdl(kernel, dim3((unsigned)(page_ctas + q_ctas)), dim3(kThreads), 0, stream, p);
    };
    const bool half = rope_layout == WC_ROPE_HALF;
    if (code == WC_CODE_INT8) {
        if (act == WC_ACT_BF16)
            return half ? go(block_append_kernel<WC_CODE_INT8, true, true>) : go(block_append_kernel<WC_CODE_INT8, true, false>);
        return half ? go(block_append_kernel<WC_CODE_INT8, false, true>) : go(block_append_kernel<WC_CODE_INT8, false, false>);
    }
    if (act == WC_ACT_BF16)
        return half ? go(block_append_kernel<WC_CODE_E4M3, true, true>) : go(block_append_kernel<WC_CODE_E4M3, true, false>);
    return half ? go(block_append_kernel<WC_CODE_E4M3, false, true>) : go(block_append_kernel<WC_CODE_E4M3, false, false>);
}

}  // namespace wc
