// Append to the block-scaled cache: rotation, page scales, 8-bit codes; queries rotated beside.
#include "block_common.cuh"

namespace wc {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kQHeads = 8;   // query heads of one token that a warp rotates

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
    s.n = hi - s.lo;
    s.start = ctx - s.n;
    if (s.lo < 0 || hi < s.lo || hi > p.n_tok) {
        if (kTell) report(p, WC_DEV_BAD_ROWS);
        return false;
    }
    if (s.n > 0 && (s.start < 0 || ctx > (long long)p.max_pages * kPage)) {
        if (kTell) report(p, WC_DEV_BAD_CTX);
        return false;
    }
    return s.n > 0;
}

// A lane's eight channels 8 i .. 8 i + 7 of a row as fp32, rotated if they are among the first
// rotary_dim: its channels and, for the half layout, their partners' come from global memory (the
// second read hits L1), so any rotary_dim takes the same path.  Products are rounded one by
// one: the result does not depend on what the compiler contracts.
template <bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void load_rotated(const void* row, int i, int rot, const float* cos_row, const float* sin_row,
                                             float (&y)[8]) {
    const uint4* src = static_cast<const uint4*>(row);
    const uint4 own = load_dep(src + i);
    const uint32_t w[4] = {own.x, own.y, own.z, own.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = act2_to_float2<kBf16>(w[j]);
        y[2 * j] = f.x;
        y[2 * j + 1] = f.y;
    }
    if (8 * i >= rot) return;
    if constexpr (kHalfLayout) {
        const int half = rot >> 4;            // 16-byte chunks of half the rotated channels
        const bool upper = i >= half;
        const uint4 other = load_dep(src + (upper ? i - half : i + half));
        const uint32_t o[4] = {other.x, other.y, other.z, other.w};
        const int j0 = 8 * (upper ? i - half : i);
        const float4* c4 = reinterpret_cast<const float4*>(cos_row + j0);
        const float4* s4 = reinterpret_cast<const float4*>(sin_row + j0);
        const float4 ca = load_dep(c4), cb = load_dep(c4 + 1), sa = load_dep(s4), sb = load_dep(s4 + 1);
        const float c[8] = {ca.x, ca.y, ca.z, ca.w, cb.x, cb.y, cb.z, cb.w};
        const float s[8] = {sa.x, sa.y, sa.z, sa.w, sb.x, sb.y, sb.z, sb.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = act2_to_float2<kBf16>(o[j]);
            const float ot[2] = {f.x, f.y};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = 2 * j + k;
                const float a = __fmul_rn(y[e], c[e]), b = __fmul_rn(ot[k], s[e]);
                y[e] = upper ? __fadd_rn(a, b) : __fsub_rn(a, b);
            }
        }
    } else {
        const float4 c4 = load_dep(reinterpret_cast<const float4*>(cos_row) + i);
        const float4 s4 = load_dep(reinterpret_cast<const float4*>(sin_row) + i);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = y[2 * j], b = y[2 * j + 1];
            y[2 * j] = __fsub_rn(__fmul_rn(a, c[j]), __fmul_rn(b, s[j]));
            y[2 * j + 1] = __fadd_rn(__fmul_rn(b, c[j]), __fmul_rn(a, s[j]));
        }
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

// One warp: the new rows of one page and KV head, keys (side 0) or values.  A half warp holds
// a row, eight channels a lane, and a lane the same channels of every second row, so the page's amax
// is one warp reduction and the rows are read once.
template <int kCode, bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void append_page(const BlockAppendParams& p, int task, int head, int side) {
    const int lane = threadIdx.x & 31, half = lane >> 4, i = lane & 15;
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

    float y[kPage / 2][8];
    bool mine[kPage / 2];
    uint32_t amax = 0;
    const char* rows = static_cast<const char*>(p.x[side]);
#pragma unroll
    for (int j = 0; j < kPage / 2; ++j) {
        const int t = page * kPage + 2 * j + half;
        mine[j] = t >= t0 && t < t1;
        const int row = s.lo + t - s.start;
        long long at = 0;
        if (rot && mine[j]) {
            at = p.positions ? load_dep(p.positions + row) : t;
            if (at < 0 || at >= p.num_positions) {
                report(p, WC_DEV_BAD_POSITION);
                mine[j] = false;
            }
        }
        if (mine[j]) {
            const size_t trig = (size_t)at * (rot >> 1);
            load_rotated<kBf16, kHalfLayout>(rows + 2 * ((size_t)row * p.x_stride[side] + (size_t)head * kHeadDim), i, rot,
                                             p.cos_table + trig, p.sin_table + trig, y[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(y[j][e]) & 0x7FFFFFFFu);
        }
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    const uint32_t now = max(scale_bits<kCode>(amax), had);
    const bool finite = now < 0x7F800000u;
    const float scale = __uint_as_float(now), inv = now && finite ? __fdiv_rn(1.0f, scale) : 0.0f;
    uint8_t* codes = p.codes[side] + block * (kPage * kHeadDim) + 8 * i;
#pragma unroll
    for (int j = 0; j < kPage / 2; ++j) {
        if (!mine[j]) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = finite ? __fmul_rn(y[j][e], inv) : 0.0f;
        *reinterpret_cast<uint2*>(codes + (2 * j + half) * kHeadDim) =
            make_uint2(encode4<kCode>(v[0], v[1], v[2], v[3]), encode4<kCode>(v[4], v[5], v[6], v[7]));
    }
    if (now > had) {
        if (lane == 0) p.scale[side][block] = scale;
        const float ratio = finite ? __fdiv_rn(__uint_as_float(had), scale) : 0.0f;
        for (int r = half; r < keep; r += 2) {   // older tokens: the page's scale grew
            uint2* at = reinterpret_cast<uint2*>(codes + r * kHeadDim);
            const uint2 c = load_dep(at);
            uint32_t h[4];
            codes4_to_h2<kCode>(c.x, h[0], h[1]);
            codes4_to_h2<kCode>(c.y, h[2], h[3]);
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = h2_to_float2(h[e]);
                v[2 * e] = finite ? __fmul_rn(f.x, ratio) : 0.0f;
                v[2 * e + 1] = finite ? __fmul_rn(f.y, ratio) : 0.0f;
            }
            *at = make_uint2(encode4<kCode>(v[0], v[1], v[2], v[3]), encode4<kCode>(v[4], v[5], v[6], v[7]));
        }
    } else if (!keep && lane == 0) {
        p.scale[side][block] = scale;   // a page begun with zeros
    }
}

// One warp: kQHeads query heads of one token.
template <bool kBf16, bool kHalfLayout>
__device__ __forceinline__ void rotate_queries(const BlockAppendParams& p, int row, int head0) {
    const int lane = threadIdx.x & 31, half = lane >> 4, i = lane & 15;
    const int rot = p.rotary_dim;
    long long at = 0;
    int b = row;
    if (p.cu_new) b = warp_find_last(p.batch, row, [&](int s) { return (long long)load_dep(p.cu_new + s); });
    Sequence s;
    if (!sequence(p, b, s) || row < s.lo || row >= s.lo + s.n) return;
    if (rot) at = p.positions ? load_dep(p.positions + row) : s.start + row - s.lo;
    const bool bad = rot && (at < 0 || at >= p.num_positions);
    if (bad && lane == 0) report(p, WC_DEV_BAD_POSITION);
    const size_t trig = (size_t)(bad ? 0 : at) * (rot >> 1);
    const char* src = static_cast<const char*>(p.q) + 2 * (size_t)row * p.q_stride;
    char* dst = static_cast<char*>(p.q_out) + 2 * (size_t)row * p.num_q_heads * kHeadDim;
#pragma unroll
    for (int j = 0; j < kQHeads / 2; ++j) {
        const int h = head0 + 2 * j + half;
        if (h >= p.num_q_heads) continue;
        float y[8] = {};
        if (!bad)
            load_rotated<kBf16, kHalfLayout>(src + 2 * (size_t)h * kHeadDim, i, rot, p.cos_table + trig, p.sin_table + trig, y);
        reinterpret_cast<uint4*>(dst + 2 * (size_t)h * kHeadDim)[i] =
            make_uint4(float2_to_act2<kBf16>(y[0], y[1]), float2_to_act2<kBf16>(y[2], y[3]), float2_to_act2<kBf16>(y[4], y[5]),
                       float2_to_act2<kBf16>(y[6], y[7]));
    }
}

template <int kCode, bool kBf16, bool kHalfLayout>
__global__ void __launch_bounds__(kThreads) block_append_kernel(const __grid_constant__ BlockAppendParams p) {
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
        const int per = (p.num_q_heads + kQHeads - 1) / kQHeads;
        const long long row = t / per;
        if (row >= p.n_tok) return;
        rotate_queries<kBf16, kHalfLayout>(p, (int)row, (int)(t - row * per) * kQHeads);
    }
}

}  // namespace

cudaError_t launch_block_append(const BlockAppendParams& params, int code, int act, int rope_layout, cudaStream_t stream) {
    BlockAppendParams p = params;
    const long long pages = p.cu_new ? (long long)p.n_tok / kPage + 2LL * p.batch : p.batch;
    const long long page_ctas = (pages * 2 * p.num_kv_heads + 1 + kWarps - 1) / kWarps;
    const long long q_ctas = p.q ? ((long long)p.n_tok * ((p.num_q_heads + kQHeads - 1) / kQHeads) + kWarps - 1) / kWarps : 0;
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
