// Append to the block-scaled cache: rotation, page scales, 8-bit codes; queries rotated beside.
//
// Eight lanes hold a row, sixteen channels each (block_rotate.cuh), so that pairs and norms never leave a warp's quarter and every
// lane's loads are 16 bytes.  A warp takes four rows at a time.  A page's rows are turned twice, for its amax and for its codes,
// and loaded again for the second time (from L1): kept in registers they would take a quarter of the SM's warps, as fp32 half.
// CTAs of pages lie among those that rotate queries: a page is a chain of loads, which the others' bytes hide (a 32k prompt
// 95 us; pages first, then queries: 103).  Normed queries and others have a loop each (with
// norms 106.5 us; one loop for both 114.5).
//
// The norm of keys is summed in two floats (block_rotate.cuh): scales and codes hang on the factor's last bit.  With the norm the
// page's loops are not unrolled: its instructions would stop fitting the cache (a 32k prompt 143 us instead of 121); what the loop
// will load is asked for ahead (118 us without the prefetches, 114.5 with).  Both were measured on earlier forms.
//
// GB300, 28 query / 4 KV heads: a prompt of 32768 tokens 94 us, 6.3 TB/s of the 587 MB that it has to move (0.92 of the
// measured copy rate), 16 ragged chunks of up to 1023 tokens (40 / 8 heads) 37 us; with norms 106.5 (0.81) and 44 us: its
// 77 million warp instructions take 59% of the issue slots, its warps wait for loads for half of their time; one token 3 us in a row
// of calls, 9 by itself, all of it launch and a chain of four loads (context, block table, scale; rows and angles beside them).
#include "block_rotate.cuh"

namespace wc {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;

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

// A warp's page task, KV head and side: (task, head, side) of the launch's heads, side fastest.  group: of its CTA among those of pages.
struct PageWork {
    unsigned task;
    int head, side;
    __device__ __forceinline__ PageWork(const BlockAppendParams& p, unsigned group, unsigned warp) {
        const unsigned t = group * kWarps + warp, per = 2 * p.page_heads;
        task = t / per;
        const unsigned rest = t - task * per;
        head = p.page_head0 + (int)(rest >> 1);
        side = rest & 1;
    }
};

enum class Norm { kNone, kUsual, kWide };   // kWide: factors in 64 bits
template <int kCode, bool kBf16, bool kHalfLayout, Norm kOf>
__device__ __forceinline__ void append_page(const BlockAppendParams& p, int task, int head, int side);

// A warp's page anew, with factors in 64 bits.  A function of its own, which finds its task again: usual pages have no register for
// what it takes (a 32k prompt with norms 114.8 us as without it; inlined, or with the task passed on, 117.6).
template <int kCode, bool kBf16, bool kHalfLayout>
__device__ __noinline__ void append_wide_page(const BlockAppendParams& p) {
    unsigned cta, thread;   // read again, not kept
    asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(cta));
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(thread));
    const PageWork w(p, cta / (unsigned)p.page_stride, __shfl_sync(0xffffffffu, thread >> 5, 0));
    append_page<kCode, kBf16, kHalfLayout, Norm::kWide>(p, (int)w.task, w.head, w.side);
}

// One warp: the new rows of one page and KV head, keys (side 0) or values.  A lane takes its channels of every
// fourth row, so the page's amax is one warp reduction.
template <int kCode, bool kBf16, bool kHalfLayout, Norm kOf>
__device__ __forceinline__ void append_page(const BlockAppendParams& p, int task, int head, int side) {
    constexpr bool kNorm = kOf != Norm::kNone;
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
    const int rot = side == 0 ? p.rotary_dim : 0;

    const Chunks<kHalfLayout> at(i, rot);
    constexpr int kSteps = kPage / 4;
    const char* rows = static_cast<const char*>(p.x[side]) + 2 * ((size_t)head * kHeadDim);
    const bool normed = kNorm && side == 0 && p.k_norm;
    auto there = [&](int j) {
        const int t = page * kPage + 4 * j + sub;
        return t >= t0 && t < t1;
    };
    auto load = [&](int j) {
        return there(j) ? load_raw(rows + 2 * ((size_t)(s.lo + page * kPage + 4 * j + sub - s.start) * p.x_stride[side]), at.a, at.b) : Raw{};
    };
    auto position_of = [&](int j) {
        const int t = page * kPage + 4 * j + sub;
        return p.rotary_dim && p.positions && there(j) ? load_dep(p.positions + s.lo + t - s.start) : t;
    };
    // rows and angles are asked for before the block table answers
    Raw next = load(0);
    if constexpr (kNorm) {
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            if (!there(j)) continue;
            const char* row = rows + 2 * ((size_t)(s.lo + page * kPage + 4 * j + sub - s.start) * p.x_stride[side]);
            if (j > 0) {
                prefetch_l1(row + 16 * at.a);
                prefetch_l1(row + 16 * at.b);
            }
            if (p.positions || page * kPage + 4 * j + sub >= p.num_positions) continue;
#pragma unroll
            for (int part = 0; part < (kHalfLayout ? 1 : 2); ++part) {
                if (!at.rotated(part)) continue;
                const size_t off = (size_t)(page * kPage + 4 * j + sub) * (p.rotary_dim >> 1) + at.first_pair(part);
                prefetch_l1(p.cos_table + off);
                prefetch_l1(p.sin_table + off);
            }
        }
    }
    if (phys < 0 || phys >= p.num_pages) {
        if (lane == 0) report(p, WC_DEV_BAD_PAGE);
        return;
    }
    const int keep = local == 0 ? t0 - page * kPage : 0;   // older tokens in the page
    const size_t block = (size_t)phys * p.num_kv_heads + head;
    const uint32_t had = keep ? __float_as_uint(load_dep(p.scale[side] + block)) : 0u;
    auto turned = [&](const Raw& raw, int position, float factor, int part, float (&y)[8]) {
        Trig trig;
        if (at.rotated(part)) load_trig(p.cos_table, p.sin_table, (size_t)position * (p.rotary_dim >> 1) + at.first_pair(part), trig);
        unpack<kBf16, kHalfLayout>(raw, part, y);
        if constexpr (kNorm) {
            if (normed) scale_part<kHalfLayout>(p.k_norm, at.a, at.b, part, factor, y);
        }
        if (at.rotated(part)) rotate<kHalfLayout>(trig, y);
    };
    // The page's amax, then its codes: rows are loaded again (from L1) and turned again.
    uint32_t mine = 0;             // bit j: step j has a row of this lane
    float most = 0.0f;
    float factors = 1.0f;          // lane i: of step i
#pragma unroll (kNorm ? 1 : kSteps)
    for (int j = 0; j < kSteps; ++j) {
        Raw raw = next;
        if (j + 1 < kSteps) next = load(j + 1);
        const int position = position_of(j);
        float factor = 1.0f;
        if constexpr (kNorm) {
            if (normed) {
                if constexpr (kOf == Norm::kWide) factor = wide_factor<kBf16>(raw, p.norm_eps);
                else factor = norm_factor<kBf16>(raw, p.norm_eps);
                if (i == j) factors = factor;
                forget(raw);
            }
        }
        if (!there(j)) continue;
        if (p.rotary_dim && (position < 0 || position >= p.num_positions)) {
            report(p, WC_DEV_BAD_POSITION);
            continue;
        }
        mine |= 1u << j;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            float y[8];
            turned(raw, position, factor, part, y);
#pragma unroll
            for (int e = 0; e < 8; e += 2) most = most_of(most, y[e], y[e + 1]);
        }
    }
    if constexpr (kOf == Norm::kUsual) {
        if (__any_sync(0xffffffffu, far_factor(factors))) return append_wide_page<kCode, kBf16, kHalfLayout>(p);
    }
    const uint32_t amax = __reduce_max_sync(0xffffffffu, __float_as_uint(most));   // bits order like the magnitudes, NaN above all
    const uint32_t now = max(scale_bits<kCode>(amax), had);
    const bool finite = now < 0x7F800000u;
    const float scale = __uint_as_float(now), inv = now && finite ? __fdiv_rn(1.0f, scale) : 0.0f;
    uint8_t* codes = p.codes[side] + block * (kPage * kHeadDim);
#pragma unroll (kNorm ? 1 : kSteps / 2)
    for (int j = 0; j < kSteps; ++j) {
        const float factor = kNorm ? __shfl_sync(0xffffffffu, factors, (lane & 24) + j) : 1.0f;
        if (!(mine >> j & 1)) continue;
        const Raw again = load(j);
        const int position = position_of(j);
        uint32_t a[2], b[2];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            float v[8];
            turned(again, position, factor, part, v);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float2 z = __fmul2_rn(make_float2(v[e], v[e + 1]), make_float2(inv, inv));
                v[e] = z.x;
                v[e + 1] = z.y;
            }
            place<kHalfLayout>(a, b, part, encode4<kCode>(v[0], v[1], v[2], v[3]), encode4<kCode>(v[4], v[5], v[6], v[7]));
        }
        if (!finite) a[0] = a[1] = b[0] = b[1] = 0;
        uint2* dst = reinterpret_cast<uint2*>(codes + (4 * j + sub) * kHeadDim);
        dst[at.a] = make_uint2(a[0], a[1]);
        dst[at.b] = make_uint2(b[0], b[1]);
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
template <bool kBf16, bool kHalfLayout, bool kNorm>
__device__ __forceinline__ void rotate_queries(const BlockAppendParams& p, int row, int head0) {
    const int lane = threadIdx.x & 31, sub = lane >> 3, i = lane & 7;
    const int rot = p.rotary_dim, end = min(head0 + p.q_heads, p.num_q_heads);
    const Chunks<kHalfLayout> at(i, rot);
    const char* src = static_cast<const char*>(p.q) + 2 * ((size_t)row * p.q_stride + sub * kHeadDim);
    char* dst = static_cast<char*>(p.q_out) + 2 * (((size_t)row * p.num_q_heads + sub) * kHeadDim);
    constexpr int kAhead = 2;   // steps of four heads in flight
    Raw raw[kAhead];
    auto load = [&](int h0) { return h0 + sub < end ? load_raw(src + h0 * (2 * kHeadDim), at.a, at.b) : Raw{}; };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) raw[j] = load(head0 + 4 * j);   // the rows do not wait for whose they are
    int b = row;
    if (p.cu_new) b = warp_find_last(p.batch, row, [&](int s) { return (long long)load_dep(p.cu_new + s); });
    Sequence s;
    if (!sequence(p, b, s) || row < s.lo || row >= s.lo + s.n) return;   // reported elsewhere
    int position = s.start + row - s.lo;
    if (rot && p.positions) position = load_dep(p.positions + row);
    const bool bad = rot && (position < 0 || position >= p.num_positions);
    if (bad && lane == 0) report(p, WC_DEV_BAD_POSITION);
    Trig trig[2];
#pragma unroll
    for (int part = 0; part < 2; ++part)
        if (at.rotated(part) && !bad) load_trig(p.cos_table, p.sin_table, (size_t)position * (rot >> 1) + at.first_pair(part), trig[part]);
    const float* weight = kNorm && !bad ? p.q_norm : nullptr;   // a bad row's are zeros
    auto rows = [&](auto with) {
        constexpr bool normed = decltype(with)::value;
        for (int h0 = head0; h0 < end; h0 += 4 * kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                float factor = 1.0f;
                if constexpr (normed) factor = quick_factor<kBf16>(raw[j], p.norm_eps);   // the warp together
                if (bad) raw[j] = {};
                uint4 a, b;
                finished_row<normed, kBf16, kBf16>(raw[j], at, weight, factor, !bad, trig, a, b);
                raw[j] = load(h0 + 4 * (j + kAhead));
                if (h0 + 4 * j + sub >= end) continue;
                uint4* out = reinterpret_cast<uint4*>(dst + (h0 + 4 * j) * (2 * kHeadDim));
                out[at.a] = a;
                out[at.b] = b;
            }
        }
    };
    if constexpr (kNorm) {
        if (weight) return rows(std::true_type{});
    }
    rows(std::false_type{});
}

template <int kCode, bool kBf16, bool kHalfLayout, bool kNorm>
__global__ void __launch_bounds__(kThreads, kNorm ? 7 : 8) block_append_kernel(const __grid_constant__ BlockAppendParams p) {
    grid_dep_launch();
    grid_dep_wait();
    const unsigned warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    // CTAs of pages lie among those of queries: theirs is a chain of loads, which the others' bytes hide
    const unsigned group = blockIdx.x / (unsigned)p.page_stride, member = blockIdx.x - group * p.page_stride;
    if (member == 0 && group < (unsigned)p.page_ctas) {
        const PageWork w(p, group, warp);
        if (w.task == (unsigned)p.page_tasks && w.head == 0 && w.side == 0) {   // one warp more reports the sequences that the others skip
            Sequence s;
            for (int b = threadIdx.x & 31; b < p.batch; b += 32) sequence<true>(p, b, s);
        }
        if (w.task >= (unsigned)p.page_tasks) return;
        append_page<kCode, kBf16, kHalfLayout, kNorm ? Norm::kUsual : Norm::kNone>(p, (int)w.task, w.head, w.side);
    } else {
        const unsigned t = (blockIdx.x - min(group + 1, (unsigned)p.page_ctas)) * kWarps + warp;
        const unsigned per = (p.num_q_heads + p.q_heads - 1) / p.q_heads, row = t / per;
        if (row >= (unsigned)p.n_tok) return;
        rotate_queries<kBf16, kHalfLayout, kNorm>(p, (int)row, (int)(t - row * per) * p.q_heads);
    }
}

}  // namespace

cudaError_t launch_block_append(const BlockAppendParams& params, int code, int act, int rope_layout, cudaStream_t stream) {
    BlockAppendParams p = params;
    const long long pages = p.cu_new ? (long long)p.n_tok / kPage + 2LL * p.batch : p.batch;
    // few tokens: eight heads a warp, in parallel; many: 32, behind one read of the angles
    p.q_heads = (long long)p.n_tok * p.num_q_heads >= 16384 ? 32 : 8;
    long long q_ctas = p.q ? ((long long)p.n_tok * ((p.num_q_heads + p.q_heads - 1) / p.q_heads) + kWarps - 1) / kWarps : 0;
    // A launch counts its warps in 32 bits: where pages times heads are more, it takes some of the heads.
    const long long most = (0x7FFFFFFFLL - q_ctas * kWarps - 2 * kWarps) / (2 * pages);
    if (most < 1) return cudaErrorInvalidConfiguration;
    p.page_tasks = (int)pages;
    long long page_ctas = 0;
    auto go = [&](auto code_of, auto bf16, auto half, auto norm) {
        return launch_pdl(block_append_kernel<code_of.value, bf16.value, half.value, norm.value>, dim3((unsigned)(page_ctas + q_ctas)), dim3(kThreads), 0,
                          stream, p);
    };
    auto pick = [](bool on, auto next) { return on ? next(std::true_type{}) : next(std::false_type{}); };
    auto with = [&](auto code_of) {
        return pick(act == WC_ACT_BF16, [&](auto bf16) {
            return pick(rope_layout == WC_ROPE_HALF, [&](auto half) {
                return pick(p.k_norm || p.q_norm, [&](auto norm) { return go(code_of, bf16, half, norm); });
            });
        });
    };
    for (p.page_head0 = 0; p.page_head0 < p.num_kv_heads; p.page_head0 += p.page_heads) {
        p.page_heads = (int)std::min<long long>(most, p.num_kv_heads - p.page_head0);
        page_ctas = (pages * 2 * p.page_heads + 1 + kWarps - 1) / kWarps;
        p.page_ctas = (int)page_ctas;
        p.page_stride = (int)((page_ctas + q_ctas) / page_ctas);
        const cudaError_t e = code == WC_CODE_INT8 ? with(std::integral_constant<int, WC_CODE_INT8>{}) : with(std::integral_constant<int, WC_CODE_E4M3>{});
        if (e != cudaSuccess) return e;
        q_ctas = 0;   // with the first heads
    }
    return cudaSuccess;
}

}  // namespace wc
