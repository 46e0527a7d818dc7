// Queries and keys normed for each head and rotated, ahead of a cache whose write takes keys as they are to be stored.
//
// A head's row r of 128 channels becomes rot(r w / sqrt(mean r^2 + eps)): one pass, bound by the bytes of the rows in and
// out.  Eight lanes hold a row (block_rotate.cuh) and a warp takes four heads of a token a step; a step's registers are loaded
// for the step two on as soon as it is written out, and 64 registers a thread leave 32 warps an SM.  Query and key heads are one
// list of steps, so that keys, of which there are few, do not leave a warp with a single load in flight.
//
// GB300, 28 query / 4 KV heads, 32768 tokens, fp16: 82 us, 6.75 TB/s of the 554 MB that it has to move (0.99 of the measured
// copy rate).  Tried: steps fetched two at a time, both written before the next two (86 us), three ahead with 24 warps an SM
// (90), four with 24 and spilled rows (89); 32 tokens of 32 heads 2.5 us between launches.  Rows without a
// norm have a path of their own.
#include "block_rotate.cuh"

namespace wc {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;

template <bool kBf16, bool kOutBf16, bool kHalfLayout>
__global__ void __launch_bounds__(kThreads, 8) qk_norm_rotate_kernel(const __grid_constant__ QkNormParams p) {
    grid_dep_launch();
    grid_dep_wait();
    const int lane = threadIdx.x & 31, sub = lane >> 3;
    const int q_steps = (p.heads[0] + 3) >> 2, all = q_steps + ((p.heads[1] + 3) >> 2), per = (all + p.warp_steps - 1) / p.warp_steps;
    const unsigned t = blockIdx.x * kWarps + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), row = t / (unsigned)per;
    if (row >= (unsigned)p.n_tok) return;
    const int step0 = (int)(t - row * per) * p.warp_steps, end = min(step0 + p.warp_steps, all);
    const Chunks<kHalfLayout> at(lane & 7, p.rotary_dim);
    constexpr int kAhead = 2;   // steps in flight
    // a lane's row of its first query head, its first key head
    auto rows = [&](auto* base, int64_t stride) { return base + 2 * (row * stride + sub * kHeadDim); };
    const char *q_src = rows(static_cast<const char*>(p.x[0]), p.x_stride[0]), *k_src = rows(static_cast<const char*>(p.x[1]), p.x_stride[1]);
    char *q_dst = rows(static_cast<char*>(p.out[0]), p.out_stride[0]), *k_dst = rows(static_cast<char*>(p.out[1]), p.out_stride[1]);
    Raw raw[kAhead];
    auto load = [&](int s) {
        const bool key = s >= q_steps;
        const int step = key ? s - q_steps : s;
        return s < end && 4 * step + sub < (key ? p.heads[1] : p.heads[0]) ? load_raw((key ? k_src : q_src) + step * (8 * kHeadDim), at.a, at.b) : Raw{};
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) raw[j] = load(step0 + j);
    const int position = p.rotary_dim ? load_dep(p.positions + row) : 0;
    const bool bad = p.rotary_dim && (position < 0 || position >= p.num_positions);
    if (bad && step0 == 0 && lane == 0 && p.dev_status) atomicOr(p.dev_status, WC_DEV_BAD_POSITION);
    Trig trig[2];
#pragma unroll
    for (int part = 0; part < 2; ++part)
        if (at.rotated(part) && !bad) load_trig(p.cos_table, p.sin_table, (size_t)position * (p.rotary_dim >> 1) + at.first_pair(part), trig[part]);
    for (int s0 = step0; s0 < end; s0 += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int s = s0 + j;
            const bool key = s >= q_steps;
            const int step = key ? s - q_steps : s;
            const float* weight = bad ? nullptr : key ? p.weight[1] : p.weight[0];   // a bad row's are zeros
            if (bad) raw[j] = {};
            uint4 a, b;
            if (weight) finished_row<true, kBf16, kOutBf16>(raw[j], at, weight, quick_factor<kBf16>(raw[j], p.eps), true, trig, a, b);
            else finished_row<false, kBf16, kOutBf16>(raw[j], at, nullptr, 1.0f, !bad, trig, a, b);
            raw[j] = load(s + kAhead);
            if (s >= end || 4 * step + sub >= (key ? p.heads[1] : p.heads[0])) continue;
            uint4* out = reinterpret_cast<uint4*>((key ? k_dst : q_dst) + step * (8 * kHeadDim));
            out[at.a] = a;
            out[at.b] = b;
        }
    }
}

}  // namespace

cudaError_t launch_qk_norm_rotate(const QkNormParams& params, int act, int out_act, int rope_layout, cudaStream_t stream) {
    QkNormParams p = params;
    const long long all = (p.heads[0] + 3) / 4 + (p.heads[1] + 3) / 4;
    // few rows: two steps a warp, in parallel; many: eight, behind one read of the angles
    p.warp_steps = p.n_tok * all >= 4096 ? 8 : 2;
    const long long ctas = (p.n_tok * ((all + p.warp_steps - 1) / p.warp_steps) + kWarps - 1) / kWarps;
    if (ctas * kWarps > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;   // tasks are counted in 32 bits
    auto pick = [](bool on, auto next) { return on ? next(std::true_type{}) : next(std::false_type{}); };
    return pick(act == WC_ACT_BF16, [&](auto bf16) {
        return pick(out_act == WC_ACT_BF16, [&](auto out_bf16) {
            return pick(rope_layout == WC_ROPE_HALF, [&](auto half) {
                return launch_pdl(qk_norm_rotate_kernel<bf16.value, out_bf16.value, half.value>, dim3((unsigned)ctas), dim3(kThreads), 0, stream, p);
            });
        });
    });
}

}  // namespace wc
