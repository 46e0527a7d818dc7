// Attention over the block-scaled cache, one CTA per (query token, KV head).
#include "block_common.cuh"

namespace wc {

namespace {

constexpr int kWarps = 4;

template <int kCode>
__global__ void __launch_bounds__(kWarps * 32) block_attention_simple_kernel(const __grid_constant__ BlockAttentionParams p) {
    grid_dep_launch();
    grid_dep_wait();
    __shared__ float q[kHeadDim], part[kWarps][kHeadDim + 2];
    const int row = blockIdx.x, head = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int b = row, lo = row, hi = row + 1;
    if (p.cu_q) {
        if (row == 0 && head == 0)   // one CTA reports the ranges that cannot be
            for (int s = threadIdx.x; s < p.batch; s += blockDim.x) {
                const int x = load_dep(p.cu_q + s), y = load_dep(p.cu_q + s + 1);
                if (x < 0 || y < x || y > p.n_tok) atomicOr(p.status, WC_DEV_BAD_ROWS);
            }
        b = warp_find_last(p.batch, row, [&](int s) { return (long long)load_dep(p.cu_q + s); });
        lo = load_dep(p.cu_q + b);
        hi = load_dep(p.cu_q + b + 1);
    }
    if (lo < 0 || hi > p.n_tok || row < lo || row >= hi) return;
    int ctx = load_dep(p.ctx_lens + b);
    if (ctx < 0 || ctx > (long long)p.max_pages * kPage) {
        if (threadIdx.x == 0) atomicOr(p.status, WC_DEV_BAD_CTX);
        ctx = 0;
    }
    const int end = p.cu_q && p.causal ? max(0, ctx - (hi - lo) + (row - lo) + 1) : ctx;   // keys seen
    for (int g = 0; g < p.group; ++g) {
        const int hq = head * p.group + g;
        __syncthreads();
        const uint16_t raw = static_cast<const uint16_t*>(p.q)[(size_t)row * p.q_stride + (size_t)hq * kHeadDim + threadIdx.x];
        q[threadIdx.x] = p.bf16 ? __uint_as_float((uint32_t)raw << 16) : __half2float(__ushort_as_half(raw));
        __syncthreads();
        float m = -INFINITY, l = 0.0f, acc[4] = {};
        for (int page = warp; page * kPage < end; page += kWarps) {
            const int phys = load_dep(p.block_table + (size_t)b * p.max_pages + page);
            if (phys < 0 || phys >= p.num_pages) {
                if (lane == 0) atomicOr(p.status, WC_DEV_BAD_PAGE);
                continue;
            }
            const size_t block = (size_t)phys * p.num_kv_heads + head;
            const float ks = p.scale[0] ? load_dep(p.scale[0] + block) : 1.0f, vs = p.scale[1] ? load_dep(p.scale[1] + block) : 1.0f;
            const uint32_t* kc = reinterpret_cast<const uint32_t*>(p.codes[0] + (block * kPage + (lane >> 1)) * kHeadDim) + 16 * (lane & 1);
            float t = 0.0f;
            for (int w = 0; w < 16; ++w) {
                uint32_t a, c;
                codes4_to_h2<kCode>(load_dep(kc + w), a, c);
                const float2 x = h2_to_float2(a), y = h2_to_float2(c);
                const float* qw = q + 64 * (lane & 1) + 4 * w;
                t += x.x * qw[0] + x.y * qw[1] + y.x * qw[2] + y.y * qw[3];
            }
            t += __shfl_xor_sync(0xffffffffu, t, 1);
            t *= ks * p.scale_log2;
            if (page * kPage + (lane >> 1) >= end) t = -INFINITY;
            float top = t;
#pragma unroll
            for (int o = 2; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float next = fmaxf(m, top), at = next == -INFINITY ? 0.0f : next;
            const float again = exp2f(m - at), e = exp2f(t - at);
            m = next;
            l = l * again + (lane & 1 ? 0.0f : e);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] *= again;
            const uint32_t* vc = reinterpret_cast<const uint32_t*>(p.codes[1] + block * kPage * kHeadDim) + lane;
            for (int r = 0; r < min(kPage, end - page * kPage); ++r) {
                const float pr = __shfl_sync(0xffffffffu, e, 2 * r) * vs;
                uint32_t a, c;
                codes4_to_h2<kCode>(load_dep(vc + r * (kHeadDim / 4)), a, c);
                const float2 x = h2_to_float2(a), y = h2_to_float2(c);
                acc[0] += pr * x.x;
                acc[1] += pr * x.y;
                acc[2] += pr * y.x;
                acc[3] += pr * y.y;
            }
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) part[warp][4 * lane + j] = acc[j];
        if (lane == 0) part[warp][kHeadDim] = m, part[warp][kHeadDim + 1] = l;
        __syncthreads();
        float top = -INFINITY, sum = 0.0f, o = 0.0f;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, part[w][kHeadDim]);
        for (int w = 0; w < kWarps; ++w) {
            const float f = exp2f(part[w][kHeadDim] - (top == -INFINITY ? 0.0f : top));
            sum += f * part[w][kHeadDim + 1];
            o += f * part[w][threadIdx.x];
        }
        o = sum == 0.0f ? 0.0f : o / sum;
        const size_t cell = (size_t)row * p.num_q_heads + hq;
        static_cast<uint16_t*>(p.out)[cell * kHeadDim + threadIdx.x] =
            p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(o)) : __half_as_ushort(__float2half_rn(o));
        if (p.lse && threadIdx.x == 0) p.lse[cell] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace

cudaError_t launch_block_attention_simple(const BlockAttentionParams& p, int code, cudaStream_t stream) {
    const dim3 grid(p.n_tok, p.num_kv_heads), block(kWarps * 32);
    return code == WC_CODE_INT8 ? launch_pdl(block_attention_simple_kernel<WC_CODE_INT8>, grid, block, 0, stream, p)
                                : launch_pdl(block_attention_simple_kernel<WC_CODE_E4M3>, grid, block, 0, stream, p);
}

}  // namespace wc
