// The block-scaled 8-bit cache: launch parameters and device helpers of its kernels.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>

#include "wc_kernels.cuh"

namespace wc {

struct BlockAppendParams {
    const void* x[2];          // new keys and values, rows of x_stride elements per token
    int64_t x_stride[2];
    const void* q;             // queries to rotate, nullptr: none
    int64_t q_stride;
    void* q_out;
    const int32_t* cu_new;     // nullptr: one token per sequence
    const int32_t* block_table;
    const int32_t* ctx_lens;
    const int32_t* positions;  // nullptr: the logical positions
    const float* cos_table;
    const float* sin_table;
    uint8_t* codes[2];
    float* scale[2];
    uint32_t* dev_status;      // optional
    int32_t n_tok, batch, max_pages, num_pages, num_q_heads, num_kv_heads, num_positions, rotary_dim;
    int32_t page_tasks;        // upper bound of the pages written, over all sequences
    int32_t page_ctas;         // CTAs of the page tasks; those after them rotate queries
    int32_t q_heads;           // query heads of one token that a warp takes
};

struct BlockAttentionParams {
    const void* q;
    int64_t q_stride;
    const int32_t* cu_q;       // nullptr: one token per sequence
    const int32_t* block_table;
    const int32_t* ctx_lens;
    const uint8_t* codes[2];
    const float* scale[2];     // nullptr: 1
    void* out;
    float* lse;                // optional
    uint32_t* status;
    float* partials;
    float scale_log2;          // softmax_scale * log2(e)
    int32_t n_tok, batch, max_pages, num_pages, num_q_heads, num_kv_heads, group, causal;
    int32_t bf16;              // element type of q and out
};

cudaError_t launch_block_append(const BlockAppendParams& p, int code, int act, int rope_layout, cudaStream_t stream);
// Sequences of one launch of the decode: their page counts' sums sit in shared memory.
constexpr int kDecodeBatch = 2048;
// A workspace: status word (256 bytes), the decode's arrival counts (a place of their own: they are 0 between
// calls), then what either kernel needs.
inline size_t block_arrived_bytes(int num_sms) { return ((size_t)num_sms * sizeof(int) + 255) & ~(size_t)255; }
size_t block_decode_workspace(int group, int num_sms);
cudaError_t launch_block_decode(const BlockAttentionParams& p, int code, int num_sms, cudaStream_t stream);   // group <= kMaxGroup
size_t block_extend_workspace(int n_tok, int num_q_heads, int num_sms);
cudaError_t launch_block_extend(const BlockAttentionParams& p, int code, int num_sms, cudaStream_t stream);

// ---- device helpers ---------------------------------------------------------------------------

__device__ __forceinline__ float2 h2_to_float2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// Two elements of act_type (fp16 or bf16) as fp32: exact.
template <bool kBf16>
__device__ __forceinline__ float2 act2_to_float2(uint32_t w) {
    if constexpr (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    else return h2_to_float2(w);
}

template <bool kBf16>
__device__ __forceinline__ uint32_t float2_to_act2(float lo, float hi) {
    if constexpr (kBf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        return pack_h2(lo, hi);
    }
}

// Four codes of a word as two exact half2 (codes 0, 1 and 2, 3).
template <int kCode>
__device__ __forceinline__ void codes4_to_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (kCode == WC_CODE_INT8) {
        const uint32_t x = w ^ 0x80808080u;
        lo = s8x2_to_h2(x, 0x4140u);
        hi = s8x2_to_h2(x, 0x4342u);
    } else {
        lo = e4m3x2_to_h2(w);
        hi = e4m3x2_to_h2(w >> 16);
    }
}

__device__ __forceinline__ uint16_t float_to_act(float x, bool bf16) {
    return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}

// A page's value scale below this (0, as a rule; the append makes none) counts as 0: its codes are taken as 0.  Smaller
// ones' reciprocals could take the sum of weights past fp32's range.  The kernels work with a scale's
// logarithm and reciprocal, so a small one stands in for it: its page's weights enter the running maximum of weighted values
// multiplied by it, and the sum of weights divided by it again.  A page of scale s keeps the maximum unless the other's
// logits (log2) are 80 + log2(s) above its own (with 1 for a stand-in, a sink of zero values took usual weights out of
// fp16's range), and the sum of weights holds what is above 2^(log2(s) - 53) of its own.
constexpr float kLeastValueScale = 0x1p-100f, kNoValueScale = 0x1p-80f;

// Weights 2^(y - m) are rounded to fp16 for the second product.  The frame m is put kHeadroom below the largest y, and moves
// when one passes it by kTopWeight: the largest weight lies in [2^7, 2^15], and others keep all their bits down to 2^-21
// of it, some to 2^-32 (from 1 on: 2^-14 and 2^-25, and what a sharp head gives to many tokens in all was lost below).  2^15
// leaves fp16's range a factor of 2 for what fp32 rounds off exponents: those of logits up to 2^22.
constexpr float kHeadroom = 7.0f, kTopWeight = 15.0f;
// The sum of weights l is kept times 2^-10: with value scales from 2^-100 on and 2^20 tokens it stays within fp32's range, and
// so do the reciprocals of the largest scales.
constexpr float kSumUnit = 0x1p-10f;

// log(sum of 2^m l), -inf for an empty sum.
__device__ __forceinline__ float log_sum(float m, float l) {
    return l == 0.0f ? -INFINITY : (m + 10.0f + log2f(l)) * 0.6931471805599453f;
}
// What sums of weighted values are multiplied with.
__device__ __forceinline__ float output_factor(float l) { return l == 0.0f ? 0.0f : __frcp_rn(l) * kSumUnit; }

// A warp's output row: four channels a lane, divided by the sum of weights.
__device__ __forceinline__ void store_output(const BlockAttentionParams& p, size_t cell, int lane, float4 o, float m, float l) {
    const float f = output_factor(l);
    const uint32_t lo = p.bf16 ? float2_to_act2<true>(o.x * f, o.y * f) : pack_h2(o.x * f, o.y * f);
    const uint32_t hi = p.bf16 ? float2_to_act2<true>(o.z * f, o.w * f) : pack_h2(o.z * f, o.w * f);
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + cell * kHeadDim)[lane] = make_uint2(lo, hi);
    if (p.lse && lane == 0) p.lse[cell] = log_sum(m, l);
}

// bf16 rows as fp16: times a power of two that puts the row's largest value below 2^15, so that all of bf16's
// bits stay but those below 2^-39 of the largest.  top: the largest of the row's words without signs, per half (as
// integers).  Rows of zeros, infinities and NaN are converted as they are.  undo: the inverse factor.
__device__ __forceinline__ float bf16_scale(uint32_t top, float& undo) {
    top = max(top << 16, top & 0xFFFF0000u);
    int e = (int)(top >> 23) - 127;   // the largest is below 2^(e + 1)
    if (top == 0 || e == 128) e = 14;
    const int shift = max(min(14 - e, 126), -126);
    undo = __uint_as_float((uint32_t)(127 - shift) << 23);
    return __uint_as_float((uint32_t)(127 + shift) << 23);
}
__device__ __forceinline__ uint32_t scaled_bf16(uint32_t w, float by) {
    const float2 f = act2_to_float2<true>(w);
    return pack_h2(f.x * by, f.y * by);
}

// The sequence whose first[b] is the last one <= x, for ascending first(0) <= x; a warp searches together.  Where first does
// not ascend, the last one of those that begin with first(0) and are <= x, so that ranges that cannot be do not hide the ones
// before them (of up to 32).
template <typename F>
__device__ __forceinline__ int warp_find_last(int n, long long x, F first) {
    int lo = 0;
    for (int len = n; len > 1;) {
        const int step = (len + 31) / 32;
        const int at = lo + (threadIdx.x & 31) * step;
        const bool le = at < lo + len && first(at) <= x;
        const int k = __clz(__brev(~__ballot_sync(0xffffffffu, le))) - 1;   // lane 0 holds by assumption
        const int next = lo + max(k, 0) * step;
        len = min(step, lo + len - next);
        lo = next;
    }
    return lo;
}

}  // namespace wc
