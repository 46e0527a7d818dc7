// extern "C" boundary of the block-scaled cache: host-side argument checks and kernel launches.
#include <cmath>

#include "api_checks.h"
#include "block_common.cuh"

using wc::aligned16;
using wc::cuda_fail;
using wc::fail;

namespace {

constexpr int kMaxBlockGroup = 128;
// The kernels' int32 positions reach up to a tile of keys past a context's end.
constexpr int kMaxTablePages = (1 << 27) - 64;
constexpr double kLog2e = 1.4426950408889634;

wc_status check_block_desc(const wc_block_desc* d) {
    if (!d) return fail(WC_ERR_INVALID_ARG, "desc is NULL");
    if (d->head_dim != wc::kHeadDim) return fail(WC_ERR_UNSUPPORTED, "head_dim must be 128 (got %d)", d->head_dim);
    if (d->page_size != wc::kPage) return fail(WC_ERR_UNSUPPORTED, "page_size must be 16 (got %d)", d->page_size);
    if (d->num_kv_heads < 1 || d->num_kv_heads > 65535)
        return fail(WC_ERR_INVALID_ARG, "num_kv_heads must be in [1, 65535] (got %d)", d->num_kv_heads);
    if (d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads != 0)
        return fail(WC_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)",
                    d->num_q_heads, d->num_kv_heads);
    if (d->num_q_heads / d->num_kv_heads > kMaxBlockGroup)
        return fail(WC_ERR_UNSUPPORTED, "num_q_heads / num_kv_heads must be at most %d (got %d)", kMaxBlockGroup,
                    d->num_q_heads / d->num_kv_heads);
    if (d->num_pages < 1) return fail(WC_ERR_INVALID_ARG, "num_pages must be positive (got %d)", d->num_pages);
    if ((long long)d->num_pages * wc::kPage > 0x7FFFFFFFLL || (long long)d->num_pages * d->num_kv_heads > 0x7FFFFFFFLL)
        return fail(WC_ERR_UNSUPPORTED, "num_pages * 16 and num_pages * num_kv_heads must fit in int32");
    if (d->code != WC_CODE_INT8 && d->code != WC_CODE_E4M3) return fail(WC_ERR_UNSUPPORTED, "unknown code %d", d->code);
    if (d->rope_layout != WC_ROPE_HALF && d->rope_layout != WC_ROPE_INTERLEAVED)
        return fail(WC_ERR_UNSUPPORTED, "unknown rope_layout %d", d->rope_layout);
    if (d->rotary_dim < 0 || d->rotary_dim > wc::kHeadDim || d->rotary_dim % 16 != 0)
        return fail(WC_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 up to 128 (got %d)", d->rotary_dim);
    return WC_OK;
}

wc_status check_positions(const wc_block_desc* d, int32_t n_tok, int32_t max_pages) {
    if ((long long)max_pages * d->num_kv_heads > 0x7FFFFFFFLL)
        return fail(WC_ERR_UNSUPPORTED, "max_pages * num_kv_heads must fit in int32");
    if ((long long)n_tok * d->num_q_heads > 0x7FFFFFFFLL)
        return fail(WC_ERR_UNSUPPORTED, "n_tok * num_q_heads must fit in int32");
    return WC_OK;
}

wc_status check_sizes(int32_t act_type, int32_t batch, int32_t n_tok, int32_t max_pages) {
    if (act_type != WC_ACT_FP16 && act_type != WC_ACT_BF16) return fail(WC_ERR_UNSUPPORTED, "unknown act_type %d", act_type);
    if (batch < 0 || batch > 65535) return fail(WC_ERR_INVALID_ARG, "batch must be in [0, 65535] (got %d)", batch);
    if (n_tok < 0) return fail(WC_ERR_INVALID_ARG, "n_tok must be >= 0 (got %d)", n_tok);
    if (max_pages < 1) return fail(WC_ERR_INVALID_ARG, "max_pages must be positive (got %d)", max_pages);
    if (max_pages > kMaxTablePages)
        return fail(WC_ERR_UNSUPPORTED, "max_pages must be at most %d (got %d)", kMaxTablePages, max_pages);
    return WC_OK;
}

// Rows of `heads` heads, `stride` elements from one token to the next.
wc_status check_rows(const char* name, const void* x, int64_t stride, int32_t heads) {
    if (!x) return fail(WC_ERR_INVALID_ARG, "%s must not be NULL", name);
    if (!aligned16(x)) return fail(WC_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    if (stride < (int64_t)heads * wc::kHeadDim || stride % 8 != 0 || stride > (int64_t(1) << 40))
        return fail(WC_ERR_INVALID_ARG, "%s's token stride must be a multiple of 8 of at least %lld elements (got %lld)", name,
                    (long long)heads * wc::kHeadDim, (long long)stride);
    return WC_OK;
}

wc_status check_block_cache(const void* kc, const void* vc, const float* ks, const float* vs) {
    if (!kc || !vc) return fail(WC_ERR_INVALID_ARG, "cache pointers must not be NULL");
    if (!aligned16(kc) || !aligned16(vc)) return fail(WC_ERR_INVALID_ARG, "cache arrays must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(ks) & 3u) || (reinterpret_cast<uintptr_t>(vs) & 3u))
        return fail(WC_ERR_INVALID_ARG, "k_scale and v_scale must be 4-byte aligned");
    return WC_OK;
}

// The same for fewer sequences, tokens and pages or less.
size_t workspace_bytes_for(const wc_block_desc* desc, int32_t n_tok, int num_sms) {
    const int group = desc->num_q_heads / desc->num_kv_heads;
    const size_t decode = group <= wc::kMaxGroup ? wc::block_decode_workspace(group, num_sms) : 0;
    const size_t extend = wc::block_extend_workspace(n_tok, desc->num_q_heads, num_sms);
    return (256 + wc::block_arrived_bytes(num_sms) + std::max(decode, extend) + 255) & ~(size_t)255;
}

wc_status attention(const wc_block_desc* desc, int32_t act_type, const void* q, int64_t q_stride, int32_t n_tok,
                    const int32_t* cu_q, bool ragged, const int32_t* block_table, int32_t max_pages, const int32_t* ctx_lens,
                    int32_t batch, const void* k_codes, const void* v_codes, const float* k_scale, const float* v_scale,
                    float softmax_scale, int32_t causal, void* out, float* lse, void* workspace, size_t workspace_bytes,
                    void* stream) {
    if (wc_status st = check_block_desc(desc)) return st;
    if (wc_status st = check_sizes(act_type, batch, n_tok, max_pages)) return st;
    if (wc_status st = check_positions(desc, n_tok, max_pages)) return st;
    if (!(softmax_scale > 0.0f) || !std::isfinite(softmax_scale))
        return fail(WC_ERR_INVALID_ARG, "softmax_scale must be positive and finite (got %g)", (double)softmax_scale);
    if (!k_scale != !v_scale) return fail(WC_ERR_INVALID_ARG, "k_scale and v_scale are NULL together or not at all");
    if (!k_scale && desc->code != WC_CODE_E4M3)
        return fail(WC_ERR_INVALID_ARG, "k_scale and v_scale may be NULL for e4m3 codes only");
    if (batch == 0 || n_tok == 0) return WC_OK;
    if (wc_status st = check_rows("q", q, q_stride, desc->num_q_heads)) return st;
    if (!block_table || !ctx_lens || !out || !workspace || (ragged && !cu_q))
        return fail(WC_ERR_INVALID_ARG, "%sblock_table, ctx_lens, out, workspace must not be NULL", ragged ? "cu_q, " : "");
    if (!aligned16(out)) return fail(WC_ERR_INVALID_ARG, "out must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
        return fail(WC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (wc_status st = check_block_cache(k_codes, v_codes, k_scale, v_scale)) return st;
    int sms = 0;
    if (wc::current_sm_count(&sms) != 0) return fail(WC_ERR_CUDA, "cannot query the current device");
    const size_t need = workspace_bytes_for(desc, n_tok, sms);
    if (workspace_bytes < need) return fail(WC_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", workspace_bytes, need);
    wc::BlockAttentionParams p = {};
    p.q = q;
    p.q_stride = q_stride;
    p.cu_q = cu_q;
    p.block_table = block_table;
    p.ctx_lens = ctx_lens;
    p.codes[0] = static_cast<const uint8_t*>(k_codes);
    p.codes[1] = static_cast<const uint8_t*>(v_codes);
    p.scale[0] = k_scale;
    p.scale[1] = v_scale;
    p.out = out;
    p.lse = lse;
    p.status = static_cast<uint32_t*>(workspace);
    p.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 256);
    p.scale_log2 = (float)((double)softmax_scale * kLog2e);
    p.n_tok = n_tok;
    p.batch = batch;
    p.max_pages = max_pages;
    p.num_pages = desc->num_pages;
    p.num_q_heads = desc->num_q_heads;
    p.num_kv_heads = desc->num_kv_heads;
    p.group = desc->num_q_heads / desc->num_kv_heads;
    p.causal = causal != 0;
    p.bf16 = act_type == WC_ACT_BF16;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = !ragged && p.group <= wc::kMaxGroup ? wc::launch_block_decode(p, desc->code, sms, s)
                                                               : wc::launch_block_extend(p, desc->code, sms, s);
    return e == cudaSuccess ? WC_OK : cuda_fail(e, "block attention kernel launch");
}

}  // namespace

extern "C" {

wc_status wc_block_append(const wc_block_desc* desc, int32_t act_type, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, const void* q, int64_t q_stride, void* q_out, int32_t n_tok,
                          const int32_t* cu_new, const int32_t* block_table, int32_t max_pages, const int32_t* ctx_lens,
                          int32_t batch, const int32_t* positions, const float* cos_table, const float* sin_table,
                          int32_t num_positions, void* k_codes, void* v_codes, float* k_scale, float* v_scale,
                          uint32_t* dev_status, void* stream) {
    if (wc_status st = check_block_desc(desc)) return st;
    if (wc_status st = check_sizes(act_type, batch, n_tok, max_pages)) return st;
    if (!cu_new && n_tok != batch)
        return fail(WC_ERR_INVALID_ARG, "cu_new may be NULL only with one token per sequence (n_tok %d, batch %d)", n_tok, batch);
    if (desc->rotary_dim > 0) {
        if (!cos_table || !sin_table || num_positions < 1)
            return fail(WC_ERR_INVALID_ARG, "cos_table, sin_table and num_positions are required when rotary_dim > 0");
        if (!aligned16(cos_table) || !aligned16(sin_table))
            return fail(WC_ERR_INVALID_ARG, "cos_table and sin_table must be 16-byte aligned");
    }
    if (!q != !q_out) return fail(WC_ERR_INVALID_ARG, "q and q_out are NULL together or not at all");
    if (batch == 0 || n_tok == 0) return WC_OK;
    if (wc_status st = check_rows("k", k, k_stride, desc->num_kv_heads)) return st;
    if (wc_status st = check_rows("v", v, v_stride, desc->num_kv_heads)) return st;
    if (q) {
        if (wc_status st = check_rows("q", q, q_stride, desc->num_q_heads)) return st;
        if (!aligned16(q_out)) return fail(WC_ERR_INVALID_ARG, "q_out must be 16-byte aligned");
    }
    if (!block_table || !ctx_lens) return fail(WC_ERR_INVALID_ARG, "block_table and ctx_lens must not be NULL");
    if (wc_status st = check_block_cache(k_codes, v_codes, k_scale, v_scale)) return st;
    if (!k_scale || !v_scale) return fail(WC_ERR_INVALID_ARG, "k_scale and v_scale must not be NULL");
    wc::BlockAppendParams p = {};
    p.x[0] = k;
    p.x[1] = v;
    p.x_stride[0] = k_stride;
    p.x_stride[1] = v_stride;
    p.q = q;
    p.q_stride = q_stride;
    p.q_out = q_out;
    p.cu_new = cu_new;
    p.block_table = block_table;
    p.ctx_lens = ctx_lens;
    p.positions = positions;
    p.cos_table = cos_table;
    p.sin_table = sin_table;
    p.codes[0] = static_cast<uint8_t*>(k_codes);
    p.codes[1] = static_cast<uint8_t*>(v_codes);
    p.scale[0] = k_scale;
    p.scale[1] = v_scale;
    p.dev_status = dev_status;
    p.n_tok = n_tok;
    p.batch = batch;
    p.max_pages = max_pages;
    p.num_pages = desc->num_pages;
    p.num_q_heads = desc->num_q_heads;
    p.num_kv_heads = desc->num_kv_heads;
    p.num_positions = num_positions;
    p.rotary_dim = desc->rotary_dim;
    const cudaError_t e =
        wc::launch_block_append(p, desc->code, act_type, desc->rope_layout, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? WC_OK : cuda_fail(e, "block append kernel launch");
}

size_t wc_block_workspace_size(const wc_block_desc* desc, int32_t batch, int32_t n_tok, int32_t max_pages) {
    if (check_block_desc(desc) != WC_OK || check_sizes(WC_ACT_FP16, batch, n_tok, max_pages) != WC_OK ||
        check_positions(desc, n_tok, max_pages) != WC_OK)
        return 0;
    if (batch < 1 || n_tok < 1) {
        fail(WC_ERR_INVALID_ARG, "batch and n_tok must be positive");
        return 0;
    }
    int sms = 0;
    if (wc::current_sm_count(&sms) != 0) {
        fail(WC_ERR_CUDA, "no current CUDA device to size the workspace for");
        return 0;
    }
    return workspace_bytes_for(desc, n_tok, sms);
}

wc_status wc_block_decode_attention(const wc_block_desc* desc, int32_t act_type, const void* q, int64_t q_stride,
                                    const int32_t* block_table, int32_t max_pages, const int32_t* ctx_lens, int32_t batch,
                                    const void* k_codes, const void* v_codes, const float* k_scale, const float* v_scale,
                                    float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    return attention(desc, act_type, q, q_stride, batch, nullptr, false, block_table, max_pages, ctx_lens, batch, k_codes,
                     v_codes, k_scale, v_scale, softmax_scale, 0, out, lse, workspace, workspace_bytes, stream);
}

wc_status wc_block_extend_attention(const wc_block_desc* desc, int32_t act_type, const void* q, int64_t q_stride,
                                    int32_t n_tok, const int32_t* cu_q, const int32_t* block_table, int32_t max_pages,
                                    const int32_t* ctx_lens, int32_t batch, const void* k_codes, const void* v_codes,
                                    const float* k_scale, const float* v_scale, float softmax_scale, int32_t causal,
                                    void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return attention(desc, act_type, q, q_stride, n_tok, cu_q, true, block_table, max_pages, ctx_lens, batch, k_codes,
                     v_codes, k_scale, v_scale, softmax_scale, causal, out, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
