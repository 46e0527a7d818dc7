// Attention of several query tokens per sequence over the block-scaled cache.
//
// A CTA takes two tiles of 128 rows (query tokens x the G query heads of one KV head, token major) and
// walks the context in tiles of 128 keys (8 pages).  Both products run on the fifth-generation tensor
// cores with accumulators in TMEM:
//   S = Q K^T   both operands in shared memory, K's codes expanded to exact fp16
//   O += P V    P (fp16) from TMEM, in S's columns; V's codes as exact fp16 in shared memory
// Page scales stay out of the operands: with y = S ks + log2(vs) (ks the page's key scale times
// softmax_scale log2(e) and the row's query factor) 2^(y - m) is p vs, so O sums it times V's codes, and
// the sum of weights takes 2^(y - m) / vs.
// Warps 0-3 and 4-7: softmax of a tile each, a row per thread, one tile's while the tensor cores work on
// the other's; warps 8-11: codes to fp16 operands, two stages; warp 12: the MMAs; warp 13: block table, scales
// and the codes' way to shared memory by TMA (read with ordinary loads in rows of 64 bytes, the shape in which
// the operands are written without bank conflicts, they cost the MMAs' operand fetch a third of its time).
// A softmax thread moves its frame m (and its row of O) only when a weight would pass 2^15.
// Values that are NaN count as 0 in the second product wherever a row may not see them (its weight of 0 would not silence
// them); the rows that do see them get theirs at the end.
//
// GB300, 28 query / 4 KV heads: 4096 tokens at the end of 32k, int8 codes, fp16: 1208 us, 1493 TFLOP/s (0.79 of the
// measured cuBLAS bf16 rate); an 8k prompt from e4m3, bf16: 370 us, 1300 TFLOP/s (11 us of a CTA's 65 pass
// before its first and after its last product); 16 sequences of 5 drafted tokens at 4k to 8k 65.5 us, where
// one tile of rows leaves its softmax (1450 cycles a step) and its products (1100) to follow each other.  A step of two
// tiles costs 3050 cycles against the MMAs' 2050: what the issuing warp waits for is not hidden, as few MMAs queue.
// Tried and slower: a warp per tile issuing MMAs (1480 us, taking turns by a barrier 1391), the copies'
// addresses prefetched to L2 (1390), codes by ordinary loads (1610).
#include "block_common.cuh"
#include "decode_common.cuh"

namespace wc {

namespace {

constexpr int kTile = 128;                 // rows of a query tile, keys of a context tile
constexpr int kPages = kTile / kPage;      // pages of a context tile
constexpr int kTiles = 2;                  // query tiles of a CTA
constexpr int kSoftmaxWarps = 4 * kTiles, kConvertWarps = 4;
constexpr int kMmaWarp = kSoftmaxWarps + kConvertWarps, kLoadWarp = kMmaWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 4);
// Registers: 128 a thread at launch, 512 threads; a softmax thread holds 64 packed weights and 32 logits and
// takes what the others give: 256 x 176 + 128 x 80 + 128 x 80 = 512 x 128.
constexpr int kSoftmaxRegs = 176, kConvertRegs = 80, kMmaRegs = 80;
static_assert(kSoftmaxWarps * 32 * kSoftmaxRegs + kConvertWarps * 32 * kConvertRegs + 4 * 32 * kMmaRegs <= kThreads * 128);
constexpr int kOperand = kTile * kHeadDim * 2;   // bytes of a [128][128] fp16 operand: two blocks of 64 channels
constexpr int kBlock = kOperand / 2;
constexpr int kCodes = kTile * kHeadDim;         // bytes of a context tile's keys, or values
constexpr int kMetaStages = 4;
constexpr float kNoMax = -3e38f;
constexpr uint32_t kTmemColumns = 512, kOutColumn = 256;   // S (and P) of tile t at 128 t, O at 256 + 128 t

struct Meta {   // of a context tile's pages
    float ks[kPages], bias[kPages], inv[kPages];
    int tokens[2][kPages];   // rows of keys, of values that count (the others hold whatever was there, NaN codes among it)
};

struct Shared {
    uint64_t codes_full[2], codes_empty[2];   // staged keys, values
    uint64_t q_full, k_first, drained, k_empty[2], v_empty[2], s_full[kTiles], o_full[kTiles];
    // What the MMAs of tile t and step j wait for, in one barrier (their queue is short: what the issuing warp waits, the
    // tensor cores wait): P_t(j), V(j) and K(j + 1); by the parity of j, since the conversion runs ahead.
    uint64_t ready[kTiles][2];
    Meta meta[kMetaStages];
    uint32_t tmem;
    int abandoned;
    int any_nan, nan_page, nan_code[kHeadDim];   // positions of the first page, and of the first key in a channel, whose values are NaN
};
constexpr int kSmem = (kTiles + 4) * kOperand + 2 * kCodes + (int)sizeof(Shared) + 1024;
static_assert(kSmem <= 227 * 1024);

struct ExtendArgs {
    BlockAttentionParams p;
    CUtensorMap maps[2];   // keys, values
    int splits;
    float* part_o;    // [splits][n_tok * Hq][128]
    float2* part_ml;  // [splits][n_tok * Hq]
};

// ---- tcgen05 ------------------------------------------------------------------------------------

__device__ __forceinline__ void tmem_alloc(uint32_t* dst) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(kTmemColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* bar) {   // bar is arrived at when all MMAs so far are done
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// D (128 x 128 fp32) = or += A B, 16 deep.  Operand descriptors below.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Shared-memory operand with the 128-byte swizzle: rows of 64 channels, 8 rows in 1024 bytes.  Q and K: channels are the
// summed dimension, 64 of them a block.  V: keys are; the leading offset leads to the block of the next 64 channels.
// `low` is the descriptor's lower half (address and leading offset in units of 16 bytes).
__device__ __forceinline__ uint32_t operand_low(const void* at, uint32_t leading) { return smem_addr(at) >> 4 | (leading >> 4) << 16; }
__device__ __forceinline__ uint64_t operand(uint32_t low) {
    constexpr uint32_t kHigh = (1024 >> 4) | 1u << 14 | 2u << 29;   // 8 rows' stride, version, swizzle
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(low), "n"(kHigh));
    return d;
}
// fp16 operands, fp32 accumulator, 128 x 128; bit 16: B's rows are the summed dimension (V).
constexpr uint32_t kIdescQk = 1u << 4 | (kTile >> 3) << 17 | (kTile >> 4) << 24, kIdescPv = kIdescQk | 1u << 16;

__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 16 bytes to shared memory, of which the first `bytes` are read and the others 0.
__device__ __forceinline__ void copy_async(void* dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Bounded wait (about two seconds); once one gives up, all do.  A warp waits together and gets one answer: a lane that saw the
// barrier complete just as the others gave up would go on without them.
__device__ __forceinline__ bool wait(Shared& s, uint64_t* bar, uint32_t parity) {
    const uint32_t at = smem_addr(bar);
    uint64_t since = 0;
    for (uint32_t i = 1;; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok)
                     : "r"(at), "r"(parity)
                     : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
        if (i % 64 == 0) {
            uint64_t now;
            asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
            if (since == 0) since = now;
            const bool over = now - since > 2000000000ull;
            if (over) *reinterpret_cast<volatile int*>(&s.abandoned) = 1;
            if (__any_sync(0xffffffffu, over || *reinterpret_cast<volatile int*>(&s.abandoned))) return false;
        }
    }
}

// ---- work ---------------------------------------------------------------------------------------

// A CTA's rows: n_rows (token, query head) rows from `row0` of sequence b, which has n query rows from
// token `lo` on and ctx keys.
struct Work {
    int b, lo, n, ctx, row0, rows;
};

// Blocks first(b) = cu[b] G / 256 + b on are sequence b's (one more than its whole tile pairs).
__device__ __forceinline__ bool find_work(const BlockAttentionParams& p, int block, Work& w) {
    int tile;
    if (p.cu_q) {
        auto first = [&](int s) { return ((long long)load_dep(p.cu_q + s) * p.group) / (kTiles * kTile) + s; };
        w.b = warp_find_last(p.batch, block, first);
        tile = block - (int)first(w.b);
        w.lo = load_dep(p.cu_q + w.b);
        const int hi = load_dep(p.cu_q + w.b + 1);
        if (w.lo < 0 || hi < w.lo || hi > p.n_tok || tile < 0) return false;
        w.n = hi - w.lo;
    } else {
        w.b = w.lo = block;
        w.n = 1;
        tile = 0;
    }
    const long long row0 = (long long)tile * (kTiles * kTile), all = (long long)w.n * p.group;
    if (row0 >= all) return false;
    w.row0 = (int)row0;
    w.rows = (int)min((long long)(kTiles * kTile), all - row0);
    w.ctx = load_dep(p.ctx_lens + w.b);
    if (w.ctx < 0 || w.ctx > (long long)p.max_pages * kPage) {
        if (threadIdx.x == 0 && blockIdx.y == 0) atomicOr(p.status, WC_DEV_BAD_CTX);
        w.ctx = 0;
    }
    return true;
}

// Keys that row r of the sequence sees (those below).
__device__ __forceinline__ int keys_seen(const BlockAttentionParams& p, const Work& w, int r) {
    return p.causal ? max(0, min(w.ctx, w.ctx - w.n + r / p.group + 1)) : w.ctx;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// A tile's largest exponent alone: before a row's first tile.
__device__ __forceinline__ float first_max(uint32_t s_at, const Meta& meta, float factor, int sees) {
    float top = kNoMax;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
        uint32_t x[32];
        tmem_ld32(s_at + 32 * c, x);
        tmem_wait_ld();
        float best[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 32; i += 2)
            best[i >> 4] = max3(best[i >> 4], 32 * c + i < sees ? __uint_as_float(x[i]) : -INFINITY, 32 * c + i + 1 < sees ? __uint_as_float(x[i + 1]) : -INFINITY);
        top = max3(top, fmaf(best[0], meta.ks[2 * c] * factor, meta.bias[2 * c]), fmaf(best[1], meta.ks[2 * c + 1] * factor, meta.bias[2 * c + 1]));
    }
    return top;
}

// A row's weights for a context tile in the frame m: pairs as fp16 in y, their sum (in units of the
// weights p: value scales divided out) returned; top: the tile's largest exponent.  kMask: the row sees the first
// `sees` keys of the tile only.
template <bool kMask>
__device__ __forceinline__ float weights(uint32_t s_at, const Meta& meta, float factor, float m, int sees, uint32_t (&y)[kTile / 2], float& top) {
    float l = 0.0f;
    top = kNoMax;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t x[32];
        tmem_ld32(s_at + 32 * c, x);
        tmem_wait_ld();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = 2 * c + h;
            const float ks = meta.ks[page] * factor, bias = meta.bias[page], shift = bias - m;
            const float2 ks2 = make_float2(ks, ks), shift2 = make_float2(shift, shift);
            float best = -INFINITY;
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < kPage; i += 2) {
                const float2 v = make_float2(__uint_as_float(x[16 * h + i]), __uint_as_float(x[16 * h + i + 1]));
                const float2 e = __ffma2_rn(v, ks2, shift2);
                float2 pr = make_float2(fast_exp2(e.x), fast_exp2(e.y));
                if constexpr (kMask) {
                    const bool in0 = 16 * page + i < sees, in1 = 16 * page + i + 1 < sees;
                    best = max3(best, in0 ? v.x : -INFINITY, in1 ? v.y : -INFINITY);
                    pr.x = in0 ? pr.x : 0.0f;
                    pr.y = in1 ? pr.y : 0.0f;
                } else {
                    best = max3(best, v.x, v.y);
                }
                sum = __fadd2_rn(sum, pr);
                y[8 * page + i / 2] = pack_h2(pr.x, pr.y);
            }
            top = fmaxf(top, fmaf(best, ks, bias));
            l = fmaf(sum.x + sum.y, meta.inv[page], l);
        }
    }
    return l;
}

template <int kCode>
__global__ void __launch_bounds__(kThreads, 1) block_extend_kernel(const __grid_constant__ ExtendArgs args) {
    const BlockAttentionParams& p = args.p;
    extern __shared__ uint8_t raw[];
    uint8_t* ops = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    uint8_t *q_op = ops, *k_op = ops + kTiles * kOperand, *v_op = k_op + 2 * kOperand;
    uint8_t* staged = v_op + 2 * kOperand;
    Shared& s = *reinterpret_cast<Shared*>(staged + 2 * kCodes);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, head = blockIdx.y;   // warp: uniform
    if (threadIdx.x == 0) {
        mbar_init(&s.q_full, kSoftmaxWarps * 32);
        mbar_init(&s.drained, 1);
        mbar_init(&s.k_first, kConvertWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.codes_full[i], 1);
            mbar_init(&s.codes_empty[i], kConvertWarps);
            mbar_init(&s.k_empty[i], 1);
            mbar_init(&s.v_empty[i], 1);
            mbar_init(&s.s_full[i], 1);
            for (int k = 0; k < 2; ++k) mbar_init(&s.ready[i][k], 128 + 2 * kConvertWarps);
            mbar_init(&s.o_full[i], 1);
        }
        s.nan_page = INT_MAX;
        s.any_nan = s.abandoned = 0;
        fence_barrier_init();
    }
    if (threadIdx.x < kHeadDim) s.nan_code[threadIdx.x] = INT_MAX;
    grid_dep_wait();
    grid_dep_launch();
    if (p.cu_q && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)   // one CTA reports the ranges that cannot be
        for (int i = threadIdx.x; i < p.batch; i += kThreads) {
            const int x = load_dep(p.cu_q + i), y = load_dep(p.cu_q + i + 1);
            if (x < 0 || y < x || y > p.n_tok) atomicOr(p.status, WC_DEV_BAD_ROWS);
        }
    Work w;
    // the blocks of a sequence's last rows come first: with a causal mask theirs is the most work
    if (!find_work(p, gridDim.x - 1 - blockIdx.x, w)) return;
    const int tiles_q = w.rows > kTile ? 2 : 1;
    const int keys = keys_seen(p, w, w.row0 + w.rows - 1), context_tiles = (keys + kTile - 1) / kTile;
    const int t0 = (int)((long long)context_tiles * blockIdx.z / args.splits);
    const int t1 = (int)((long long)context_tiles * (blockIdx.z + 1) / args.splits), n = t1 - t0;
    if (warp == kMmaWarp && n > 0) tmem_alloc(&s.tmem);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, n > 0 ? s.tmem : 0, 0);

    if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int t = warp >> 2, thread = threadIdx.x & 127;
        // A warp moves whole rows: a half warp a row, every second one.  The first one's token and head; two rows on.
        const int chunk = lane & 15, warp_row = 32 * (warp & 3) + (lane >> 4);
        struct Row {
            int token, hq;   // hq: of the group
        };
        auto row_at = [&](int row) {
            const int r = w.row0 + t * kTile + row, i = (unsigned)r / (unsigned)p.group;
            return Row{w.lo + i, r - i * p.group};
        };
        const int step_token = 2u / (unsigned)p.group, step_hq = 2 - step_token * p.group;
        auto next_row = [&](Row& r) {
            r.token += step_token;
            r.hq += step_hq;
            if (r.hq >= p.group) {
                r.hq -= p.group;
                ++r.token;
            }
        };
        const int rows = w.rows - t * kTile;   // of this tile
        float m = kNoMax, l = 0.0f;
        bool ok = true;
        if (n > 0) {
            // Q by asynchronous copies (rows past the last: zeros); bf16 rows are then scaled by a power of two into
            // fp16's range, a lane a row.  Short loops: this code runs once, from a cold instruction cache.
            uint8_t* dst = q_op + t * kOperand + (chunk >> 3) * kBlock;
            Row at = row_at(warp_row);
#pragma unroll 2
            for (int i = 0; i < 16; ++i) {
                const int r = warp_row + 2 * i;
                const bool there = r < rows;
                const uint16_t* src = static_cast<const uint16_t*>(p.q) + (there ? (size_t)at.token * p.q_stride + (head * p.group + at.hq) * kHeadDim + 8 * chunk : 0);
                copy_async(dst + r * 128 + 16 * ((chunk & 7) ^ (r & 7)), src, there ? 16 : 0);
                next_row(at);
            }
            copy_async_wait();
            __syncwarp();
            float factor = 1.0f;
            if (p.bf16) {
                uint8_t* row = q_op + t * kOperand + thread * 128;
                auto word4 = [&](int i) { return reinterpret_cast<uint4*>(row + (i >> 3) * kBlock + 16 * ((i & 7) ^ (thread & 7))); };
                uint32_t top = 0;
#pragma unroll 8
                for (int i = 0; i < 16; ++i) {
                    const uint4 x = *word4(i);
                    top = __vmaxu2(__vmaxu2(top, __vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu)), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
                }
                const float up = bf16_scale(top, factor);
#pragma unroll 4
                for (int i = 0; i < 16; ++i) {
                    uint4* at = word4(i);
                    const uint4 x = *at;
                    *at = make_uint4(scaled_bf16(x.x, up), scaled_bf16(x.y, up), scaled_bf16(x.z, up), scaled_bf16(x.w, up));
                }
            }
            fence_async();
            arrive(&s.q_full);
            const bool live = thread < rows;
            const int seen = live ? keys_seen(p, w, w.row0 + t * kTile + thread) : 0;
            const int least = __reduce_min_sync(0xffffffffu, live ? seen : w.ctx);   // of the warp's rows
            if (!live) m = -kNoMax;   // rows past the last (zeros): nothing passes their frame, so they hold no warp up
            const uint32_t lanes = (uint32_t)(warp & 3) << 21, s_at = tmem + t * kTile + lanes, o_at = tmem + kOutColumn + t * kTile + lanes;
            if (t < tiles_q) {
                for (int j = 0; j < n && ok; ++j) {
                    ok = wait(s, &s.s_full[t], j & 1);   // and the O += P V before it is done
                    if (!ok) break;
                    fence_after();
                    const Meta& meta = s.meta[j % kMetaStages];
                    const int key0 = (t0 + j) * kTile, sees = seen - key0;
                    const bool masked = least < key0 + kTile;
                    uint32_t y[kTile / 2];
                    float sum;
                    if (j == 0) m = fmaxf(m, first_max(s_at, meta, factor, sees) - kHeadroom);
                    for (;;) {   // again where a logit passed the frame by too much: rarely
                        float top;
                        sum = masked ? weights<true>(s_at, meta, factor, m, sees, y, top) : weights<false>(s_at, meta, factor, m, sees, y, top);
                        if (!__any_sync(0xffffffffu, top > m + kTopWeight)) break;
                        const float now = fmaxf(m, top - kHeadroom), f = fast_exp2(m - now);
                        m = now;
                        l *= f;
                        if (j == 0) continue;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t x[32];
                            tmem_ld32(o_at + 32 * c, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
                            tmem_st32(o_at + 32 * c, x);
                        }
                    }
                    l += sum;
                    // P takes the place of S's first columns
                    tmem_st32(s_at, reinterpret_cast<const uint32_t(&)[32]>(y[0]));
                    tmem_st32(s_at + 32, reinterpret_cast<const uint32_t(&)[32]>(y[32]));
                    tmem_wait_st();
                    fence_before();
                    arrive(&s.ready[t][j & 1]);
                }
                ok = ok && wait(s, &s.o_full[t], 0);
                fence_after();
            }
        }
        const bool live = thread < rows, split = args.splits > 1;
        const Row mine = row_at(thread);
        const size_t cell = (size_t)mine.token * p.num_q_heads + head * p.group + mine.hq;
        const size_t part = (size_t)blockIdx.z * p.n_tok * p.num_q_heads + cell;
        if (ok && n > 0 && t < tiles_q) {
            const float f = output_factor(l);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t x[32];
                tmem_ld32(tmem + kOutColumn + t * kTile + ((uint32_t)(warp & 3) << 21) + 32 * c, x);
                tmem_wait_ld();
                if (live && split) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        reinterpret_cast<uint4*>(args.part_o + part * kHeadDim + 32 * c)[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                } else if (!split) {   // to Q's place, which the MMAs are done with
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t o[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float a = l == 0.0f ? 0.0f : __uint_as_float(x[8 * i + 2 * k]) * f;
                            const float b = l == 0.0f ? 0.0f : __uint_as_float(x[8 * i + 2 * k + 1]) * f;
                            o[k] = p.bf16 ? float2_to_act2<true>(a, b) : pack_h2(a, b);
                        }
                        *reinterpret_cast<uint4*>(q_op + t * kOperand + thread * 256 + 16 * ((4 * c + i) ^ (thread & 7))) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                }
            }
            if (!split) {
                __syncwarp();
                Row at = row_at(warp_row);
#pragma unroll 4
                for (int i = 0; i < 16; ++i) {
                    const int r = warp_row + 2 * i;
                    if (r < rows)
                        reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + ((size_t)at.token * p.num_q_heads + head * p.group + at.hq) * kHeadDim)[chunk] =
                            *reinterpret_cast<const uint4*>(q_op + t * kOperand + r * 256 + 16 * (chunk ^ (r & 7)));
                    next_row(at);
                }
            }
        } else if (n == 0 && live && !split) {   // no key in sight
            uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + cell * kHeadDim);
            for (int i = 0; i < 16; ++i) out[i] = make_uint4(0, 0, 0, 0);
        }
        if (live && split) args.part_ml[part] = make_float2(m, l);
        else if (live && p.lse) p.lse[cell] = log_sum(m, l);
        if (!ok && lane == 0) atomicOr(p.status, WC_DEV_TIMEOUT);
        fence_before();
    } else if (warp < kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kConvertRegs));
        const int cw = warp - kSoftmaxWarps, row = lane & 7, chunk = lane >> 3;   // a warp has two pages of the tile
        const int src0 = row * kHeadDim + 16 * (chunk ^ row), src1 = row * kHeadDim + 16 * ((chunk + 4) ^ row);
        const int dst0 = (32 * cw + row) * 128 + 16 * ((2 * chunk) ^ row), dst1 = (32 * cw + row) * 128 + 16 * ((2 * chunk + 1) ^ row);
        // 16 codes a lane and step (8 rows of 4 chunks, conflict-free in both layouts)
        const int all_see = keys_seen(p, w, w.row0);   // keys that every row sees
        // key0: position of the warp's first key
        auto expand = [&](int side, uint8_t* op, const int* tokens, int key0) {
            const int have0 = tokens[2 * cw], have1 = tokens[2 * cw + 1];
            uint8_t* src = staged + side * kCodes + cw * (2 * kPage * kHeadDim);
            uint4 x[8];   // read first: the compiler cannot tell the stores from the loads
            for (;;) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const uint4*>(src + (i >> 1) * 1024 + (i & 1 ? src1 : src0));
                if (min(have0, have1) < kPage) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (8 * ((i >> 1) & 1) + row >= (i < 4 ? have0 : have1)) x[i] = make_uint4(0, 0, 0, 0);
                }
                if (kCode != WC_CODE_E4M3 || side == 0 || key0 + 2 * kPage <= all_see) break;
                // a NaN among the values would reach the rows that do not see it, times 0
                uint32_t nan = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) nan |= (word_of(x[i], k) & 0x7F7F7F7Fu) + 0x01010101u;
                if (!__any_sync(0xffffffffu, nan & 0x80808080u)) break;
                s.any_nan = 1;   // rarely: it counts as 0 here, and is noted for the rows that see it
#pragma unroll 1
                for (int i = 0; i < 8 * 16; ++i) {
                    const int r = 8 * ((i >> 5) & 3) + row, c = chunk + 4 * ((i >> 4) & 1);   // row of the two pages, chunk of the row
                    uint8_t* code = src + r * kHeadDim + 16 * (c ^ row) + (i & 15);
                    if ((*code & 0x7F) != 0x7F) continue;
                    *code = 0;
                    if ((r & 15) < (r < kPage ? have0 : have1)) atomicMin(&s.nan_code[16 * c + (i & 15)], key0 + r);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t h[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) codes4_to_h2<kCode>(word_of(x[i], k), h[2 * k], h[2 * k + 1]);
                uint8_t* at = op + (i & 1) * kBlock + (i >> 1) * 1024;
                *reinterpret_cast<uint4*>(at + dst0) = make_uint4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<uint4*>(at + dst1) = make_uint4(h[4], h[5], h[6], h[7]);
            }
        };
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const int st = j & 1;
            const Meta& meta = s.meta[j % kMetaStages];
#pragma unroll 1
            for (int side = 0; side < 2 && ok; ++side) {
                if (j >= 2) ok = wait(s, side ? &s.v_empty[st] : &s.k_empty[st], ((j >> 1) - 1) & 1);
                ok = ok && wait(s, &s.codes_full[side], j & 1);
                if (!ok) break;
                expand(side, (side ? v_op : k_op) + st * kOperand, meta.tokens[side], (t0 + j) * kTile + 32 * cw);
                fence_async();
                __syncwarp();
                if (lane == 0) {
                    arrive(&s.codes_empty[side]);
                    if (side == 0 && j == 0) {
                        arrive(&s.k_first);
                    } else {   // V(j) for step j, K(j) for the step before
                        arrive(&s.ready[0][side ? st : st ^ 1]);
                        arrive(&s.ready[1][side ? st : st ^ 1]);
                    }
                }
            }
            if (!ok) break;
        }
        if (ok && n > 0 && lane == 0) {   // after the last step there are no keys to wait for
            arrive(&s.ready[0][(n - 1) & 1]);
            arrive(&s.ready[1][(n - 1) & 1]);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));
        if (warp == kMmaWarp && n > 0) {
            // the warp walks together, so that operands stay in uniform registers; one lane issues
            const uint32_t q_low = operand_low(q_op, 16), k_low = operand_low(k_op, 16), v_low = operand_low(v_op, kBlock);
            auto qk = [&](int t, int st) {
                const uint32_t q = q_low + t * (kOperand >> 4), k = k_low + st * (kOperand >> 4), d = tmem + t * kTile;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t off = ((i >> 2) * kBlock + (i & 3) * 32) >> 4;
                    mma_ss(d, operand(q + off), operand(k + off), kIdescQk, i > 0);
                }
                commit(&s.s_full[t]);
            };
            bool ok = wait(s, &s.q_full, 0) && wait(s, &s.k_first, 0);
            if (ok) {
                fence_after();
                if (elect_one()) {
                    qk(0, 0);
                    if (tiles_q > 1) qk(1, 0);
                    commit(&s.k_empty[0]);
                }
            }
#pragma unroll 1
            for (int j = 0; j < n && ok; ++j) {
                const int st = j & 1;
                const bool more = j + 1 < n;
#pragma unroll 1
                for (int t = 0; t < tiles_q && ok; ++t) {
                    ok = wait(s, &s.ready[t][st], (j >> 1) & 1);
                    if (!ok) break;
                    fence_after();
                    if (elect_one()) {
                        const uint32_t v = v_low + st * (kOperand >> 4), pr = tmem + t * kTile, d = pr + kOutColumn;
                        mma_ts(d, pr, operand(v), kIdescPv, j > 0);   // 16 keys each: 8 columns of P, 16 rows of V
#pragma unroll
                        for (int i = 1; i < 8; ++i) mma_ts(d, pr + 8 * i, operand(v + i * (2048 >> 4)), kIdescPv, true);
                        if (more) qk(t, st ^ 1);
                        else commit(&s.o_full[t]);
                        if (t == tiles_q - 1) {
                            commit(&s.v_empty[st]);
                            if (more) commit(&s.k_empty[st ^ 1]);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!ok) {   // what was issued ends before the accumulators are given back
                if (elect_one()) commit(&s.drained);
                (void)mbar_wait_bounded(&s.drained, 0);
            }
        } else if (warp == kLoadWarp && n > 0) {
            // lane i < 8 looks after page i of the tile: page numbers are read two tiles ahead, scales one
            const int page0 = t0 * kPages + lane, pages = lane < kPages ? min((w.ctx + kPage - 1) >> 4, t1 * kPages) : 0;
            const int32_t* table = p.block_table + (size_t)w.b * p.max_pages;
            auto number = [&](int j) { return page0 + j * kPages < pages ? load_dep(table + page0 + j * kPages) : 0; };
            auto valid = [&](int j, int phys) { return page0 + j * kPages < pages && phys >= 0 && phys < p.num_pages; };
            auto scale_at = [&](const float* scale, int phys, bool there) {
                return there && scale ? load_dep(scale + (size_t)phys * p.num_kv_heads + head) : 1.0f;
            };
            int phys = number(0), next = number(1);
            bool there = valid(0, phys), ok = true;
            float ks = scale_at(p.scale[0], phys, there), vs = scale_at(p.scale[1], phys, there);
            for (int j = 0; j < n; ++j) {
                const bool next_there = valid(j + 1, next);
                const float next_ks = scale_at(p.scale[0], next, next_there), next_vs = scale_at(p.scale[1], next, next_there);
                const int after = number(j + 2);
                const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, there)) * (kPage * kHeadDim);
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    if (j > 0) ok = ok && wait(s, &s.codes_empty[side], (j - 1) & 1);
                    if (!ok) break;
                    if (side == 0 && lane < kPages) {   // four tiles' worth: the tile four back is done with
                        Meta& meta = s.meta[j % kMetaStages];
                        const bool outside = !there && page0 + j * kPages < pages;
                        const int tokens = there ? min(kPage, w.ctx - (page0 + j * kPages) * kPage) : 0;
                        const bool lost = !(vs < INFINITY), no_values = lost || vs < kLeastValueScale;   // lost: infinity or NaN
                        const float of = no_values ? kNoValueScale : vs;
                        meta.ks[lane] = ks * p.scale_log2;
                        meta.bias[lane] = outside ? -INFINITY : log2f(of);
                        meta.inv[lane] = __frcp_rn(of) * kSumUnit;
                        meta.tokens[0][lane] = tokens;
                        meta.tokens[1][lane] = no_values ? 0 : tokens;
                        if (lost) {
                            atomicMin(&s.nan_page, (page0 + j * kPages) * kPage);
                            s.any_nan = 1;
                        }
                        if (outside) atomicOr(p.status, WC_DEV_BAD_PAGE);
                    }
                    __syncwarp();
                    if (elect_one()) mbar_arrive_expect_tx(&s.codes_full[side], bytes);
                    __syncwarp();
                    if (there) tma_page(staged + side * kCodes + lane * (kPage * kHeadDim), &args.maps[side], phys * p.num_kv_heads + head, &s.codes_full[side]);
                }
                if (!ok) break;
                phys = next;
                there = next_there;
                ks = next_ks;
                vs = next_vs;
                next = after;
            }
            // copies in flight end before the CTA does (bounded): the last tile's, or whichever there are where a wait gave up; the
            // conversion may have given up since the last one was issued
            for (int side = 0; side < 2; ++side) {
                if (ok) (void)mbar_wait_bounded<64>(&s.codes_full[side], (n - 1) & 1);
                else for (int parity = 0; parity < 2; ++parity) (void)mbar_wait_bounded<64>(&s.codes_full[side], parity);
            }
        }
    }
    __syncthreads();
    if (warp == kMmaWarp && n > 0) {
        fence_after();
        tmem_free(tmem);
    }
    // Rows that see values that are NaN, rarely: the products took them as 0, for the rows that do not see them.  Written here,
    // where no role's registers have to hold what it needs.
    if (s.any_nan) {
        for (int i = threadIdx.x; i < w.rows * kHeadDim; i += kThreads) {
            const int row = i / kHeadDim, r = w.row0 + row;
            if (keys_seen(p, w, r) <= min(s.nan_page, s.nan_code[i % kHeadDim])) continue;
            const size_t at = ((size_t)(w.lo + r / p.group) * p.num_q_heads + head * p.group + r % p.group) * kHeadDim + i % kHeadDim;
            if (args.splits > 1) args.part_o[(size_t)blockIdx.z * p.n_tok * p.num_q_heads * kHeadDim + at] = NAN;
            else static_cast<uint16_t*>(p.out)[at] = 0x7FFF;   // in both types
        }
    }
}

// Splits of a row merged: a warp per row, four channels a lane.
__global__ void __launch_bounds__(256) block_extend_merge_kernel(const __grid_constant__ ExtendArgs args) {
    const BlockAttentionParams& p = args.p;
    grid_dep_wait();
    grid_dep_launch();
    const int lane = threadIdx.x & 31;
    const size_t cells = (size_t)p.n_tok * p.num_q_heads, cell = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (cell >= cells) return;
    if (p.cu_q) {   // rows outside every sequence's range are not written
        const int row = (int)(cell / p.num_q_heads);
        const int b = warp_find_last(p.batch, row, [&](int s) { return (long long)load_dep(p.cu_q + s); });
        const int lo = load_dep(p.cu_q + b), hi = load_dep(p.cu_q + b + 1);
        if (lo < 0 || hi > p.n_tok || row < lo || row >= hi) return;
    }
    float m = kNoMax, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = 0; i < args.splits; ++i) {
        const float2 ml = args.part_ml[i * cells + cell];
        if (ml.y == 0.0f) continue;   // no key in sight: its sums were not written
        const float4 x = reinterpret_cast<const float4*>(args.part_o + (i * cells + cell) * kHeadDim)[lane];
        const float now = fmaxf(m, ml.x), f = fast_exp2(m - now), g = fast_exp2(ml.x - now);
        m = now;
        l = l * f + g * ml.y;
        o.x = o.x * f + g * x.x;
        o.y = o.y * f + g * x.y;
        o.z = o.z * f + g * x.z;
        o.w = o.w * f + g * x.w;
    }
    store_output(p, cell, lane, o, m, l);
}

constexpr int kMaxSplits = 64, kMaxCtas = 4;   // of a row; of a call that splits rows, per SM

struct ExtendPlan {
    long long blocks;   // tile pairs, an upper bound: find_work's numbering leaves some to nobody
    int splits;
    ExtendPlan(bool ragged, int batch, int n_tok, int num_kv_heads, int group, int max_pages, int num_sms) {
        blocks = ragged ? (long long)n_tok * group / (kTiles * kTile) + batch : batch;
        // the split count that takes the fewest tile steps: waves x (tiles of a split + a fixed part of about two)
        const long long ctas = blocks * num_kv_heads;
        const int tiles = (max_pages + kPages - 1) / kPages;
        long long best = -1;
        splits = 1;
        for (int s = 1; s <= std::min(tiles, kMaxSplits) && (s == 1 || ctas * s <= (long long)kMaxCtas * num_sms); ++s) {
            const long long waves = (ctas * s + num_sms - 1) / num_sms, cost = waves * ((tiles + s - 1) / s + 2) + (s > 1 ? 2 : 0);
            if (best < 0 || cost < best) best = cost, splits = s;
        }
    }
};

size_t part_ml_bytes(long long cells, int splits) { return ((size_t)cells * splits * sizeof(float2) + 255) & ~(size_t)255; }

}  // namespace

// For calls of up to n_tok tokens, whatever their batch and context: a CTA holds at most two tiles of rows.
size_t block_extend_workspace(int n_tok, int num_q_heads, int num_sms) {
    const long long rows = std::min((long long)n_tok * num_q_heads * kMaxSplits, (long long)kTiles * kTile * kMaxCtas * num_sms);
    return part_ml_bytes(rows, 1) + (size_t)rows * kHeadDim * sizeof(float);
}

cudaError_t launch_block_extend(const BlockAttentionParams& p, int code, int num_sms, cudaStream_t stream) {
    static PerDevice<Configured, cudaError_t> configured[2];
    auto* kernel = code == WC_CODE_INT8 ? block_extend_kernel<WC_CODE_INT8> : block_extend_kernel<WC_CODE_E4M3>;
    if (cudaError_t e = configure(configured[code == WC_CODE_INT8], kernel, kSmem)) return e;
    const ExtendPlan plan(p.cu_q != nullptr, p.batch, p.n_tok, p.num_kv_heads, p.group, p.max_pages, num_sms);
    const long long cells = (long long)p.n_tok * p.num_q_heads;
    ExtendArgs args;
    args.p = p;
    for (int side = 0; side < 2; ++side)
        if (!encode_page_map(&args.maps[side], p.codes[side], p.num_pages, p.num_kv_heads)) return cudaErrorInvalidValue;
    args.splits = plan.splits;
    float* scratch = p.partials + block_arrived_bytes(num_sms) / sizeof(float);
    args.part_ml = reinterpret_cast<float2*>(scratch);
    args.part_o = scratch + part_ml_bytes(cells, plan.splits) / sizeof(float);
    if (cudaError_t e = launch_pdl(kernel, dim3((unsigned)plan.blocks, p.num_kv_heads, plan.splits), dim3(kThreads), kSmem, stream, args))
        return e;
    if (plan.splits == 1) return cudaSuccess;
    static PerDevice<Configured, cudaError_t> merge_configured;
    if (cudaError_t e = configure(merge_configured, block_extend_merge_kernel, 0)) return e;
    return launch_pdl(block_extend_merge_kernel, dim3((unsigned)((cells + 7) / 8)), dim3(256), 0, stream, args);
}

}  // namespace wc
