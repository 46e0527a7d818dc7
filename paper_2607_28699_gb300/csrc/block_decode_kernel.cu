// Decode attention over the block-scaled cache: one query token per sequence.
//
// A unit is one (KV head, sequence); the pages that its row sees (all of them, or the sinks' and the window's) of all units laid
// end to end (head by head) are cut into equal shares, a CTA's range and in it a warp's, so that any mix of lengths keeps every
// SM busy.  A warp streams its pages through its own ring (a page: two TMA copies of 2 KB with the
// 128-byte swizzle) and holds the unit's softmax state in registers:
//   S (16 tokens x 8 heads) = K q^T, one mma.m16n8k16 per 16 channels, codes as exact fp16;
//   y = S ks + log2(vs), ks the page's key scale times softmax_scale log2(e): the value scale
//     is an offset in the exponent, so 2^(y - m) is p vs at no cost, and O sums it times V's
//     codes; the sum of weights takes p = 2^(y - m) / vs;
//   O^T (128 x 8) += V^T P^T, 8 mma, V transposed by ldmatrix on bytes.
// The frame m follows the running maximum lazily: it moves only when a weight would pass 2^15 (one vote a page).
// A unit inside one warp's range is finished there, one inside a CTA's by the CTA; the CTAs of a unit
// that reaches over several leave partial results, and the last of them to arrive merges these
// (in the order of the pages, so the result does not depend on which one it is).
//
// GB300, 4 KV heads of 7 query heads, a call by itself: 32 sequences of 4k to 32k 106 us (5.7 TB/s, 0.84 of the measured copy rate:
// the page loop reads 7 TB/s, the rest is the first pages' latency and the merges), 16 of 4k to 8k 33 us, one of 32k 20 us
// (6 us page loop at the copy rate; launch and block table before it, merges in the CTA and over 38 CTAs after it).  In a row of
// calls, whose launches overlap, 102, 28 and 16 us (what fits the L2 read from there; with other inputs each time 31 and 19).
// 16 warps on one CTA an SM (with three pages in flight each: 111 / 35 / 20.5 us; 8 warps on two CTAs 110 / 35 / 26, twice the
// partial results; on one 131 / 37 / 23); several shares per SM, taken as SMs come free, 121 / 45 / 41 (each has its own
// prologue and merge).
// With a window of 4096 tokens and 64 sinks, in a row of calls, 32 sequences 30 us (4.5 TB/s: 128 CTAs with a sequence and head
// each, whole units; 12 us are launch, first pages and the merge in the CTA), 16 with a window of 1000 12 us, one with 512 9 us.
#include "block_common.cuh"
#include "decode_common.cuh"

namespace wc {

namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32;
// Pages of a warp in flight: 128 KB an SM saturate the memory; with three, what others load (block tables, partial
// results) waits a microsecond longer behind the copies (111 / 35 us for the batches below, 107 / 33 with two).
constexpr int kStages = 2;
constexpr int kPageBytes = kPage * kHeadDim;           // one head's page of keys, or of values
constexpr int kStageBytes = 2 * kPageBytes;
constexpr int kRow = kHeadDim + 4;                     // floats of a merge row in shared memory
constexpr int kMinPages = 1;                           // per warp, before a launch takes more CTAs
constexpr float kNoMax = -3e38f;                       // the frame before the first logit
// The units of windowed calls have about as many pages each.  Shares of whole units need no merges between CTAs, but leave SMs
// without work; they are taken where the longest is at most this many pages above an equal share.  Whole against cut shares, us in a
// row of calls (28 / 4 heads, 38 shares a head, units of n sequences; pages above):
//   window 1024   n 1 (52) 11.9 / 10.3   4 (50) 12.2 / 12.8   12 (45) 12.3 / 13.9   16 (38) 12.3 / 14.3
//   window 2048   n 16 (75) 17.6 / 16.4  20 (62) 17.6 / 18.1  24 (48) 17.7 / 18.9   27 (38) 17.7 / 19.5
//   window 4096   n 24 (95) 29.1 / 26.7  28 (68) 29.7 / 29.8  31 (48) 30.4 / 33.5   32 (41) 30.4 / 34.0
//   window 8192   n 27 (149) 51.8 / 47.8 31 (95) 51.9 / 54.7  36 (27) 53.0 / 59.4
// Up to 41 above whole shares were never behind.  What the merges cost grows with sequences and pages, so one number has to miss some:
// at 44 one or two short units stay cut (1.6 us), and 28 to 31 sequences of 4096 too, which lose up to 3.1 us by it.  The kernel finds
// the shares from the lengths (0.2 us): by the window alone one sequence of 258 pages among 31 of 2 would have a CTA to itself (26.7
// us instead of 16.0).
constexpr int kWholePages = 44;

struct DecodeArgs {
    BlockAttentionParams p;
    CUtensorMap k_map, v_map;
    // Of the unit that begins in CTA c and reaches past it: CTAs that left a partial result; 0 between
    // calls.  Its place does not depend on a call's sizes.
    int* arrived;
    int by_head;             // the shares are of one head's pages
    int whole;               // most units of a share of whole units; 0: none are formed
    float* partials;         // [grid][2 + kWarps] slots: of the CTA's first and last unit, of a warp's first
};

// A unit (head, sequence), its pages' positions and the CTAs that read them.
struct Unit {
    int id, start, end, c0, c1;
};
constexpr int kSequenceBits = 11;
static_assert(kDecodeBatch <= 1 << kSequenceBits);   // id: head << kSequenceBits | sequence

struct Shared {
    int prefix[kDecodeBatch + 1];   // pages of one head before each sequence
    int ctx[kDecodeBatch];
    int warp_sum[kWarps];
    int entry[2 * kWarps];   // units of the warps' unfinished results (a warp's first, its last), -1: none
    Unit ends[2];            // the units of the CTA's first and last page
    int open[2];             // slot 0, 1 holds a partial result of ends[0], ends[1]; then: to be merged here
    uint64_t bars[kWarps][kStages];
};
constexpr int kRingBytes = kWarps * kStages * kStageBytes;
constexpr int kSmem = kRingBytes + (int)sizeof(Shared) + 1024;
static_assert(kMaxGroup * kRow * 4 <= kStages * kStageBytes, "a warp's last result takes its ring's place");

// A partial result: [group][128] sums, [group] (m, l); 16-byte aligned.
__host__ __device__ __forceinline__ size_t slot_floats(int group) { return ((size_t)group * (kHeadDim + 2) + 3) & ~(size_t)3; }

// How [0, total) is cut: the first `more` CTAs take len + 1 pages, the others len; total < 2^31.
// Where the grid is a multiple of the heads, or one sequence is all there is, each head's pages are
// cut by themselves (no CTA then reads two units of one sequence), else all heads' laid end to end.
struct Shares {
    int used, len, more;
    __device__ __forceinline__ Shares(int total, int grid) {
        used = max(1, min(grid, (int)(((unsigned)total + kWarps * kMinPages - 1) / (kWarps * kMinPages))));
        len = (unsigned)total / (unsigned)used;
        more = total - len * used;
    }
    __device__ __forceinline__ int begin(int c) const { return c * len + min(c, more); }
    __device__ __forceinline__ int cta_at(int x) const {
        const int head = (len + 1) * more;
        return x < head ? (unsigned)x / (unsigned)(len + 1) : more + (unsigned)(x - head) / (unsigned)len;
    }
};
__device__ __forceinline__ int warp_begin(int a, int e, int w) { return a + (int)((unsigned)(e - a) / kWarps * w + (unsigned)(e - a) % kWarps * w / kWarps); }

// Context of sequence b, 0 for a length that cannot be.
__device__ __forceinline__ int context(const BlockAttentionParams& p, int b, bool tell) {
    const int ctx = load_dep(p.ctx_lens + b);
    if (ctx < 0 || ctx > (long long)p.max_pages * kPage) {
        if (tell) atomicOr(p.status, WC_DEV_BAD_CTX);
        return 0;
    }
    return ctx;
}

// What the last token of a context sees: its last `window` positions and the first `sinks`.  The pages that hold any of them
// are counted without the ones between: page v of those is logical page v before the gap, v + skip from there on.
struct Seen {
    int window = 0x7FFFFFFF, sinks = 0;
    __device__ __forceinline__ int low(int ctx) const { return max(0, ctx - window); }
    __device__ __forceinline__ int head(int ctx) const { return (min(sinks, ctx) + kPage - 1) / kPage; }
    __device__ __forceinline__ int skip(int ctx) const { return max(0, low(ctx) / kPage - head(ctx)); }
    __device__ __forceinline__ int pages(int ctx) const { return ((ctx + kPage - 1) >> 4) - skip(ctx); }
};

// Contexts and exclusive prefix sums of the pages seen.  Up to 32 sequences each warp finds them by itself and goes on
// without a barrier: a place is written once by each, with the sum that every warp writes there, since others may be
// reading it.  More are shared out over the CTA.
__device__ __forceinline__ void page_prefix(const BlockAttentionParams& p, Shared& s, bool tell, Seen seen = {}) {
    const int tid = threadIdx.x, lane = tid & 31;
    const bool by_warp = p.batch <= 32;
    const int per = by_warp ? 1 : (p.batch + kThreads - 1) / kThreads;
    const int b0 = min((by_warp ? lane : tid) * per, p.batch), b1 = min(b0 + per, p.batch);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int ctx = context(p, b, tell);
        s.ctx[b] = ctx;
        if (!by_warp) s.prefix[b] = mine;
        mine += seen.pages(ctx);
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (by_warp) {
        if (lane < p.batch) s.prefix[lane] = incl - mine;
        if (lane == 31) s.prefix[p.batch] = incl;
        __syncwarp();
        return;
    }
    if (lane == 31) s.warp_sum[tid >> 5] = incl;
    __syncthreads();
    int before = incl - mine;
    for (int w = 0; w < (tid >> 5); ++w) before += s.warp_sum[w];
    for (int b = b0; b < b1; ++b) s.prefix[b] += before;
    if (tid == kThreads - 1) s.prefix[p.batch] = before + mine;
    __syncthreads();
}

// The sequence that holds page r of one head's pages.
__device__ __forceinline__ int sequence_at(const Shared& s, int batch, int r) {
    int lo = 0, hi = batch;   // prefix[lo] <= r < prefix[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.prefix[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// What a lane knows of one page of its warp's range.  Found in two steps, so that no step waits for a load that it
// has just issued: where the page is in the block table, then (page_resolve) its scales.
struct PageEntry {
    int row;       // page number, then (page, head) index of the code arrays
    int unit;      // Unit::id
    int info;      // a bit for each token that counts | kFirst | kLast
    float ks, vs;  // key scale, value scale
};
constexpr int kTokens = 0xFFFF, kFirst = 1 << 16, kLast = 1 << 17;
__device__ __forceinline__ int tokens_below(int n) { return n >= kPage ? kTokens : (1 << max(n, 0)) - 1; }

__device__ __forceinline__ PageEntry page_find(const BlockAttentionParams& p, const Shared& s, int head0, int per_head, int at, int first, int last) {
    PageEntry e = {0, head0 << kSequenceBits, 0, 0.0f, 1.0f};
    if (at >= last) return e;
    const int k = at < per_head ? 0 : (int)((unsigned)at / (unsigned)per_head), r = at - k * per_head;
    const int b = sequence_at(s, p.batch, r), page = r - s.prefix[b], ctx = s.ctx[b];
    const Seen seen = {p.window, p.sinks};
    const int logical = page < seen.head(ctx) ? page : page + seen.skip(ctx), start = logical * kPage;
    e.row = load_dep(p.block_table + (size_t)b * p.max_pages + logical);
    e.unit = (head0 + k) << kSequenceBits | b;
    e.info = (tokens_below(ctx - start) & (~tokens_below(seen.low(ctx) - start) | tokens_below(p.sinks - start))) |
             (page == 0 || at == first ? kFirst : 0) | (page + 1 == s.prefix[b + 1] - s.prefix[b] || at + 1 == last ? kLast : 0);
    return e;
}

__device__ __forceinline__ void page_resolve(const BlockAttentionParams& p, PageEntry& e) {
    const int phys = e.row;
    const bool there = phys >= 0 && phys < p.num_pages;
    if (!there) {
        atomicOr(p.status, WC_DEV_BAD_PAGE);
        e.info &= ~kTokens;
    }
    e.row = (there ? phys * p.num_kv_heads : 0) + (e.unit >> kSequenceBits);
    if (there && p.scale[0]) {
        e.ks = load_dep(p.scale[0] + e.row);
        e.vs = load_dep(p.scale[1] + e.row);
    } else {
        e.ks = 1.0f;
    }
}

// A head's query row as B fragments: lane (g, t) holds channels 32 t .. 32 t + 31 of query head g, in
// the order in which the K rows are read.  bf16 rows are scaled by a power of two into fp16's range,
// which keeps every bit that fp32 products would keep; returns the factor that undoes it.
__device__ __forceinline__ float load_queries(const BlockAttentionParams& p, int b, int head, uint32_t (&q)[16]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint4 w[4] = {};
    if (g < p.group) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.q) + (size_t)b * p.q_stride +
                                                          (size_t)(head * p.group + g) * kHeadDim + 32 * t);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = load_dep(src + i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = word_of(w[i >> 2], i & 3);
    if (!p.bf16) return 1.0f;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __vmaxu2(top, q[i] & 0x7FFF7FFFu);
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float undo;
    const float up = bf16_scale(top, undo);
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = scaled_bf16(q[i], up);
    return undo;
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ void fma4(float4& o, float f, float4 x) {
    o.x = fmaf(f, x.x, o.x);
    o.y = fmaf(f, x.y, o.y);
    o.z = fmaf(f, x.z, o.z);
    o.w = fmaf(f, x.w, o.w);
}

// The adds of a CTA whose other threads' writes this thread has seen (behind a barrier), and the reads after it.
__device__ __forceinline__ int add_acq_rel(int* at, int x) {
    int old;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(old) : "l"(at), "r"(x) : "memory");
    return old;
}

template <int kCode>
__global__ void __launch_bounds__(kThreads, 1) block_decode_kernel(const __grid_constant__ DecodeArgs args) {
    const BlockAttentionParams& p = args.p;
    extern __shared__ uint8_t raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    Shared& s = *reinterpret_cast<Shared*>(ring + kRingBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if (lane == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(&s.bars[warp][i], 1);
        fence_barrier_init();
        if (warp == 0) {
            prefetch_map(&args.k_map);
            prefetch_map(&args.v_map);
        }
    }
    grid_dep_wait();
    grid_dep_launch();
    page_prefix(p, s, blockIdx.x == 0, {p.window, p.sinks});
    const int per_head = s.prefix[p.batch];
    // sequences without context: nothing to add up
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
        if (s.prefix[b + 1] > s.prefix[b]) continue;
        for (int i = threadIdx.x; i < p.num_q_heads * (kHeadDim / 2); i += kThreads)
            static_cast<uint32_t*>(p.out)[(size_t)b * p.num_q_heads * (kHeadDim / 2) + i] = 0;
        for (int i = threadIdx.x; p.lse && i < p.num_q_heads; i += kThreads) p.lse[(size_t)b * p.num_q_heads + i] = -INFINITY;
    }
    if (per_head == 0) return;
    const bool by_head = args.by_head;
    const int heads = by_head ? 1 : p.num_kv_heads, per_part = by_head ? gridDim.x / p.num_kv_heads : gridDim.x;
    const int part0 = by_head ? blockIdx.x / per_part : 0, cta0 = part0 * per_part, head0 = part0;   // this part's first CTA and head
    const Shares shares(per_head * heads, per_part);
    const int cta = blockIdx.x - cta0;
    bool whole = args.whole > 0;
    if (whole) {   // every warp finds it for itself
        int longest = 0;
        for (int b = lane; b < p.batch; b += 32) longest = max(longest, s.prefix[b + 1] - s.prefix[b]);
        whole = (long long)args.whole * __reduce_max_sync(0xffffffffu, longest) <= shares.len + kWholePages;
    }
    if (!whole && cta >= shares.used) return;
    auto unit_begin = [&](unsigned c) {
        const unsigned u = (unsigned)(heads * p.batch) * c / per_part, k = by_head ? 0 : u / (unsigned)p.batch;
        return (int)k * per_head + s.prefix[u - k * p.batch];
    };
    const int a = whole ? unit_begin(cta) : shares.begin(cta), e = whole ? unit_begin(cta + 1) : shares.begin(cta + 1);
    if (a == e) return;
    const int first = warp_begin(a, e, warp), last = warp_begin(a, e, warp + 1), n = last - first;
    float* cta_slots = args.partials + (size_t)blockIdx.x * (2 + kWarps) * slot_floats(p.group);
    if (lane < 2) s.entry[2 * warp + lane] = -1;   // read after the CTA's next barrier
    if (threadIdx.x < 2) s.open[threadIdx.x] = 0;
    __syncwarp();
    uint8_t* stage0 = ring + warp * kStages * kStageBytes;
    PageEntry cur = page_find(p, s, head0, per_head, first + lane, first, last), next = {};
    page_resolve(p, cur);
    int issued = 0;
    auto issue = [&](int i, int row) {   // page i of the warp's range
        issued = i + 1;
        if (elect_one()) {
            uint64_t* bar = &s.bars[warp][i % kStages];
            uint8_t* dst = stage0 + (i % kStages) * kStageBytes;
            mbar_arrive_expect_tx(bar, kStageBytes);
            tma_page(dst, &args.k_map, row, bar);
            tma_page(dst + kPageBytes, &args.v_map, row, bar);
        }
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
        const int row = __shfl_sync(0xffffffffu, cur.row, i);
        if (i < n) issue(i, row);
    }
    if (n > 32) next = page_find(p, s, head0, per_head, first + 32 + lane, first, last);   // while the first pages come
    if (warp == kWarps - 1 && lane < 2) {
        const int at = lane ? e - 1 : a, k = at < per_head ? 0 : (int)((unsigned)at / (unsigned)per_head);
        const int b = sequence_at(s, p.batch, at - k * per_head);
        Unit u = {(head0 + k) << kSequenceBits | b, k * per_head + s.prefix[b], k * per_head + s.prefix[b + 1], 0, 0};
        if (!whole) {
            u.c0 = shares.cta_at(u.start);
            u.c1 = shares.cta_at(u.end - 1);
        }
        s.ends[lane] = u;
    }
    __syncwarp();

    uint32_t q[16];
    float acc[8][4];
    float m[2] = {kNoMax, kNoMax}, l[2] = {0.0f, 0.0f}, qf[2] = {1.0f, 1.0f};
    bool ok = true;
    int seg = first;   // where the current unit's pages of this warp begin
    const int trow = tok_row(g);

    for (int i = 0; i < n; ++i) {
        const int from = i & 31;
        const int info = __shfl_sync(0xffffffffu, cur.info, from);
        const float ks = __shfl_sync(0xffffffffu, cur.ks, from) * p.scale_log2;
        float vs = __shfl_sync(0xffffffffu, cur.vs, from);
        const bool lost = !(vs < INFINITY), no_values = lost || vs < kLeastValueScale;   // lost: infinity or NaN
        if (no_values) vs = kNoValueScale;
        if (info & kFirst) {
            const int unit = __shfl_sync(0xffffffffu, cur.unit, from);
            const float f = load_queries(p, unit & ((1 << kSequenceBits) - 1), unit >> kSequenceBits, q);
            qf[0] = __shfl_sync(0xffffffffu, f, 8 * t);       // of head 2 t
            qf[1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);   // of head 2 t + 1
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[j][c] = 0.0f;
            m[0] = m[1] = kNoMax;
            l[0] = l[1] = 0.0f;
            seg = first + i;
        }
        if (ok && !__all_sync(0xffffffffu, mbar_wait_bounded(&s.bars[warp][i % kStages], (i / kStages) & 1))) {
            if (lane == 0) atomicOr(p.status, WC_DEV_TIMEOUT);
            ok = false;
        }
        const uint8_t* kp = stage0 + (i % kStages) * kStageBytes;
        float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        {
            const uint4* lo = reinterpret_cast<const uint4*>(kp);
            const uint4 k00 = lo[trow * 8 + ((2 * t) ^ (trow & 7))], k01 = lo[trow * 8 + ((2 * t + 1) ^ (trow & 7))];
            const int trow8 = trow + 2;   // tok_row(g + 8)
            const uint4 k10 = lo[trow8 * 8 + ((2 * t) ^ (trow8 & 7))], k11 = lo[trow8 * 8 + ((2 * t + 1) ^ (trow8 & 7))];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t af[4];
                codes4_to_h2<kCode>(word_of(j < 4 ? k00 : k01, j & 3), af[0], af[2]);
                codes4_to_h2<kCode>(word_of(j < 4 ? k10 : k11, j & 3), af[1], af[3]);
                mma16816(sc, af, q[2 * j], q[2 * j + 1]);
            }
        }
        const int tokens = info & kTokens;
        const float bias = log2f(vs);
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = fmaf(sc[c], ks * qf[c & 1], bias);
        if (tokens != kTokens) {
            if (!(tokens >> trow & 1)) y[0] = y[1] = -INFINITY;
            if (!(tokens >> (trow + 2) & 1)) y[2] = y[3] = -INFINITY;
        }
        const float top0 = fmaxf(y[0], y[2]), top1 = fmaxf(y[1], y[3]);
        if (__any_sync(0xffffffffu, top0 - m[0] > kTopWeight || top1 - m[1] > kTopWeight)) {
            float top[2] = {top0, top1};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], o));
                const float now = fmaxf(m[h], top[h] - kHeadroom), f = fast_exp2(m[h] - now);
                m[h] = now;
                l[h] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    acc[j][h] *= f;
                    acc[j][h + 2] *= f;
                }
            }
        }
        float pr[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) pr[c] = fast_exp2(y[c] - m[c & 1]);
        const float inv = __frcp_rn(vs) * kSumUnit;
        l[0] = fmaf(pr[0] + pr[2], inv, l[0]);
        l[1] = fmaf(pr[1] + pr[3], inv, l[1]);
        const uint32_t b0 = movmatrix_t(pack_h2(pr[0], pr[1])), b1 = movmatrix_t(pack_h2(pr[2], pr[3]));
        const bool clean = tokens != kTokens || no_values;   // codes that must not count, NaN among them
#pragma unroll
        for (int j = 0; j < 4; ++j) {   // 32 channels
            uint32_t d[4];
            ldsm_t_b8_x2(d, kp + kPageBytes + swz(lane & 15, 2 * j + (lane >> 4)));
            if (clean) {
                const uint32_t have = no_values ? 0u : tokens >> (4 * t) & 15;   // of this lane's four tokens, a bit each
                const uint32_t keep = (have * 0x204081u & 0x01010101u) * 0xFFu;   // a byte each
#pragma unroll
                for (int c = 0; c < 4; ++c) d[c] &= keep;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t af[4];
                codes4_to_h2<kCode>(d[2 * h], af[0], af[2]);
                codes4_to_h2<kCode>(d[2 * h + 1], af[1], af[3]);
                mma16816(acc[2 * j + h], af, b0, b1);
            }
        }
        if (lost) {   // the output is; the sum of weights does not depend on values
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[j][c] = NAN;
        }
        __syncwarp();
        // the stage is free: the page kStages on
        const int ahead = i + kStages;
        const int row = __shfl_sync(0xffffffffu, (ahead >> 5) == (i >> 5) ? cur.row : next.row, ahead & 31);
        if (ok && ahead < n) issue(ahead, row);
        if (info & kLast) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
            const int unit = __shfl_sync(0xffffffffu, cur.unit, from), head = unit >> kSequenceBits, b = unit & ((1 << kSequenceBits) - 1);
            const int start = (head - head0) * per_head + s.prefix[b], end = (head - head0) * per_head + s.prefix[b + 1];
            const bool whole = start == seg && end == first + i + 1, final = i == n - 1;
            if (whole) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int hq = 2 * t + h;
                    if (hq >= p.group) continue;
                    const size_t cell = (size_t)b * p.num_q_heads + head * p.group + hq;
                    const float f = output_factor(l[h]);
                    uint16_t* out = static_cast<uint16_t*>(p.out) + cell * kHeadDim;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        out[16 * j + g] = float_to_act(acc[j][h] * f, p.bf16);
                        out[16 * j + 8 + g] = float_to_act(acc[j][h + 2] * f, p.bf16);
                    }
                    if (p.lse && g == 0) p.lse[cell] = log_sum(m[h], l[h]);
                }
            } else {
                // the warp's last result takes the place of its ring (every page of it has been read), a first one
                // that others follow waits in global memory
                float* rows = final ? reinterpret_cast<float*>(stage0) : cta_slots + (2 + warp) * slot_floats(p.group);
                const int pitch = final ? kRow : kHeadDim;
                float* ml = final ? rows + kHeadDim : rows + p.group * kHeadDim;
                const int ml_pitch = final ? kRow : 2;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int hq = 2 * t + h;
                    if (hq >= p.group) continue;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        rows[hq * pitch + 16 * j + g] = acc[j][h];
                        rows[hq * pitch + 16 * j + 8 + g] = acc[j][h + 2];
                    }
                    if (g == 0) *reinterpret_cast<float2*>(ml + hq * ml_pitch) = make_float2(m[h], l[h]);
                }
                if (lane == 0) s.entry[2 * warp + final] = unit;
            }
        }
        if (from == 15 && i + 17 < n) page_resolve(p, next);
        if (from == 31) {
            cur = next;
            if (i + 33 < n) next = page_find(p, s, head0, per_head, first + i + 33 + lane, first, last);
        }
    }
    if (!ok) {   // copies still in flight end before the CTA does (bounded again)
        for (int i = max(0, issued - kStages); i < issued; ++i)
            (void)mbar_wait_bounded<64>(&s.bars[warp][i % kStages], (i / kStages) & 1);
    }
    __syncthreads();

    // the CTA's unfinished results (lane k looks after entry k; those of one unit follow each other): a query head per
    // warp, and as many units at a time as there are warps for
    const int parts = kWarps / p.group, part = warp / p.group, hq = warp - part * p.group;   // warps per query head
    auto finish = [&](int unit, int hq, float4 o, float m, float l) {
        const int head = unit >> kSequenceBits, b = unit & ((1 << kSequenceBits) - 1);
        store_output(p, (size_t)b * p.num_q_heads + head * p.group + hq, lane, o, m, l);
    };
    if (part < parts) {
        const int mine = lane < 2 * kWarps ? s.entry[lane] : -1;
        const float* rows = reinterpret_cast<const float*>(ring) + hq * kRow;   // of the warps' last results
        constexpr int kPitch = kStages * kStageBytes / 4;
        int turn = 0;
        for (uint32_t left = __ballot_sync(0xffffffffu, mine >= 0); left;) {
            const int unit = __shfl_sync(0xffffffffu, mine, __ffs(left) - 1);
            const bool member = mine == unit;
            const uint32_t members = __ballot_sync(0xffffffffu, member);
            left &= ~members;
            const bool other = turn != part;
            turn = turn + 1 == parts ? 0 : turn + 1;
            if (other) continue;
            float2 ml = make_float2(kNoMax, 0.0f);
            if (member)
                ml = lane & 1 ? *reinterpret_cast<const float2*>(rows + (lane >> 1) * kPitch + kHeadDim)
                              : *reinterpret_cast<const float2*>(cta_slots + (2 + (lane >> 1)) * slot_floats(p.group) + p.group * kHeadDim + 2 * hq);
            const float top = warp_max(ml.x), f = fast_exp2(ml.x - top), sum = warp_sum(f * ml.y);
            float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {   // no branches: sixteen loads in flight
                float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (members >> (2 * w + 1) & 1) x = *reinterpret_cast<const float4*>(rows + w * kPitch + 4 * lane);
                fma4(o, __shfl_sync(0xffffffffu, f, 2 * w + 1), x);
            }
            for (uint32_t rest = members & 0x55555555u; rest; rest &= rest - 1) {
                const int k = __ffs(rest) - 1;
                fma4(o, __shfl_sync(0xffffffffu, f, k), *reinterpret_cast<const float4*>(cta_slots + (2 + (k >> 1)) * slot_floats(p.group) + hq * kHeadDim + 4 * lane));
            }
            const bool before = unit == s.ends[0].id && s.ends[0].start < a, after = unit == s.ends[1].id && s.ends[1].end > e;
            if (!before && !after) {
                finish(unit, hq, o, top, sum);
                continue;
            }
            const int which = before ? 0 : 1;
            float* slot = cta_slots + which * slot_floats(p.group);
            *reinterpret_cast<float4*>(slot + hq * kHeadDim + 4 * lane) = o;
            if (lane == 0) {
                *reinterpret_cast<float2*>(slot + p.group * kHeadDim + 2 * hq) = make_float2(top, sum);
                if (hq == 0) s.open[which] = 1;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < 2 && s.open[threadIdx.x]) {
        const Unit& u = s.ends[threadIdx.x];
        int* arrived = args.arrived + cta0 + u.c0;
        if (add_acq_rel(arrived, 1) == u.c1 - u.c0) *arrived = 0;
        else s.open[threadIdx.x] = 0;
    }
    __syncthreads();
    float* rows = reinterpret_cast<float*>(ring);
    for (int which = 0; which < 2; ++which) {
        if (!s.open[which]) continue;
        const int unit = s.ends[which].id, c0 = cta0 + s.ends[which].c0, c1 = cta0 + s.ends[which].c1;
        float m = kNoMax, l = 0.0f;
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (part < parts) {
            // CTA c0 left its result in its second slot, the others in their first
            const int slot = (int)slot_floats(p.group), pitch = (2 + kWarps) * slot, ml_at = p.group * kHeadDim + 2 * hq, o_at = hq * kHeadDim + 4 * lane;
            const float* base = args.partials + c0 * pitch;
            if (part == 0) {
                const float2 ml = __ldcg(reinterpret_cast<const float2*>(base + slot + ml_at));
                o = __ldcg(reinterpret_cast<const float4*>(base + slot + o_at));
                m = ml.x;
                l = ml.y;
            }
            base += (1 + part) * pitch;
            const int step = parts * pitch, mine = c1 - c0 > part ? (c1 - c0 - part - 1) / parts + 1 : 0;   // results of this warp
#pragma unroll 1
            for (int k0 = 0; k0 < mine; k0 += 32, base += 32 * step) {
                const int count = min(32, mine - k0);
                float2 ml = make_float2(kNoMax, 0.0f);
                if (lane < count) ml = __ldcg(reinterpret_cast<const float2*>(base + lane * step + ml_at));
                float4 x[16];   // sixteen results in flight
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j < count) x[j] = __ldcg(reinterpret_cast<const float4*>(base + j * step + o_at));
                const float top = fmaxf(m, warp_max(ml.x)), f = fast_exp2(ml.x - top), again = fast_exp2(m - top);
                m = top;
                l = l * again + warp_sum(f * ml.y);
                o = make_float4(o.x * again, o.y * again, o.z * again, o.w * again);
#pragma unroll 1
                for (int k = 0;;) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (k + j < count) fma4(o, __shfl_sync(0xffffffffu, f, k + j), x[j]);
                    if ((k += 16) >= count) break;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (k + j < count) x[j] = __ldcg(reinterpret_cast<const float4*>(base + (k + j) * step + o_at));
                }
            }
            *reinterpret_cast<float4*>(rows + warp * kRow + 4 * lane) = o;
            if (lane == 0) *reinterpret_cast<float2*>(rows + warp * kRow + kHeadDim) = make_float2(m, l);
        }
        __syncthreads();
        if (warp < p.group) {
            for (int k = 1; k < parts; ++k) {
                const float* other = rows + (warp + k * p.group) * kRow;
                const float2 ml = *reinterpret_cast<const float2*>(other + kHeadDim);
                const float top = fmaxf(m, ml.x), again = fast_exp2(m - top), f = fast_exp2(ml.x - top);
                m = top;
                l = l * again + f * ml.y;
                o = make_float4(o.x * again, o.y * again, o.z * again, o.w * again);
                fma4(o, f, *reinterpret_cast<const float4*>(other + 4 * lane));
            }
            finish(unit, warp, o, m, l);
        }
        __syncthreads();
    }
}

struct DecodeGrid {
    int ctas;
    bool by_head;
    DecodeGrid(int batch, int num_kv_heads, int max_pages, int num_sms) {
        const long long most = ((long long)batch * num_kv_heads * max_pages + kWarps * kMinPages - 1) / (kWarps * kMinPages);
        ctas = (int)std::max(1LL, std::min<long long>(num_sms, most));
        by_head = num_kv_heads <= num_sms && (batch == 1 || num_sms % num_kv_heads == 0);
        if (by_head) ctas = std::max(num_kv_heads, ctas / num_kv_heads * num_kv_heads);
    }
};

}  // namespace

size_t block_decode_workspace(int group, int num_sms) {   // the grid never exceeds the SMs
    return sizeof(float) * (size_t)num_sms * (2 + kWarps) * slot_floats(group);
}

cudaError_t launch_block_decode(const BlockAttentionParams& params, int code, int num_sms, cudaStream_t stream) {
    DecodeArgs args;
    args.p = params;
    if (!encode_page_map(&args.k_map, params.codes[0], params.num_pages, params.num_kv_heads) ||
        !encode_page_map(&args.v_map, params.codes[1], params.num_pages, params.num_kv_heads))
        return cudaErrorInvalidValue;
    static PerDevice<Configured, cudaError_t> configured[2];
    auto* kernel = code == WC_CODE_INT8 ? block_decode_kernel<WC_CODE_INT8> : block_decode_kernel<WC_CODE_E4M3>;
    if (cudaError_t e = configure(configured[code == WC_CODE_INT8], kernel, kSmem)) return e;
    // a launch holds the page sums of kDecodeBatch sequences; positions, pages times heads, stay below 2^31
    const int pages = seen_pages(params, params.max_pages, 1);
    const long long one = (long long)pages * params.num_kv_heads;
    if (one > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;   // refused by the caller
    const int each = (int)std::min<long long>(kDecodeBatch, 0x7FFFFFFFLL / one);
    for (int b0 = 0; b0 < params.batch; b0 += each) {
        BlockAttentionParams& p = args.p;
        p.batch = std::min(each, params.batch - b0);
        p.q = static_cast<const uint16_t*>(params.q) + (size_t)b0 * params.q_stride;
        p.block_table = params.block_table + (size_t)b0 * params.max_pages;
        p.ctx_lens = params.ctx_lens + b0;
        p.out = static_cast<uint16_t*>(params.out) + (size_t)b0 * params.num_q_heads * kHeadDim;
        p.lse = params.lse ? params.lse + (size_t)b0 * params.num_q_heads : nullptr;
        const DecodeGrid grid(p.batch, p.num_kv_heads, pages, num_sms);
        args.by_head = grid.by_head;
        const long long units = (long long)(grid.by_head ? 1 : p.num_kv_heads) * p.batch, ctas = grid.by_head ? grid.ctas / p.num_kv_heads : grid.ctas;
        args.whole = p.windowed() && units * (ctas + 1) <= 0x7FFFFFFFLL ? (int)((units + ctas - 1) / ctas) : 0;
        args.arrived = reinterpret_cast<int*>(p.partials);
        args.partials = p.partials + block_arrived_bytes(num_sms) / sizeof(float);
        if (cudaError_t e = launch_pdl(kernel, dim3(grid.ctas), dim3(kThreads), kSmem, stream, args)) return e;
    }
    return cudaSuccess;
}

}  // namespace wc
