"""How the block append is cut into launches (launch_block_append and PageWork in csrc/block_append_kernel.cu): their own text compiled
for the host.  Whatever the sizes, each page task of each KV head and side is one warp's, each token's queries are, and warps are
counted in 32 bits (no GPU needed)."""

import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_28699_gb300", "csrc")

HOST = r"""
#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <vector>
#define __device__
#define __forceinline__ inline
enum { WC_CODE_INT8 = 0, WC_CODE_E4M3 = 1, WC_ACT_BF16 = 1, WC_ROPE_HALF = 0 };
enum cudaError_t { cudaSuccess = 0, cudaErrorInvalidConfiguration = 9 };
typedef void* cudaStream_t;
struct dim3 { unsigned x, y = 1, z = 1; dim3(unsigned a) : x(a) {} };
constexpr int kPage = 16, kThreads = 128, kWarps = kThreads / 32;
@PARAMS@
@WORK@
struct Launch { unsigned ctas; BlockAppendParams p; };
static std::vector<Launch> launches;
template <int kCode, bool kBf16, bool kHalf, bool kNorm> void block_append_kernel(const BlockAppendParams&) {}
template <typename K> cudaError_t launch_pdl(K, dim3 grid, dim3, int, cudaStream_t, const BlockAppendParams& p) {
    launches.push_back({grid.x, p});
    return cudaSuccess;
}
@LAUNCH@
extern "C" int plan(int ragged, int q, int n_tok, int batch, int hq, int hkv, int64_t* out) {   // count, then per launch seven numbers
    BlockAppendParams p = {};
    static int32_t cu;
    p.cu_new = ragged ? &cu : nullptr;
    p.q = q ? &cu : nullptr;
    p.n_tok = n_tok, p.batch = batch, p.num_q_heads = hq, p.num_kv_heads = hkv;
    launches.clear();
    if (launch_block_append(p, 0, 0, 0, nullptr)) return -1;
    for (auto& l : launches)
        for (int64_t x : {(int64_t)l.ctas, (int64_t)l.p.page_head0, (int64_t)l.p.page_heads, (int64_t)l.p.page_ctas, (int64_t)l.p.page_stride, (int64_t)l.p.page_tasks,
                          (int64_t)l.p.q_heads}) *out++ = x;
    return (int)launches.size();
}
extern "C" void work(int head0, int heads, unsigned group, unsigned warp, int64_t* out) {
    BlockAppendParams p = {};
    p.page_head0 = head0, p.page_heads = heads;
    const PageWork w(p, group, warp);
    out[0] = w.task, out[1] = w.head, out[2] = w.side;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    kernel, common = (open(os.path.join(CSRC, f)).read() for f in ("block_append_kernel.cu", "block_common.cuh"))
    find = lambda pattern, text: re.search(pattern, text, re.S | re.M).group(0)  # noqa: E731
    text = HOST.replace("@PARAMS@", find(r"^struct BlockAppendParams \{.*?^};\n", common)).replace("@WORK@", find(r"^struct PageWork \{.*?^};\n", kernel))
    text = text.replace("@LAUNCH@", find(r"^cudaError_t launch_block_append\(.*?^}\n", kernel))
    d = tmp_path_factory.mktemp("launches")
    (d / "t.cpp").write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC", "-o", str(d / "t.so"), str(d / "t.cpp")],
                   check=True)
    return ctypes.CDLL(str(d / "t.so"))


@pytest.mark.parametrize("ragged,q,n_tok,batch,hq,hkv", [
    (0, 1, 1, 1, 8, 2), (0, 1, 32, 32, 28, 4), (1, 1, 32768, 1, 28, 4), (1, 0, 5, 3, 1, 1), (0, 0, 7, 7, 71, 1), (1, 1, 3, 65535, 64, 8),
    # more than 2^31 warps of pages: some 8200 sequences on, with the most KV heads; with queries beside them
    (1, 0, 1, 8191, 65535, 65535), (1, 0, 1, 8193, 65535, 65535), (1, 1, 3, 9000, 65535, 65535), (0, 1, 65535, 65535, 128 * 256, 256),
    (1, 1, 65535, 65535, 65535, 65535), (1, 0, 2 ** 31 - 1, 65535, 65535, 65535), (1, 1, 2 ** 30, 2, 1, 1)])
def test_every_task_once(lib, ragged, q, n_tok, batch, hq, hkv):
    out = np.zeros(7 * 16384, np.int64)     # a launch takes seven heads or more of the most pages
    n = lib.plan(ragged, q, n_tok, batch, hq, hkv, out.ctypes.data_as(ctypes.c_void_p))
    assert n >= 1
    tasks, head = n_tok // 16 + 2 * batch if ragged else batch, 0
    got = np.zeros(3, np.int64)
    for i, (ctas, head0, heads, page_ctas, stride, page_tasks, q_heads) in enumerate(out[:7 * n].reshape(n, 7).tolist()):
        assert head0 == head and heads >= 1 and page_tasks == tasks and 4 * ctas < 2 ** 31 and stride >= 1 and page_ctas * stride <= ctas
        head += heads
        warps = tasks * 2 * heads
        assert page_ctas == (warps + 1 + 3) // 4     # and one that reports
        for t in {0, 1, warps // 3, warps // 2, warps - 2, warps - 1, warps}:
            lib.work(head0, heads, t // 4, t % 4, got.ctypes.data_as(ctypes.c_void_p))
            assert got.tolist() == [t // (2 * heads), head0 + t // 2 % heads, t % 2]
        row_warps = (hq + q_heads - 1) // q_heads
        assert ctas - page_ctas == ((n_tok * row_warps + 3) // 4 if q and i == 0 else 0)
    assert head == hkv
    row_warps = n_tok * ((hq + q_heads - 1) // q_heads) if q else 0
    assert (n == 1) == (2 * tasks * hkv + row_warps < 2 ** 31 - 16)


@pytest.mark.parametrize("n_tok,hq,hkv", [(2 ** 31 - 1, 1, 1), (65535, 128 * 65535, 65535)])
def test_more_queries_than_warps(lib, n_tok, hq, hkv):
    """550 GB of queries and more: refused, not wrapped around."""
    out = np.zeros(7, np.int64)
    assert lib.plan(1, 1, n_tok, 1, hq, hkv, out.ctypes.data_as(ctypes.c_void_p)) == -1
