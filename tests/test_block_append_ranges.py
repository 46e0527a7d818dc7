"""Which rows and lengths the block append takes (sequence() in csrc/block_append_kernel.cu): its own text compiled for the
host, over lengths and row ranges to the ends of int32, and the same lengths through the call."""

import ctypes
import itertools
import os
import re
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_28699_gb300", "csrc")
HOST = r"""
#include <cstdint>
#define __device__
#define __forceinline__ inline
constexpr int kPage = 16;
constexpr unsigned WC_DEV_BAD_CTX = 4, WC_DEV_BAD_ROWS = 128;
struct BlockAppendParams { const int32_t *cu_new, *ctx_lens; uint32_t* dev_status; int32_t n_tok, max_pages; };
template <typename T> T load_dep(const T* p) { return *p; }
static void report(const BlockAppendParams& p, uint32_t bit) { *p.dev_status |= bit; }
@CODE@
extern "C" int run(int lo, int hi, int ctx, int n_tok, int max_pages, int32_t* out, uint32_t* status) {
    const int32_t cu[2] = {lo, hi}, len = ctx;
    const BlockAppendParams p = {cu, &len, status, n_tok, max_pages};
    Sequence s = {};
    const bool taken = sequence<true>(p, 0, s);
    out[0] = s.lo, out[1] = s.n, out[2] = s.start;
    return taken;
}
"""
LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    text = open(os.path.join(CSRC, "block_append_kernel.cu")).read()
    code = re.search(r"^struct Sequence \{.*?^__device__ __forceinline__ bool sequence\(.*?^}\n", text, re.S | re.M)
    d = tmp_path_factory.mktemp("sequence")
    (d / "t.cpp").write_text(HOST.replace("@CODE@", code.group(0)))
    # integers wrap on the GPU
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-o", str(d / "t.so"), str(d / "t.cpp")], check=True)
    return ctypes.CDLL(str(d / "t.so"))


@pytest.mark.parametrize("n_tok,max_pages", [(0, 1), (1, 1), (40, 3), (40, 2 ** 26)])
def test_rows_and_lengths(lib, n_tok, max_pages):
    edges = sorted({LEAST, LEAST + 1, LEAST + 39, -41, -1, 0, 1, 16, 39, 40, 41, 48, 49, 16 * max_pages, 16 * max_pages + 1, MOST - 1, MOST})
    out, status = np.zeros(3, np.int32), np.zeros(1, np.uint32)
    for lo, hi, ctx in itertools.product(edges, edges, edges):
        status[0] = 0
        taken = lib.run(lo, hi, ctx, n_tok, max_pages, out.ctypes.data_as(ctypes.c_void_p), status.ctypes.data_as(ctypes.c_void_p))
        rows = 0 <= lo <= hi <= n_tok
        n = hi - lo
        fits = n <= ctx <= 16 * max_pages
        assert status[0] == (128 if not rows else 4 if n and not fits else 0), (lo, hi, ctx)
        assert bool(taken) == (rows and n > 0 and fits), (lo, hi, ctx)
        if taken:
            assert out.tolist() == [lo, n, ctx - n]


@pytest.mark.gpu
@pytest.mark.parametrize("ctx", [LEAST, LEAST + 2, -1, 2, 33, MOST])
def test_lengths_that_cannot_be(ctx):
    import paper_2607_28699_gb300 as wc
    desc = wc.BlockDesc(num_q_heads=2, num_kv_heads=1, num_pages=4, rotary_dim=0)
    cache = wc.BlockCache.empty(desc)
    rows, word = torch.ones(3, 1, 128, device="cuda").half(), torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    q = torch.ones(3, 2, 128, device="cuda").half()
    out = torch.full_like(q, 7.0)
    wc.block_append(desc, rows, rows, i32(ctx), i32(0, 1)[None], cache, cu_new=i32(0, 3), q=q, q_out=out, dev_status=word)
    assert wc.read_status(word) == wc.DEV_BAD_CTX
    assert all(not t.any() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)) and (out == 7).all()
