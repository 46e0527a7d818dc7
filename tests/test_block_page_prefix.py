"""The block decode's page sums (page_prefix in csrc/block_decode_kernel.cu), its own text compiled for the host with a
thread per lane: the sums for every batch, and for batches whose warps each find them without a barrier that no
place of the shared array ever holds anything but its final sum, since other warps read it meanwhile."""

import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_28699_gb300", "csrc")
HOST = r"""
#include <algorithm>
#include <atomic>
#include <barrier>
#include <cstdint>
#include <memory>
#include <mutex>
#include <thread>
#include <vector>
#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
constexpr int kPage = 16, kWarps = 16, kThreads = 512, kDecodeBatch = 2048;
constexpr unsigned WC_DEV_BAD_CTX = 4;
struct BlockAttentionParams { const int32_t* ctx_lens; uint32_t* status; int32_t batch, max_pages; };
struct Cell {     // every value that was ever stored
    std::mutex lock;
    std::vector<int> stored;
    Cell& operator=(int x) { std::lock_guard<std::mutex> g(lock); stored.push_back(x); return *this; }
    Cell& operator+=(int x) { std::lock_guard<std::mutex> g(lock); stored.push_back(stored.back() + x); return *this; }
};
struct Shared { Cell prefix[kDecodeBatch + 1]; std::atomic<int> ctx[kDecodeBatch]; int warp_sum[kWarps]; };
struct Warp { std::barrier<> all{32}; int value[32]; };
static thread_local struct { int x; } threadIdx;
static thread_local Warp* warp_of;
static thread_local std::barrier<>* cta;
template <typename T> T load_dep(const T* p) { return *p; }
static void atomicOr(uint32_t* p, uint32_t bit) { __atomic_fetch_or(p, bit, __ATOMIC_SEQ_CST); }
static int __shfl_up_sync(unsigned, int x, int o) {
    const int lane = threadIdx.x & 31;
    warp_of->value[lane] = x;
    warp_of->all.arrive_and_wait();
    const int y = warp_of->value[lane >= o ? lane - o : lane];
    warp_of->all.arrive_and_wait();
    return y;
}
static void __syncwarp() { warp_of->all.arrive_and_wait(); }
static void __syncthreads() { cta->arrive_and_wait(); }
@CODE@
extern "C" int run(const int32_t* ctx, int batch, int max_pages, int32_t* sums, int32_t* others, uint32_t* status) {
    auto s = std::make_unique<Shared>();
    const BlockAttentionParams p = {ctx, status, batch, max_pages};
    std::vector<Warp> warps(kWarps);
    std::barrier<> all(kThreads);
    std::vector<std::thread> threads;
    for (int t = 0; t < kThreads; ++t)
        threads.emplace_back([&, t] {
            threadIdx.x = t;
            warp_of = &warps[t / 32];
            cta = &all;
            page_prefix(p, *s, true);
        });
    for (auto& t : threads) t.join();
    for (int b = 0; b <= batch; ++b) {
        if (s->prefix[b].stored.empty()) return 1;
        sums[b] = s->prefix[b].stored.back();
        others[b] = 0;
        for (int x : s->prefix[b].stored) others[b] += x != sums[b];
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    text = open(os.path.join(CSRC, "block_decode_kernel.cu")).read()
    code = re.search(r"^__device__ __forceinline__ int context\(.*?^}\n.*?^__device__ __forceinline__ void page_prefix\(.*?^}\n", text, re.S | re.M)
    d = tmp_path_factory.mktemp("page_prefix")
    (d / "t.cpp").write_text(HOST.replace("@CODE@", code.group(0)))
    subprocess.run(["g++", "-std=c++20", "-O1", "-pthread", "-shared", "-fPIC", "-o", str(d / "t.so"), str(d / "t.cpp")], check=True)
    return ctypes.CDLL(str(d / "t.so"))


@pytest.mark.parametrize("batch", [1, 2, 3, 31, 32, 33, 513, 2048])
def test_page_sums(lib, batch):
    ctx = np.random.default_rng(batch).integers(1, 400, batch).astype(np.int32)
    ctx[5::5] = 0
    bad = batch > 6
    if bad:
        ctx[1], ctx[2] = -1, 401     # lengths that cannot be count as none
    sums, others, status = np.zeros(batch + 1, np.int32), np.zeros(batch + 1, np.int32), np.zeros(1, np.uint32)
    assert lib.run(*(a.ctypes.data_as(ctypes.c_void_p) if isinstance(a, np.ndarray) else a for a in (ctx, batch, 25, sums, others, status))) == 0
    pages = np.where((ctx < 0) | (ctx > 400), 0, (ctx + 15) // 16)
    assert np.array_equal(sums, np.concatenate([[0], np.cumsum(pages)]))
    assert status[0] == (4 if bad else 0)
    if batch <= 32:      # no barrier of the CTA before the sums are read
        assert not others.any(), others
