"""The bounded waits of the block kernels, where they run out: all lanes of a warp get one answer, since what follows (elected lanes,
warp barriers) needs all of them.  The extend's own text is compiled for the host with a thread per lane and a barrier
that some lanes see complete at the very poll at which the others give up."""

import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_28699_gb300", "csrc")
HOST = r"""
#include <atomic>
#include <barrier>
#include <cstdint>
#include <thread>
#include <vector>
#define __device__
#define __forceinline__ inline
struct Shared { int abandoned; };
struct Warp { std::barrier<> all{32}; std::atomic<unsigned> bits{0}; };
static thread_local Warp* warp_of;
static thread_local int lane, polls, done_at, late_at;
static unsigned ballot(bool x) {
    if (x) warp_of->bits |= 1u << lane;
    warp_of->all.arrive_and_wait();
    const unsigned r = warp_of->bits;
    warp_of->all.arrive_and_wait();
    warp_of->bits = 0;
    warp_of->all.arrive_and_wait();
    return r;
}
static bool __all_sync(unsigned, bool x) { return ballot(x) == 0xffffffffu; }
static bool __any_sync(unsigned, bool x) { return ballot(x) != 0; }
static uint32_t smem_addr(const void*) { return 0; }
static uint32_t host_try() { return ++polls >= done_at; }
static uint64_t host_time() { return polls >= late_at ? 5000000000ull : 1000000000ull; }
@CODE@
extern "C" void run(const int32_t* done, int late, int abandoned, int32_t* got) {
    Shared s = {abandoned};
    Warp w;
    std::vector<std::thread> threads;
    for (int i = 0; i < 32; ++i)
        threads.emplace_back([&, i] {
            warp_of = &w, lane = i, polls = 0, done_at = done[i], late_at = late;
            got[i] = wait(s, nullptr, 0);
        });
    for (auto& t : threads) t.join();
    got[32] = s.abandoned;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    text = open(os.path.join(CSRC, "block_extend_kernel.cu")).read()
    code = re.search(r"^__device__ __forceinline__ bool wait\(.*?^}\n", text, re.S | re.M).group(0)
    code, n = re.subn(r'asm volatile\("\{[^;]*;[^)]*try_wait.*?"memory"\);', "ok = host_try();", code, flags=re.S)
    code, m = re.subn(r'asm volatile\("mov\.u64 %0, %globaltimer;".*?\);', "now = host_time();", code, flags=re.S)
    assert n == 1 and m == 1
    d = tmp_path_factory.mktemp("wait")
    (d / "t.cpp").write_text(HOST.replace("@CODE@", code))
    subprocess.run(["g++", "-std=c++20", "-O1", "-pthread", "-shared", "-fPIC", "-o", str(d / "t.so"), str(d / "t.cpp")], check=True)
    return ctypes.CDLL(str(d / "t.so"))


NEVER = 10 ** 9


@pytest.mark.parametrize("done,late,abandoned,want,left", [
    ([1] * 32, NEVER, 0, True, 0),                          # there already
    ([1] * 31 + [7], NEVER, 0, True, 0),                    # one lane sees it a little later
    ([200] * 32, NEVER, 0, True, 0),
    ([NEVER] * 32, 100, 0, False, 1),                       # it never comes
    ([NEVER] * 32, NEVER, 1, False, 1),                     # another warp gave up
    ([128] * 16 + [NEVER] * 16, 100, 0, False, 1),          # half the lanes see it as the others give up
    ([128] + [NEVER] * 31, NEVER, 1, False, 1),
    ([NEVER] * 31 + [64], NEVER, 1, False, 1)])
def test_one_answer(lib, done, late, abandoned, want, left):
    got = np.full(33, -1, np.int32)
    d = np.array(done, np.int32)
    lib.run(d.ctypes.data_as(ctypes.c_void_p), late, abandoned, got.ctypes.data_as(ctypes.c_void_p))
    assert got[:32].tolist() == [int(want)] * 32 and got[32] == left


def test_the_decode_votes_on_its_waits():
    code = open(os.path.join(CSRC, "block_decode_kernel.cu")).read()
    uses = re.findall(r"[^\n]*mbar_wait_bounded[^\n]*", code)
    assert len(uses) == 2
    assert "__all_sync(0xffffffffu, mbar_wait_bounded(" in uses[0]
    assert "(void)mbar_wait_bounded" in uses[1]     # at the end, with nothing of the warp after it
