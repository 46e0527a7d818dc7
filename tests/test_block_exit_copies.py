"""No CTA of the block extend ends with copies into its shared memory in flight: the warp that issued them waits for the last ones
itself, whether or not the warps that read them gave up, before the CTA's last barrier."""

import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_loading_warp_waits_for_its_last_copies():
    code = open(os.path.join(ROOT, "paper_2607_28699_gb300", "csrc", "block_extend_kernel.cu")).read()
    role = code[code.index("warp == kLoadWarp"):]
    role = role[:role.index("__syncthreads();")]
    assert role.count("tma_page(") == 1
    tail = role[role.index("next = after;"):]
    loop, body = re.search(r"\n *(for \(int side = 0; side < 2; \+\+side\)) \{\n(.*)", tail, re.S).groups()
    before = tail[:tail.index(loop)]
    assert "if" not in "\n".join(line.split("//")[0] for line in before.splitlines())      # not only where a wait gave up
    assert re.search(r"if \(ok\) \(void\)mbar_wait_bounded<\d+>\(&s\.codes_full\[side\], \(n - 1\) & 1\);", body)
    assert re.search(r"else for \(int parity = 0; parity < 2; \+\+parity\) \(void\)mbar_wait_bounded<\d+>\(&s\.codes_full\[side\], parity\);", body)
