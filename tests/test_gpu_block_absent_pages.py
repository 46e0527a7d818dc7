"""Block table entries outside the pool: their tokens are left out, and nothing of any page stands in for them."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [None, [5, 6]])
@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_page_outside_the_pool(new, code):
    """The pool's first page, which no sequence has, holds NaN."""
    import paper_2607_28699_gb300 as wc

    def edit(cache, bt, q):
        free = sorted(set(range(len(cache["k_scale"]))) - set(bt[bt >= 0].tolist()))[0]
        bt[bt == 0] = free
        for n in "kv":
            cache[n + "_scale"][0] = np.nan
            cache[n + "_codes"][0] = 0x7F
        bt[0, 1], bt[1, 0] = 10 ** 6, -1
    out, lse, status = run(54, code, torch.float16, [90, 70], 4, 2, new=new, edit=edit, extra=1)
    assert status == wc.DEV_BAD_PAGE and torch.isfinite(out).all() and torch.isfinite(lse).all()
