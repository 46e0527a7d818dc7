"""Attention where every logit is far below or above 0, up to near fp32's ends: the softmax is of their differences."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup
from test_gpu_block_value_ranges import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("size", [-2.0 ** 120, -2.0 ** 100, -2.0 ** 96, 2.0 ** 120])
@pytest.mark.parametrize("hq,new", [(7, None), (12, None), (7, [3, 2])])
def test_equal_keys(code, size, hq, new):
    """Logits of 8.5 times size.  One page a sequence: at these sizes fp32 holds no difference between pages' value scales beside them."""
    ctx = [16, 5]
    wc, desc, bt, cache, q = setup(95, code, torch.bfloat16, ctx, hq, 1, new)
    q[...] = 0
    q[..., 0] = size
    cache["k_codes"][:] = 0
    cache["k_codes"][:, :, :, 0] = R.encode(np.array([96.0]), code)[0]
    cache["k_scale"][:] = 1.0
    out, lse = attend(wc, desc, cache, bt, ctx, q, None if new is None else [0] + np.cumsum(new).tolist(), code)
    n = [1, 1] if new is None else new
    for b in range(2):
        v = R.decode(cache["v_codes"][bt[b, 0], 0], code) * float(cache["v_scale"][bt[b, 0], 0])
        for i in range(n[b]):
            row, see = sum(n[:b]) + i, ctx[b] - n[b] + i + 1
            want = v[:see].mean(0)
            # fp16 weights and fp32 sums of them, out rounded to bf16
            tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * np.abs(v[:see]).mean(0)
            assert np.all(np.abs(out[row].double().cpu().numpy() - want) <= tol)
            assert np.allclose(lse[row].cpu().numpy(), SCALE * 96 * size, rtol=1e-5)
