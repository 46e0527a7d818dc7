"""Attention with value scales near the ends of their range: the sum of weights, which holds the scales' reciprocals, neither
overflows nor vanishes.  From 2^-100 on values count, below it they are 0; lse does not depend on them."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup

pytestmark = pytest.mark.gpu


def attend(wc, desc, cache, bt, ctx, q, cu, code):
    gpu, ws = R.to_gpu(cache, code), wc.BlockWorkspace(desc, len(ctx), q.shape[0], bt.shape[1])
    ctx_g, bt_g = torch.tensor(ctx, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda()
    if cu is None:
        out, lse = wc.block_decode_attention(desc, q.cuda(), bt_g, ctx_g, gpu, ws, return_lse=True)
    else:
        out, lse = wc.block_extend_attention(desc, q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), bt_g, ctx_g, gpu, ws, return_lse=True)
    assert wc.read_status(ws) == 0
    return out, lse


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("exponent", [-126, -125, -110, -101, -100, -60, 118])
@pytest.mark.parametrize("hq,hkv,new", [(7, 1, None), (9, 1, None), (4, 2, [40, 3])])
@pytest.mark.parametrize("rising", [False, True])
def test_all_pages_at(code, exponent, hq, hkv, new, rising):
    """rising: the logits of the pages after a context's first 128 tokens lie above the first ones', by up to what the running maximum
    lets pass."""
    ctx = [700, 150]
    wc, desc, bt, cache, q = setup(61, code, torch.bfloat16, ctx, hq, hkv, new)
    top = 127.0 if code == R.INT8 else 448.0
    cache["v_scale"][:] = 2.0 ** exponent if exponent < 0 else np.float32(2.0 ** 127 / top / 4)
    if rising:
        q[...] = q.abs() * 0.01
        q[..., 0] = 1.0
        for b in range(2):
            for j, page in enumerate(bt[b]):
                if page >= 0:
                    cache["k_codes"][page, :, :, 0] = R.encode(np.array([100.0]), code)
                    cache["k_scale"][page] = 0.0 if j < 8 else 0.6
    cu = None if new is None else [0] + np.cumsum(new).tolist()
    out, lse = attend(wc, desc, cache, bt, ctx, q, cu, code)
    args = (q.double().numpy(), list(range(3)) if cu is None else cu, bt, ctx, cache["k_codes"], cache["v_codes"], cache["k_scale"])
    # the tolerance has an absolute part for fp16's subnormals: values as if their scale were 1 / top
    scale = cache["v_scale"].copy()
    assert torch.isfinite(lse).all()
    if exponent < -100:
        assert out.abs().max() == 0
        scale[:] = 0
    else:
        out = (out.double() / float(scale.flat[0]) / top)
        scale[:] = 1 / top
    ref = R.attention(*args, scale, code, SCALE, new is not None)
    R.check_attention(out, lse, ref, torch.bfloat16)
