"""Attention whose logits lie millions apart, beyond what fp32 resolves of them: the output stays an average of the values that are
seen, and lse near the largest logit.  The extend kernel, which takes more than 8 heads' decode too, up to logits of 2^22, the
decode kernel at any size."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup
from test_gpu_block_value_ranges import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("hq,new,size", [(7, None, s) for s in (20, 23, 25, 26, 27, 28, 30, 32, 60, 110)] +
                         [(h, n, s) for h, n in ((12, None), (7, [40, 3])) for s in (14, 16, 18)])
@pytest.mark.parametrize("near", [False, True])
def test_outputs_are_averages(code, size, hq, new, near):
    """near: all logits of one size that differ in their last bits only."""
    ctx = [700, 150]
    wc, desc, bt, cache, q = setup(97, code, torch.bfloat16, ctx, hq, 1, new)
    q *= 2.0 ** size
    if near:
        q[...] = q.abs() * 2.0 ** -12
        q[..., 0] = 2.0 ** size
        cache["k_codes"][:, :, :, 0] = R.encode(np.array([100.0]), code)[0]
        cache["k_scale"][:] = 0.5
    cu = None if new is None else [0] + np.cumsum(new).tolist()
    out, lse = attend(wc, desc, cache, bt, ctx, q, cu, code)
    causal, cu = new is not None, list(range(3)) if cu is None else cu
    _, want_lse, _, big = R.attention(q.double().numpy(), cu, bt, ctx, cache["k_codes"], cache["v_codes"], cache["k_scale"], cache["v_scale"],
                                      code, SCALE, causal)
    assert new is None and hq <= 8 or np.abs(want_lse).max() < 2.0 ** 22
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for b, c in enumerate(ctx):
        pages = bt[b, :(c + 15) // 16]
        v = (R.decode(cache["v_codes"][pages, 0], code) * cache["v_scale"][pages, 0].astype(np.float64)[:, None, None]).reshape(-1, 128)[:c]
        most = np.abs(v).max(0) * (1 + 2.0 ** -7)
        assert np.all(np.abs(out[cu[b]:cu[b + 1]].double().cpu().numpy()) <= most)
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse) <= big * 2.0 ** -17 + 2.0 ** -18 * (1 + np.abs(want_lse)))


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_decode_compares_exactly(code):
    """Exponents of 2^24 + 10 and 2^24 + 20 in turn, where fp32 holds every second number: a frame set by the first is passed by 16
    by the second, though the frame plus 15 rounds to that."""
    ctx = [256] * 300
    wc, desc, bt, cache, q = setup(98, code, torch.float16, ctx, 2, 1)
    q[...] = 0
    q[..., 0] = 64.0
    cache["k_codes"][:] = 0
    cache["k_codes"][:, :, :, 0] = R.encode(np.array([64.0]), code)[0]
    cache["v_codes"][:] = R.encode(np.array([1.0]), code)[0]
    cache["v_scale"][:] = 1.0
    for b in range(len(ctx)):
        cache["k_scale"][bt[b, 0::2]] = 2.0 ** 12 + 10 * 2.0 ** -12
        cache["k_scale"][bt[b, 1::2]] = 2.0 ** 12 + 20 * 2.0 ** -12
    gpu, ws = R.to_gpu(cache, code), wc.BlockWorkspace(desc, len(ctx), len(ctx), bt.shape[1])
    out = wc.block_decode_attention(desc, q.cuda(), torch.from_numpy(bt).cuda(), torch.tensor(ctx, dtype=torch.int32).cuda(), gpu, ws,
                                    softmax_scale=float(np.log(2)))
    assert (out - 1).abs().max() <= 2.0 ** -10
