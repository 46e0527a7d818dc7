"""Weights far below a row's largest still count: one sharp key over tokens that each weigh 2^-26.3 of it, in channels where its own
value is 0."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup
from test_gpu_block_value_ranges import attend

pytestmark = pytest.mark.gpu
BATCH, CTX, DOWN = 600, 512, 26.3


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,new", [(7, None), (1, 1), (12, None)])
@pytest.mark.parametrize("last", [False, True])
def test_sharp_key(code, act, hq, new, last):
    """So many sequences that a warp (decode) or a CTA has pages beside the sharp key's; it comes first or last."""
    ctx = [CTX] * BATCH
    wc, desc, bt, cache, q = setup(71, code, act, ctx, hq, 1, None if new is None else [1] * BATCH)
    q[...] = 0
    q[..., 0] = 1.0
    sharp, some = R.encode(np.array([96.0]), code)[0], R.encode(np.array([64.0]), code)[0]
    cache["k_codes"][:] = 0
    cache["k_scale"][:] = 1.0
    cache["v_codes"][:] = some
    cache["v_scale"][:] = 64.0
    for b in range(BATCH):
        page, at = (bt[b, -1], 15) if last else (bt[b, 0], 0)
        cache["k_codes"][page, 0, at, 0] = sharp
        cache["k_scale"][page] = np.float32(DOWN * np.log(2) / (SCALE * 96))
        cache["v_codes"][page, 0, at, :64] = 0
    cu = None if new is None else list(range(BATCH + 1))
    out, lse = attend(wc, desc, cache, bt, ctx, q, cu, code)
    want, want_lse, mass, big = R.attention(q.double().numpy(), list(range(BATCH + 1)), bt, ctx, cache["k_codes"], cache["v_codes"],
                                            cache["k_scale"], cache["v_scale"], code, SCALE, False)
    # as _block_ref's bound; for the absolute part: a weight's fp16 subnormals are 2^-24 where the largest weight is 2^7 at least
    u, d = 2.0 ** -11 if act == torch.float16 else 2.0 ** -8, big * 2.0 ** -17
    tol = u * np.abs(want) + (1 + u) * ((2.0 ** -11 + 2.0 ** -18 + 2 * d)[..., None] * mass + 2.0 ** -32 * CTX * 64 * 64)
    got = out.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:3], want[bad][:3], tol[bad][:3])
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse) <= d + 2.0 ** -18 * (1 + np.abs(want_lse)))
