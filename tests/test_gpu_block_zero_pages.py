"""Attention where a page of zero values holds most of the softmax mass (an attention sink): it counts in the sum of weights,
and the other pages' weights keep their bits beside it."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup

pytestmark = pytest.mark.gpu


def check(out, lse, ref, cache, bt, ctx, cu, code, act):
    """_block_ref's bound without its absolute term, but for what fp16 outputs' subnormals round off.  In its place: a weight is rounded to fp16 in units in which the largest
    weighted value scale p vs of its row is at least 1, so by no more than 2^-25 of that where it is subnormal."""
    want, want_lse, mass, big, share = ref      # share: the softmax mass of the pages with values, no less than their largest p
    u = 2.0 ** -11 if act == torch.float16 else 2.0 ** -8
    d = (big * 2.0 ** -17)[..., None]
    largest = np.zeros(want.shape[:2])
    for b, c in enumerate(ctx):
        vs = np.repeat(cache["v_scale"][bt[b, :(c + 15) // 16]].max(-1), 16)[:c].max()
        largest[cu[b]:cu[b + 1]] = vs * c * (127 if code == R.INT8 else 448)
    tol = u * np.abs(want) + (1 + u) * ((2.0 ** -11 + 2.0 ** -18 + 2 * d) * mass + 2.0 ** -25 * (largest * share)[..., None])
    tol += 2.0 ** -25 if act == torch.float16 else 0.0
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), float(np.linalg.norm(got - want) / np.linalg.norm(want))
    assert np.all(np.abs(got_lse - want_lse) <= d[..., 0] + 2.0 ** -18 * (1 + np.abs(want_lse)))


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("hq,hkv,new", [(7, 1, None), (4, 2, None), (12, 1, None), (7, 1, [40, 3]), (4, 2, [130, 20])])
@pytest.mark.parametrize("down", [0, 12, 55])
@pytest.mark.parametrize("above", [8.0, 16.0])
@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
def test_sink_of_zero_values(code, hq, hkv, new, down, above, act):
    if act == torch.float16 and down:
        pytest.skip("such outputs are below fp16's normal numbers")
    # a decode of up to 8 heads: so many sequences that a warp has several of a sequence's pages
    ctx = [400] * 300 if new is None and hq // hkv <= 8 else [700, 150]
    wc, desc, bt, cache, q = setup(41, code, act, ctx, hq, hkv, new)
    q[..., 0] = 8.0
    hundred = R.encode(np.array([100.0]), code)
    cache["v_scale"] *= np.float32(2.0 ** -down)
    for b in range(len(ctx)):     # the first page's fourth key: a logit of `above`, the others' are around 0
        sink = bt[b, 0]
        cache["k_codes"][sink] = 0
        cache["k_codes"][sink, :, 3, 0] = hundred
        cache["k_scale"][sink] = np.float32(above / (SCALE * 8.0 * R.decode(hundred, code)[0]))
        cache["v_scale"][sink] = 0      # the codes stay: a scale of 0 silences them
    cu = list(range(len(ctx) + 1)) if new is None else [0] + np.cumsum(new).tolist()
    gpu = R.to_gpu(cache, code)
    ws = wc.BlockWorkspace(desc, len(ctx), q.shape[0], bt.shape[1])
    ctx_g, bt_g = torch.tensor(ctx, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda()
    if new is None:
        out, lse = wc.block_decode_attention(desc, q.cuda(), bt_g, ctx_g, gpu, ws, return_lse=True)
    else:
        out, lse = wc.block_extend_attention(desc, q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), bt_g, ctx_g, gpu, ws, return_lse=True)
    assert wc.read_status(ws) == 0
    args = (q.double().numpy(), cu, bt, ctx, cache["k_codes"])
    ref = R.attention(*args, cache["v_codes"], cache["k_scale"], cache["v_scale"], code, SCALE, new is not None)
    # values of 1 in the pages with values: their share of the softmax
    ones, scales = np.broadcast_to(R.encode(np.array([1.0]), code), cache["v_codes"].shape), (cache["v_scale"] > 0).astype(np.float32)
    mass = R.attention(*args, ones, cache["k_scale"], scales, code, SCALE, new is not None)[0].max(-1)
    check(out, lse, (*ref, mass), cache, bt, ctx, cu, code, act)
