"""Infinities and NaN among a block-scaled cache's page scales reach the rows that see their page and no others; lse does not
depend on values."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (7, 1)])
@pytest.mark.parametrize("ctx,new,page", [([300, 40], [300, 40], 9), ([5000], [40], 311), ([200], [3], 2)])
def test_page_scales(code, side, value, hq, hkv, ctx, new, page):
    """A page as the append leaves it after a row with NaN: a prompt, rows over a context that is split, rows all after it."""
    def edit(cache, bt, q):
        cache[side + "_scale"][bt[0, page]] = value
        cache[side + "_codes"][bt[0, page]] = 0
    out, lse, _ = run(51, code, torch.float16, ctx, hq, hkv, new=new, edit=edit)
    before = max(0, page * 16 - (ctx[0] - new[0]))      # rows that see nothing of the page
    assert torch.isfinite(out[:before]).all() and torch.isnan(out[before:new[0]]).all() and torch.isfinite(out[new[0]:]).all()
    assert torch.isfinite(lse[:before]).all() and torch.isfinite(lse[new[0]:]).all()
    assert (torch.isnan(lse[before:new[0]]) if side == "k" else torch.isfinite(lse)).all()


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("ctx", [[200], [400] * 300])
def test_decode_value_scales(code, value, ctx):
    def edit(cache, bt, q):
        cache["v_scale"][bt[0, 2]] = value
        cache["v_codes"][bt[0, 2]] = 0
    out, lse, _ = run(53, code, torch.float16, ctx, 7, 1, edit=edit)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1:]).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_a_prompt_with_a_nan_row(code):
    """Appended and attended to as a server does: the tokens before its page are as without it."""
    import paper_2607_28699_gb300 as wc
    n, hq, hkv = 400, 4, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, hq + 2 * hkv, 128, generator=g, device="cuda").half()
    desc = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=25, code=code, rotary_dim=0)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    table, ctx, cu = torch.arange(25, dtype=torch.int32, device="cuda")[None].contiguous(), i32(n), i32(0, n)
    outs = []
    for bad in (False, True):
        y = x.clone()
        if bad:
            y[150, hq + hkv, 3] = float("nan")      # a value of KV head 0
        cache, ws = wc.BlockCache.empty(desc), wc.BlockWorkspace(desc, 1, n, 25)
        wc.block_append(desc, y[:, hq:hq + hkv], y[:, hq + hkv:], ctx, table, cache, cu_new=cu)
        outs.append(wc.block_extend_attention(desc, y[:, :hq], cu, table, ctx, cache, ws, softmax_scale=SCALE).float())
    clean, got = outs
    assert torch.isnan(got[144:, :2]).all()
    # both are within 2^-10 of the output and of sum p |v| (<= max |v|) of the definition
    for rows, heads in ((slice(0, 144), slice(0, 4)), (slice(0, n), slice(2, 4))):
        assert (got[rows, heads] - clean[rows, heads]).abs().max() <= 2.0 ** -9 * float(x[:, hq + hkv:].abs().max())
