"""NaN among raw e4m3 codes reaches the rows that see its token and no others."""

import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (7, 1)])
@pytest.mark.parametrize("ctx,new", [([300, 40], [300, 40]), ([5000], [40]), ([9000, 700], [2, 30])])
@pytest.mark.parametrize("causal", [True, False])
def test_codes(scaled, hq, hkv, ctx, new, causal):
    """A NaN code among the values is NaN in its channel for the rows that see its token, one among the keys everywhere for these."""
    at = ctx[0] - max(1, new[0] // 2)

    def edit(cache, bt, q):
        def put(name, position, head, channel, byte):
            cache[name][bt[0, position // 16], head, position % 16, channel] = byte
        put("v_codes", at, 0, 5, 0x7F)
        put("v_codes", at, 0, 77, 0xFF)
        put("v_codes", max(at - 4, 0), hkv - 1, 127, 0x7F)
        put("v_codes", ctx[0] - 1, hkv - 1, 0, 0xFF)
        put("k_codes", ctx[0] - 1, 0, 64, 0x7F)
    out, lse, _ = run(52, R.E4M3, torch.bfloat16, ctx, hq, hkv, new=new, scaled=scaled, edit=edit, causal=causal)
    if causal:
        row = at - (ctx[0] - new[0])
        assert torch.isnan(out[row, 0, [5, 77]]).all() and torch.isfinite(out[:new[0] - 1, 0, :5]).all()
        assert torch.isfinite(lse[:new[0] - 1]).all() and torch.isfinite(out[new[0]:]).all()
