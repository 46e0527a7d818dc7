"""Rows that are not normed are rotated the same in every call: products rounded one by one, as wc_block_append has it, whether the
other side is normed or not, and alone."""

import pytest
import torch

import _block_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [128, 48])
def test_same_bits(act, interleaved, rot):
    import paper_2607_28699_gb300 as wc
    n, hq, hkv = 1024, 28, 4     # 3.7 million values: a rounding less would change some hundreds of them
    g = torch.Generator(device="cuda").manual_seed(rot)
    x = torch.randn(n, hq + 2 * hkv, 128, generator=g, device="cuda").to(act)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    cos, sin = (torch.from_numpy(t).cuda() for t in R.tables(rot=rot, n=n))
    w = 1 + 0.5 * torch.rand(128, generator=g, device="cuda")
    layout = wc.ROPE_INTERLEAVED if interleaved else wc.ROPE_HALF
    desc = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=n // 16, code=wc.CODE_INT8, rope_layout=layout, rotary_dim=rot)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    table, at = torch.arange(n // 16, dtype=torch.int32, device="cuda")[None], torch.arange(n, dtype=torch.int32, device="cuda")

    def append(**norms):
        cache = wc.BlockCache.empty(desc)
        out = wc.block_append(desc, k, v, i32(n), table, cache, cu_new=i32(0, n), cos=cos, sin=sin, q=q, **norms)
        return out, cache

    want, plain = append()
    got, _ = append(k_norm=w)
    assert torch.equal(got, want)
    got, cache = append(q_norm=w)
    assert not torch.equal(got, want)
    assert torch.equal(cache.k_codes, plain.k_codes) and torch.equal(cache.k_scale, plain.k_scale)
    for norms in ({}, {"k_norm": w}):
        got, _ = wc.qk_norm_rotate(q, k, at, cos, sin, rope_layout=layout, **norms)
        assert torch.equal(got, want)
    # as keys, beside normed queries
    _, got = wc.qk_norm_rotate(q, q, at, cos, sin, q_norm=w, rope_layout=layout)
    assert torch.equal(got, want)
    # decode's form: few rows
    one = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=n // 16, code=wc.CODE_INT8, rope_layout=layout, rotary_dim=rot)
    few = [wc.block_append(one, k[-64:], v[-64:], at[-64:] + 1, torch.arange(64, dtype=torch.int32, device="cuda")[:, None].expand(64, n // 16).contiguous(),
                           wc.BlockCache.empty(one), cos=cos, sin=sin, q=q[-64:], **norms) for norms in ({}, {"k_norm": w})]
    assert torch.equal(few[0], want[-64:]) and torch.equal(few[1], want[-64:])
