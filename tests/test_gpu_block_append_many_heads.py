"""An append whose pages times KV heads pass 2^31: one new token in the last of 9000 sequences, 65535 KV heads, in two launches (some
600 million blocks, nearly all with nothing to do: seconds)."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_last_sequence_of_many():
    import paper_2607_28699_gb300 as wc
    heads, batch = 65535, 9000
    desc = wc.BlockDesc(num_q_heads=heads, num_kv_heads=heads, num_pages=1, rotary_dim=0)
    x = torch.randn(1, heads, 128, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    want, got = wc.BlockCache.empty(desc), wc.BlockCache.empty(desc)
    q = wc.block_append(desc, x, -x, i32(1), i32(0)[None], want, q=x)
    cu, ctx, table = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (batch + 1, batch, batch))
    cu[-1] = ctx[-1] = 1
    table[:-1] = -1
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    many = wc.block_append(desc, x, -x, ctx, table[:, None], got, cu_new=cu, q=x, dev_status=word)
    assert wc.read_status(word) == 0 and torch.equal(q, many) and torch.equal(q, x)
    for name in ("k_codes", "v_codes"):     # the token's, first of 16: others are as they were allocated
        a, b = (getattr(c, name).view(heads, 16, 128)[:, 0] for c in (want, got))
        assert torch.equal(a, b) and bool(a.any(-1).all())
    assert torch.equal(want.k_scale, got.k_scale) and torch.equal(want.v_scale, got.v_scale)
