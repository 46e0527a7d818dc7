"""The binding refuses a block cache whose tensors hold another kind of code than the descriptor names (no GPU needed)."""

import pytest
import torch


@pytest.fixture(scope="module")
def wc():
    import paper_2607_28699_gb300 as w
    return w


def calls(wc, desc, cache):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    k, q = torch.zeros(1, 2, 128, dtype=torch.float16), torch.zeros(1, 4, 128, dtype=torch.float16)
    table = torch.zeros(1, 1, dtype=torch.int32)
    stream = torch.Stream("cpu")
    yield lambda: wc.block_append(desc, k, k, i32(1), table, cache, stream=stream)
    yield lambda: wc.block_decode_attention(desc, q, table, i32(1), cache, None, stream=stream)
    yield lambda: wc.block_extend_attention(desc, q, i32(0, 1), table, i32(1), cache, None, stream=stream)


@pytest.mark.parametrize("name,k_type,v_type", [
    ("CODE_E4M3", torch.int8, torch.int8), ("CODE_E4M3", torch.uint8, torch.int8), ("CODE_E4M3", torch.int8, torch.float8_e4m3fn),
    ("CODE_E4M3", torch.float8_e5m2, torch.float8_e5m2), ("CODE_E4M3", torch.bool, torch.bool), ("CODE_INT8", torch.uint8, torch.uint8),
    ("CODE_INT8", torch.float8_e4m3fn, torch.float8_e4m3fn), ("CODE_INT8", torch.int8, torch.uint8)])
def test_refused(wc, name, k_type, v_type):
    desc = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=3, rotary_dim=0, code=getattr(wc, name))
    codes = [torch.zeros(3, 2, 16, 128, dtype=torch.uint8).view(t) for t in (k_type, v_type)]
    cache = wc.BlockCache(*codes, torch.zeros(3, 2), torch.zeros(3, 2))
    for call in calls(wc, desc, cache):
        with pytest.raises(ValueError, match="codes"):
            call()


@pytest.mark.parametrize("name,types", [("CODE_INT8", (torch.int8,)), ("CODE_E4M3", (torch.uint8, torch.float8_e4m3fn))])
def test_taken(wc, name, types):
    desc = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=3, code=getattr(wc, name))
    for t in types:
        cache = wc.BlockCache(*(torch.zeros(3, 2, 16, 128, dtype=torch.uint8).view(t) for _ in range(2)), torch.zeros(3, 2), torch.zeros(3, 2))
        assert len(wc._block_cache(desc, cache)) == 4
    wc._block_cache(desc, wc.BlockCache.empty(desc, device="cpu"))
