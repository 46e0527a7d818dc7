"""A token whose rotary position is outside the tables is not written by the block append: neither its key nor its value, and
neither takes part in its page's scales."""

import numpy as np
import pytest
import torch

import _block_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("given", [True, False])
def test_neither_half_is_written(code, interleaved, given):
    """Positions that are given, or contexts that reach past the tables."""
    import paper_2607_28699_gb300 as wc
    n, start = 40, 5
    rng = np.random.default_rng(81)
    bt = np.array([[3, 0, 2]], np.int32)
    cache = R.random_cache(rng, 4, 2, code)
    if code == R.E4M3:
        for m in ("k_scale", "v_scale"):
            cache[m] = np.exp2(np.round(np.log2(cache[m]))).astype(np.float32)
    before = {m: a.copy() for m, a in cache.items()}
    gpu = R.to_gpu(cache, code)
    cos, sin = R.tables(n=64 if given else 38)
    positions = np.arange(start, start + n) if not given else rng.integers(0, 64, n)
    if given:
        positions[[2, 17, 30]] = [-1, 64, 2 ** 31 - 1]
    bad = (positions < 0) | (positions >= len(cos))
    k, v = (torch.from_numpy(rng.standard_normal((n, 2, 128)).astype(np.float32)).half() for _ in range(2))
    k[bad], v[bad] = 100.0, 100.0     # would set their pages' scales
    desc = wc.BlockDesc(num_q_heads=2, num_kv_heads=2, num_pages=4, code=code, rope_layout=wc.ROPE_INTERLEAVED if interleaved else wc.ROPE_HALF)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    wc.block_append(desc, k.cuda(), v.cuda(), i32(start + n), torch.from_numpy(bt).cuda(), gpu, cu_new=i32(0, n), cos=torch.from_numpy(cos).cuda(),
                    sin=torch.from_numpy(sin).cuda(), positions=i32(*positions.tolist()) if given else None, dev_status=word)
    assert wc.read_status(word) == wc.DEV_BAD_POSITION
    # the definition with rows of zeros in the bad ones' place, which have no part in a scale; their codes stay
    f = [x.float().numpy() * ~bad[:, None, None] for x in (k, v)]
    R.append(cache, code, *f, [start + n], [n], bt, cos, sin, 128, interleaved, np.where(bad, 0, positions))
    for t in np.flatnonzero(bad) + start:
        for m in ("k_codes", "v_codes"):
            cache[m][bt[0, t // 16], :, t % 16] = before[m][bt[0, t // 16], :, t % 16]
    for m in ("k_scale", "v_scale"):
        assert np.array_equal(getattr(gpu, m).cpu().numpy(), cache[m]), m
    for m in ("k_codes", "v_codes"):
        assert np.array_equal(R.decode(getattr(gpu, m).cpu().numpy().view(np.uint8), code), R.decode(cache[m], code)), m
