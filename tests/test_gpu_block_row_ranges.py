"""Row ranges that are not ascending: the sequences before the first bad one are as ever, the bad one's rows are not written."""

import numpy as np
import pytest
import torch

import _block_ref as R
from test_gpu_block_attention import SCALE, setup

pytestmark = pytest.mark.gpu
N = 24
BAD = [([0, 8, 25], 1), ([0, 8, 4], 1), ([0, 25, 24], 0), ([0, 8, 16, -100000, 24], 2), ([0, 5, 5, 9, 2 ** 31 - 1, 24], 3),
       ([0, 1, 8, -2 ** 31, -2 ** 31, 3, 9], 2), ([8, 16, -5, 20, 24], 1)]


@pytest.mark.parametrize("cu,good", BAD)
@pytest.mark.parametrize("hq,hkv", [(4, 2), (14, 1)])
@pytest.mark.parametrize("wide", [4, 200])
def test_extend(cu, good, hq, hkv, wide):
    """wide: block tables for which the contexts are split, so that another kernel writes the rows."""
    batch = len(cu) - 1
    ctx = [64] * batch
    wc, desc, bt, cache, _ = setup(91, R.INT8, torch.float16, ctx, hq, hkv, max_pages=wide)
    q = torch.from_numpy(np.random.default_rng(91).standard_normal((N, hq, 128)).astype(np.float32)).half()
    ws = wc.BlockWorkspace(desc, batch, N, wide)
    ws.view[256:].fill_(0xFF)      # partial results that nobody left are NaN
    ws.view[256:2048].fill_(0)     # (the decode's counts are not)
    out, lse = torch.full((N, hq, 128), 3.0, device="cuda").half(), torch.full((N, hq), 3.0, device="cuda")
    wc.block_extend_attention(desc, q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(),
                              torch.tensor(ctx, dtype=torch.int32).cuda(), R.to_gpu(cache, R.INT8), ws, out=out, lse=lse)
    assert wc.read_status(ws) == wc.DEV_BAD_ROWS
    ref = R.attention(q.double().numpy(), cu[:good + 1], bt, ctx[:good], cache["k_codes"], cache["v_codes"], cache["k_scale"], cache["v_scale"],
                      R.INT8, SCALE, True)
    ranges = np.zeros(N, int)      # that are valid by themselves and hold a row
    for lo, hi in zip(cu, cu[1:]):
        if 0 <= lo <= hi <= N:
            ranges[lo:hi] += 1
    # a row of two such ranges, one of them behind the bad one, may get either's result
    rows = np.flatnonzero((ranges == 1) & (np.arange(N) >= cu[0]) & (np.arange(N) < cu[good]))
    R.check_attention(out[rows], lse[rows], [x[rows] for x in ref], torch.float16)
    assert (out[ranges == 0] == 3).all() and (lse[ranges == 0] == 3).all()


@pytest.mark.parametrize("cu,good", BAD)
def test_append(cu, good):
    import paper_2607_28699_gb300 as wc
    batch, rng = len(cu) - 1, np.random.default_rng(92)
    bt, pages = R.page_tables(rng, [32] * batch)
    cache = R.random_cache(rng, pages, 2, R.INT8)
    gpu = R.to_gpu(cache, R.INT8)
    desc = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=pages)
    k, v = (torch.from_numpy(rng.standard_normal((N, 2, 128)).astype(np.float32)).half() for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((N, 4, 128)).astype(np.float32)).half()
    cos, sin = R.tables(n=64)
    word, q_out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((N, 4, 128), 3.0, device="cuda").half()
    wc.block_append(desc, k.cuda(), v.cuda(), torch.full((batch,), 32, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(), gpu,
                    cu_new=torch.tensor(cu, dtype=torch.int32).cuda(), cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda(),
                    q=q.cuda(), q_out=q_out, dev_status=word)
    assert wc.read_status(word) == wc.DEV_BAD_ROWS
    new = np.diff(cu[:good + 1]).tolist()
    rows = slice(cu[0], cu[good])
    R.append(cache, R.INT8, k[rows].float().numpy(), v[rows].float().numpy(), [32] * good, new, bt, cos, sin, 128, False)
    for b in range(good):
        for n in ("k_scale", "v_scale", "k_codes", "v_codes"):
            assert np.array_equal(getattr(gpu, n).cpu().numpy().view(cache[n].dtype)[bt[b]], cache[n][bt[b]]), (b, n)
    at = np.concatenate([np.arange(32 - n, 32) for n in new] or [np.zeros(0)]).astype(int)
    want = R.rotate(q[rows].float().numpy(), cos[at][:, None], sin[at][:, None], 128, False)
    assert torch.equal(q_out[rows].cpu(), torch.from_numpy(want).half())
