"""Append to the block-scaled cache: codes, scales and rotated queries, bit for bit the definition's
float32 operations, and near the rotation in float64."""

import numpy as np
import pytest
import torch

import _block_ref as R

pytestmark = pytest.mark.gpu


def run(seed, code, act, ctx, new, hkv=2, hq=4, rot=128, interleaved=False, positions=None, packed=False, edit=None,
        decode_form=False, batches=1, queries=True):
    import paper_2607_28699_gb300 as wc
    rng = np.random.default_rng(seed)
    bt, pages = R.page_tables(rng, ctx, extra=2)
    cache = R.random_cache(rng, pages, hkv, code)
    if code == R.E4M3:
        for n in ("k_scale", "v_scale"):
            cache[n] = np.exp2(np.round(np.log2(cache[n]))).astype(np.float32)
    n = sum(new)
    x = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, 128)).astype(np.float32))
    x *= torch.from_numpy(np.exp(rng.standard_normal((n, hq + 2 * hkv, 1))).astype(np.float32))
    if edit is not None:
        edit(x, hq, hkv)
    x = x.to(act)
    cos, sin = R.tables(rot=rot, n=max(max(ctx), 64))
    desc = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=pages, code=code,
                        rope_layout=wc.ROPE_INTERLEAVED if interleaved else wc.ROPE_HALF, rotary_dim=rot)
    gpu = R.to_gpu(cache, code)
    g = x.cuda()
    q, k, v = g[:, :hq], g[:, hq:hq + hkv], g[:, hq + hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(batches):
        q_out = wc.block_append(desc, k, v, torch.tensor(ctx, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(), gpu,
                                cu_new=None if decode_form else cu, cos=torch.from_numpy(cos).cuda() if rot else None,
                                sin=torch.from_numpy(sin).cuda() if rot else None,
                                positions=None if positions is None else torch.tensor(positions, dtype=torch.int32).cuda(),
                                q=q if queries else None, dev_status=word)
    f = x.float().numpy()
    for _ in range(batches):
        R.append(cache, code, f[:, hq:hq + hkv], f[:, hq + hkv:], ctx, new, bt, cos, sin, rot, interleaved, positions)
    assert wc.read_status(word) == 0
    for name in ("k_scale", "v_scale"):
        assert np.array_equal(getattr(gpu, name).cpu().numpy(), cache[name], equal_nan=True), name
    for name in ("k_codes", "v_codes"):
        got = getattr(gpu, name).cpu().numpy().view(np.uint8)
        # a zero's sign is no part of the value
        a, b = R.decode(got, code), R.decode(cache[name], code)
        assert np.array_equal(a, b, equal_nan=True), (name, int((a != b).sum()))
    at = np.concatenate([np.arange(c - m, c) for c, m in zip(ctx, new)]).astype(int) if positions is None else np.asarray(positions)
    if queries:
        want = R.rotate(f[:, :hq], cos[at][:, None], sin[at][:, None], rot, interleaved) if rot else f[:, :hq]
        with np.errstate(over="ignore"):
            assert torch.equal(q_out.cpu(), torch.from_numpy(want).to(act))
        exact = R.rotate(f[:, :hq].astype(np.float64), cos[at].astype(np.float64)[:, None], sin[at].astype(np.float64)[:, None], rot, interleaved)
        u = 2.0 ** -11 if act == torch.float16 else 2.0 ** -8
        size = np.abs(f[:, :hq]).max(-1, keepdims=True)
        got, held = q_out.double().cpu().numpy(), np.abs(exact) < torch.finfo(act).max     # past it: infinity, or the largest
        assert np.all(np.abs(got - exact)[held] <= (u * np.abs(exact) + 2.0 ** -22 * size + 2.0 ** -25)[held])
        assert np.all(np.abs(got)[~held] >= torch.finfo(act).max)
    return cache, gpu


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_ragged_batches(code, act, interleaved):
    """Sequences with no new token, one, a page, a page and a bit, and starts inside a page."""
    ctx = [0, 1, 16, 17, 33, 40, 100, 64, 15, 31]
    new = [0, 1, 16, 1, 33, 7, 70, 0, 3, 16]
    run(1, code, act, ctx, new, interleaved=interleaved)


@pytest.mark.parametrize("rot", [0, 16, 64, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_dims(rot, interleaved):
    run(2, R.INT8, torch.float16, [50, 9], [20, 9], rot=rot, interleaved=interleaved)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (28, 4), (40, 8), (13, 13), (71, 1)])
def test_one_token_each(code, hq, hkv):
    ctx = [1, 2, 16, 17, 18, 32, 33, 48, 4000, 100, 31, 30] * 3
    run(3, code, torch.bfloat16, ctx, [1] * len(ctx), hkv=hkv, hq=hq, decode_form=True, packed=True)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_positions_and_packed_rows(code):
    run(4, code, torch.float16, [20, 40], [5, 20], positions=[3, 0, 63, 7, 7] + list(range(20)), packed=True)


def test_many_sequences():
    """More sequences than one search step of a warp sees, most of them empty."""
    rng = np.random.default_rng(5)
    new = [int(n) for n in rng.integers(0, 3, 1500) * (rng.random(1500) < 0.3)]
    ctx = [n + int(c) for n, c in zip(new, rng.integers(0, 20, 1500))]
    run(5, R.INT8, torch.float16, ctx, new, hkv=1, hq=1)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_extremes(code):
    """Rows of zeros, the largest and the least values, and rows with infinities or NaN."""
    def edit(x, hq, hkv):
        x[0] = 0
        x[1] = 65504.0
        x[2] = 2.0 ** -24
        x[20, hq] = float("inf")
        x[40, hq + hkv] = float("nan")
    run(6, code, torch.float16, [60], [60], edit=edit)
    run(6, code, torch.float16, [63], [60], edit=edit, batches=2)
    run(7, code, torch.float16, [19, 4], [1, 4], edit=lambda x, hq, hkv: x.zero_())

    def tiny(x, hq, hkv):
        x *= 2.0 ** -120
        x[3:] *= 2.0 ** -10
    run(8, code, torch.bfloat16, [30], [30], edit=tiny)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_growing_page(code):
    """Token by token, each larger than all before: the page's scale grows with every call."""
    import paper_2607_28699_gb300 as wc
    rng = np.random.default_rng(9)
    cos, sin = R.tables(n=64)
    bt = np.array([[2, 0]], np.int32)
    cache = R.random_cache(rng, 3, 1, code)
    gpu = R.to_gpu(cache, code)
    desc = wc.BlockDesc(num_q_heads=1, num_kv_heads=1, num_pages=3, code=code)
    rows = torch.from_numpy(rng.standard_normal((20, 2, 128)).astype(np.float32) * 1.3 ** np.arange(20)[:, None, None].astype(np.float32)).half()
    for t in range(20):
        k, v = rows[t:t + 1, :1].contiguous(), rows[t:t + 1, 1:].contiguous()
        wc.block_append(desc, k.cuda(), v.cuda(), torch.tensor([t + 1], dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(), gpu,
                        cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda())
        R.append(cache, code, k.float().numpy(), v.float().numpy(), [t + 1], [1], bt, cos, sin, 128, False)
        for name in ("k", "v"):
            assert np.array_equal(getattr(gpu, name + "_scale").cpu().numpy(), cache[name + "_scale"])
            assert np.array_equal(R.decode(getattr(gpu, name + "_codes"), code), R.decode(cache[name + "_codes"], code))
    # what was stored: 15 roundings of half a step each at most, steps growing
    x = rows[:16, 1].double().numpy()
    got = R.decode(cache["v_codes"], code)[2, 0] * float(cache["v_scale"][2, 0])
    step = float(cache["v_scale"][2, 0])
    assert np.all(np.abs(got - x) <= (8 * step if code == R.INT8 else 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * step))


def test_rejected_drafts_are_replaced():
    """A token appended again at an earlier position: the ones after it are gone."""
    run(10, R.INT8, torch.float16, [21], [2], batches=3)


def test_status_reports():
    import paper_2607_28699_gb300 as wc
    desc = wc.BlockDesc(num_q_heads=2, num_kv_heads=1, num_pages=4)
    cache = wc.BlockCache.empty(desc)
    before = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
    cos, sin = (torch.from_numpy(x).cuda() for x in R.tables(n=40))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    rows = torch.randn(4, 1, 128, device="cuda").half()
    q = torch.randn(4, 2, 128, device="cuda").half()
    word = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(ctx, cu, table, positions=None):
        out = torch.full_like(q, 7.0)
        wc.block_append(desc, rows, rows, i32(*ctx), torch.tensor(table, dtype=torch.int32).cuda(), cache, cu_new=i32(*cu),
                        cos=cos, sin=sin, positions=positions, q=q, q_out=out, dev_status=word)
        return wc.read_status(word), out

    def untouched():
        return all(torch.equal(a, b) for a, b in zip(before, (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)))

    assert call([4], [0, 4], [[4, 0]])[0] == wc.DEV_BAD_PAGE and untouched()
    assert call([4], [0, 4], [[-1, 0]])[0] == wc.DEV_BAD_PAGE and untouched()
    assert call([33], [0, 4], [[0, 1]])[0] == wc.DEV_BAD_CTX and untouched()
    assert call([3], [0, 4], [[0, 1]])[0] == wc.DEV_BAD_CTX and untouched()
    assert call([4, 4], [0, 5, 4], [[0, 1], [2, 3]])[0] == wc.DEV_BAD_ROWS and untouched()
    assert call([4, 4], [-1, 0, 0], [[0, 1], [2, 3]])[0] == wc.DEV_BAD_ROWS and untouched()
    st, out = call([4], [0, 4], [[0, 1]], i32(0, 40, 1, -1))
    assert st == wc.DEV_BAD_POSITION
    assert out[1].abs().max() == 0 and out[3].abs().max() == 0 and out[0].abs().max() > 0
    assert cache.k_codes[0, 0, 1].abs().max() == 0 and cache.k_codes[0, 0, 2].abs().max() > 0


def test_other_stream_and_graph():
    import paper_2607_28699_gb300 as wc
    desc = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=8)
    cos, sin = (torch.from_numpy(x).cuda() for x in R.tables(n=64))
    k, v = (torch.randn(3, 2, 128, device="cuda").half() for _ in range(2))
    q = torch.randn(3, 4, 128, device="cuda").half()
    ctx = torch.tensor([5, 17, 33], dtype=torch.int32).cuda()
    bt = torch.tensor([[0, -1, -1], [1, 2, -1], [3, 4, 5]], dtype=torch.int32).cuda()
    results = []
    for how in ("plain", "stream", "graph"):
        cache = wc.BlockCache.empty(desc)
        out = torch.empty_like(q)
        go = lambda: wc.block_append(desc, k, v, ctx, bt, cache, cos=cos, sin=sin, q=q, q_out=out)  # noqa: E731
        if how == "plain":
            go()
        else:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            if how == "stream":
                wc.block_append(desc, k, v, ctx, bt, cache, cos=cos, sin=sin, q=q, q_out=out, stream=side)
            else:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    go()
                graph.replay()
            torch.cuda.synchronize()
        results.append((out, cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale))
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))
