"""Attention over the block-scaled cache, decode and extend, against the definition in float64."""

import math

import numpy as np
import pytest
import torch

import _block_ref as R

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def setup(seed, code, act, ctx, hq, hkv, new=None, scaled=True, extra=0, max_pages=None, q_size=1.0, stale=True):
    import paper_2607_28699_gb300 as wc
    rng = np.random.default_rng(seed)
    bt, pages = R.page_tables(rng, ctx, extra, max_pages)
    cache = R.random_cache(rng, pages, hkv, code, scaled)
    if stale:   # whatever was in memory past the context: any byte, NaN codes among them
        for b, c in enumerate(ctx):
            if c % 16:
                for n in ("k_codes", "v_codes"):
                    tail = cache[n][bt[b, c // 16], :, c % 16:]
                    tail[...] = rng.integers(0, 256, tail.shape, dtype=np.uint8)
                    tail[..., 0] = 0x7F
    n = sum(new) if new is not None else len(ctx)
    q = (torch.from_numpy(rng.standard_normal((n, hq, 128)).astype(np.float32)) * q_size).to(act)
    desc = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=pages, code=code)
    return wc, desc, bt, cache, q


def run(seed, code, act, ctx, hq, hkv, new=None, causal=True, scale=SCALE, edit=None, packed=False, **kw):
    """new None: the decode call."""
    wc, desc, bt, cache, q = setup(seed, code, act, ctx, hq, hkv, new, **kw)
    if edit is not None:
        edit(cache, bt, q)
    gpu = R.to_gpu(cache, code)
    ws = wc.BlockWorkspace(desc, len(ctx), q.shape[0], bt.shape[1])
    ctx_g, bt_g = torch.tensor(ctx, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda()
    qg = q.cuda()
    if packed:
        wide = torch.full((q.shape[0], hq + 3, 128), float("nan"), dtype=act, device="cuda")
        wide[:, 1:hq + 1] = qg
        qg = wide[:, 1:hq + 1]
    if new is None:
        cu = list(range(len(ctx) + 1))
        call = lambda: wc.block_decode_attention(desc, qg, bt_g, ctx_g, gpu, ws, softmax_scale=scale, return_lse=True)  # noqa: E731
        causal = False
    else:
        cu = [0] + np.cumsum(new).tolist()
        cu_g = torch.tensor(cu, dtype=torch.int32).cuda()
        call = lambda: wc.block_extend_attention(desc, qg, cu_g, bt_g, ctx_g, gpu, ws, softmax_scale=scale, causal=causal, return_lse=True)  # noqa: E731
    out, lse = call()
    again = call()
    status = wc.read_status(ws)
    ref = R.attention(q.double().numpy(), cu, bt, ctx, cache["k_codes"], cache["v_codes"], cache["k_scale"], cache["v_scale"], code, scale, causal)
    R.check_attention(out, lse, ref, act)
    bits = lambda t: t.view(torch.int16 if t.element_size() == 2 else torch.int32)  # noqa: E731
    assert torch.equal(bits(out), bits(again[0])) and torch.equal(bits(lse), bits(again[1]))     # the same bits each time
    assert out.dtype == act
    return out, lse, status


EDGES = [0, 1, 15, 16, 17, 31, 33, 128, 129, 255, 257]


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (28, 4), (8, 1), (3, 3), (16, 1)])
def test_decode_heads(code, act, hq, hkv):
    assert run(1, code, act, EDGES, hq, hkv)[2] == 0


@pytest.mark.parametrize("group", [2, 5, 6, 9, 17, 64, 71, 128])
def test_decode_groups(group):
    run(2, R.E4M3, torch.float16, [5, 300, 77], group, 1)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("ctx", [[1], [16], [1000], [4099], [700, 3, 5000, 1, 0, 64], [0], [0, 0]])
def test_decode_lengths(code, ctx):
    run(3, code, torch.float16, ctx, 7, 1)


def test_decode_wide_tables():
    """Tables much wider than any context, and many sequences."""
    run(4, R.INT8, torch.bfloat16, [40, 0, 7], 4, 2, max_pages=3000)
    rng = np.random.default_rng(4)
    run(5, R.INT8, torch.float16, [int(c) for c in rng.integers(0, 60, 700)], 4, 1)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("act", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (14, 2), (8, 1), (16, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_extend_heads(code, act, hq, hkv, causal):
    ctx = [0, 1, 16, 17, 40, 130, 257, 64]
    new = [0, 1, 16, 3, 40, 2, 130, 0]
    assert run(6, code, act, ctx, hq, hkv, new=new, causal=causal)[2] == 0


@pytest.mark.parametrize("group", [1, 3, 7, 12, 33, 71, 128])
def test_extend_groups(group):
    run(7, R.INT8, torch.float16, [150, 40], group, 1, new=[20, 6])


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("ctx,new", [([1], [1]), ([300], [300]), ([1030], [2]), ([2000], [129]), ([700, 90], [257, 90])])
def test_extend_lengths(code, ctx, new):
    run(8, code, torch.bfloat16, ctx, 4, 2, new=new)


@pytest.mark.parametrize("causal", [True, False])
def test_rows_before_the_start(causal):
    """More query rows than context: causal rows before position 0 attend to nothing."""
    out, lse, _ = run(9, R.INT8, torch.float16, [5, 0, 20], 4, 2, new=[9, 3, 4], causal=causal)
    if causal:
        assert torch.isneginf(lse[:4]).all() and out[:4].abs().max() == 0
    assert torch.isneginf(lse[9:12]).all() and out[9:12].abs().max() == 0


def test_extend_many_sequences():
    rng = np.random.default_rng(10)
    new = [int(n) for n in rng.integers(0, 5, 300)]
    run(10, R.E4M3, torch.float16, [n + int(c) for n, c in zip(new, rng.integers(0, 40, 300))], 4, 2, new=new)


@pytest.mark.parametrize("new", [None, [1, 30]])
def test_without_scales(new):
    """The raw-cast fp8 layout: scale 1."""
    run(11, R.E4M3, torch.float16, [77, 300], 4, 2, new=new, scaled=False)


@pytest.mark.parametrize("new", [None, [30, 60, 9]])
def test_page_scales_far_apart(new):
    """Scales of 2^-40 to 2^10 in one context, and pages of zeros with scale 0."""
    def edit(cache, bt, q):
        rng = np.random.default_rng(1)
        for n in ("k_scale", "v_scale"):
            cache[n] *= np.exp2(rng.integers(-40, 3 if n[0] == "k" else 11, cache[n].shape)).astype(np.float32)
        zero = bt[0, 1]
        for n in "kv":
            cache[n + "_scale"][zero] = 0
            cache[n + "_codes"][zero] = 0
        cache["v_scale"][bt[1, 0]] = 0     # codes that a scale of 0 silences
    run(12, R.INT8, torch.bfloat16, [130, 260, 40], 6, 2, new=new, edit=edit)


@pytest.mark.parametrize("new", [None, [40]])
def test_all_values_zero(new):
    def edit(cache, bt, q):
        cache["v_scale"][:] = 0
    out, _, _ = run(13, R.E4M3, torch.float16, [100], 4, 2, new=new, edit=edit)
    assert out.abs().max() == 0


@pytest.mark.parametrize("act,size", [(torch.bfloat16, 2.0 ** 60), (torch.bfloat16, 2.0 ** -60), (torch.float16, 2.0 ** 9), (torch.float16, 2.0 ** -14)])
@pytest.mark.parametrize("new", [None, [21]])
def test_query_sizes(act, size, new):
    """Queries far from 1 with a softmax scale to match: logits of the usual size."""
    run(14, R.INT8, act, [150], 8, 1, new=new, q_size=size, scale=SCALE / size)


@pytest.mark.parametrize("new", [None, [21]])
def test_sharp_softmax(new):
    """Logits of hundreds: one key takes all; running maxima that jump."""
    run(15, R.INT8, torch.float16, [900], 4, 1, new=new, scale=SCALE * 40)


@pytest.mark.parametrize("new", [None, [50, 20]])
def test_rising_logits(new):
    """Each page's keys larger than the last's: the running maximum moves in every tile."""
    def edit(cache, bt, q):
        q[...] = q.abs()
        for b in range(2):
            for j, p in enumerate(bt[b]):
                if p >= 0:
                    cache["k_codes"][p] = 100
                    cache["k_scale"][p] = 0.01 * (j + 1)
    run(16, R.INT8, torch.float16, [700, 330], 7, 1, new=new, edit=edit, stale=False)


@pytest.mark.parametrize("new", [None, [40, 30]])
def test_nan_spreads_only_to_its_sequence(new):
    def edit(cache, bt, q):
        cache["k_scale"][bt[0, 1]] = np.nan
    out, lse, _ = run(17, R.INT8, torch.float16, [200, 90], 4, 2, new=new, edit=edit)
    n = 1 if new is None else new[0]
    assert torch.isnan(out[:n]).all() and torch.isfinite(out[n:]).all()


@pytest.mark.parametrize("new", [None, [5, 6, 7]])
def test_bad_pages_and_lengths(new):
    """A page outside the pool is left out, a context past the table is taken as none; both are reported."""
    import paper_2607_28699_gb300 as wc

    def edit(cache, bt, q):
        bt[0, 1], bt[1, 0] = 10 ** 6, -3
    out, _, status = run(18, R.INT8, torch.float16, [90, 16, 300], 4, 2, new=new, edit=edit)
    assert status == wc.DEV_BAD_PAGE
    wc_, desc, bt, cache, q = setup(19, R.INT8, torch.float16, [64, 64, 64], 4, 2, new)
    gpu = R.to_gpu(cache, R.INT8)
    ws = wc.BlockWorkspace(desc, 3, q.shape[0], 4)
    for bad in (65, -1):
        ctx = torch.tensor([64, bad, 64], dtype=torch.int32).cuda()
        btg = torch.from_numpy(bt).cuda()
        if new is None:
            out, lse = wc.block_decode_attention(desc, q.cuda(), btg, ctx, gpu, ws, return_lse=True)
            rows = slice(1, 2)
        else:
            cu = torch.tensor([0, 5, 11, 18], dtype=torch.int32).cuda()
            out, lse = wc.block_extend_attention(desc, q.cuda(), cu, btg, ctx, gpu, ws, return_lse=True)
            rows = slice(5, 11)
        assert wc.read_status(ws) == wc.DEV_BAD_CTX
        assert out[rows].abs().max() == 0 and torch.isneginf(lse[rows]).all()
        assert torch.isfinite(lse[:rows.start]).all() and torch.isfinite(lse[rows.stop:]).all()


def test_bad_row_ranges():
    import paper_2607_28699_gb300 as wc
    _, desc, bt, cache, q = setup(20, R.INT8, torch.float16, [64, 64], 4, 2, [8, 8])
    gpu = R.to_gpu(cache, R.INT8)
    ws = wc.BlockWorkspace(desc, 2, 16, 4)
    for cu in ([0, 17, 16], [0, 8, 17], [0, 8, 4], [-1, 8, 16]):
        out = torch.full((16, 4, 128), 3.0, device="cuda").half()
        wc.block_extend_attention(desc, q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(),
                                  torch.tensor([64, 64], dtype=torch.int32).cuda(), gpu, ws, out=out)
        assert wc.read_status(ws) == wc.DEV_BAD_ROWS


@pytest.mark.parametrize("new", [None, [9, 20]])
def test_strided_queries(new):
    run(21, R.E4M3, torch.bfloat16, [100, 60], 6, 2, new=new, packed=True)


def test_pool_past_32_bits():
    """A pool of more than 4 GiB of codes whose last pages are the ones in use."""
    import paper_2607_28699_gb300 as wc
    hkv, pages = 4, 2 ** 19 + 2 ** 14
    rng = np.random.default_rng(22)
    small = R.random_cache(rng, 20, hkv, R.INT8)
    desc = wc.BlockDesc(num_q_heads=8, num_kv_heads=hkv, num_pages=pages)
    cache = wc.BlockCache(*(torch.empty(pages, hkv, 16, 128, dtype=torch.int8, device="cuda") for _ in range(2)),
                          *(torch.empty(pages, hkv, device="cuda") for _ in range(2)))
    at = pages - 20
    for n in ("k_codes", "v_codes", "k_scale", "v_scale"):
        t = torch.from_numpy(small[n].view(np.int8) if n.endswith("codes") else small[n])
        getattr(cache, n)[at:] = t.cuda()
    bt = rng.permutation(20).astype(np.int32)[None]
    q = torch.from_numpy(rng.standard_normal((6, 8, 128)).astype(np.float32)).half()
    ctx = torch.tensor([310], dtype=torch.int32).cuda()
    table = torch.from_numpy(bt + at).cuda()
    ws = wc.BlockWorkspace(desc, 1, 6, 20)
    args = (small["k_codes"], small["v_codes"], small["k_scale"], small["v_scale"], R.INT8, SCALE)
    out, lse = wc.block_decode_attention(desc, q[:1].cuda(), table, ctx, cache, ws, return_lse=True)
    R.check_attention(out, lse, R.attention(q[:1].double().numpy(), [0, 1], bt, [310], *args, False), torch.float16)
    cu = torch.tensor([0, 6], dtype=torch.int32).cuda()
    out, lse = wc.block_extend_attention(desc, q.cuda(), cu, table, ctx, cache, ws, return_lse=True)
    R.check_attention(out, lse, R.attention(q.double().numpy(), [0, 6], bt, [310], *args, True), torch.float16)
    cos, sin = (torch.from_numpy(x).cuda() for x in R.tables(n=400))
    k = torch.from_numpy(rng.standard_normal((2, hkv, 128)).astype(np.float32)).half()
    wc.block_append(desc, k.cuda(), k.cuda(), ctx, table, cache, cu_new=torch.tensor([0, 2], dtype=torch.int32).cuda(), cos=cos, sin=sin)
    R.append(small, R.INT8, k.float().numpy(), k.float().numpy(), [310], [2], bt, cos.cpu().numpy(), sin.cpu().numpy(), 128, False)
    assert np.array_equal(cache.k_codes[at:].cpu().numpy().view(np.uint8), small["k_codes"])
    assert np.array_equal(cache.v_scale[at:].cpu().numpy(), small["v_scale"])


def test_other_stream_and_graph():
    wc, desc, bt, cache, q = setup(23, R.INT8, torch.float16, [200, 31], 8, 2, [30, 12])
    gpu = R.to_gpu(cache, R.INT8)
    ws = wc.BlockWorkspace(desc, 2, 42, bt.shape[1])
    ctx, btg, cu = torch.tensor([200, 31], dtype=torch.int32).cuda(), torch.from_numpy(bt).cuda(), torch.tensor([0, 30, 42], dtype=torch.int32).cuda()
    qg, q1 = q.cuda(), q[:2].cuda()
    both = lambda **kw: (wc.block_extend_attention(desc, qg, cu, btg, ctx, gpu, ws, **kw),  # noqa: E731
                         wc.block_decode_attention(desc, q1, btg, ctx, gpu, ws, **kw))
    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = both(stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = both()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_reads_the_fp8_layer_cache():
    """Extend attention over a cache that the framework's fp8 write filled: the metered decode of the last token agrees."""
    import paper_2607_28699_gb300 as wc
    pages, ctx = 20, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(ctx, 2, 128, generator=g, device="cuda").half() for _ in range(2))
    q = torch.randn(8, 4, 128, generator=g, device="cuda").half()
    d = wc.CacheDesc(num_q_heads=4, num_kv_heads=2, num_pages=pages, scheme=wc.SCHEME_FP8_E4M3)
    layer = wc.LayerCache.empty(d)
    wc.kv_quantize_witness(d, 0, k, v, torch.arange(ctx, dtype=torch.int32, device="cuda"), layer)
    bt = torch.arange(19, dtype=torch.int32, device="cuda")[None].contiguous()
    lens = torch.tensor([ctx], dtype=torch.int32, device="cuda")
    want = wc.metered_decode_attention(d, 0, q[-1:].contiguous(), bt, lens, layer, wc.Workspace(d, 1, 19))[0]
    bd = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=pages, code=wc.CODE_E4M3)
    bc = wc.BlockCache(layer.k_codes, layer.v_codes, None, None)
    ws = wc.BlockWorkspace(bd, 1, 8, 19)
    got = wc.block_extend_attention(bd, q, torch.tensor([0, 8], dtype=torch.int32, device="cuda"), bt, lens, bc, ws)
    # both are within 2^-11 of the output and of sum p |v| (<= max |v|) of the definition
    assert (got[-1].float() - want[0]).abs().max() <= 2.0 ** -9 * float(v.abs().max())
    got = wc.block_decode_attention(bd, q[-1:], bt, lens, bc, ws)
    assert (got[0].float() - want[0]).abs().max() <= 2.0 ** -9 * float(v.abs().max())


@pytest.mark.parametrize("hkv", [5, 160])
def test_decode_heads_and_shares(hkv):
    """Head counts that do not divide the SMs, or exceed them, with one sequence and with several."""
    run(24, R.INT8, torch.float16, [260], hkv, hkv)
    run(25, R.E4M3, torch.bfloat16, [100, 0, 37, 300], hkv, hkv)


def test_decode_thousands_of_sequences():
    """More sequences than one launch holds."""
    rng = np.random.default_rng(26)
    run(26, R.INT8, torch.float16, [int(c) for c in rng.integers(0, 40, 2600)], 2, 1)


@pytest.mark.parametrize("hq,hkv", [(7, 1), (16, 1)])
def test_extend_splits(hq, hkv):
    """Few rows over a long context: the context is split over many CTAs, at lengths that do not divide evenly."""
    run(27, R.E4M3, torch.float16, [9001], hq, hkv, new=[3])
    run(28, R.INT8, torch.bfloat16, [4100, 130, 2000], hq, hkv, new=[2, 1, 5], causal=False)


def test_one_workspace_for_all_calls():
    """A workspace of the largest call serves smaller ones of other shapes, in any order."""
    wc, desc, bt, cache, q = setup(29, R.INT8, torch.float16, [700, 900, 40, 333], 8, 2, [60, 20, 40, 3])
    gpu = R.to_gpu(cache, R.INT8)
    ws = wc.BlockWorkspace(desc, 4, q.shape[0], bt.shape[1])
    args = (cache["k_codes"], cache["v_codes"], cache["k_scale"], cache["v_scale"], R.INT8, SCALE)
    ctx = [700, 900, 40, 333]

    def decode(pick):
        qd, btd, cd = q[:len(pick)].clone(), bt[pick], [ctx[b] for b in pick]
        out, lse = wc.block_decode_attention(desc, qd.cuda(), torch.from_numpy(btd).cuda(), torch.tensor(cd, dtype=torch.int32).cuda(), gpu, ws, return_lse=True)
        R.check_attention(out, lse, R.attention(qd.double().numpy(), list(range(len(pick) + 1)), btd, cd, *args, False), torch.float16)

    def extend(pick, new):
        n = sum(new)
        cu = [0] + np.cumsum(new).tolist()
        qd, btd, cd = q[:n].clone(), bt[pick], [ctx[b] for b in pick]
        out, lse = wc.block_extend_attention(desc, qd.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.from_numpy(btd).cuda(),
                                             torch.tensor(cd, dtype=torch.int32).cuda(), gpu, ws, return_lse=True)
        R.check_attention(out, lse, R.attention(qd.double().numpy(), cu, btd, cd, *args, True), torch.float16)

    decode([0, 1, 2, 3])
    extend([1], [3])
    decode([1])
    extend([0, 1, 2, 3], [60, 20, 40, 3])
    decode([3, 0])
    extend([1, 0], [20, 1])
    decode([1, 2, 3])
    assert wc.read_status(ws) == 0


@pytest.mark.parametrize("group", [1, 7])
def test_extend_mostly_empty_batches(group):
    """Far fewer query tokens than sequences, the ones with tokens among the last."""
    ctx = [20] * 300
    new = [0] * 300
    ctx[150], new[150], ctx[298], new[298], ctx[299], new[299] = 400, 2, 33, 1, 700, 30
    run(30, R.INT8, torch.float16, ctx, group, 1, new=new)


@pytest.mark.parametrize("new", [None, [33]])
def test_subnormal_value_scales(new):
    """Value scales below the least normal number: the page's values count as 0 (they are, next to the others), its keys do not."""
    def edit(cache, bt, q):
        cache["v_scale"][bt[0, ::2]] = 1e-40
    run(31, R.INT8, torch.float16, [300], 4, 1, new=new, edit=edit)
