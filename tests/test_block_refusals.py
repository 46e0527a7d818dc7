"""Calls of the block-scaled cache that are refused before any launch (no GPU needed)."""

import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def wc():
    import paper_2607_28699_gb300 as w
    return w


P = ctypes.c_void_p(256)


def desc(wc, **kw):
    d = wc.BlockDesc(num_q_heads=8, num_kv_heads=2, num_pages=4).c()
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def append(wc, d=None, **kw):
    a = dict(act=0, k=P, ks=256, v=P, vs=256, q=None, qs=0, qo=None, n=3, cu=P, bt=P, mp=4, ctx=P, batch=2, pos=None, cos=P, sin=P,
             npos=64, kc=P, vc=P, ksc=P, vsc=P, word=None)
    assert set(kw) <= set(a)
    a.update(kw)
    d = desc(wc) if d is None else d
    return wc.lib.wc_block_append(ctypes.byref(d), a["act"], a["k"], a["ks"], a["v"], a["vs"], a["q"], a["qs"], a["qo"], a["n"], a["cu"], a["bt"],
                                  a["mp"], a["ctx"], a["batch"], a["pos"], a["cos"], a["sin"], a["npos"], a["kc"], a["vc"], a["ksc"],
                                  a["vsc"], a["word"], None), wc.lib.wc_last_error()


def attend(wc, d=None, extend=False, **kw):
    a = dict(act=0, q=P, qs=1024, n=3, cu=P, bt=P, mp=4, ctx=P, batch=2, kc=P, vc=P, ks=P, vs=P, scale=0.1, causal=1, out=P, lse=None, ws=P,
             bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    d = desc(wc) if d is None else d
    f = ctypes.c_float(a["scale"])
    if extend:
        st = wc.lib.wc_block_extend_attention(ctypes.byref(d), a["act"], a["q"], a["qs"], a["n"], a["cu"], a["bt"], a["mp"], a["ctx"], a["batch"],
                                              a["kc"], a["vc"], a["ks"], a["vs"], f, a["causal"], a["out"], a["lse"], a["ws"], a["bytes"], None)
    else:
        st = wc.lib.wc_block_decode_attention(ctypes.byref(d), a["act"], a["q"], a["qs"], a["bt"], a["mp"], a["ctx"], a["batch"], a["kc"], a["vc"],
                                              a["ks"], a["vs"], f, a["out"], a["lse"], a["ws"], a["bytes"], None)
    return st, wc.lib.wc_last_error()


def test_descriptors(wc):
    for field, value, status in (("head_dim", 64, 2), ("page_size", 32, 2), ("num_kv_heads", 0, 1), ("num_q_heads", 7, 1),
                                 ("num_q_heads", 2 * 129, 2), ("num_pages", 0, 1), ("num_pages", 1 << 28, 2), ("code", 2, 2),
                                 ("rope_layout", 2, 2), ("rotary_dim", 24, 2), ("rotary_dim", 144, 2), ("rotary_dim", -16, 2)):
        d = desc(wc, **{field: value})
        for st, message in (append(wc, d), attend(wc, d), attend(wc, d, extend=True)):
            assert st == status and field.encode() in message, (field, value, st, message)
        assert wc.lib.wc_block_workspace_size(ctypes.byref(d), 1, 1, 1) == 0
    assert wc.lib.wc_block_workspace_size(None, 1, 1, 1) == 0


@pytest.mark.parametrize("call", [append, attend, lambda wc, **kw: attend(wc, extend=True, **kw)])
def test_sizes(wc, call):
    assert call(wc, act=2)[0] == 2
    assert call(wc, batch=-1)[0] == 1 and call(wc, batch=65536)[0] == 1
    assert call(wc, mp=0)[0] == 1 and call(wc, mp=1 << 27)[0] == 2
    assert call(wc, bt=None)[0] == 1 and call(wc, ctx=None)[0] == 1
    assert call(wc, kc=None)[0] == 1 and call(wc, vc=ctypes.c_void_p(8))[0] == 1


def test_append(wc):
    assert append(wc, n=-1)[0] == 1
    st, m = append(wc, cu=None)
    assert st == 1 and b"cu_new" in m
    for n in ("k", "v"):
        st, m = append(wc, **{n: None})
        assert st == 1 and m.startswith(n.encode())
        assert append(wc, **{n: ctypes.c_void_p(8)})[0] == 1
        for stride in (255, 252, -256, 260):
            st, m = append(wc, **{n + "s": stride})
            assert st == 1 and b"stride" in m
    assert append(wc, q=P, qs=1024)[0] == 1 and append(wc, qo=P)[0] == 1
    assert append(wc, q=P, qs=1016, qo=P)[0] == 1 and append(wc, q=P, qs=1024, qo=ctypes.c_void_p(8))[0] == 1
    assert append(wc, cos=None)[0] == 1 and append(wc, sin=None)[0] == 1 and append(wc, npos=0)[0] == 1
    assert append(wc, cos=ctypes.c_void_p(4))[0] == 1
    assert append(wc, ksc=None)[0] == 1 and append(wc, vsc=ctypes.c_void_p(2))[0] == 1
    assert append(wc, n=0)[0] == 0 and append(wc, n=0, batch=0, cu=None)[0] == 0      # nothing to do


@pytest.mark.parametrize("extend", [False, True])
def test_attention(wc, extend):
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        st, m = attend(wc, extend=extend, scale=bad)
        assert st == 1 and b"softmax_scale" in m
    assert attend(wc, extend=extend, q=None)[0] == 1 and attend(wc, extend=extend, q=ctypes.c_void_p(24))[0] == 1
    assert attend(wc, extend=extend, qs=1016)[0] == 1 and attend(wc, extend=extend, qs=1028)[0] == 1
    assert attend(wc, extend=extend, out=None)[0] == 1 and attend(wc, extend=extend, out=ctypes.c_void_p(2))[0] == 1
    assert attend(wc, extend=extend, ws=None)[0] == 1 and attend(wc, extend=extend, ws=ctypes.c_void_p(128))[0] == 1
    assert attend(wc, extend=extend, ks=None)[0] == 1 and attend(wc, extend=extend, vs=None)[0] == 1
    st, m = attend(wc, extend=extend, ks=None, vs=None)
    assert st == 1 and b"e4m3" in m
    assert attend(wc, extend=extend, ks=ctypes.c_void_p(6))[0] == 1
    assert attend(wc, extend=extend, batch=0)[0] == 0
    if extend:
        assert attend(wc, extend=True, cu=None)[0] == 1 and attend(wc, extend=True, n=-1)[0] == 1
        assert attend(wc, extend=True, n=0)[0] == 0


def test_binding_checks_tensors(wc):
    d = wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=3)
    c = wc.BlockCache.empty(d, device="cpu")
    k = torch.zeros(5, 2, 128, dtype=torch.float16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    ok = dict(ctx_lens=i32(3, 2), block_table=torch.zeros(2, 1, dtype=torch.int32), cache=c, cu_new=i32(0, 3, 5),
              cos=torch.zeros(8, 64), sin=torch.zeros(8, 64))
    for k2, v2, kw in ((k.float(), k, {}), (k, k.bfloat16(), {}), (k[:, :1], k, {}), (k, k[:4], {}), (k, k[..., ::2], {}),
                       (k, k, {"ctx_lens": torch.tensor([3, 2])}), (k, k, {"cu_new": i32(0, 5)}), (k, k, {"cos": torch.zeros(8, 32)}),
                       (k, k, {"sin": None}), (k, k, {"positions": i32(0)}), (k, k, {"q": torch.zeros(5, 2, 128, dtype=torch.float16)}),
                       (k, k, {"cache": wc.BlockCache.empty(wc.BlockDesc(num_q_heads=4, num_kv_heads=2, num_pages=2), device="cpu")})):
        with pytest.raises(ValueError):
            wc.block_append(d, k2, v2, **{**ok, **kw}, stream=torch.Stream("cpu"))
    for bad in ((c.k_codes[:2], c.v_codes, c.k_scale, c.v_scale), (c.k_codes, c.v_codes, c.k_scale.half(), c.v_scale),
                (c.k_codes.half(), c.v_codes, c.k_scale, c.v_scale), (c.k_codes, c.v_codes.transpose(2, 3), None, None)):
        with pytest.raises(ValueError):
            wc.BlockCache(*bad)
    q = torch.zeros(2, 4, 128, dtype=torch.float16)
    for q2, kw in ((q.float(), {}), (q[:1], {}), (q, {"out": q[:1]}), (q, {"lse": torch.zeros(3)}), (q[:, :2], {})):
        with pytest.raises(ValueError):
            wc.block_decode_attention(d, q2, ok["block_table"], ok["ctx_lens"], c, None, stream=torch.Stream("cpu"), **kw)
