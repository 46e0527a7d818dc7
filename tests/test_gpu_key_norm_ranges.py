"""The append's norm of keys at the ends of fp32: rows whose squares or whose norm_eps are near the largest and the least that fp32
holds have the factor, and so the scales and codes, of the definition; only rows whose sum of squares passes fp32's range are lost."""

import numpy as np
import pytest
import torch

import _block_ref as R
import _norm_ref as N
from test_gpu_qk_norm import append_case

pytestmark = pytest.mark.gpu


def append(x, weight, eps, code):
    """Keys x [n, 2, 128] (a page a token: nothing shares a scale) appended with their norm: cache, and what it should hold."""
    import paper_2607_28699_gb300 as wc
    n = x.shape[0]
    desc = wc.BlockDesc(num_q_heads=2, num_kv_heads=2, num_pages=n, code=code, rotary_dim=0)
    cache = wc.BlockCache.empty(desc)
    table = torch.randperm(n, generator=torch.Generator().manual_seed(n)).int()[:, None]
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = x.cuda()
    wc.block_append(desc, g, g, torch.ones(n, dtype=torch.int32, device="cuda"), table.cuda(), cache, dev_status=word,
                    k_norm=torch.from_numpy(weight).cuda(), norm_eps=eps)
    assert wc.read_status(word) == 0
    at = table[:, 0].long()
    codes, scale = cache.k_codes.cpu().view(torch.uint8).view(n, 2, 16, 128)[at, :, 0].numpy(), cache.k_scale.cpu().view(n, 2)[at].numpy()
    y = N.norm(x.float().numpy(), weight, eps)
    return codes, scale, y


def check(codes, scale, y, code):
    want = np.array([[R.scale_for(np.nan if np.isnan(r).any() else np.abs(r).max(), code) for r in rows] for rows in y], np.float32)
    assert np.array_equal(scale, want, equal_nan=True)
    good = np.isfinite(want) & (want > 0)
    with np.errstate(all="ignore"):
        z = y * (np.float32(1) / want)[..., None]
    assert np.array_equal(R.decode(codes, code)[good], R.decode(R.encode(z, code), code)[good])


def rows(seed, n, act, size):
    x = np.random.default_rng(seed).standard_normal((n, 2, 128)) * size
    return torch.from_numpy(x.astype(np.float32)).to(act)


WEIGHT = (1 + 0.5 * np.random.default_rng(1).standard_normal(128)).astype(np.float32)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
def test_large_rows(code):
    """bf16 rows whose largest squares reach 2^127 and past it, their sums of squares below 2^128."""
    x = rows(2, 40, torch.bfloat16, 1.0)
    x[:8] *= 2.0 ** 56
    x[8:16] *= 2.0 ** 58
    x[16:24] *= 2.0 ** 59
    x[24:] *= 2.0 ** 30
    x[0], x[1] = 0, 0
    x[0, :, 5] = 1.203125 * 2.0 ** 63        # a square of 0.36 x 2^128
    x[1, :, 77] = -1.40625 * 2.0 ** 63       # 0.494 x 2^128, and half as much
    x[1, 0, 78] = 2.0 ** 63
    x[2, 1] = 0
    x[2, 1, ::2] = 2.0 ** 60                 # 64 squares in a few lanes: 2^126
    x[24, :, 3] = 1.375 * 2.0 ** 63
    sums = (x.double() ** 2).sum(-1)
    assert float(sums.max()) < 2.0 ** 128 * (1 - 2.0 ** -20)
    codes, scale, y = append(x, WEIGHT, 1e-6, code)
    assert np.isfinite(scale).all()
    check(codes, scale, y, code)


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("act,size", [(torch.bfloat16, 2.0 ** -70), (torch.bfloat16, 2.0 ** -64), (torch.bfloat16, 2.0 ** -62),
                                      (torch.bfloat16, 1.0), (torch.bfloat16, 2.0 ** 50), (torch.float16, 2.0 ** -22), (torch.float16, 1.0),
                                      (torch.float16, 2.0 ** 13)])
@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** -122, 2.0 ** -61, 2.0 ** 60, 1e25, 3e38])
def test_eps(code, act, size, eps):
    x = rows(3, 200, act, size)
    x[0] = 0
    x[1, :, 1:] = 0
    codes, scale, y = append(x, WEIGHT, eps, code)
    check(codes, scale, y, code)


def test_rows_past_the_range_are_lost_alone():
    """In one warp with usual rows (four rows of a page): a sum of squares of 2^128, infinities, NaN; and the page of each of them only."""
    x = rows(4, 12, torch.bfloat16, 1.0)
    x[3, 0, :] = 2.0 ** 61            # 128 x 2^122
    x[4, 1, 9] = 2.0 ** 64
    x[5, 0, 0] = float("inf")
    x[6, 1, 127] = float("nan")
    x[7, :, ::3] = torch.finfo(torch.bfloat16).max
    lost = np.zeros((12, 2), bool)
    lost[3, 0] = lost[4, 1] = lost[5, 0] = lost[6, 1] = lost[7] = True
    codes, scale, y = append(x, WEIGHT, 1e-6, R.INT8)
    assert np.isnan(scale[lost]).all() and np.isfinite(scale[~lost]).all()
    y[lost] = np.nan
    check(codes, scale, y, R.INT8)
    # the same rows on one page: the others' norms do not change, the page is lost by the definition
    import paper_2607_28699_gb300 as wc
    desc = wc.BlockDesc(num_q_heads=2, num_kv_heads=2, num_pages=2, code=R.INT8, rotary_dim=0)
    cache = wc.BlockCache.empty(desc)
    g = x.cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    wc.block_append(desc, g, g, i32(12), i32(1)[None], cache, cu_new=i32(0, 12), k_norm=torch.from_numpy(WEIGHT).cuda())
    assert torch.isnan(cache.k_scale.view(2, 2)[1]).all()


@pytest.mark.parametrize("code", [R.INT8, R.E4M3])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("decode_form", [False, True])
def test_among_usual_rows(code, interleaved, decode_form, monkeypatch):
    """Such rows on pages with usual and older ones, rotated, packed; appended twice.  Rows whose sum of squares passes fp32's range are
    NaN by definition, which the plain form in float64 does not have of itself."""
    plain = N.norm
    monkeypatch.setattr(N, "norm", lambda x, w, eps: np.where((x.astype(np.float64) ** 2).sum(-1, keepdims=True) < 2.0 ** 128, plain(x, w, eps), np.float32(np.nan)))

    def edit(x, hq, hkv):
        keys = x[:, hq:hq + hkv]
        keys[::5] *= 2.0 ** 57
        keys[3::7, 0] = 0
        keys[3::7, 0, 9] = 1.3125 * 2.0 ** 63
        keys[4::9, 1] *= 2.0 ** -66
    ctx, new = ([60, 35, 17, 1, 16], [57, 20, 1, 1, 0]) if not decode_form else ([60, 35, 17, 1, 16, 33, 64] * 2, [1] * 14)
    append_case(5, code, torch.bfloat16, ctx, new, hkv=3, hq=6, interleaved=interleaved, edit=edit, packed=True, decode_form=decode_form, batches=2)
