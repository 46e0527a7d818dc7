"""Plain implementations of the block-scaled cache for its tests: attention in float64, the append
token by token in float32 with IEEE operations (numpy), where the definition is a sequence of them."""

import numpy as np
import torch

PAGE, DIM = 16, 128
INT8, E4M3 = 0, 1


def decode(codes, code):
    """Stored bytes as the numbers they stand for, float64."""
    t = torch.from_numpy(np.ascontiguousarray(codes)) if isinstance(codes, np.ndarray) else codes.cpu()
    return (t.view(torch.int8) if code == INT8 else t.view(torch.uint8).view(torch.float8_e4m3fn).float()).double().numpy()


def encode(y, code):
    """Codes (uint8 bytes) nearest to the float32 array y, ties to even."""
    y = np.asarray(y, np.float32)
    if code == INT8:
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    return torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def rotate(x, cos, sin, rot, interleaved):
    """One row [.., 128] float32 -> float32, each product rounded."""
    y = x.copy()
    if rot:
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def scale_for(amax, code):
    """The least scale a page of this largest magnitude may have (float32)."""
    amax = np.float32(amax)
    if amax == 0 or not np.isfinite(amax):
        return amax
    least = np.float32(2.0 ** -100)
    if code == INT8:
        return max(amax * np.float32(1 / 127), least)
    e = -100
    while float(amax) > 448.0 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def append(cache, code, k, v, ctx, new, bt, cos, sin, rot, interleaved, positions=None):
    """cache: dict of k_codes, v_codes (uint8 [pages, H, 16, 128]) and k_scale, v_scale (float32), updated in place.
    k, v float32 arrays [n, H, 128] of the new tokens."""
    row = 0
    with np.errstate(all="ignore"):
        for b, (c, n) in enumerate(zip(ctx, new)):
            first = c - n
            for page in range(first // PAGE, (c + PAGE - 1) // PAGE if n else 0):
                t0, t1 = max(first, page * PAGE), min(c, page * PAGE + PAGE)
                phys, keep = bt[b][page], t0 - page * PAGE
                rows = slice(row + t0 - first, row + t1 - first)
                at = np.arange(t0, t1) if positions is None else np.asarray(positions[rows])
                for h in range(k.shape[1]):
                    for name, x in (("k", k), ("v", v)):
                        y = x[rows, h]
                        if name == "k" and rot:
                            y = rotate(y, cos[at], sin[at], rot, interleaved)
                        a = np.abs(y)
                        amax = np.float32(np.nan) if np.isnan(a).any() else a.max()
                        old = cache[name + "_scale"][phys, h] if keep else np.float32(0)
                        s = scale_for(amax, code)
                        s = s if np.isnan(s) or s > old else old
                        grew = np.isnan(s) or s > old
                        codes = cache[name + "_codes"][phys, h]
                        if grew and keep and not np.isnan(old):
                            had = decode(codes[:keep], code).astype(np.float32)
                            codes[:keep] = encode(had * np.float32(old / s), code) if np.isfinite(s) else 0
                        inv = np.float32(1) / s if s > 0 and np.isfinite(s) else np.float32(0)
                        codes[t0 - page * PAGE:t1 - page * PAGE] = encode(y * inv, code) if np.isfinite(s) else 0
                        if not np.isnan(old):
                            cache[name + "_scale"][phys, h] = s
            row += n


def attention(q, cu, bt, ctx, k_codes, v_codes, k_scale, v_scale, code, scale, causal):
    """float64 out [n, Hq, 128], lse [n, Hq], and per cell sum_t p |v| and the largest sum |scale q k|: what the
    tolerances are made of.  q float64 [n, Hq, 128]."""
    n_tok, hq, _ = q.shape
    hkv = k_codes.shape[1]
    G = hq // hkv
    out, lse = np.zeros((n_tok, hq, DIM)), np.full((n_tok, hq), -np.inf)
    mass, big = np.zeros((n_tok, hq, DIM)), np.zeros((n_tok, hq))
    for b, c in enumerate(ctx):
        n = cu[b + 1] - cu[b]
        pages = [p for p in bt[b][:(c + PAGE - 1) // PAGE]]
        if not pages or not n:
            continue
        ok = np.repeat([0 <= p < k_codes.shape[0] for p in pages], PAGE)[:c]
        use = [p if 0 <= p < k_codes.shape[0] else 0 for p in pages]
        for h in range(hkv):
            k = (decode(k_codes[use, h], code) * (1.0 if k_scale is None else k_scale[use, h].astype(np.float64)[:, None, None])).reshape(-1, DIM)[:c]
            v = (decode(v_codes[use, h], code) * (1.0 if v_scale is None else v_scale[use, h].astype(np.float64)[:, None, None])).reshape(-1, DIM)[:c]
            k, v = np.where(ok[:, None], k, 0), np.where(ok[:, None], v, 0)
            for i in range(n):
                end = max(0, c - n + i + 1) if causal else c
                see = ok[:end]
                if not see.any():
                    continue
                r = cu[b] + i
                for g in range(h * G, (h + 1) * G):
                    with np.errstate(invalid="ignore"):
                        t = np.where(see, scale * (k[:end] @ q[r, g]), -np.inf)
                        m = t.max()
                        e = np.exp(t - m)
                        l = e.sum()
                        out[r, g] = (e / l) @ v[:end]
                        mass[r, g] = (e / l) @ np.abs(v[:end])
                        lse[r, g] = m + np.log(l)
                        big[r, g] = (np.abs(k[:end]) @ np.abs(q[r, g])).max() * scale
    return out, lse, mass, big


def check_attention(out, lse, ref, act, what=""):
    """Derived bounds: out is rounded once (2^-11 or 2^-8 of it); each weight may be rounded to fp16 (2^-11 of sum p |v|);
    a logit of 128 fp32 products carries 2^-17 of their absolute sum, which moves a weight and the sum of weights; 2^-18 for
    the exponentials and fp32 sums.  lse carries the logit's and the sum's."""
    want, want_lse, mass, big = ref
    u = 2.0 ** -11 if act == torch.float16 else 2.0 ** -8
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    d = big * 2.0 ** -17
    tol = u * np.abs(want) + (1 + u) * (2.0 ** -11 + 2.0 ** -18 + 2 * d)[..., None] * mass + 2.0 ** -24
    bad = ~(np.abs(got - want) <= tol)
    bad &= ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], tol[bad][:3])
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got_lse - want_lse) <= d + 2.0 ** -18 * (1 + np.abs(want_lse)))
    bad &= ~((got_lse == want_lse) | (np.isnan(got_lse) & np.isnan(want_lse)))
    assert not bad.any(), (what, "lse", int(bad.sum()), np.argwhere(bad)[:3].tolist(), got_lse[bad][:3], want_lse[bad][:3])


def tables(base=1e4, rot=128, n=4096):
    ang = np.arange(n)[:, None] * base ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def random_cache(rng, pages, hkv, code, scale=True):
    x = rng.standard_normal((2, pages, hkv, PAGE, DIM)).astype(np.float32)
    codes = [encode(a * (30 if code == INT8 else 80), code) for a in x]
    s = np.exp(0.5 * rng.standard_normal((2, pages, hkv))).astype(np.float32) / (30 if code == INT8 else 80)
    if not scale:
        return {"k_codes": encode(x[0], code), "v_codes": encode(x[1], code), "k_scale": None, "v_scale": None}
    return {"k_codes": codes[0], "v_codes": codes[1], "k_scale": s[0], "v_scale": s[1]}


def page_tables(rng, ctx, extra=0, max_pages=None):
    """Shuffled pages; entries past a sequence's pages are -1."""
    per = [(c + PAGE - 1) // PAGE for c in ctx]
    pages = sum(per) + extra
    order = rng.permutation(max(pages, 1))
    bt = np.full((len(ctx), max(1, max_pages or max(per, default=1))), -1, np.int32)
    at = 0
    for b, n in enumerate(per):
        bt[b, :n] = order[at:at + n]
        at += n
    return bt, max(pages, 1)


def to_gpu(cache, code):
    import paper_2607_28699_gb300 as wc
    dt = np.int8 if code == INT8 else np.uint8
    t = lambda x, d=None: None if x is None else torch.from_numpy(x.view(d) if d else x).cuda()  # noqa: E731
    return wc.BlockCache(t(cache["k_codes"], dt), t(cache["v_codes"], dt), t(cache["k_scale"]), t(cache["v_scale"]))
