"""The block-scaled 8-bit cache, as timed cases: appending to it, decoding from it, and extending a context over it.

Three kinds of pass over one layer's paged cache (pages of 16 tokens, 8-bit codes, one fp32 scale for each page and KV head):

``append``  rotate a step's (or a prompt's) new keys and queries to their positions and store keys and values
``decode``  attention of one query token per sequence over its whole context
``extend``  causal attention of several new query tokens per sequence (a prompt, a chunk of one, drafted tokens to verify)

Head shapes and context lengths are those of the repository's workloads and tests (28 query / 4 KV heads, 8 / 2, 40 / 8, 32 / 8; 4k to
128k tokens; batches of 16 x 4k-8k and 32 x 4k-32k).
"""

import math

import torch

own = False

PAGE, DIM = 16, 128
TINY = 2.0 ** -100


def _case(name, kind, code, act, batch, lo, hi, hq, hkv, new_lo=1, new_hi=1, rope="half", rot=128, packed=False):
    return {"name": name, "kind": kind, "code": code, "act": act, "batch": batch, "ctx_lo": lo, "ctx_hi": hi, "new_lo": new_lo,
            "new_hi": new_hi, "hq": hq, "hkv": hkv, "rope": rope, "rot": rot, "packed": packed}


def listed():
    return [
        # One new token of one short sequence: what a single user's decode step writes; latency.
        _case("append-token", "append", "int8", "fp16", 1, 4096, 4096, 8, 2),
        # One new token of each of 32 ragged sequences, straight from the packed output of a QKV projection.
        _case("append-batch32", "append", "e4m3", "bf16", 32, 4096, 32768, 28, 4, packed=True),
        # Ragged chunks of 16 prompts in flight, partial interleaved rotation.
        _case("append-chunks", "append", "e4m3", "bf16", 16, 700, 6001, 40, 8, new_lo=1, new_hi=1023, rope="interleaved", rot=64),
        # A whole 32k prompt.
        _case("append-prompt-32k", "append", "int8", "fp16", 1, 32768, 32768, 28, 4, new_lo=32768, new_hi=32768),
        # The first call anybody makes: one short sequence; latency.
        _case("decode-4k", "decode", "int8", "fp16", 1, 4096, 4096, 8, 2),
        # A 7B-class layer's decode at 32k.
        _case("decode-32k", "decode", "e4m3", "bf16", 1, 32768, 32768, 28, 4),
        # Serving: 16 ragged sequences of 4k to 8k.
        _case("decode-batch16", "decode", "int8", "bf16", 16, 4096, 8192, 28, 4, packed=True),
        # The largest batch: 32 sequences of 4k to 32k.
        _case("decode-batch32", "decode", "e4m3", "fp16", 32, 4096, 32768, 28, 4),
        # Five drafted tokens of each of 16 sequences are verified.
        _case("extend-verify", "extend", "int8", "fp16", 16, 4096, 8192, 28, 4, new_lo=5, new_hi=5),
        # Ragged chunks of 8 prompts, some of a few tokens; four query heads per KV head.
        _case("extend-ragged", "extend", "e4m3", "bf16", 8, 1000, 16001, 32, 8, new_lo=3, new_hi=1021, packed=True),
        # A whole 8k prompt.
        _case("extend-prompt-8k", "extend", "e4m3", "bf16", 1, 8192, 8192, 28, 4, new_lo=8192, new_hi=8192),
        # The last 4096 tokens of a 32k prompt processed in chunks.
        _case("extend-chunk-32k", "extend", "int8", "fp16", 1, 32768, 32768, 28, 4, new_lo=4096, new_hi=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "decode", "extend"])
    batch = rng.choice([1, 1, 2, 3, 5, 8, 16, 32])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    if hq > 64:
        hq = 8 * hkv
    hi = _log(rng, 16, 524288 // batch // hkv)
    hi = min(hi, 131072)
    lo = hi if batch == 1 else hi // rng.choice([1, 2, 8, hi + 1])
    new_lo = new_hi = 1
    if kind == "append":
        new_hi = rng.choice([1, _log(rng, 1, min(hi, max(1, 524288 // batch // (hq + 2 * hkv))))])
        new_lo = new_hi // rng.choice([1, 2, 8, new_hi + 1])
    elif kind == "extend":
        # the largest listed pass: 4096 new tokens, 28 heads, 32768 tokens of context
        most = min(4096 * 32768 * 28 // (batch * hi * hq), 32768 // batch)
        new_hi = min(hi, _log(rng, 2, max(2, most)))
        new_lo = new_hi // rng.choice([1, 2, 8, new_hi + 1])
    c = _case("", kind, rng.choice(["int8", "e4m3"]), rng.choice(["fp16", "bf16"]), batch, lo, hi, hq, hkv, new_lo, new_hi,
              rng.choice(["half", "interleaved"]), rng.choice([128, 128, 64, 32]), rng.random() < 0.4)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _spread(lo, hi, n):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lens(case, seed=0):
    """Context length after the step and new tokens of every sequence."""
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])
    new = [min(n, c) for n, c in zip(_spread(case["new_lo"], case["new_hi"], case["batch"]), ctx)]
    if case["kind"] == "decode":
        new = [1] * case["batch"]
    at = seed % case["batch"]
    return ctx[at:] + ctx[:at], new[at:] + new[:at]


def _codes(g, shape, code):
    """Codes of normal rows whose page's largest value takes the format's range, with heavier channels."""
    sigma = torch.exp(0.3 * torch.randn(shape[1], 1, DIM, generator=g, device="cuda"))
    x = torch.randn(shape, generator=g, device="cuda").mul_(sigma)
    if code == "int8":
        return x.mul_(30.0).round_().clamp_(-127, 127).to(torch.int8)
    return x.mul_(80.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1_000_003 + 17)
    h = torch.Generator().manual_seed(seed * 31 + 5)
    B, hq, hkv, code = case["batch"], case["hq"], case["hkv"], case["code"]
    act = torch.float16 if case["act"] == "fp16" else torch.bfloat16
    ctx, new = _lens(case, seed)
    per = [(c + PAGE - 1) // PAGE for c in ctx]
    most = max(1, max(per))
    pages = sum(per) + 1
    order = torch.randperm(pages, generator=h).int()
    bt = torch.full((B, most), -1, dtype=torch.int32)       # what is past a sequence's pages is never looked at
    at = 0
    for b, n in enumerate(per):
        bt[b, :n] = order[at:at + n]
        at += n
    n_tok = sum(new)
    heads = hq + 2 * hkv
    x = torch.randn(n_tok, heads, DIM, generator=g, device="cuda")
    x *= torch.exp(0.3 * torch.randn(heads, DIM, generator=g, device="cuda"))
    x = x.to(act)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not case["packed"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    shape = (pages, hkv, PAGE, DIM)
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.tensor(new).cumsum(0)
    s = {"case": case, "q": q, "k": k, "v": v, "bt": bt.cuda(), "ctx": torch.tensor(ctx, dtype=torch.int32).cuda(),
         "cu": cu.cuda(), "n_tok": n_tok, "new_max": max(new), "free": int(order[-1])}
    for n in ("k", "v"):
        s[n + "_codes"] = _codes(g, shape, code)
        s[n + "_scale"] = torch.exp(0.2 * torch.randn(pages, hkv, generator=g, device="cuda")) * (1 / 30 if code == "int8" else 1 / 80)
    if code == "e4m3":      # this format's scales are powers of two
        for n in ("k_scale", "v_scale"):
            s[n] = torch.exp2(torch.round(torch.log2(s[n])))
    # places past the context hold whatever was there, NaN codes among them
    last = torch.tensor([b for b in range(B) if ctx[b] % PAGE], dtype=torch.long)
    if len(last) and case["kind"] != "append":
        page = bt[last, torch.tensor(ctx)[last] // PAGE].long().cuda()
        stale = torch.arange(PAGE, device="cuda")[None] >= (torch.tensor(ctx)[last] % PAGE).cuda()[:, None]
        junk = torch.randint(0, 256, (len(last), hkv, PAGE, DIM), generator=g, device="cuda", dtype=torch.uint8).view(s["k_codes"].dtype)
        for n in ("k_codes", "v_codes"):
            s[n][page] = torch.where(stale[:, None, :, None], junk, s[n][page])
    if case["kind"] == "append":
        rot = case["rot"]
        ang = torch.arange(case["ctx_hi"], device="cuda", dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
    if own:
        import paper_2607_28699_gb300 as wc
        s["wc"] = wc
        s["desc"] = wc.BlockDesc(num_q_heads=hq, num_kv_heads=hkv, num_pages=pages, code=wc.CODE_INT8 if code == "int8" else wc.CODE_E4M3,
                                 rope_layout=wc.ROPE_HALF if case["rope"] == "half" else wc.ROPE_INTERLEAVED, rotary_dim=case["rot"])
        s["cache"] = wc.BlockCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"])
        if case["kind"] != "append":
            s["ws"] = wc.BlockWorkspace(s["desc"], B, n_tok, most)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the passes


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        wc = s["wc"]
        if kind == "append":
            cu = None if s["case"]["new_lo"] == s["case"]["new_hi"] == 1 and s["n_tok"] == s["case"]["batch"] else s["cu"]
            q = wc.block_append(s["desc"], s["k"], s["v"], s["ctx"], s["bt"], s["cache"], cu_new=cu, cos=s["cos"], sin=s["sin"], q=s["q"])
            return _appended(s, q)
        if kind == "decode":
            out, lse = wc.block_decode_attention(s["desc"], s["q"], s["bt"], s["ctx"], s["cache"], s["ws"], return_lse=True)
        else:
            out, lse = wc.block_extend_attention(s["desc"], s["q"], s["cu"], s["bt"], s["ctx"], s["cache"], s["ws"], return_lse=True)
        return {"out": out, "lse": lse}
    return _plain_append(s) if kind == "append" else _plain_attention(s)


def _appended(s, q):
    e4m3 = s["case"]["code"] == "e4m3"
    codes = {n: s[n].view(torch.float8_e4m3fn) if e4m3 else s[n] for n in ("k_codes", "v_codes")}
    return {"q": q, "k_scale": s["k_scale"], "v_scale": s["v_scale"], **codes}


def _rotate(x, cos, sin, rope, rot):
    """x [n, heads, 128] in 32 bits; cos, sin [n, 1, rot / 2]."""
    if rope == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _scale_of(amax, code):
    if code == "int8":
        s = (amax / 127.0).clamp_min(TINY)
    else:       # the least power of two with amax / s <= 448 = 1.75 * 2^8
        m, e = torch.frexp(amax)        # amax = m 2^e, m in [0.5, 1)
        e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-100)
        s = ((e + 127) << 23).view(torch.float32)
    return torch.where(amax > 0, s, torch.zeros_like(s))


def _encode(y, code):
    """The nearest code of y (already divided by its scale), ties to even."""
    if code == "int8":
        return y.round().clamp_(-127, 127).to(torch.int8)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(c, code):
    return c.float() if code == "int8" else c.view(torch.float8_e4m3fn).float()


def _plain_append(s):
    case = s["case"]
    code, B = case["code"], case["batch"]
    cu, ctx = s["cu"].long(), s["ctx"].long()
    new = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), new, output_size=s["n_tok"])
    pos = torch.arange(s["n_tok"], device="cuda") - cu[seq] + (ctx - new)[seq]
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    q = _rotate(s["q"].float(), cos, sin, case["rope"], case["rot"]).to(s["q"].dtype)
    page, off = s["bt"][seq, pos // PAGE].long(), pos % PAGE
    # each sequence's first page may hold older tokens
    start = ctx - new
    keep = torch.where(new > 0, start % PAGE, torch.zeros_like(start))
    at = s["bt"].gather(1, (start // PAGE).clamp(max=s["bt"].shape[1] - 1)[:, None])[:, 0].long()
    old_page = torch.where(keep > 0, at, torch.full_like(at, s["free"]))        # none: a page in nobody's table
    held = (torch.arange(PAGE, device="cuda")[None] < keep[:, None])[:, None, :, None]      # places of older tokens
    for x, n in ((_rotate(s["k"].float(), cos, sin, case["rope"], case["rot"]), "k"), (s["v"].float(), "v")):
        codes, scale = s[n + "_codes"], s[n + "_scale"]
        amax = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
        had = scale[old_page]
        to = _scale_of(amax, code)
        to[old_page] = torch.maximum(to[old_page], had)
        ratio = torch.where(to[old_page] > 0, had / to[old_page], torch.zeros_like(had))
        again = _encode(_decode(codes[old_page], code) * ratio[:, :, None, None], code)
        kept = torch.where(held, again, codes[old_page])
        inv = torch.where(to > 0, 1.0 / to, torch.zeros_like(to))[page]
        codes[old_page] = kept
        codes[page, :, off] = _encode(x * inv[..., None], code)
        scale[page] = to[page]
    return _appended(s, q)


def _plain_attention(s):
    case = s["case"]
    code, B, hq, hkv = case["code"], case["batch"], case["hq"], case["hkv"]
    G = hq // hkv
    ctx, cu, n = s["ctx"].long(), s["cu"].long(), s["new_max"]
    S = s["bt"].shape[1] * PAGE
    table = s["bt"].long().clamp(min=0)
    place = torch.arange(S, device="cuda")
    valid = place[None] < ctx[:, None]
    kv = []
    for name in ("k", "v"):
        x = _decode(s[name + "_codes"][table], code)                                    # [B, pages, hkv, 16, 128]
        x *= s[name + "_scale"][table][..., None, None]
        x = x.transpose(1, 2).reshape(B, hkv, S, DIM)
        kv.append(x.masked_fill_(~valid[:, None, :, None], 0.0))
    new = cu[1:] - cu[:-1]
    i = torch.arange(n, device="cuda")
    row = (cu[:-1, None] + i[None]).clamp(max=s["n_tok"] - 1)
    q = s["q"][row].float()                                                             # [B, n, hq, 128]
    q = q.view(B, n, hkv, G, DIM).permute(0, 2, 3, 1, 4).reshape(B, hkv, G * n, DIM)
    t = torch.matmul(q, kv[0].transpose(-1, -2)).mul_(1 / math.sqrt(DIM)).view(B, hkv, G, n, S)
    seen = place[None, None] <= (ctx - new)[:, None, None] + i[None, :, None]           # [B, n, S]
    t.masked_fill_(~(seen & valid[:, None])[:, None, None], -math.inf)
    m = t.amax(-1, keepdim=True).clamp_min(-1e30)
    l = t.sub_(m).exp_().sum(-1, keepdim=True)
    o = torch.matmul(t.view(B, hkv, G * n, S), kv[1]).view(B, hkv, G, n, DIM)
    o = torch.where(l > 0, o / l, torch.zeros_like(o))
    lse = (m + l.log())[..., 0]
    mine = torch.repeat_interleave(torch.arange(B, device="cuda"), new, output_size=s["n_tok"])
    at = torch.arange(s["n_tok"], device="cuda") - cu[mine]
    out = o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, DIM)[mine, at].to(s["q"].dtype)
    return {"out": out, "lse": lse.permute(0, 3, 1, 2).reshape(B, n, hq)[mine, at]}


# ---------------------------------------------------------------------------------------------------------------------


def work(case):
    ctx, new = _lens(case)
    hq, hkv = case["hq"], case["hkv"]
    n = sum(new)
    tables = 4 * sum((c + PAGE - 1) // PAGE for c in ctx)
    if case["kind"] == "append":
        moved = n * (2 * hq + 2 * hkv) * DIM * 2 + n * hkv * 2 * DIM + n * case["rot"] * 4
        return {"bytes": moved + 8 * hkv * sum((a + PAGE - 1) // PAGE for a in new), "flops": n * DIM * (3 * hq + 6 * hkv)}
    # keys that a token's row sees, summed over the rows
    seen = sum(a * (c - a) + a * (a + 1) // 2 for c, a in zip(ctx, new))
    if case["kind"] == "decode":
        seen = sum(ctx)
    read = sum(ctx) * hkv * 2 * DIM + 2 * hkv * tables + tables
    return {"bytes": read + n * hq * (2 * DIM * 2 + 4), "flops": 4 * DIM * hq * seen}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, a sequence at a time


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s) if case["kind"] == "append" else _exact_attention(s)


def _values(codes, code):
    return codes.double() if code == "int8" else codes.view(torch.float8_e4m3fn).double()


def _turn(x, pos, case):
    """x [heads, 128] in 64 bits, turned pair by pair in the complex plane by the tables' angles."""
    rot, (cos, sin) = case["rot"], pos
    by = torch.complex(cos.double(), sin.double())
    if case["rope"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * by
        y = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * by
        y = torch.view_as_real(z).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _exact_append(s):
    case = s["case"]
    ctx, new = s["ctx"].tolist(), (s["cu"][1:] - s["cu"][:-1]).tolist()
    scales = {n: s[n + "_scale"].double() for n in "kv"}
    qs, at = [], 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        if n == 0:
            continue
        rows, first = slice(at, at + n), c - n
        at += n
        trig = s["cos"][first:c][:, None], s["sin"][first:c][:, None]
        qs.append(_turn(s["q"][rows].double(), trig, case))
        lead = first % PAGE
        for name, x in (("k", _turn(s["k"][rows].double(), trig, case)), ("v", s["v"][rows].double())):
            most = x.abs().amax(-1)                                             # [n, hkv]
            whole = torch.zeros(-(-(lead + n) // PAGE) * PAGE, most.shape[1], dtype=torch.float64, device="cuda")
            whole[lead:lead + n] = most
            most = whole.view(-1, PAGE, most.shape[1]).amax(1)
            if case["code"] == "int8":
                need = (most / 127).clamp_min(TINY)
            else:
                m, e = torch.frexp(most / 448)      # m in [0.5, 1): the least power of two is 2^e, or 2^(e - 1) at m = 0.5
                need = torch.tensor([math.ldexp(1.0, x) for x in torch.where(m == 0.5, e - 1, e).clamp(min=-100).flatten().tolist()],
                                    dtype=torch.float64, device="cuda").view_as(most)
            page = s["bt"][b, first // PAGE:(c + PAGE - 1) // PAGE].long()
            if lead:
                need[0] = torch.maximum(need[0], scales[name][page[0]])
            scales[name][page] = need
    q = torch.cat(qs) if qs else s["q"].double()
    # a code is a rounding of these: where its argument lies next to a tie, 64 bits do not say which neighbour 32 bits find
    return {"q": q, "k_scale": scales["k"], "v_scale": scales["v"], "k_codes": None, "v_codes": None}


def _exact_attention(s):
    case = s["case"]
    G, hkv, code = case["hq"] // case["hkv"], case["hkv"], case["code"]
    if work(case)["flops"] > 3e12:
        return None
    out = torch.zeros(s["n_tok"], case["hq"], DIM, dtype=torch.float64, device="cuda")
    lse = torch.full((s["n_tok"], case["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    ctx, cu = s["ctx"].tolist(), s["cu"].tolist()
    for b, c in enumerate(ctx):
        n = cu[b + 1] - cu[b]
        if n == 0 or c == 0:
            continue
        pages = s["bt"][b, :(c + PAGE - 1) // PAGE].long()
        for h in range(hkv):
            k, v = ((_values(s[x + "_codes"][pages, h], code) * s[x + "_scale"][pages, h, None, None].double()).view(-1, DIM)[:c] for x in "kv")
            for i in range(cu[b], cu[b + 1], 1024):
                j = min(i + 1024, cu[b + 1])
                last = c - n + torch.arange(i, j, device="cuda") - cu[b]
                hidden = torch.arange(c, device="cuda")[None] > last[:, None]
                for g in range(h * G, (h + 1) * G):
                    t = (s["q"][i:j, g].double() @ k.T / math.sqrt(DIM)).masked_fill_(hidden, -math.inf)
                    lse[i:j, g] = torch.logsumexp(t, -1)
                    out[i:j, g] = torch.softmax(t, -1).nan_to_num_(0.0) @ v
    return {"out": out, "lse": lse}
