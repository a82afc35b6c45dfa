"""Workloads of the operators around the ternary GEMVs of a decoder layer: the paged key/value cache
(written with rotation and quantisation, read back), the attention of a chunk of new tokens over it,
and the norms before and after a block with its gate and residual scale.

`run` computes an operator either in its plain form (elementary torch operations in 32 bits, rounded
once at the end) or, with `own`, through the framework's entry points. The batch of a case is text:
"ctx" holds each sequence's length with its new tokens, "q" the number of its new tokens.

Cache formats: "f16" (fp16 rows), "fp8" (E4M3 codes) and "fp4" (E2M1 codes, two per byte, the lower
element in the low nibble), the last two with one power of two per 32 elements of a row: the smallest
2^e, -14 <= e, with the block's largest magnitude at most 448 * 2^e (fp8) or 6 * 2^e (fp4), held as
the byte e + 127. Pages are [n_pages][kv heads][page_size][head_dim].
"""
import math

import torch

own = False

_KV = ("f16", "fp8", "fp4")
_BLOCK = 32
_TOP = {"fp8": 448.0, "fp4": 6.0}
_E_MAX = {"fp8": 7, "fp4": 13}


# ------------------------------------------------------------------------------------------ cases


def listed():
    return [
        # one user's decode step, short context: what counts is latency
        dict(name="att_decode_one_f16", op="attention", fmt="f16", q="1", ctx="517", hq=32, hkv=8, dim=128, page=16,
             window=0),
        # a serving batch of decode steps, ragged contexts, one sequence of a single token
        dict(name="att_decode_batch_fp8", op="attention", fmt="fp8", q="1,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1",
             ctx="8192,7013,1,655,3001,4096,129,8191,2500,6400,77,5120,1023,1024,7777,333", hq=40, hkv=8, dim=128,
             page=64, window=0),
        # one long document, a decode step over the smallest cache format
        dict(name="att_decode_long_fp4", op="attention", fmt="fp4", q="1", ctx="131071", hq=64, hkv=8, dim=128,
             page=128, window=0),
        # 16 tokens a sequence (the largest batch of one GEMV call): drafted tokens or a small chunk
        dict(name="att_chunk16_fp8", op="attention", fmt="fp8", q="16,16,16,16,16,16,16,16",
             ctx="16384,9001,16001,12345,16,8192,15000,11111", hq=64, hkv=8, dim=128, page=64, window=0),
        # two prompts' chunks packed together over what their caches already hold: compute-bound
        dict(name="att_prompt_f16", op="attention", fmt="f16", q="2048,1000", ctx="16384,5001", hq=32, hkv=8, dim=128,
             page=32, window=0),
        # a decode step's 16 tokens written into an 8-bit cache, with rotation
        dict(name="append_decode_fp8", op="append", fmt="fp8", q="1,1,1,1,1,1,1,1,1,1,1,1,1,1,1,1",
             ctx="2048,7013,1,655,3001,4096,129,2047,2500,6400,77,5120,1023,1024,7777,333", hq=40, hkv=8, dim=128,
             page=64, src="f32", rotate=True, qk_norm=False),
        # prompts' tokens written into a 16-bit cache, with the per-head norms of q and k
        dict(name="append_prompt_f16", op="append", fmt="f16", q="5000,3192", ctx="5000,8000", hq=32, hkv=8, dim=128,
             page=16, src="f32", rotate=True, qk_norm=True),
        # a sequence's cache read back (to move it, or to hand it to other code)
        dict(name="read_long_fp8", op="read", fmt="fp8", q="1", ctx="100003", hq=32, hkv=8, dim=128, page=64),
        # a chunk written into a 4-bit cache and the sequences read back
        dict(name="write_read_fp4", op="write_read", fmt="fp4", q="509,1,258", ctx="2045,1000,258", hq=32, hkv=8,
             dim=128, page=32, src="f16", rotate=True, qk_norm=False),
        # one decode token: the norm before a block, nothing else (hidden size of the Llama3-8B layer)
        dict(name="norm_one", op="norm", rows=1, cols=4096, y="none", post=False, gate="none", h="f32"),
        # 16 tokens, norms on both sides of a block (hidden size of the Qwen3-14B layer)
        dict(name="norm_16_sandwich", op="norm", rows=16, cols=5120, y="f32", post=True, gate="channel", h="f32"),
        # a prompt's tokens with a gate for each token (hidden size of the Llama3-70B layer)
        dict(name="norm_prompt", op="norm", rows=8192, cols=8192, y="f32", post=True, gate="token", h="f32"),
    ]


def _size(n):
    return n - (n == 3072)  # none of the framework's own configurations has this size


def _log(rng, lo, hi):
    return _size(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """A case of the same ranges: decode steps, small chunks, prompts; every cache format."""
    op = rng.choice(("attention", "attention", "attention", "append", "read", "write_read", "norm"))
    if op == "norm":
        cols = _log(rng, 64, 8192)
        if rng.random() < 0.7:  # hidden sizes are mostly multiples of 64, a few are not
            cols = _size(cols // 64 * 64)
        rows = _log(rng, 1, max(1, min(8192, 40_000_000 // cols)))
        y = rng.choice(("f32", "f32", "f16", "none"))
        return dict(op="norm", rows=rows, cols=cols, y=y, post=y != "none" and rng.random() < 0.6,
                    gate=rng.choice(("none", "channel", "token")) if y != "none" else "none",
                    h=rng.choice(("f32", "f32", "f16")))
    hq, hkv = rng.choice(((32, 8), (40, 8), (64, 8), (16, 16), (24, 2), (8, 1)))
    dim = rng.choice((128, 128, 64))
    page = rng.choice((16, 32, 64, 128))
    fmt = rng.choice(_KV)
    if op == "attention":
        kind = rng.choice(("decode", "decode", "few", "chunk"))
        seqs = _log(rng, 1, 24) if kind != "chunk" else rng.randint(1, 2)
        longest = max(1, min(100_000, 150_000 // seqs)) if kind != "chunk" else 6000
        top = {"decode": 1, "few": 16, "chunk": 1000}[kind]
        q = [1 if kind == "decode" else _log(rng, 1, top) for _ in range(seqs)]
        ctx = [max(n, _log(rng, 1, longest)) for n in q]
        return dict(op=op, fmt=fmt, q=_text(q), ctx=_text(ctx), hq=hq, hkv=hkv, dim=dim, page=page,
                    window=rng.choice((0, 0, 0, _log(rng, 16, 4096))))
    if op == "read":
        seqs = _log(rng, 1, 12)
        ctx = [_log(rng, 1, max(1, 60_000 // seqs)) for _ in range(seqs)]
        return dict(op=op, fmt=fmt, q=_text([1] * seqs), ctx=_text(ctx), hq=hq, hkv=hkv, dim=dim, page=page)
    if op == "append":
        fmt = rng.choice(("f16", "fp8"))
    seqs = _log(rng, 1, 24)
    q = [_log(rng, 1, max(1, 6000 // seqs)) if rng.random() < 0.6 else 1 for _ in range(seqs)]
    ctx = [_size(n + (0 if rng.random() < 0.3 else _log(rng, 1, 3000))) for n in q]
    return dict(op=op, fmt=fmt, q=_text(q), ctx=_text(ctx), hq=hq, hkv=hkv, dim=dim, page=page,
                src=rng.choice(("f32", "f16")), rotate=rng.random() < 0.8,
                qk_norm=op == "append" and fmt == "f16" and rng.random() < 0.4)


def _text(v):
    return ",".join(str(x) for x in v)


def _list(case, key):
    return [int(x) for x in case[key].split(",")]


def _row_bytes(fmt, dim):
    """Bytes of one cached row of one head: its elements and the bytes of its scales."""
    return {"f16": 2 * dim, "fp8": dim + dim // _BLOCK, "fp4": dim // 2 + dim // _BLOCK}[fmt]


def work(case):
    """Bytes read and written once, and operations (two per multiply-add of the matrix products)."""
    if case["op"] == "norm":
        m, n = case["rows"], case["cols"]
        size = {"f32": 4, "f16": 2, "none": 0}
        has_y = case["y"] != "none"
        per = size[case["h"]] * (2 if has_y else 1) + size[case["y"]] + 2 + (2 if case["gate"] == "token" else 0)
        vec = 2 + (2 if case["post"] else 0) + (2 if case["gate"] == "channel" else 0)
        return dict(bytes=m * n * per + n * vec, flops=m * n * 10)
    q, ctx = _list(case, "q"), _list(case, "ctx")
    hq, hkv, dim, page = case["hq"], case["hkv"], case["dim"], case["page"]
    tables = 4 * (2 * len(q) + 1 + sum(-(-c // page) for c in ctx))
    row = 2 * hkv * _row_bytes(case["fmt"], dim)
    if case["op"] == "attention":
        w = case["window"]
        pairs = keys = 0
        for n, c in zip(q, ctx):
            first = c - n + 1  # keys that the first new token sees
            if w:
                pairs += sum(min(first + i, w) for i in range(n))
                keys += c - max(0, first - w)
            else:
                pairs += n * first + n * (n - 1) // 2
                keys += c
        return dict(bytes=keys * row + 2 * 2 * sum(q) * hq * dim + tables, flops=4 * dim * hq * pairs)
    if case["op"] == "read":
        return dict(bytes=sum(ctx) * (row + 2 * hkv * dim * 2) + tables, flops=sum(ctx) * 2 * hkv * dim)
    t, src = sum(q), 4 if case["src"] == "f32" else 2
    moved = t * (hq + 2 * hkv) * dim * src + t * hq * dim * 2 + t * row + tables
    if case["rotate"]:
        moved += min(t, max(ctx)) * dim * 4
    flops = 6 * t * (hq + hkv) * dim + 4 * t * hkv * dim
    if case["op"] == "write_read":
        moved += sum(ctx) * (row + 2 * hkv * dim * 2)
    return dict(bytes=moved, flops=flops)


# ----------------------------------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    types = {"f32": torch.float32, "f16": torch.float16}
    if case["op"] == "norm":
        m, n = case["rows"], case["cols"]
        s = dict(case=case, h=randn(m, n, scale=3.0, dtype=types[case["h"]]), weight=(1 + randn(n, scale=0.2)).half(),
                 y=None, post=None, gate=None, res_scale=1.0, eps=1e-6)
        s["x"] = torch.empty(m, n, dtype=torch.float16, device="cuda")
        if case["y"] != "none":
            # one channel in 64 is a hundred times larger, as the massive activations of real models
            y = randn(m, n) * (1 + 99 * (torch.arange(n, device="cuda") % 64 == 5))
            s.update(y=y.to(types[case["y"]]), res_scale=0.7, h_out=torch.empty_like(s["h"]))
        if case["post"]:
            s["post"] = (1 + randn(n, scale=0.2)).half()
        if case["gate"] != "none":
            shape = (m, n) if case["gate"] == "token" else (n,)
            s["gate"] = torch.sigmoid(randn(*shape)).half()
        return s

    q, ctx = _list(case, "q"), _list(case, "ctx")
    hq, hkv, dim, page, fmt = case["hq"], case["hkv"], case["dim"], case["page"], case["fmt"]
    tokens = sum(q)
    counts = [-(-c // page) for c in ctx]
    n_pages = sum(counts) + 3
    # a sequence's pages lie anywhere in the pool; unused entries of its table are never looked at
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    pages = torch.full((len(q), max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(counts):
        pages[i, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in q:
        starts.append(starts[-1] + n)
    rows = [0]
    for n in ctx:
        rows.append(rows[-1] + n)
    s = dict(case=case, q_start=torch.tensor(starts, dtype=torch.int32, device="cuda"),
             ctx_len=torch.tensor(ctx, dtype=torch.int32, device="cuda"), pages=pages, max_q=max(q), tokens=tokens,
             row_start=torch.tensor(rows, dtype=torch.int32, device="cuda"), rows=rows[-1], max_ctx=max(ctx))
    for name in ("k", "v"):
        # keys with a few large channels, the usual case that rotation leaves in place
        x = randn(n_pages, hkv, page, dim)
        if name == "k":
            x *= 1 + 4 * (torch.arange(dim, device="cuda") % 32 == 7)
        s[name + "_pages"], s[name + "_scale"] = _encode(x, fmt)
        del x
    if case["op"] == "attention":
        s["q"] = randn(tokens, hq, dim, dtype=torch.float16)
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = dim ** -0.5
    elif case["op"] != "read":
        src = types[case["src"]]
        s["q"], s["k"], s["v"] = (randn(tokens, h * dim, dtype=src) for h in (hq, hkv, hkv))
        s["q_out"] = torch.empty(tokens, hq, dim, dtype=torch.float16, device="cuda")
        s["cos"] = s["sin"] = s["q_norm"] = s["k_norm"] = None
        s["eps"] = 1e-6
        if case["rotate"]:
            rate = 500000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
            angle = torch.arange(max(ctx), device="cuda", dtype=torch.float64)[:, None] * rate
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if case["qk_norm"]:
            s["q_norm"], s["k_norm"] = ((1 + randn(dim, scale=0.2)).half() for _ in range(2))
    if case["op"] in ("read", "write_read"):
        s["k_out"], s["v_out"] = (torch.empty(rows[-1], hkv, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    if own:  # the cache and batch handles that a program makes once and keeps with these tensors
        import paper_2609_00224_gb300 as qt
        s["cache"] = qt.KVCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"],
                                fmt={"f16": qt.QTEA_KV_F16, "fp8": qt.QTEA_KV_FP8, "fp4": qt.QTEA_KV_FP4}[fmt])
        s["batch"] = qt.KVBatch(s["q_start"], s["ctx_len"], s["pages"], n_tokens=tokens, max_q_len=max(q))
    return s


# ------------------------------------------------------------------------------------------ passes


def run(state):
    op = state["case"]["op"]
    return _own(op, state) if own else _plain(op, state)


def _own(op, s):
    import paper_2609_00224_gb300 as qt
    if op == "norm":
        x = qt.qtea_norm(s["h"], s["weight"], y=s["y"], post_weight=s["post"], gate=s["gate"],
                         res_scale=s["res_scale"], eps=s["eps"], h_out=s.get("h_out"), x=s["x"])
        return dict(x=x, h=s["h_out"]) if s["y"] is not None else dict(x=x)
    cache, batch = s["cache"], s["batch"]
    if op == "attention":
        return qt.qtea_attention(cache, batch, s["q"], scale=s["scale"], window=s["case"]["window"], out=s["out"])
    if op == "read":
        return qt.qtea_kv_read(cache, batch, s["row_start"], k_out=s["k_out"], v_out=s["v_out"])
    q = qt.qtea_kv_append(cache, batch, s["k"], s["v"], q=s["q"], cos=s["cos"], sin=s["sin"], q_norm=s["q_norm"],
                          k_norm=s["k_norm"], eps=s["eps"], q_out=s["q_out"])
    if op == "write_read":
        k, v = qt.qtea_kv_read(cache, batch, s["row_start"], k_out=s["k_out"], v_out=s["v_out"])
        return dict(q=q, k=k, v=v)
    return dict(q=q, **_held(s))


def _held(s):
    """The cache's contents as the values that they stand for (before their powers of two), and those."""
    if s["case"]["fmt"] == "f16":
        return dict(k=s["k_pages"], v=s["v_pages"])
    f8 = torch.float8_e4m3fn
    return dict(k=s["k_pages"].view(f8), v=s["v_pages"].view(f8), k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain(op, s):
    if op == "norm":
        return _plain_norm(s)
    if op == "attention":
        return _plain_attention(s)
    if op == "read":
        return _plain_read(s)
    q = _plain_append(s)
    if op == "write_read":
        k, v = _plain_read(s)
        return dict(q=q, k=k, v=v)
    return dict(q=q, **_held(s))


def _encode(x, fmt):
    """fp32 rows in a cache format: (codes, bytes of the scales or None)."""
    if fmt == "f16":
        return x.half(), None
    b = x.unflatten(-1, (-1, _BLOCK))
    top = b.abs().amax(-1)
    # the smallest e with top <= limit * 2^e: frexp gives top / limit's exponent up to one, then compare
    e = (torch.frexp(top)[1] - (9 if fmt == "fp8" else 3)).clamp(-14, _E_MAX[fmt])
    e = torch.where((top > _TOP[fmt] * torch.exp2(e.float())) & (e < _E_MAX[fmt]), e + 1, e)
    e = torch.where(top > 0, e, -14)
    v = (b * torch.exp2(-e.float())[..., None]).clamp(-_TOP[fmt], _TOP[fmt])
    scale = (e + 127).to(torch.uint8)
    if fmt == "fp8":
        return v.to(torch.float8_e4m3fn).flatten(-2).view(torch.uint8), scale
    # E2M1 to nearest, ties to even: how many of these the magnitude passes (or reaches, for odd codes)
    m = v.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    code = (code | (torch.signbit(v).to(torch.uint8) << 3)).flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), scale


def _decode(codes, scale, fmt):
    """fp32 rows from a cache format."""
    if fmt == "f16":
        return codes.float()
    if fmt == "fp8":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
        x = torch.where(c >= 8, -table[c & 7], table[c & 7])
    f = torch.exp2(scale.float() - 127)
    return (x.unflatten(-1, (-1, _BLOCK)) * f[..., None]).flatten(-2)


def _gathered(s, name):
    """Every sequence's rows of one side of the cache: fp32 [sequences][kv heads][tokens][dim]."""
    p = s["pages"].clamp(min=0).long()
    scale = s[name + "_scale"]
    x = _decode(s[name + "_pages"][p], None if scale is None else scale[p], s["case"]["fmt"])
    return x.transpose(1, 2).flatten(2, 3)


def _tokens(s):
    """Of each new token: its sequence, its place among that sequence's new tokens, its position."""
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    i = t - s["q_start"].long()[seq]
    n = s["q_start"].long().diff()[seq]
    return seq, i, s["ctx_len"].long()[seq] - n + i


def _plain_attention(s):
    c = s["case"]
    hq, hkv, dim, w = c["hq"], c["hkv"], c["dim"], c["window"]
    seq, i, pos = _tokens(s)
    n_seqs, most = s["ctx_len"].numel(), s["max_q"]
    q = torch.zeros(n_seqs, most, hq, dim, device="cuda")
    q[seq, i] = s["q"].float()
    q = q.view(n_seqs, most, hkv, hq // hkv, dim).transpose(1, 2).flatten(2, 3)
    k = _gathered(s, "k")
    logits = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    del k
    last = torch.full((n_seqs, most), -1, device="cuda", dtype=torch.long)
    last[seq, i] = pos
    last = last.repeat_interleave(hq // hkv, 1)[:, None, :, None]
    j = torch.arange(logits.shape[-1], device="cuda")
    hidden = j > last
    if w:
        hidden |= j <= last - w
    logits.masked_fill_(hidden, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = logits.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _gathered(s, "v")) / torch.where(total > 0, total, 1.0)
    o = o.view(n_seqs, hkv, most, hq // hkv, dim).transpose(1, 2).reshape(n_seqs, most, hq, dim)
    return o[seq, i].half()


def _plain_read(s):
    r = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["row_start"][1:].long(), r, right=True)
    p = r - s["row_start"].long()[seq]
    return tuple(_gathered(s, name).transpose(1, 2)[seq, p].half() for name in ("k", "v"))


def _rotated(x, weight, s, pos):
    """The per-head norm, then the rotation of the pairs (i, i + dim/2) by the position's angles."""
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
    if s["cos"] is None:
        return x
    c, d = s["cos"][pos][:, None], s["sin"][pos][:, None]
    a, b = x.chunk(2, -1)
    return torch.cat((a * c - b * d, b * c + a * d), -1)


def _plain_append(s):
    c = s["case"]
    seq, i, pos = _tokens(s)
    page = s["pages"].long()[seq, pos // c["page"]]
    off = pos % c["page"]
    k = _rotated(s["k"].float().unflatten(-1, (c["hkv"], c["dim"])), s["k_norm"], s, pos)
    v = s["v"].float().unflatten(-1, (c["hkv"], c["dim"]))
    for name, x in (("k", k), ("v", v)):
        codes, scale = _encode(x, c["fmt"])
        s[name + "_pages"][page, :, off] = codes
        if scale is not None:
            s[name + "_scale"][page, :, off] = scale
    return _rotated(s["q"].float().unflatten(-1, (c["hq"], c["dim"])), s["q_norm"], s, pos).half()


def _plain_norm(s):
    def rms(t, w):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + s["eps"]) * w.float()

    h = s["h"].float()
    if s["y"] is None:
        return dict(x=rms(h, s["weight"]).half())
    t = s["y"].float()
    if s["post"] is not None:
        t = rms(t, s["post"])
    if s["gate"] is not None:
        t = t * s["gate"].float()
    h = h + s["res_scale"] * t
    return dict(x=rms(h, s["weight"]).half(), h=h.to(s["h"].dtype))


# ------------------------------------------------------------------------------- the same in 64 bits


def exact(case, seed):
    """run()'s outputs from the operators' definitions in 64 bits, a sequence at a time."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "attention":
        return _exact_attention(s)
    if case["op"] == "read":
        return _exact_read(s)
    if case["op"] == "append":
        return _exact_append(s)
    return None  # codes of 4 bits read back: a value at a rounding's edge has no one answer


def _value(s, name, i):
    """Sequence i's cached rows in 64 bits: [context][kv heads][dim]."""
    c = s["case"]
    n = int(s["ctx_len"][i])
    used = s["pages"][i, :-(-n // c["page"])].tolist()
    codes = torch.cat([s[name + "_pages"][p].transpose(0, 1) for p in used])[:n]
    if c["fmt"] == "f16":
        return codes.double()
    power = torch.cat([s[name + "_scale"][p].transpose(0, 1) for p in used])[:n].double() - 127
    if c["fmt"] == "fp8":
        bits = torch.arange(256)
        e, m = (bits >> 3) & 15, bits & 7
        table = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10).double())
        table = torch.where(bits >= 128, -table, table).to(codes.device)
        x = table[codes.long()]
    else:
        table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                             device=codes.device)
        x = torch.empty(*codes.shape[:-1], c["dim"], dtype=torch.float64, device=codes.device)
        x[..., 0::2], x[..., 1::2] = table[(codes % 16).long()], table[(codes // 16).long()]
    return x * torch.repeat_interleave(2.0 ** power, _BLOCK, -1)


def _exact_attention(s):
    c = s["case"]
    group = c["hq"] // c["hkv"]
    out = torch.zeros(s["tokens"], c["hq"], c["dim"], dtype=torch.float64, device="cuda")
    for i in range(s["ctx_len"].numel()):
        a, b, n = int(s["q_start"][i]), int(s["q_start"][i + 1]), int(s["ctx_len"][i])
        k, v = _value(s, "k", i), _value(s, "v", i)
        pos = torch.arange(n - (b - a), n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        seen = j <= pos
        if c["window"]:
            seen &= j > pos - c["window"]
        for h in range(c["hq"]):
            z = (s["q"][a:b, h].double() @ k[:, h // group].T) * s["scale"]
            z = torch.where(seen, z, -math.inf)
            out[a:b, h] = torch.softmax(z, -1) @ v[:, h // group]
    return out


def _exact_read(s):
    k, v = (torch.cat([_value(s, name, i) for i in range(s["ctx_len"].numel())]) for name in ("k", "v"))
    return k, v


def _exact_append(s):
    c = s["case"]
    dim, half = c["dim"], c["dim"] // 2
    held = {n: (s[n + "_pages"] if c["fmt"] == "f16" else s[n + "_pages"].view(torch.float8_e4m3fn)).double()
            for n in ("k", "v")}
    q_out = torch.empty(s["tokens"], c["hq"], dim, dtype=torch.float64, device="cuda")
    for i in range(s["ctx_len"].numel()):
        a, b, n = int(s["q_start"][i]), int(s["q_start"][i + 1]), int(s["ctx_len"][i])
        pos = torch.arange(n - (b - a), n, device="cuda")
        page, off = s["pages"][i].long()[pos // c["page"]], pos % c["page"]
        for name, heads in (("q", c["hq"]), ("k", c["hkv"]), ("v", c["hkv"])):
            x = s[name][a:b].double().view(b - a, heads, dim)
            w = s.get(name + "_norm")
            if w is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / dim + s["eps"]).sqrt() * w.double()
            if s["cos"] is not None and name != "v":
                z = torch.complex(x[..., :half], x[..., half:])
                z = z * torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]
                x = torch.cat((z.real, z.imag), -1)
            if name == "q":
                q_out[a:b] = x
                continue
            if c["fmt"] == "fp8":
                top = x.view(b - a, heads, -1, _BLOCK).abs().amax(-1).clamp(min=448 * 2.0 ** -14)
                e = torch.ceil(torch.log2(top / 448)).clamp(-14, 7)
                x = x / torch.repeat_interleave(2.0 ** e, _BLOCK, -1)
            held[name][page, :, off] = x
    got = dict(q=q_out, k=held["k"], v=held["v"])
    return got if c["fmt"] == "f16" else dict(got, k_scale=None, v_scale=None)


def _exact_norm(s):
    def rms(t, w):
        return t / (t.pow(2).sum(-1, keepdim=True) / t.shape[-1] + s["eps"]).sqrt() * w.double()

    h = s["h"].double()
    if s["y"] is None:
        return dict(x=rms(h, s["weight"]))
    t = s["y"].double()
    if s["post"] is not None:
        t = rms(t, s["post"])
    if s["gate"] is not None:
        t = t * s["gate"].double()
    h = h + s["res_scale"] * t
    return dict(x=rms(h, s["weight"]), h=h)
