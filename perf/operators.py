"""The operators of a serving loop around the package's attention, as they are timed: rotary positions, a paged key/value
cache that is quantised as it is written, attention of the newest tokens over that cache, and the same for a batch whose
sequences share a long prefix.

Each comes in a plain form (elementary torch operations in 32 bits, 64 where angles need them) and, where `own` is true, as
the package's own call.  Sizes are those of the package's own benchmark and tests (32/8, 16/16, 12/12 and 64/8 heads, head dims
64/64, 128/128 and 192/128, its decoding lengths) or generic ones of the same ranges.

Layouts: Q [B, H_q, n, D_qk], K and V [B, H_kv, L, D]; cache pages [n_pages, H_kv, page, D]; a position of the cache is the slot
page_number * page + place.  An 8-bit cache holds e4m3 values and, for every cached row of a head, a power of two as its biased exponent:
the smallest 2^k (k >= -126) for which the row's largest finite magnitude fits 448.
"""
import math
import random

import torch

own = False


# ---- the cases ----------------------------------------------------------------------------------------------------
def _rotary(name, B, H_q, H_kv, L, D, rot, **kw):
    c = dict(name=name, op="rotary", B=B, H_q=H_q, H_kv=H_kv, L=L, D=D, rot=rot, layout="half", scaling="none", factor=1.0,
             start=0, backward=False, dtype="bf16", order="blhd")
    c.update(kw)
    return c


def _write(name, B, H_kv, L, D_qk, D_v, **kw):
    c = dict(name=name, op="write", B=B, H_kv=H_kv, L=L, D_qk=D_qk, D_v=D_v, page=64, cache="fp8", order="blhd")
    c.update(kw)
    return c


def _attend(name, B, H_q, H_kv, n, L, D_qk, D_v, **kw):
    c = dict(name=name, op="attend", B=B, H_q=H_q, H_kv=H_kv, n=n, L=L, D_qk=D_qk, D_v=D_v, page=64, cache="bf16", prefix=0, ragged=0)
    c.update(kw)
    return c


def listed():
    return [
        # One new token of one sequence, grouped heads: the smallest call of a decoding loop, where latency is all.
        _rotary("rotary_token_1x32x8", 1, 32, 8, 1, 128, 128, start=7000),
        # Prompts of a batch in the order a fused projection leaves them, frequencies blended for a long context.
        _rotary("rotary_prompt_4x32x8x2048", 4, 32, 8, 2048, 128, 128, scaling="by_parts", factor=8.0, start=100000),
        # Gradients of a training step as the attention's backward pass hands them on (32 bits), neighbouring pairs, a third of the head rotated.
        _rotary("rotary_bwd_2x16x1023", 2, 16, 16, 1023, 192, 64, layout="interleaved", backward=True, dtype="f32", order="bhld"),
        # One new token of each of 64 sequences into an 8-bit cache.
        _write("write_fp8_64x8x1", 64, 8, 1, 128, 128),
        # Whole prompts into an 8-bit cache.
        _write("write_fp8_4x8x4096", 4, 8, 4096, 128, 128),
        # One token of one sequence over a short cache with small pages: latency.
        _attend("attend_1x32x8_777", 1, 32, 8, 1, 777, 128, 128, page=16),
        # A decoding batch of uneven lengths over an 8-bit cache.
        _attend("attend_fp8_32x32x8_5003", 32, 32, 8, 1, 5003, 128, 128, cache="fp8", ragged=1),
        # Four tokens at once (drafted tokens that are being verified), heads of their own keys, 192/128.
        _attend("attend_16x16x16_n4_2500", 16, 16, 16, 4, 2500, 192, 128, ragged=2),
        # Few sequences over a very long context.
        _attend("attend_4x64x8_131072", 4, 64, 8, 1, 131072, 128, 128),
        # A small batch behind a common instruction of odd length, small heads.
        _attend("prefix_8x12x12_1000", 8, 12, 12, 1, 150, 64, 64, prefix=1000, page=32, ragged=3),
        # A batch of requests behind a long common document.
        _attend("prefix_64x32x8_8192", 64, 32, 8, 1, 300, 128, 128, prefix=8192, ragged=4),
        # The largest: 256 requests, a very long common document, an 8-bit cache.
        _attend("prefix_fp8_256x64x8_32768", 256, 64, 8, 1, 1024, 128, 128, prefix=32768, cache="fp8", ragged=5),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm; a third of them round, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n >= 128 and rng.random() < 0.33:
        n = n // 64 * 64
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["rotary", "write", "attend", "attend", "prefix"])
    H_q, H_kv = rng.choice([(32, 8), (16, 16), (12, 12), (64, 8), (32, 32)])
    D_qk, D_v = rng.choice([(64, 64), (128, 128), (128, 128), (192, 128)])
    if op == "rotary":
        D, B, L = D_qk, _log_int(rng, 1, 64), _log_int(rng, 1, 8192)
        while B * L * (H_q + H_kv) * D > 4e8:
            L = max(1, L * 2 // 3)
        scaling = rng.choice(["none", "linear", "ntk", "by_parts"])
        c = _rotary("", B, H_q, H_kv, L, D, rng.choice([D, D, D // 2, 32]), layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]), start=rng.choice([0, 0, 5000, 1000000]),
                    backward=rng.random() < 0.4, dtype=rng.choice(["bf16", "bf16", "f32"]), order=rng.choice(["bhld", "blhd"]))
    elif op == "write":
        B, L = _log_int(rng, 1, 256), _log_int(rng, 1, 8192)
        while B * L * H_kv * (D_qk + D_v) > 1e8:
            L = max(1, L * 2 // 3)
        c = _write("", B, H_kv, L, D_qk, D_v, page=rng.choice([16, 32, 64, 128]), cache=rng.choice(["fp8", "fp8", "bf16"]),
                   order=rng.choice(["bhld", "blhd"]))
    else:
        prefix = _log_int(rng, 100, 32768) if op == "prefix" else 0
        B, n = _log_int(rng, 2 if prefix else 1, 256), rng.choice([1, 1, 1, 2, 3, 4, 8])
        L = max(n, _log_int(rng, 1, 1024 if prefix else 131072))
        while B * L * H_kv * (D_qk + D_v) > 8e8:
            L = max(n, L * 2 // 3)
        while B * n * H_q * prefix * (D_qk + D_v) > 1e11:
            prefix = prefix * 2 // 3
        c = _attend("", B, H_q, H_kv, n, L, D_qk, D_v, page=rng.choice([16, 32, 64, 128]), cache=rng.choice(["fp8", "bf16"]),
                    prefix=prefix, ragged=rng.randrange(0, 1000) if rng.random() < 0.8 else 0)
    del c["name"]
    return c


# ---- what follows from a case ---------------------------------------------------------------------------------------
def _lengths(c):
    """Cached tokens of each sequence, the newest ones among them: all L, or spread between a quarter and all of it."""
    if not c["ragged"]:
        return [c["L"]] * c["B"]
    rng = random.Random(c["ragged"])
    return [max(c["n"], rng.randint((c["L"] + 3) // 4, c["L"])) for _ in range(c["B"])]


def _frequencies(c):
    """Angle per position of each pair, and the factor on the rotated part.  Linear: positions shrink by the factor; ntk: the base grows so
    that the slowest pair shrinks by it; by_parts: pairs that turn less than once in 4096 positions shrink, those that turn 32 times or
    more stay, linear between, and the rotated part grows by 0.1 ln(factor) + 1."""
    half, base, s = c["rot"] // 2, 10000.0, c["factor"]
    if c["scaling"] == "ntk":
        base *= s ** (c["rot"] / (c["rot"] - 2))
    f = [base ** (-i / half) for i in range(half)]
    if c["scaling"] == "linear":
        return [x / s for x in f], 1.0
    if c["scaling"] == "by_parts":
        keep = [min(1.0, max(0.0, (4096 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
        return [x * k + x / s * (1 - k) for x, k in zip(f, keep)], 0.1 * math.log(s) + 1.0
    return f, 1.0


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _heads(g, order, B, H, L, D, dtype):
    """[B, H, L, D]: contiguous, or a view of [B, L, H, D]."""
    if order == "blhd":
        return _normal(g, B, L, H, D).to(dtype).transpose(1, 2)
    return _normal(g, B, H, L, D).to(dtype)


def _row_scale(x):
    """Biased exponent of the power of two of each row (last dimension), from the row's largest magnitude (inputs here are finite)."""
    m, e = torch.frexp(x.abs().amax(-1))
    return torch.where(m > 0, (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126), torch.full_like(e, -126)) + 127


def _two_to(e):
    """2^(e - 127) in 32 bits from biased exponents (1 to 254): the exponent's own bits, as a power function may be a unit off."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _quantised(x):
    e = _row_scale(x)
    return (x / _two_to(e).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.uint8)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "rotary":
        dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        f, amp = _frequencies(c)
        pos = torch.arange(c["L"], device="cuda").repeat(c["B"], 1) + c["start"]
        pos = pos + torch.randint(0, 1000, (c["B"], 1), generator=g, device="cuda")  # every sequence is somewhere else
        q, k = (_heads(g, c["order"], c["B"], h, c["L"], c["D"], dtype) for h in (c["H_q"], c["H_kv"]))
        return dict(case=c, q=q, k=k, pos=pos.to(torch.int32), f=f, amp=amp, f64=torch.tensor(f, dtype=torch.float64, device="cuda"))
    page = c["page"]
    if c["op"] == "write":
        pages_each = -(-c["L"] // page)
        n_pages = c["B"] * pages_each + 3
        own_pages = torch.randperm(n_pages, generator=g, device="cuda")[: c["B"] * pages_each].view(c["B"], pages_each)
        at = torch.arange(c["L"], device="cuda")
        slots = (own_pages[:, at // page] * page + at % page).to(torch.int32)
        k, v = (_heads(g, c["order"], c["B"], c["H_kv"], c["L"], d, torch.bfloat16) for d in (c["D_qk"], c["D_v"]))
        s = dict(case=c, k=k, v=v, slots=slots)
    else:
        lens = _lengths(c)
        width, own_width = -(-c["prefix"] // page), -(-max(lens) // page)
        n_pages = width + c["B"] * own_width + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        s = dict(case=c, prefix_table=order[:width].contiguous(), table=order[width:width + c["B"] * own_width].view(c["B"], own_width).contiguous(),
                 lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                 q=_heads(g, "blhd", c["B"], c["H_q"], c["n"], c["D_qk"], torch.bfloat16), scale=c["D_qk"] ** -0.5)
    for name, d in (("kc", c["D_qk"]), ("vc", c["D_v"])):
        if c["op"] == "write":
            x = torch.zeros(n_pages, c["H_kv"], page, d, device="cuda")
        else:
            x = _normal(g, n_pages, c["H_kv"], page, d).to(torch.bfloat16)
        if c["cache"] == "bf16":
            s[name] = x.to(torch.bfloat16)
        else:
            s[name], s[name + "_e"] = _quantised(x.float())
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------
def _plain_rotary(s, x):
    c, half = s["case"], s["case"]["rot"] // 2
    a = s["pos"].to(torch.float64).unsqueeze(-1) * s["f64"]  # angles of far positions: 64 bits
    cos, sin = ((t(a) * s["amp"]).to(torch.float32).unsqueeze(1) for t in (torch.cos, torch.sin))
    if c["backward"]:
        sin = -sin
    r, rest = x[..., : 2 * half].to(torch.float32), x[..., 2 * half:]
    x1, x2 = (r[..., :half], r[..., half:]) if c["layout"] == "half" else (r[..., 0::2], r[..., 1::2])
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.cat((y1, y2), -1) if c["layout"] == "half" else torch.stack((y1, y2), -1).flatten(-2)
    return torch.cat((y.to(x.dtype), rest), -1)


def _plain_written(s, x, name):
    """Writes x's rows at their slots, and reads them back."""
    c, n = s["case"], s["slots"].numel()
    rows = x.transpose(1, 2).reshape(n, c["H_kv"], -1)
    page, place = s["slots"].view(-1) // c["page"], s["slots"].view(-1) % c["page"]
    if c["cache"] == "bf16":
        s[name][page, :, place] = rows
        y = s[name][page, :, place]
    else:
        q, e = _quantised(rows.to(torch.float32))
        s[name].view(torch.uint8)[page, :, place] = q.view(torch.uint8)
        s[name + "_e"][page, :, place] = e
        back = s[name].view(torch.uint8)[page, :, place].view(torch.float8_e4m3fn)
        y = (back.to(torch.float32) * _two_to(s[name + "_e"][page, :, place]).unsqueeze(-1)).to(torch.bfloat16)
    return y.view(c["B"], c["L"], c["H_kv"], -1).transpose(1, 2)


def _plain_pages(s, name, table):
    """The pages of a table [..., width] as rows [..., H_kv, width * page, D] in 32 bits."""
    t = table.long()
    x = s[name][t] if s["case"]["cache"] == "bf16" else s[name].view(torch.uint8)[t].view(torch.float8_e4m3fn)
    x = x.to(torch.float32)
    if s["case"]["cache"] != "bf16":
        x = x * _two_to(s[name + "_e"][t]).unsqueeze(-1)
    return x.transpose(-4, -3).flatten(-3, -2)


def _plain_attend(s):
    c = s["case"]
    B, n, H_kv, g = c["B"], c["n"], c["H_kv"], c["H_q"] // c["H_kv"]
    q = s["q"].to(torch.float32).reshape(B, H_kv, g * n, c["D_qk"])  # rows: (head of the group, token)
    k, v = _plain_pages(s, "kc", s["table"]), _plain_pages(s, "vc", s["table"])
    x = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    seen = s["lengths"].view(B, 1) - n + 1 + torch.arange(n, device="cuda")  # keys that token t of a sequence sees
    seen = seen.repeat(1, g).view(B, 1, g * n, 1)
    x = torch.where(torch.arange(x.shape[-1], device="cuda") < seen, x, -math.inf)
    if c["prefix"]:
        pk, pv = (_plain_pages(s, m, s["prefix_table"])[:, : c["prefix"]] for m in ("kc", "vc"))
        rows = q.transpose(0, 1).reshape(H_kv, B * g * n, -1)  # the prefix is read once for all sequences
        px = torch.matmul(rows, pk.transpose(-1, -2)) * s["scale"]
        x = torch.cat((px.view(H_kv, B, g * n, -1).transpose(0, 1), x), -1)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w[..., c["prefix"]:], v)
    if c["prefix"]:
        pw = w[..., : c["prefix"]].transpose(0, 1).reshape(H_kv, B * g * n, -1)
        o = o + torch.matmul(pw, pv).view(H_kv, B, g * n, -1).transpose(0, 1)
    return (o / total).to(torch.bfloat16).view(B, c["H_q"], n, -1), (top + torch.log(total)).view(B, c["H_q"], n)


# ---- the package's calls ------------------------------------------------------------------------------------------------
def _own_rotary(s):
    from paper_2502_15349_amd import ae_attn as A

    c = s["case"]
    if "plan" not in s:  # a program keeps the handle of its step, and the step's output buffers
        s["out"] = [torch.empty_like(x) for x in (s["q"], s["k"])]
        s["plan"] = A.RotaryPlan(s["q"], s["k"], s["pos"], *s["out"], freqs=s["f"], amplitude=s["amp"], layout=c["layout"])
    step = s["plan"].backward if c["backward"] else s["plan"].forward
    step(s["q"], s["k"], s["pos"], *s["out"])
    return s["out"]


def _own_cache(s):
    from paper_2502_15349_amd import ae_attn as A

    if "cache" not in s:
        s["cache"] = A.PagedCache(s["kc"], s["vc"], s.get("kc_e"), s.get("vc_e"))
    return s["cache"]


def _own_write(s):
    cache = _own_cache(s)
    cache.append(s["k"], s["v"], s["slots"])
    return cache.read(s["slots"])


def _own_attend(s):
    from paper_2502_15349_amd import ae_attn as A

    c = s["case"]
    if "plan" not in s:
        s["out"] = torch.empty(c["B"], c["H_q"], c["n"], c["D_v"], dtype=torch.bfloat16, device="cuda")
        s["stats"] = torch.empty(c["B"], c["H_q"], c["n"], device="cuda")
        s["plan"] = A.CachedAttentionPlan(_own_cache(s), s["q"], s["out"], max_length=max(_lengths(c)), table_width=s["table"].shape[1],
                                          prefix_length=c["prefix"], scale=s["scale"])
    s["plan"].forward(s["q"], s["table"], s["lengths"], s["out"], stats=s["stats"], prefix_table=s["prefix_table"] if c["prefix"] else None)
    return s["out"], s["stats"]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"rotary": _own_rotary, "write": _own_write, "attend": _own_attend}[op](state)
    if op == "rotary":
        return [_plain_rotary(state, x) for x in (state["q"], state["k"])]
    if op == "write":
        return [_plain_written(state, state[x], x + "c") for x in ("k", "v")]
    return _plain_attend(state)


# ---- the work of a pass ----------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "rotary":
        n = c["B"] * c["L"] * (c["H_q"] + c["H_kv"])
        return {"bytes": 2 * n * c["D"] * (4 if c["dtype"] == "f32" else 2) + 4 * c["B"] * c["L"], "flops": 3 * n * c["rot"]}
    size, extra = (2, 0) if c["cache"] == "bf16" else (1, 2)
    row = (c["D_qk"] + c["D_v"]) * size + extra  # a cached key and value of one head
    if c["op"] == "write":
        n = c["B"] * c["L"] * c["H_kv"]
        return {"bytes": n * (2 * 2 * (c["D_qk"] + c["D_v"]) + 2 * row) + 8 * c["B"] * c["L"], "flops": 3 * n * (c["D_qk"] + c["D_v"])}
    lens, n, D = _lengths(c), c["n"], c["D_qk"] + c["D_v"]
    seen = sum(n * x - n * (n - 1) // 2 for x in lens) + c["B"] * n * c["prefix"]
    return {"bytes": (sum(lens) + c["prefix"]) * c["H_kv"] * row + c["B"] * c["H_q"] * n * (2 * D + 4), "flops": 2 * seen * c["H_q"] * D}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------
def _exact_rotary(s, x):
    """Pairs as complex numbers, times amplitude * e^(i angle)."""
    c, half = s["case"], s["case"]["rot"] // 2
    turn = torch.polar(torch.full((), s["amp"], dtype=torch.float64, device="cuda"), s["pos"].double()[:, None, :, None] * s["f64"])
    if c["backward"]:
        turn = turn.conj()
    y = x.double().clone()
    first, second = (slice(0, half), slice(half, 2 * half)) if c["layout"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _pow2(k):
    """2^k in 64 bits, from the exponent's bits."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_written(x, cache):
    """The nearest e4m3 value (3 bits behind the leading one, exponents from -6, ties to even) on the row's power of two."""
    x = x.double()
    if cache == "bf16":
        return x
    top = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448.0)).clamp(min=-126)
    k = torch.where(top <= 448.0 * _pow2(k - 1), k - 1, k).clamp(min=-126)  # (the logarithm may have been rounded up)
    y = x * _pow2(-k)
    step = _pow2(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step * _pow2(k)


def _exact_row(s, name, table):
    """Keys or values of one page list, [H_kv, tokens, D], in 64 bits."""
    t = table.long()
    x = s[name].view(torch.uint8 if s["case"]["cache"] != "bf16" else torch.bfloat16)
    if s["case"]["cache"] == "bf16":
        y = x.index_select(0, t).double()
    else:
        y = x.index_select(0, t).view(torch.float8_e4m3fn).float().double()
        y = y * _pow2(s[name + "_e"].index_select(0, t).long() - 127).unsqueeze(-1)
    return y.permute(1, 0, 2, 3).reshape(y.shape[1], -1, y.shape[3])


def _exact_attend(s):
    """Sequence by sequence, head by head of the keys: softmax over the prefix's keys and those of the sequence that a token sees."""
    c = s["case"]
    n, g, lens = c["n"], c["H_q"] // c["H_kv"], _lengths(c)
    out = torch.zeros(c["B"], c["H_q"], n, c["D_v"], dtype=torch.float64, device="cuda")
    stats = torch.zeros(c["B"], c["H_q"], n, dtype=torch.float64, device="cuda")
    pk, pv = (_exact_row(s, m, s["prefix_table"])[:, : c["prefix"]] for m in ("kc", "vc")) if c["prefix"] else (None, None)
    for b in range(c["B"]):
        k, v = (_exact_row(s, m, s["table"][b])[:, : lens[b]] for m in ("kc", "vc"))
        if c["prefix"]:
            k, v = torch.cat((pk, k), 1), torch.cat((pv, v), 1)
        for t in range(n):
            end = k.shape[1] - n + 1 + t
            q = s["q"][b, :, t].double().view(c["H_kv"], g, -1)
            x = (k[:, :end] @ q.transpose(1, 2)) * s["scale"]  # [H_kv, keys, g]
            lse = torch.logsumexp(x, 1)
            stats[b, :, t] = lse.flatten()
            out[b, :, t] = (torch.exp(x - lse.unsqueeze(1)).transpose(1, 2) @ v[:, :end]).flatten(0, 1)
    return out, stats


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return [_exact_rotary(s, x) for x in (s["q"], s["k"])]
    if case["op"] == "write":
        return [_exact_written(s[x], case["cache"]) for x in ("k", "v")]
    return _exact_attend(s)
