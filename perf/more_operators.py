"""Attention over spans of keys, forward and backward, its scores optionally capped by a tanh or biased by distance; the same scores over the
paged cache; and the eviction of cached tokens by the attention that they have received, as they are timed.

Each comes in a plain form (elementary torch operations in 32 bits) and, where `own` is true, as the package's own call.  Sizes are
those of the package's own benchmark and tests (32/8, 16/16, 12/12 and 64/8 heads, head dims 64/64, 128/128 and 192/128) or generic ones of the
same ranges.

Span attention: row i of batch entry b sees the keys begin[b, i] <= j < end[b, i]; documents packed behind each other, prefixes that are
seen both ways, windows and the causal mask are such spans.  With s = scale q k, a score is cap tanh(s / cap) where there is a cap, less
slope_h |i + L_k - L_q - j| where there are slopes; then softmax over the span.

Eviction: every cached entry of a k/v head carries a weight, the sum of the probabilities that the queries so far gave it, and the
position of its token.  An eviction keeps the entries of the newest positions and of the first ones, and of the others those with the most
weight (equal ones: the first of the list), `keep` in all; kept entries beyond place `keep` move, in their order, to the places below it
that have become free.

Layouts: Q [B, H_q, L, D_qk], K and V [B, H_kv, L, D]; cache pages [n_pages, H_kv, page, D] with, in 8 bits, a power of two per cached row of
a head as its biased exponent; weights and positions [B, H_kv, capacity].
"""
import math
import random

import torch

own = False


# ---- the cases ----------------------------------------------------------------------------------------------------
def _span(name, op, B, H_q, H_kv, L, D_qk, D_v, mask, **kw):
    c = dict(name=name, op=op, B=B, H_q=H_q, H_kv=H_kv, L_q=L, L=L, D_qk=D_qk, D_v=D_v, mask=mask, window=0, docs=0, cap=0.0, slopes=False)
    c.update(kw)
    return c


def _cached(name, op, B, H_q, H_kv, n, L, D_qk, D_v, **kw):
    c = dict(name=name, op=op, B=B, H_q=H_q, H_kv=H_kv, n=n, L=L, D_qk=D_qk, D_v=D_v, page=64, cache="bf16", ragged=0, cap=0.0)
    c.update(kw)
    return c


def _evict(name, B, H_kv, L, keep, D_qk, D_v, **kw):
    c = dict(name=name, op="evict", B=B, H_kv=H_kv, L=L, keep=keep, recent=keep // 4, sinks=4, D_qk=D_qk, D_v=D_v, page=64, cache="bf16", ragged=0)
    c.update(kw)
    return c


def listed():
    return [
        # A short causal prompt with capped scores: the smallest call, where latency is all.
        _span("fwd_cap_1x12x12_100", "forward", 1, 12, 12, 100, 64, 64, "causal", cap=30.0),
        # A long row of packed documents with some padding behind the last one.
        _span("fwd_docs_1x32x8_8192", "forward", 1, 32, 8, 8192, 128, 128, "docs", docs=11),
        # Heads of their own keys, biased by distance, in a window, of odd length.
        _span("fwd_slopes_2x16x16_2500", "forward", 2, 16, 16, 2500, 192, 128, "window", window=1000, slopes=True),
        # Gradients behind prefixes that are seen both ways, small heads, odd length.
        _span("bwd_prefix_2x12x12_1023", "backward", 2, 12, 12, 1023, 64, 64, "prefix", docs=12, slopes=True),
        # Gradients of a training step, capped scores, grouped heads.
        _span("bwd_cap_2x32x8_4096", "backward", 2, 32, 8, 4096, 128, 128, "causal", cap=50.0),
        # Gradients of packed documents, heads of 192/128.
        _span("bwd_docs_1x16x16_4000", "backward", 1, 16, 16, 4000, 192, 128, "docs", docs=13),
        # One token of one sequence over a short cache with small pages, capped scores: latency.
        _cached("cached_cap_1x32x8_777", "cached", 1, 32, 8, 1, 777, 128, 128, page=16, cap=50.0, slopes=False),
        # A decoding batch of uneven lengths over an 8-bit cache, scores biased by distance.
        _cached("cached_slopes_fp8_32x32x8_5003", "cached", 32, 32, 8, 1, 5003, 128, 128, cache="fp8", ragged=1, slopes=True),
        # The weights of a decoding batch after one more token.
        _cached("weigh_16x32x8_2048", "weigh", 16, 32, 8, 1, 2048, 128, 128, ragged=2),
        # The weights of a prompt's piece of 500 tokens, 8-bit cache, capped scores.
        _cached("weigh_cap_fp8_4x16x16_n500_8000", "weigh", 4, 16, 16, 500, 8000, 128, 128, cache="fp8", cap=50.0),
        # A decoding batch that has grown a little over its room.
        _evict("evict_16x8_1100_to_1024", 16, 8, 1100, 1024, 128, 128),
        # Long prompts cut down to an eighth, 8-bit cache.
        _evict("evict_fp8_8x8_16384_to_2048", 8, 8, 16384, 2048, 128, 128, cache="fp8"),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm; a third of them round, the others as they fall."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n >= 128 and rng.random() < 0.33:
        n = n // 64 * 64
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "cached", "weigh", "evict"])
    H_q, H_kv = rng.choice([(32, 8), (16, 16), (12, 12), (64, 8), (32, 32)])
    D_qk, D_v = rng.choice([(64, 64), (128, 128), (128, 128), (192, 128)])
    cap, slopes = rng.choice([(0.0, False), (0.0, False), (30.0, False), (50.0, False), (0.0, True), (50.0, True)])
    cache, page = rng.choice(["fp8", "bf16"]), rng.choice([16, 32, 64, 128])
    if op in ("forward", "backward"):
        B, L = _log_int(rng, 1, 16), _log_int(rng, 1, 8192)
        while B * H_q * L * L > (2.1e9 if op == "forward" else 1.0e9):
            L = max(1, L * 2 // 3)
        mask = rng.choice(["none", "causal", "window", "docs", "docs", "docs_both", "prefix"])
        c = _span("", op, B, H_q, H_kv, L, D_qk, D_v, mask, cap=cap, slopes=slopes)
        if mask == "window":
            c["window"] = _log_int(rng, 1, L)
        if mask in ("docs", "docs_both", "prefix"):
            c["docs"] = rng.randrange(1, 1000)
        elif rng.random() < 0.3:
            c["L_q"] = _log_int(rng, 1, L)
    elif op == "evict":
        B, L = _log_int(rng, 1, 64), _log_int(rng, 2, 32768)
        while B * L * H_kv * (D_qk + D_v) > 3e8:
            L = max(2, L * 2 // 3)
        keep = _log_int(rng, max(1, L // 16), L)
        sinks = min(rng.choice([0, 1, 4]), keep)
        c = _evict("", B, H_kv, L, keep, D_qk, D_v, recent=rng.randint(0, keep - sinks), sinks=sinks, page=page, cache=cache,
                   ragged=rng.randrange(0, 1000) if rng.random() < 0.7 else 0)
    else:
        B, n = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 8])
        if op == "weigh" and rng.random() < 0.3:
            n = _log_int(rng, 16, 500)
        L = max(n, _log_int(rng, 1, 65536))
        while B * L * H_kv * (D_qk + D_v) > 5e8 or B * n * H_q * L > 2.6e8:
            L = max(n, L * 2 // 3)
            if L == n:
                B = max(1, B // 2)
        c = _cached("", op, B, H_q, H_kv, n, L, D_qk, D_v, page=page, cache=cache, cap=cap, ragged=rng.randrange(0, 1000) if rng.random() < 0.8 else 0)
        if op == "cached":
            c["slopes"] = slopes
    del c["name"]
    return c


# ---- what follows from a case ---------------------------------------------------------------------------------------
def _lengths(c):
    """Cached entries of each sequence: all L, or spread between a quarter and all of it (the newest tokens among them)."""
    if not c["ragged"]:
        return [c["L"]] * c["B"]
    rng, least = random.Random(c["ragged"]), c.get("n", 1)
    return [max(least, rng.randint((c["L"] + 3) // 4, c["L"])) for _ in range(c["B"])]


def _documents(c):
    """For each batch entry its documents as (first token, first behind, tokens of the prefix); what lies behind the last one is padding."""
    rows = []
    for b in range(c["B"]):
        rng = random.Random(c["docs"] * 1000 + b)
        used, at, docs = c["L"] - (rng.randint(0, c["L"] // 20) if c["L"] > 1 else 0), 0, []
        while at < used:
            n = min(used - at, max(1, int(math.exp(rng.uniform(math.log(max(1, c["L"] // 16)), math.log(max(1, c["L"])))))))
            docs.append((at, at + n, rng.randint(0, n) if c["mask"] == "prefix" else 0))
            at += n
        rows.append(docs)
    return rows


def _spans(c):
    """First visible key and the first behind the last one, of every query row: two lists of B lists of L_q."""
    L_q, L, off = c["L_q"], c["L"], c["L"] - c["L_q"]
    if c["mask"] == "none":
        return [[0] * L_q] * c["B"], [[L] * L_q] * c["B"]
    if c["mask"] in ("causal", "window"):
        w = c["window"] or L + L_q
        return [[max(0, i + off - w + 1) for i in range(L_q)]] * c["B"], [[i + off + 1 for i in range(L_q)]] * c["B"]
    begin, end = [[0] * L for _ in range(c["B"])], [[0] * L for _ in range(c["B"])]
    for b, docs in enumerate(_documents(c)):
        for first, behind, prefix in docs:
            for i in range(first, behind):
                begin[b][i] = first
                end[b][i] = behind if c["mask"] == "docs_both" else max(i + 1, first + prefix)
    return begin, end


def _slopes(H):
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(g, B, H, L, D, by=1.0):
    """[B, H, L, D] as a view of [B, L, H, D], the order that a projection leaves."""
    return (_normal(g, B, L, H, D) * by).to(torch.bfloat16).transpose(1, 2)


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


def _prepare_span(c, g):
    # (queries of three times unit deviation: scores that a cap of 30 or 50 bends)
    s = dict(case=c, q=_rows(g, c["B"], c["H_q"], c["L_q"], c["D_qk"], 3.0), k=_rows(g, c["B"], c["H_kv"], c["L"], c["D_qk"]),
             v=_rows(g, c["B"], c["H_kv"], c["L"], c["D_v"]), scale=c["D_qk"] ** -0.5)
    s["begin"], s["end"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in _spans(c))
    if c["slopes"]:
        s["slopes"] = torch.tensor(_slopes(c["H_q"]), device="cuda")
    if c["op"] == "backward":
        s["do"] = _rows(g, c["B"], c["H_q"], c["L_q"], c["D_v"])
        s["o"], s["stats"] = _plain_forward(s)  # (in 32 bits: next to nothing but rounding is left of dP - delta in short documents)
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] in ("forward", "backward"):
        return _prepare_span(c, g)
    page, lens = c["page"], _lengths(c)
    width = -(-max(lens) // page)
    n_pages, room = c["B"] * width + 3, width * page
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    s = dict(case=c, table=order[: c["B"] * width].view(c["B"], width).contiguous(), lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for name, d in (("kc", c["D_qk"]), ("vc", c["D_v"])):
        x = _normal(g, n_pages, c["H_kv"], page, d).to(torch.bfloat16)
        if c["cache"] == "bf16":
            s[name] = x
        else:
            s[name], s[name + "_e"] = _quantised(x.float())
    if c["op"] != "cached":
        # weights of earlier queries, a third of them on coarse steps, so that there are equal ones; tokens in the order that evictions left
        w = torch.rand(c["B"], c["H_kv"], room, generator=g, device="cuda") ** 4 * 8
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.33, torch.round(w * 16) / 16, w)
        at = torch.randint(1, 4, w.shape, generator=g, device="cuda").cumsum(-1)
        mixed = torch.rand(w.shape, generator=g, device="cuda") + (torch.arange(room, device="cuda") >= max(lens) // 2)
        s["positions"] = at.gather(-1, mixed.argsort(-1)).to(torch.int32)
    if c["op"] == "evict":
        s["weights_out"], s["positions_out"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
        s["lengths_out"] = torch.zeros_like(s["lengths"])
        kept = torch.arange(c["keep"], device="cuda")
        slots = s["table"].long()[:, (kept // page).clamp(max=width - 1)] * page + kept % page
        s["slots"] = torch.where(kept < s["lengths"].unsqueeze(1), slots, -1).to(torch.int32)
        return s
    s["q"], s["scale"] = _rows(g, c["B"], c["H_q"], c["n"], c["D_qk"], 2.0), c["D_qk"] ** -0.5
    if c.get("slopes"):
        s["slopes"] = torch.tensor(_slopes(c["H_q"]), device="cuda")
    if c["op"] == "weigh":
        s["weights_out"] = torch.zeros_like(s["weights"])
        s["new_positions"] = (3 * s["lengths"].view(-1, 1) + torch.arange(c["n"], device="cuda")).to(torch.int32)
        x = _plain_cached_scores(s)
        s["stats"] = torch.logsumexp(x, -1).view(c["B"], c["H_q"], c["n"])
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------
def _grouped(x, H_kv):
    """[B, H_q, L, D] as [B, H_kv, g L, D] in 32 bits: the rows of the heads that share a k/v head behind each other."""
    return x.to(torch.float32).reshape(x.shape[0], H_kv, -1, x.shape[3])


def _plain_scores(s, q, k):
    """Modified scores [B, H_kv, g, L_q, L] with -inf where a key is hidden, and the derivative of the cap (None without one)."""
    c = s["case"]
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).view(c["B"], c["H_kv"], -1, c["L_q"], c["L"])
    bend = None
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = c["cap"] * t
        bend = 1 - t * t if c["op"] == "backward" else None
    i, j = torch.arange(c["L_q"], device="cuda").unsqueeze(1) + (c["L"] - c["L_q"]), torch.arange(c["L"], device="cuda")
    if c["slopes"]:
        x = x - s["slopes"].view(1, c["H_kv"], -1, 1, 1) * (i - j).abs().to(torch.float32)
    seen = (j >= s["begin"].unsqueeze(-1)) & (j < s["end"].unsqueeze(-1))
    return torch.where(seen.view(-1, 1, 1, c["L_q"], c["L"]), x, -math.inf), bend


def _plain_forward(s):
    c = s["case"]
    x, _ = _plain_scores(dict(s, case=dict(c, op="forward")), _grouped(s["q"], c["H_kv"]), s["k"].to(torch.float32))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.flatten(2, 3), s["v"].to(torch.float32)).view(total.shape[:-1] + (-1,))
    o = o / torch.where(total == 0, 1.0, total)
    return o.flatten(1, 2), (top + torch.log(total)).view(c["B"], c["H_q"], c["L_q"])


def _plain_rounded(s):
    o, stats = _plain_forward(s)
    return o.to(torch.bfloat16), stats


def _plain_backward(s):
    c = s["case"]
    q, k, v = _grouped(s["q"], c["H_kv"]), s["k"].to(torch.float32), s["v"].to(torch.float32)
    do = _grouped(s["do"], c["H_kv"])
    x, bend = _plain_scores(s, q, k)
    lse = s["stats"].view(c["B"], c["H_kv"], -1, c["L_q"], 1)
    w = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)).flatten(2, 3)
    del x
    dv = torch.matmul(w.transpose(-1, -2), do)
    delta = (_grouped(s["o"], c["H_kv"]) * do).sum(-1, keepdim=True)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_(delta).mul_(w).mul_(s["scale"])
    if bend is not None:
        ds = ds.mul_(bend.flatten(2, 3))
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    return [dq.view(c["B"], c["H_q"], c["L_q"], -1).to(torch.bfloat16), dk.to(torch.bfloat16), dv.to(torch.bfloat16)]


def _plain_pages(s, name):
    """The cached rows [B, H_kv, width * page, D] of the sequences in 32 bits."""
    t = s["table"].long()
    x = s[name][t] if s["case"]["cache"] == "bf16" else s[name].view(torch.uint8)[t].view(torch.float8_e4m3fn)
    x = x.to(torch.float32)
    if s["case"]["cache"] != "bf16":
        x = x * _two_to(s[name + "_e"][t]).unsqueeze(-1)
    return x.transpose(-4, -3).flatten(-3, -2)


def _plain_cached_scores(s):
    """Modified scores [B, H_kv, g n, keys] of the newest tokens, -inf where a key is hidden."""
    c = s["case"]
    n, g = c["n"], c["H_q"] // c["H_kv"]
    x = torch.matmul(_grouped(s["q"], c["H_kv"]), _plain_pages(s, "kc").transpose(-1, -2)) * s["scale"]
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    at = s["lengths"].view(-1, 1) - n + torch.arange(n, device="cuda")  # the tokens' own places
    at = at.repeat(1, g).view(c["B"], 1, g * n, 1)
    j = torch.arange(x.shape[-1], device="cuda")
    if c.get("slopes"):
        x = x - s["slopes"].view(1, c["H_kv"], g, 1).expand(-1, -1, -1, n).reshape(1, c["H_kv"], g * n, 1) * (at - j).to(torch.float32)
    return torch.where(j <= at, x, -math.inf)


def _plain_cached(s):
    c = s["case"]
    x = _plain_cached_scores(s)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w, _plain_pages(s, "vc")) / total
    return o.to(torch.bfloat16).view(c["B"], c["H_q"], c["n"], -1), (top + torch.log(total)).view(c["B"], c["H_q"], c["n"])


def _plain_weigh(s):
    c = s["case"]
    got = torch.exp(_plain_cached_scores(s) - s["stats"].view(c["B"], c["H_kv"], -1, 1)).sum(2)  # [B, H_kv, keys]
    j, first_new = torch.arange(got.shape[-1], device="cuda"), (s["lengths"] - c["n"]).view(-1, 1, 1)
    there = j < s["lengths"].view(-1, 1, 1)
    new = there & (j >= first_new)
    s["weights_out"] = torch.where(there, got + torch.where(new, 0.0, s["weights"]), s["weights_out"])
    p = s["new_positions"].gather(1, (j - first_new.view(-1, 1)).clamp(0, c["n"] - 1)).unsqueeze(1)
    s["positions"] = torch.where(new, p, s["positions"])
    return s["weights_out"], s["positions"]


def _plain_moves(s):
    """Which entries stay: for every place below `keep` the entry that it will hold, [B, H_kv, min(keep, room)]; and how many are kept."""
    c = s["case"]
    keep, L = c["keep"], s["weights"].shape[-1]
    j, lens = torch.arange(L, device="cuda"), s["lengths"].view(-1, 1, 1)
    there, p = j < lens, s["positions"]
    newest = torch.where(there, p, -1).amax(-1, keepdim=True)
    rank = torch.where((p > newest - c["recent"]) | (p < c["sinks"]), math.inf, s["weights"])
    order = torch.sort(torch.where(there, rank, -1.0), dim=-1, descending=True, stable=True).indices  # (weights are at least 0)
    count = lens.clamp(max=keep)
    stays = torch.zeros(order.shape, dtype=torch.bool, device="cuda").scatter_(-1, order, (j < count).expand(order.shape))
    free = torch.sort((~stays & (j < count)).to(torch.int32), dim=-1, descending=True, stable=True).indices  # free places first, in order
    moved = torch.sort((stays & (j >= count)).to(torch.int32), dim=-1, descending=True, stable=True).indices
    m = (stays & (j >= count)).sum(-1, keepdim=True)
    source = j.expand(order.shape).scatter(-1, free, torch.where(j < m, moved, free))
    return source[..., :keep], count


def _plain_evict(s):
    c = s["case"]
    source, count = _plain_moves(s)
    room, page = source.shape[-1], c["page"]
    at = torch.arange(room, device="cuda")
    here = at < count
    b = torch.arange(c["B"], device="cuda").view(-1, 1, 1)
    h = torch.arange(c["H_kv"], device="cuda").view(1, -1, 1)
    for name, full in (("weights", "weights_out"), ("positions", "positions_out")):
        s[full][..., :room] = torch.where(here, s[name].gather(-1, source), s[full][..., :room])
    s["lengths_out"] = count.view(-1).to(torch.int32)
    to, source = at.expand(source.shape), torch.where(here, source, at)
    page_of = s["table"].long()
    for name in ("kc", "vc", "kc_e", "vc_e"):
        if name in s:
            x = s[name].view(torch.uint8) if c["cache"] != "bf16" else s[name]
            x[page_of[b, to // page], h, to % page] = x[page_of[b, source // page], h, source % page]
    return [s["weights_out"], s["positions_out"], s["lengths_out"], *_plain_kept(s)]


def _plain_kept(s):
    """The pages, or, in 8 bits, the kept rows as the values they stand for, [B, H_kv, keep, D]."""
    c = s["case"]
    if c["cache"] == "bf16":
        return [s["kc"], s["vc"]]
    got = []
    for name in ("kc", "vc"):
        at = s["slots"].long().clamp(min=0)
        x = s[name].view(torch.uint8)[at // c["page"], :, at % c["page"]].view(torch.float8_e4m3fn).to(torch.float32)
        x = x * _two_to(s[name + "_e"][at // c["page"], :, at % c["page"]]).unsqueeze(-1)
        got.append(torch.where((s["slots"] >= 0).view(c["B"], -1, 1, 1), x, 0.0).to(torch.bfloat16).transpose(1, 2))
    return got


# ---- the package's calls ------------------------------------------------------------------------------------------------
def _own_span(s):
    from paper_2502_15349_amd import ae_attn as A

    c = s["case"]
    backward = c["op"] == "backward"
    if "plan" not in s:  # a program keeps the plan of its layers, and the output buffers
        if not backward:
            s["o"] = torch.empty(c["B"], c["L_q"], c["H_q"], c["D_v"], dtype=torch.bfloat16, device="cuda").transpose(1, 2)
            s["stats"] = torch.empty(c["B"], c["H_q"], c["L_q"], device="cuda")
        else:
            s["grads"] = [torch.empty(x.shape, dtype=torch.bfloat16, device="cuda") for x in (s["q"], s["k"], s["v"])]
        mask = {"none": "none", "causal": "causal", "window": "sliding_window"}.get(c["mask"], "spans")
        s["plan"] = A.SpanAttentionPlan(s["q"], s["k"], s["v"], s["o"], scale=s["scale"], cap=c["cap"], slopes=_slopes(c["H_q"]) if c["slopes"] else None,
                                        mask=mask, window=c["window"])
        s["spans"] = (s["begin"], s["end"]) if mask == "spans" else None
    if not backward:
        s["plan"].forward(s["q"], s["k"], s["v"], s["o"], stats=s["stats"], spans=s["spans"])
        return s["o"], s["stats"]
    s["plan"].backward(s["q"], s["k"], s["v"], s["o"], s["do"], s["stats"], *s["grads"], spans=s["spans"])
    return s["grads"]


def _own_cache(s):
    from paper_2502_15349_amd import ae_attn as A

    if "cache" not in s:
        s["cache"] = A.PagedCache(s["kc"], s["vc"], s.get("kc_e"), s.get("vc_e"))
    return s["cache"]


def _own_cached(s):
    from paper_2502_15349_amd import ae_attn as A

    c = s["case"]
    if "plan" not in s:
        s["out"] = torch.empty(c["B"], c["H_q"], c["n"], c["D_v"], dtype=torch.bfloat16, device="cuda")
        s["stats"] = torch.empty(c["B"], c["H_q"], c["n"], device="cuda")
        s["plan"] = A.CachedAttentionPlan(_own_cache(s), s["q"], s["out"], max_length=max(_lengths(c)), table_width=s["table"].shape[1],
                                          scale=s["scale"], cap=c["cap"], slopes=_slopes(c["H_q"]) if c["slopes"] else None)
    s["plan"].forward(s["q"], s["table"], s["lengths"], s["out"], stats=s["stats"])
    return s["out"], s["stats"]


def _own_weigh(s):
    from paper_2502_15349_amd import ae_attn as A

    c = s["case"]
    if "plan" not in s:
        s["plan"] = A.CacheWeightsPlan(_own_cache(s), s["q"], s["weights"], max_length=max(_lengths(c)), table_width=s["table"].shape[1],
                                       scale=s["scale"], cap=c["cap"])
    s["plan"].forward(s["q"], s["table"], s["lengths"], s["stats"], s["weights"], s["positions"], s["new_positions"], out=s["weights_out"])
    return s["weights_out"], s["positions"]


def _own_evict(s):
    from paper_2502_15349_amd import ae_attn as A

    c, cache = s["case"], _own_cache(s)
    if "plan" not in s:
        s["plan"] = A.CacheEvictionPlan(cache, s["weights"], keep=c["keep"], recent=c["recent"], sinks=c["sinks"], max_length=max(_lengths(c)),
                                        table_width=s["table"].shape[1])
    s["plan"].forward(s["table"], s["lengths"], s["weights"], s["positions"], s["lengths_out"], weights_out=s["weights_out"],
                      positions_out=s["positions_out"])
    kept = [s["kc"], s["vc"]] if c["cache"] == "bf16" else cache.read(s["slots"])
    return [s["weights_out"], s["positions_out"], s["lengths_out"], *kept]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"forward": _own_span, "backward": _own_span, "cached": _own_cached, "weigh": _own_weigh, "evict": _own_evict}[op](state)
    return {"forward": _plain_rounded, "backward": _plain_backward, "cached": _plain_cached, "weigh": _plain_weigh, "evict": _plain_evict}[op](state)


# ---- the work of a pass ----------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] in ("forward", "backward"):
        begin, end = _spans(c)
        seen = sum(max(0, min(e, c["L"]) - b) for bs, es in zip(begin, end) for b, e in zip(bs, es)) * c["H_q"]
        rows, keys = c["B"] * c["H_q"] * c["L_q"], c["B"] * c["H_kv"] * c["L"]
        if c["op"] == "forward":
            return {"bytes": 2 * (rows + keys) * (c["D_qk"] + c["D_v"]) + 4 * rows, "flops": 2 * seen * (c["D_qk"] + c["D_v"])}
        return {"bytes": 2 * (rows * (2 * c["D_qk"] + 3 * c["D_v"]) + 2 * keys * (c["D_qk"] + c["D_v"])) + 4 * rows,
                "flops": 2 * seen * (3 * c["D_qk"] + 2 * c["D_v"])}
    lens = _lengths(c)
    size, extra = (2, 0) if c["cache"] == "bf16" else (1, 1)
    if c["op"] == "evict":
        row = (c["D_qk"] + c["D_v"]) * size + 2 * extra
        kept = sum(min(x, c["keep"]) for x in lens) * c["H_kv"]
        # a weight has to be above another's to move; about keep (L - keep) / L entries do: rows read and written
        moved = sum(max(0, x - c["keep"]) * min(1.0, c["keep"] / x) for x in lens) * c["H_kv"] * 0.7
        back = 0 if c["cache"] == "bf16" else kept * (row + 2 * (c["D_qk"] + c["D_v"]))
        return {"bytes": sum(lens) * c["H_kv"] * 8 + kept * 8 + int(moved) * 2 * row + back, "flops": sum(lens) * c["H_kv"]}
    n = c["n"]
    seen = sum(n * x - n * (n - 1) // 2 for x in lens) * c["H_q"]
    rows, keys = c["B"] * c["H_q"] * n, sum(lens) * c["H_kv"]
    if c["op"] == "cached":
        D = c["D_qk"] + c["D_v"]
        return {"bytes": keys * (D * size + 2 * extra) + rows * (2 * D + 4), "flops": 2 * seen * D}
    return {"bytes": keys * (c["D_qk"] * size + extra + 8) + rows * (2 * c["D_qk"] + 4), "flops": 2 * seen * c["D_qk"]}


# ---- 64 bits ------------------------------------------------------------------------------------------------------------------
def _exact_span(s):
    """Batch entry by batch entry, head by head: scores, softmax over the span, and the gradients of sum(O * dO)."""
    c = s["case"]
    B, H_q, L_q, L, g = c["B"], c["H_q"], c["L_q"], c["L"], c["H_q"] // c["H_kv"]
    z = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    o, stats = z(B, H_q, L_q, c["D_v"]), z(B, H_q, L_q)
    dq, dk, dv = z(*s["q"].shape), z(*s["k"].shape), z(*s["v"].shape)
    j = torch.arange(L, device="cuda")
    far = (torch.arange(L_q, device="cuda").view(-1, 1) + (L - L_q) - j).abs().double() if c["slopes"] else None
    slopes = _slopes(H_q)
    for b in range(B):
        hidden = (j < s["begin"][b].view(-1, 1)) | (j >= s["end"][b].view(-1, 1))
        for h in range(H_q):
            q, k, v = s["q"][b, h].double(), s["k"][b, h // g].double(), s["v"][b, h // g].double()
            x = (q @ k.T) * s["scale"]
            bent = torch.tanh(x / c["cap"]) if c["cap"] else None
            if c["cap"]:
                x = bent * c["cap"]
            if c["slopes"]:
                x = x - far * slopes[h]
            lse = torch.logsumexp(x.masked_fill_(hidden, -math.inf), 1, keepdim=True)
            stats[b, h] = lse[:, 0]
            w = torch.exp(x - lse).masked_fill_(hidden, 0.0)
            o[b, h] = w @ v
            if c["op"] == "backward":
                do = s["do"][b, h].double()
                dv[b, h // g] += w.T @ do
                dp = do @ v.T
                dx = w * (dp - (w * dp).sum(1, keepdim=True)) * s["scale"]
                if c["cap"]:
                    dx = dx * (1 - bent * bent)
                dq[b, h] = dx @ k
                dk[b, h // g] += dx.T @ q
    return [dq, dk, dv] if c["op"] == "backward" else (o, stats)


def _pow2(k):
    """2^k in 64 bits, from the exponent's bits."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_row(s, name, b):
    """The cached rows of one sequence, [H_kv, room, D], in 64 bits."""
    t = s["table"][b].long()
    if s["case"]["cache"] == "bf16":
        y = s[name].index_select(0, t).double()
    else:
        y = s[name].view(torch.uint8).index_select(0, t).view(torch.float8_e4m3fn).float().double()
        y = y * _pow2(s[name + "_e"].index_select(0, t).long() - 127).unsqueeze(-1)
    return y.permute(1, 0, 2, 3).reshape(y.shape[1], -1, y.shape[3])


def _exact_cached(s):
    c = s["case"]
    n, g, lens = c["n"], c["H_q"] // c["H_kv"], _lengths(c)
    weigh = c["op"] == "weigh"
    out = torch.zeros(c["B"], c["H_q"], n, c["D_v"], dtype=torch.float64, device="cuda")
    stats = torch.zeros(c["B"], c["H_q"], n, dtype=torch.float64, device="cuda")
    weights, positions = s.get("weights_out", torch.zeros(0, device="cuda")).double(), s.get("positions")
    slope = torch.tensor(_slopes(c["H_q"]), dtype=torch.float64, device="cuda").view(c["H_kv"], 1, g)
    for b in range(c["B"]):
        k = _exact_row(s, "kc", b)[:, : lens[b]]
        v = None if weigh else _exact_row(s, "vc", b)[:, : lens[b]]
        if weigh:
            first = lens[b] - n
            weights[b, :, :first] = s["weights"][b, :, :first].double()
            weights[b, :, first: lens[b]] = 0.0
            positions[b, :, first: lens[b]] = s["new_positions"][b]
        for t in range(n):
            end = lens[b] - n + 1 + t
            x = (k[:, :end] @ s["q"][b, :, t].double().view(c["H_kv"], g, -1).transpose(1, 2)) * s["scale"]  # [H_kv, keys, g]
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c.get("slopes"):
                x = x - slope * (end - 1 - torch.arange(end, device="cuda").double()).view(1, -1, 1)
            if weigh:
                weights[b, :, :end] += torch.exp(x - s["stats"][b, :, t].double().view(c["H_kv"], 1, g)).sum(-1)
                continue
            lse = torch.logsumexp(x, 1)
            stats[b, :, t] = lse.flatten()
            out[b, :, t] = (torch.exp(x - lse.unsqueeze(1)).transpose(1, 2) @ v[:, :end]).flatten(0, 1)
    return (weights, positions) if weigh else (out, stats)


def _exact_evict(s):
    """Entry by entry on the host."""
    c = s["case"]
    lens, keep, page = _lengths(c), c["keep"], c["page"]
    w, p = s["weights"].tolist(), s["positions"].tolist()
    weights, positions = s["weights_out"].double().cpu(), s["positions_out"].cpu()
    table = s["table"].tolist()
    moves = [[], [], [], []]  # page and place, of source and destination, with the head
    heads = []
    for b in range(c["B"]):
        count = min(lens[b], keep)
        for h in range(c["H_kv"]):
            ws, ps = w[b][h], p[b][h]
            newest = max(ps[: lens[b]])
            ranked = sorted(range(lens[b]), key=lambda i: (0 if ps[i] > newest - c["recent"] or ps[i] < c["sinks"] else 1, 0.0 if ps[i] > newest - c["recent"] or ps[i] < c["sinks"] else -ws[i], i))
            stay = set(ranked[:count])
            holds, behind = list(range(count)), iter(sorted(i for i in stay if i >= count))
            for i in range(count):
                if i not in stay:
                    holds[i] = next(behind)
                    for k, x in zip(moves, (table[b][holds[i] // page], holds[i] % page, table[b][i // page], i % page)):
                        k.append(x)
                    heads.append(h)
            weights[b, h, :count] = torch.tensor([ws[i] for i in holds], dtype=torch.float64)
            positions[b, h, :count] = torch.tensor([ps[i] for i in holds], dtype=torch.int32)
    sp, sl, dp, dl = (torch.tensor(x, dtype=torch.long, device="cuda") for x in moves)
    heads = torch.tensor(heads, dtype=torch.long, device="cuda")
    pages = []
    for name in ("kc", "vc"):
        x = s[name].double() if c["cache"] == "bf16" else s[name].float().double() * _pow2(s[name + "_e"].long() - 127).unsqueeze(-1)
        x[dp, heads, dl] = x[sp, heads, sl]
        if c["cache"] != "bf16":
            at = s["slots"].long()
            x = x.transpose(1, 2).reshape(-1, c["H_kv"], x.shape[3])[at.clamp(min=0)]
            x = (x * (at >= 0).view(c["B"], -1, 1, 1)).transpose(1, 2)
        pages.append(x)
    return [weights, positions, torch.tensor([min(x, keep) for x in lens], dtype=torch.int32), *pages]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("forward", "backward"):
        return _exact_span(s)
    return _exact_evict(s) if case["op"] == "evict" else _exact_cached(s)
