"""GPU parity of attention over the paged cache with capped and distance-biased scores, against the 64-bit definition on the values that the cache holds.

Bounds.  A score's sum of D products is off by at most D 2^-24 |scale| sum |q k|; a cap adds 4e-7 of itself or of the largest score, whichever is
less, a distance 2^-22 of its term; e is their sum with 2^-21 for the exponent.  A normalised weight is off by 2 e of itself and rounded once to bf16, so
|O - ref| <= (2^-8 + 2 e + 2^-20) sum_j p_j |v_j|, a bf16 output adds 2^-8 of itself, the statistic is within e + 2^-20 (1 + |stat|)."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import dequantise
from oracle.span_oracle import span_attention, spans_of

pytestmark = pytest.mark.gpu
SCORES = [dict(cap=6.0), dict(slopes=True), dict(cap=30.0, slopes=True)]


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def slopes_of(H):
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


def values(cache):
    if cache.k_exp is None:
        return [t.cpu().double().numpy() for t in (cache.k, cache.v)]
    return [dequantise(t.view(torch.uint8).cpu().numpy(), e.cpu().numpy()) for t, e in ((cache.k, cache.k_exp), (cache.v, cache.v_exp))]


def setup(A, seed, H_kv, page, lengths, dqk, dv, dtype, extra=0):
    """A cache of N(0, 1) rows with shuffled page lists; everything behind the lists' ends is NaN.  `extra`: pages for a prefix, behind them."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lengths]
    width, n_pages = max(max(need), 1) + 1, sum(need) + extra + 1
    c = A.PagedCache.empty(n_pages, H_kv, page, dqk, dv, dtype=dtype)
    k, v = (torch.randn(1, H_kv, n_pages * page, d, generator=g).to(torch.bfloat16).cuda() for d in (dqk, dv))
    c.append(k, v, torch.arange(n_pages * page, dtype=torch.int32).cuda()[None])
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table, at = torch.full((len(lengths), width), -9, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    used = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lengths):
        for j in range(n):
            used[table[b, j // page], j % page] = True
    used[order[at: at + extra].long()] = True
    rest = ~used.cuda()
    for t in (c.k, c.v):
        (t if dtype == "bf16" else t.view(torch.uint8)).transpose(1, 2)[rest] = float("nan") if dtype == "bf16" else 0x7f
    return c, table, order[at: at + extra]


def rows_of(pages, table, length):
    """[1, H, length, D] of a page list."""
    page = pages.shape[2]
    x = [pages[t] for t in table[: -(-length // page)]]
    return np.concatenate(x + [np.zeros((pages.shape[1], 0, pages.shape[3]))], 1)[None, :, :length]


def queries(seed, B, H, n, D):
    return (2 * torch.randn(B, n, H, D, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda().transpose(1, 2)


def check(O, S, Q, keys, vals, scale, cap=0.0, slopes=None):
    for b in range(Q.shape[0]):
        q = Q[b: b + 1].cpu().double().numpy()
        n, L = q.shape[2], keys[b].shape[2]
        got, stat = O[b: b + 1].cpu().double().numpy(), S[b: b + 1].cpu().double().numpy()
        if L == 0:
            assert (got == 0).all() and np.isneginf(stat).all()
            continue
        ref, lse, mag = span_attention(q, keys[b], vals[b], *spans_of("causal", 1, n, L), scale=scale, cap=cap, slopes=slopes)
        most = abs(scale) * float(np.abs(q).max((0, 1, 2)) @ np.abs(keys[b]).max((0, 1, 2)))
        e = q.shape[3] * 2.0 ** -24 * most + 4e-7 * min(cap, most) + (2.0 ** -22 * max(map(abs, slopes)) * (L + n) if slopes else 0.0) + 2.0 ** -21
        bound = (2.0 ** -8 + 2 * e + 2.0 ** -20) * mag
        if O.dtype == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        assert np.all(np.abs(got - ref) <= bound + 1e-30), (b, float(np.nanmax(np.abs(got - ref) - bound)))
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(stat), empty)
        assert np.all(np.abs(stat[~empty] - lse[~empty]) <= e + 2.0 ** -20 * (1 + np.abs(lse[~empty])))


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("H_q,H_kv,n,page,lengths,out,chunk", [
    (1, 1, 1, 16, [1], "f32", 0),
    (32, 8, 1, 64, [777, 300, 64, 1], "bf16", 0),
    (8, 1, 1, 32, [1500, 129, 128, 0], "f32", 128),
    (6, 2, 3, 16, [3, 2, 50, 33, 160], "f32", 128),
    (64, 8, 8, 128, [333, 9], "bf16", 0),
    (40, 1, 2, 16, [65, 200], "f32", 256),
])
def test_matches_definition(A, dqk, dv, dtype, score, H_q, H_kv, n, page, lengths, out, chunk):
    """Every kernel; lists cut and whole, empty ones, more new tokens than keys."""
    c, t, _ = setup(A, 1, H_kv, page, lengths, dqk, dv, dtype)
    Q, B, scale = queries(2, len(lengths), H_q, n, dqk), len(lengths), dqk ** -0.5
    kw = dict(cap=score.get("cap", 0.0), slopes=slopes_of(H_q) if score.get("slopes") else None)
    S = torch.full((B, H_q, n), 7.0, device="cuda")
    O = A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=scale, stats=S, chunk=chunk, out_dtype=torch.bfloat16 if out == "bf16" else torch.float32, **kw)
    keys, vals = ([rows_of(x, t[b].tolist(), lengths[b]) for b in range(B)] for x in values(c))
    check(O, S, Q, keys, vals, scale, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,lengths,prefix", [(8, 2, 1, [100, 1, 0, 40], 700), (16, 1, 2, [300, 2], 65), (12, 12, 1, [1], 33)])
def test_behind_a_prefix(A, dtype, H_q, H_kv, n, lengths, prefix):
    """A distance counts the prefix in front of the list."""
    page = 32
    c, t, pre = setup(A, 3, H_kv, page, lengths, 128, 128, dtype, extra=-(-prefix // page))
    Q, B = queries(4, len(lengths), H_q, n, 128), len(lengths)
    for kw in (dict(cap=9.0, slopes=None), dict(cap=0.0, slopes=slopes_of(H_q))):
        S = torch.empty(B, H_q, n, device="cuda")
        O = A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=0.09, stats=S, prefix_table=pre.cuda(), prefix_length=prefix, **kw)
        keys, vals = ([np.concatenate([rows_of(x, pre.tolist(), prefix), rows_of(x, t[b].tolist(), lengths[b])], 2) for b in range(B)] for x in values(c))
        for b in range(B):
            if lengths[b] < n:  # (its rows see the prefix, whole)
                assert torch.isfinite(O[b]).all() and torch.isfinite(S[b]).all()
                keys[b], vals[b], O[b], S[b] = keys[b][:, :, :0], vals[b][:, :, :0], 0, float("-inf")
        check(O, S, Q, keys, vals, 0.09, **kw)


@pytest.mark.parametrize("scale", [0.2, -0.2])
@pytest.mark.parametrize("cap", [0.5, 40.0, 1e6])
@pytest.mark.parametrize("n", [1, 20])
def test_caps(A, scale, cap, n):
    """Scores far beyond the cap, around it and far below; both signs of the scale; rows of one tile and of two."""
    c, t, _ = setup(A, 5, 2, 64, [300, 90], 64, 64, "bf16")
    Q, S = queries(6, 2, 4, n, 64), torch.empty(2, 4, n, device="cuda")
    O = A.attention_cached(Q, c, t.cuda(), ints([300, 90]), scale=scale, cap=cap, stats=S)
    keys, vals = ([rows_of(x, t[b].tolist(), (300, 90)[b]) for b in range(2)] for x in values(c))
    check(O, S, Q, keys, vals, scale, cap)


def test_long_list_steep_slopes_and_pages_outside(A):
    """A distance of thousands against a score of a few; pages that are not there are hidden; lengths outside the range count as its ends."""
    lengths, page = [9000, 5000], 128
    c, t, _ = setup(A, 7, 1, page, lengths, 64, 64, "bf16")
    t[1, 0], t[1, 38] = -1, c.n_pages
    Q, S, slopes = queries(8, 2, 4, 1, 64), torch.empty(2, 4, 1, device="cuda"), [3.0, 0.01, 0.0, -0.002]
    O = A.attention_cached(Q, c, t.cuda(), ints([12000, 5000]), scale=0.1, max_length=9000, slopes=slopes, stats=S)
    keys, vals = ([rows_of(x, [max(0, min(p, c.n_pages - 1)) for p in t[b].tolist()], lengths[b]) for b in range(2)] for x in values(c))
    check(O[:1], S[:1], Q[:1], keys[:1], vals[:1], 0.1, slopes=slopes)
    hidden = np.array([j // page in (0, 38) for j in range(5000)])
    x = 0.1 * np.einsum("hd,ld->hl", Q[1, :, 0].cpu().double().numpy(), np.nan_to_num(keys[1][0, 0])) - np.array(slopes)[:, None] * (4999 - np.arange(5000))
    x[:, hidden] = -np.inf
    lse = np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)) + x.max(1)
    # e = 64 2^-24 of scores up to 0.1 * 2 * 64 * 9 = 115, distances of 15000 * 2^-22, 2^-21; the statistic's own rounding 2^-20 (1 + 30)
    assert np.all(np.abs(S[1, :, 0].cpu().numpy() - lse) <= 115 * 64 * 2.0 ** -24 + 15000 * 2.0 ** -22 + 2.0 ** -21 + 31 * 2.0 ** -20)
    w = np.exp(x - lse[:, None])
    v = np.nan_to_num(vals[1][0, 0])
    assert np.all(np.abs(O[1, :, 0].cpu().numpy() - w @ v) <= (2.0 ** -8 + 9e-3) * (w @ np.abs(v)))


def test_slopes_of_zero_and_a_far_cap_change_next_to_nothing(A):
    c, t, _ = setup(A, 9, 2, 32, [700], 128, 128, "e4m3")
    Q, L = queries(10, 1, 8, 1, 128), ints([700])
    plain, S = torch.empty(1, 8, 1, device="cuda"), torch.empty(1, 8, 1, device="cuda")
    A.attention_cached(Q, c, t.cuda(), L, scale=0.1, stats=plain)
    for kw in (dict(slopes=[0.0] * 8), dict(cap=1e6)):
        A.attention_cached(Q, c, t.cuda(), L, scale=0.1, stats=S, **kw)
        # scores up to 12 or so: 2e-7 of them, and the statistics' roundings
        assert (plain - S).abs().max() <= 12 * 2e-7 + 2.0 ** -19 * 13


def test_special_values_and_same_bits(A):
    """A NaN key among the newest tokens reaches the rows that see it and no others, NaN queries their row; the same bits again."""
    c, t, _ = setup(A, 11, 1, 16, [500], 64, 64, "bf16")
    Q, kw = queries(12, 1, 4, 4, 64), dict(scale=0.125, cap=20.0, slopes=slopes_of(4), chunk=128)
    clean = A.attention_cached(Q, c, t.cuda(), ints([500]), **kw)
    for _ in range(3):
        assert torch.equal(A.attention_cached(Q, c, t.cuda(), ints([500]), **kw), clean)
    Q2 = Q.clone()
    Q2[0, 1, 2] = float("nan")
    O = A.attention_cached(Q2, c, t.cuda(), ints([500]), **kw)
    assert torch.isnan(O[0, 1, 2]).all()
    rest = torch.ones(4, 4, dtype=torch.bool)
    rest[1, 2] = False
    assert torch.equal(O[0][rest.cuda()], clean[0][rest.cuda()])
    c.k[int(t[0, 498 // 16]), 0, 498 % 16, 3] = float("nan")
    O = A.attention_cached(Q, c, t.cuda(), ints([500]), **kw)
    assert torch.equal(O[:, :, :2], clean[:, :, :2]) and torch.isnan(O[:, :, 2:]).all()


def test_captured_steps(A):
    """A captured decoding step with scores of its own, replayed on new queries and lengths between eager work."""
    lengths = [900, 333]
    c, t, _ = setup(A, 13, 2, 64, [1000, 1000], 128, 128, "bf16")
    td, L, Q = t.cuda(), ints(lengths), queries(14, 2, 8, 1, 128).contiguous()
    out, S = torch.empty(2, 8, 1, 128, device="cuda"), torch.empty(2, 8, 1, device="cuda")
    make = lambda: A.CachedAttentionPlan(c, Q, out, max_length=1000, table_width=t.shape[1], scale=0.1, cap=15.0, slopes=slopes_of(8), chunk=128)
    plan, eager = make(), make()
    assert plan.workspace is not None
    plan.forward(Q, td, L, out, stats=S)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.forward(Q, td, L, out, stats=S)
    for n in range(4):
        Q.copy_(queries(20 + n, 2, 8, 1, 128))
        L.copy_(ints([900 + 20 * n, 5 + 300 * n]))
        want = eager.forward(Q, td, L, torch.empty_like(out)).clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals_of_the_binding(A):
    c, t, _ = setup(A, 15, 2, 16, [40], 64, 64, "bf16")
    Q = queries(16, 1, 4, 1, 64)
    with pytest.raises(ValueError):
        A.attention_cached(Q, c, t.cuda(), ints([40]), scale=0.1, slopes=[1.0])
    with pytest.raises(A.AeAttnError):
        A.attention_cached(Q, c, t.cuda(), ints([40]), scale=0.1, cap=-2.0)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,prefix", [(264, 1, 1, 0), (320, 8, 2, 0), (1024, 16, 1, 0), (512, 16, 1, 100)])
def test_a_cap_with_more_heads_than_a_table_of_slopes_has(A, dtype, H_q, H_kv, n, prefix):
    """Caps come with any number of heads; the statistics of all of them are the definition's too, and what the entries receive by them adds up."""
    lengths, page = [150, 33], 32
    c, t, pre = setup(A, 17, H_kv, page, lengths, 64, 64, dtype, extra=-(-prefix // page))
    Q, L = queries(18, 2, H_q, n, 64), ints(lengths)
    kw = dict(scale=0.125, cap=8.0)
    S = torch.full((2, H_q, n), float("nan"), device="cuda")
    O = A.attention_cached(Q, c, t.cuda(), L, stats=S, prefix_table=pre.cuda() if prefix else None, prefix_length=prefix, **kw)
    keys, vals = ([np.concatenate([rows_of(x, pre.tolist(), prefix), rows_of(x, t[b].tolist(), lengths[b])], 2) for b in range(2)] for x in values(c))
    check(O, S, Q, keys, vals, **kw)
    if not prefix:  # g n rows of probabilities that sum to 1; score and statistic are within e each, 64 2^-24 of 0.125 * 64 * 8 * 4, so 2e-3 together
        W = A.cache_weights(Q, c, t.cuda(), L, S, torch.zeros(2, H_kv, 160, device="cuda"), **kw)
        assert torch.allclose(W.sum(-1), torch.full((2, H_kv), float(H_q // H_kv * n), device="cuda"), rtol=2.0 ** -8, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("cap", [2e36, 1e37])
def test_the_largest_caps_leave_the_scores(A, dtype, cap):
    """Scale / cap next to the smallest 32-bit number with all its bits: as without a cap, also for what the entries receive."""
    lengths, page = [300, 70], 32
    c, t, _ = setup(A, 19, 2, page, lengths, 64, 64, dtype)
    Q, L, got = queries(20, 2, 8, 2, 64), ints(lengths), []
    for x in (0.0, cap):
        S = torch.empty(2, 8, 2, device="cuda")
        O = A.attention_cached(Q, c, t.cuda(), L, scale=0.125, stats=S, cap=x)
        keys, vals = ([rows_of(y, t[b].tolist(), lengths[b]) for b in range(2)] for y in values(c))
        check(O, S, Q, keys, vals, 0.125, cap=x)
        got.append((S, A.cache_weights(Q, c, t.cuda(), L, S, torch.zeros(2, 2, 320, device="cuda"), scale=0.125, cap=x)))
    # scores up to 20 or so, 3e-7 of which the cap's constants are off, and the roundings of the statistic
    assert (got[0][0] - got[1][0]).abs().max() <= 20 * 3e-7 + 2.0 ** -19 * 20
    assert torch.allclose(got[0][1], got[1][1], rtol=1e-4, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,lengths,prefix", [(8, 2, 3, [0, 1, 2, 3, 50], 100), (4, 4, 8, [2, 0], 5), (16, 1, 2, [0, 300], 700)])
def test_tokens_that_their_list_is_too_short_for(A, dtype, H_q, H_kv, n, lengths, prefix):
    """Behind a prefix they see all of it, from places inside it or in front of it: keys on both sides."""
    page = 16
    c, t, pre = setup(A, 21, H_kv, page, lengths, 64, 64, dtype, extra=-(-prefix // page))
    Q, B = queries(22, len(lengths), H_q, n, 64), len(lengths)
    keys, vals = ([np.concatenate([rows_of(x, pre.tolist(), prefix), rows_of(x, t[b].tolist(), lengths[b])], 2) for b in range(B)] for x in values(c))
    for kw in (dict(slopes=slopes_of(H_q)), dict(slopes=[1.5 - h for h in range(H_q)]), dict(cap=4.0, slopes=slopes_of(H_q))):
        S = torch.empty(B, H_q, n, device="cuda")
        O = A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=0.1, stats=S, prefix_table=pre.cuda(), prefix_length=prefix, **kw)
        for b in range(B):
            q, L = Q[b: b + 1].cpu().double().numpy(), prefix + lengths[b]
            seen = np.zeros((1, n), int), np.maximum(prefix, L - n + 1 + np.arange(n))[None]
            ref, lse, mag = span_attention(q, keys[b], vals[b], *seen, scale=0.1, **kw)
            most = 0.1 * float(np.abs(q).max((0, 1, 2)) @ np.abs(keys[b]).max((0, 1, 2)))
            e = 64 * 2.0 ** -24 * most + 4e-7 * min(kw.get("cap", 0.0), most) + 2.0 ** -22 * max(map(abs, kw["slopes"])) * (L + n) + 2.0 ** -21
            assert np.all(np.abs(O[b: b + 1].cpu().double().numpy() - ref) <= (2.0 ** -8 + 2 * e + 2.0 ** -20) * mag), b
            assert np.all(np.abs(S[b: b + 1].cpu().double().numpy() - lse) <= e + 2.0 ** -20 * (1 + np.abs(lse))), b
