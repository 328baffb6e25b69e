"""GPU parity of attention over the paged cache (ae_cached_forward) against the 64-bit definition on the values that the
cache holds.

Bounds.  A weight is rounded once to bf16 (at most 2^-8 of it) before the product with the values; scores, weights and sums are 32-bit:
score error <= D 2^-24 scale sum |q k|, below 2e-5 for these inputs, which is also the weights' relative error.  So |O - ref| <= (2^-8 + 4e-5) *
sum_j p_j |v_j|, and a bf16 output adds half a step, 2^-8 |O|.  The statistic is within 1e-4 (D 2^-24 scale sum |q k| plus the logarithm's own)."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import attend, dequantise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def values(cache):
    """The cache's contents in 64 bits, [n_pages, H_kv, page, D] each."""
    if cache.k_exp is None:
        return [t.cpu().double().numpy() for t in (cache.k, cache.v)]
    return [dequantise(t.view(torch.uint8).cpu().numpy(), e.cpu().numpy()) for t, e in ((cache.k, cache.k_exp), (cache.v, cache.v_exp))]


def listed(pages, table, length):
    """Rows [H, length, D] of a page list."""
    page = pages.shape[2]
    need = -(-length // page)
    return np.concatenate([pages[t] for t in table[:need]] + [np.zeros((pages.shape[1], 0, pages.shape[3]))], axis=1)[:, :length]


def make(A, seed, n_pages, H_kv, page, dqk, dv, dtype, poison=True):
    """A cache full of N(0, 1) rows; `poison`: what no test writes afterwards is NaN (and exponents of 255)."""
    g = torch.Generator().manual_seed(seed)
    c = A.PagedCache.empty(n_pages, H_kv, page, dqk, dv, dtype=dtype)
    k, v = (torch.randn(1, H_kv, n_pages * page, d, generator=g).to(torch.bfloat16).cuda() for d in (dqk, dv))
    c.append(k, v, torch.arange(n_pages * page, dtype=torch.int32).cuda()[None])
    return c


def spoil_behind(cache, tables, lengths):
    """NaN in every row of the cache that no list holds."""
    page = cache.page_size
    used = torch.zeros(cache.n_pages * page, dtype=torch.bool)
    for t, n in zip(tables, lengths):
        for j in range(n):
            p = int(t[j // page])
            if 0 <= p < cache.n_pages:
                used[p * page + j % page] = True
    rest = ~used.view(cache.n_pages, page).cuda()
    for t in (cache.k, cache.v):
        if t.dtype == torch.bfloat16:
            t.transpose(1, 2)[rest] = float("nan")
        else:
            t.view(torch.uint8).transpose(1, 2)[rest] = 0x7f
    for e in (cache.k_exp, cache.v_exp):
        if e is not None:
            e.transpose(1, 2)[rest] = 255


def queries(seed, B, H_q, n, D):
    return torch.randn(B, n, H_q, D, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda().transpose(1, 2)


def check(got, stats, Q, keys, vals, scale, what):
    """keys, vals: per sequence, [H_kv, len, D]."""
    O, S = got.cpu().double().numpy(), None if stats is None else stats.cpu().double().numpy()
    worst = 0.0
    for b in range(Q.shape[0]):
        q = Q[b].cpu().double().numpy()
        ref, lse = attend(q, keys[b], vals[b], scale)
        mag, _ = attend(q, keys[b], np.abs(vals[b]), scale)
        bound = (2.0 ** -8 + 4e-5) * mag + 1e-30
        if got.dtype == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        err = np.abs(O[b] - ref)
        assert np.isfinite(O[b]).all(), (what, b)
        worst = max(worst, float((err / bound).max()))
        assert (err <= bound).all(), (what, b, float((err / bound).max()))
        if S is not None:
            empty = np.isneginf(lse)
            assert np.array_equal(np.isneginf(S[b]), empty), (what, b)
            assert (np.abs(S[b][~empty] - lse[~empty]) <= 1e-4).all(), (what, b)
    print(f"{what}: largest error {worst:.3f} of the bound", flush=True)


def tables_for(seed, n_pages, lengths, page, width, first=0):
    """A page list per sequence; entries behind the last needed one are numbers of no page."""
    order = torch.randperm(n_pages - first, generator=torch.Generator().manual_seed(seed)) + first
    t, at = torch.full((len(lengths), width), -7, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        need = -(-n // page)
        t[b, :need] = order[at: at + need].to(torch.int32)
        at += need
    return t


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,page,lengths,out,chunk", [
    (1, 1, 1, 16, [1], "f32", 0),
    (4, 4, 1, 16, [1, 15, 16, 17, 31, 32, 33], "bf16", 0),
    (32, 8, 1, 64, [777, 300, 64, 1], "f32", 0),
    (8, 1, 1, 32, [1500, 129, 128, 127], "bf16", 128),
    (6, 2, 3, 16, [3, 4, 50, 33, 160], "f32", 128),
    (16, 2, 4, 256, [700, 4, 513], "f32", 0),
    (64, 8, 8, 128, [333, 9], "bf16", 0),
    (12, 12, 2, 32, [2, 34, 257], "f32", 256),
    (7, 1, 5, 64, [90, 64, 5], "f32", 0),
    (40, 1, 2, 16, [65, 200], "f32", 128),
])
def test_matches_definition(A, dqk, dv, dtype, H_q, H_kv, n, page, lengths, out, chunk):
    B, width = len(lengths), -(-max(lengths) // page) + 2
    n_pages = sum(-(-x // page) for x in lengths) + 1
    c = make(A, 1, n_pages, H_kv, page, dqk, dv, dtype)
    t = tables_for(2, n_pages, lengths, page, width)
    spoil_behind(c, t, lengths)
    Q = queries(3, B, H_q, n, dqk)
    stats = torch.full((B, H_q, n), 7.0, device="cuda")
    scale = dqk ** -0.5
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=scale, stats=stats, chunk=chunk,
                           out_dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    kv = values(c)
    rows = [[listed(x, t[b].tolist(), lengths[b]) for b in range(B)] for x in kv]
    check(O, stats, Q, *rows, scale, f"{dqk}/{dv} {dtype} {H_q}/{H_kv} n {n} page {page}")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,chunk", [(1, 0), (3, 128)])
def test_lengths_of_padded_batches(A, dtype, n, chunk):
    # empty sequences, fewer keys than new tokens, lengths outside [0, max_length]
    lengths, page, width = [0, 1, 2, 200, -5, 4000, 130], 32, 8
    n_pages = len(lengths) * width
    c = make(A, 4, n_pages, 2, page, 128, 128, dtype)
    t = torch.randperm(n_pages, generator=torch.Generator().manual_seed(5)).view(len(lengths), width).to(torch.int32)
    Q = queries(6, len(lengths), 4, n, 128)
    stats = torch.empty(len(lengths), 4, n, device="cuda")
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=0.09, max_length=201, stats=stats, chunk=chunk)
    real = [min(max(x, 0), 201) for x in lengths]
    rows = [[listed(x, t[b].tolist(), real[b]) for b in range(len(real))] for x in values(c)]
    check(O, stats, Q, *rows, 0.09, f"padded {dtype} n {n}")
    assert (O[0] == 0).all() and torch.isneginf(stats[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pages_outside_the_cache(A, dtype):
    # their keys are hidden; all pages of a sequence may be bad
    page, lengths = 16, [100, 70, 40, 33]
    c = make(A, 7, 30, 2, page, 64, 64, dtype)
    t = tables_for(8, 29, lengths, page, 7)
    t[t == 0] = 29  # (page 0 is what a bad number is replaced by: it holds NaN)
    t[0, 2], t[0, 6], t[1, 0], t[1, 3], t[3, 0] = -1, 30, 2 ** 31 - 1, -2 ** 31, 99999
    t[2, :] = -1
    spoil_behind(c, t, lengths)
    Q = queries(9, 4, 4, 1, 64)
    stats = torch.empty(4, 4, 1, device="cuda")
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=0.125, stats=stats)
    rows = []
    for x in values(c):
        per = []
        for b, n in enumerate(lengths):
            live = [j for j in range(n) if 0 <= int(t[b, j // page]) < 30]
            per.append(np.stack([x[int(t[b, j // page]), :, j % page] for j in live], axis=1) if live else np.zeros((2, 0, 64)))
        rows.append(per)
    check(O, stats, Q, *rows, 0.125, f"bad pages {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_special_values_reach_only_the_rows_that_see_them(A, dtype):
    # the newest tokens hold infinities (16-bit) and NaN: earlier ones of them do not see those
    n, page, length = 4, 16, 50
    c = make(A, 10, 5, 1, page, 64, 64, dtype)
    t = torch.tensor([[3, 1, 4, 0]], dtype=torch.int32)
    Q = queries(11, 1, 2, n, 64)
    run = lambda: A.attention_cached(Q, c, t.cuda(), torch.tensor([length], dtype=torch.int32).cuda(), scale=0.125)
    clean = run()
    where = [(int(t[0, j // page]), 0, j % page) for j in range(length - n, length)]  # rows of the newest tokens
    nan = float("nan") if dtype == "bf16" else 0x7f
    V = c.v if dtype == "bf16" else c.v.view(torch.uint8)
    K = c.k if dtype == "bf16" else c.k.view(torch.uint8)
    V[where[1]][5] = nan
    if dtype == "bf16":
        V[where[2]][9], V[where[2]][10], V[where[3]][10] = float("inf"), float("-inf"), float("inf")
    K[where[3]][0] = nan
    O = run()
    assert torch.equal(O[:, :, 0], clean[:, :, 0])
    assert torch.isnan(O[0, :, 1:, 5]).all() and torch.isfinite(O[0, :, 1, :5]).all()
    others = [d for d in range(64) if d not in (5, 9, 10)]
    assert torch.equal(O[:, :, 1:3][..., others], clean[:, :, 1:3][..., others])
    assert torch.isnan(O[0, :, 3]).all()
    if dtype == "bf16":
        assert torch.isposinf(O[0, :, 2, 9]).all() and torch.isneginf(O[0, :, 2, 10]).all()


def test_infinity_in_the_last_row(A):
    # a copy of the row behind the end, weighed with zero, would make it NaN
    c = make(A, 12, 3, 1, 16, 64, 64, "bf16")
    c.v[1, 0, 4, 7] = float("inf")  # key 20 of 21
    Q = queries(13, 1, 1, 1, 64)
    O = A.attention_cached(Q, c, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), torch.tensor([21], dtype=torch.int32).cuda(), scale=0.125)
    assert torch.isposinf(O[0, 0, 0, 7]) and torch.isfinite(O[0, 0, 0, :7]).all() and torch.isfinite(O[0, 0, 0, 8:]).all()


@pytest.mark.parametrize("scale", [3.0, -0.2, 1e-4])
def test_scales(A, scale):
    # steep softmax (the reference moves often), a negative scale, a flat one.  Errors of the scores grow with the scale:
    # 64 * 2^-24 * 3 * sum |q k| (about 41) = 5e-4 of a weight, inside the bound's margin over the typical 2^-9
    c = make(A, 14, 9, 2, 64, 64, 64, "bf16")
    t = torch.randperm(9, generator=torch.Generator().manual_seed(15)).view(1, 9).to(torch.int32)
    Q = queries(16, 1, 6, 1, 64)
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor([570], dtype=torch.int32).cuda(), scale=scale)
    rows = [[listed(x, t[0].tolist(), 570)] for x in values(c)]
    check(O, None, Q, *rows, scale, f"scale {scale}")


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,page,prefix,lengths,chunk", [
    (4, 4, 1, 16, 1, [1, 2], 0),
    (12, 12, 1, 32, 1000, [150, 1, 33, 0], 0),
    (32, 8, 1, 64, 515, [90] * 9, 0),
    (8, 2, 3, 16, 129, [3, 40, 17], 128),
    (16, 1, 2, 128, 2049, [2, 130, 64, 7, 300], 256),
    (64, 8, 1, 64, 64, [5] * 20, 0),
])
def test_shared_prefix(A, dqk, dv, dtype, H_q, H_kv, n, page, prefix, lengths, chunk):
    B, width, pp = len(lengths), -(-max(lengths) // page), -(-prefix // page)
    n_pages = pp + sum(-(-x // page) for x in lengths) + 1
    c = make(A, 20, n_pages, H_kv, page, dqk, dv, dtype)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(21)).to(torch.int32)
    ptab, t, at = order[:pp].clone(), torch.full((B, width), -3, dtype=torch.int32), pp
    for b, x in enumerate(lengths):
        need = -(-x // page)
        t[b, :need] = order[at: at + need]
        at += need
    spoil_behind(c, list(t) + [ptab], lengths + [prefix])
    Q = queries(22, B, H_q, n, dqk)
    stats = torch.empty(B, H_q, n, device="cuda")
    scale = dqk ** -0.5
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=scale, prefix_table=ptab.cuda(), prefix_length=prefix,
                           stats=stats, chunk=chunk)
    kv = values(c)
    own = [[listed(x, t[b].tolist(), lengths[b]) for b in range(B)] for x in kv]
    pre = [listed(x, ptab.tolist(), prefix) for x in kv]
    if min(lengths) >= n:
        rows = [[np.concatenate((p, o), axis=1) for o in per] for p, per in zip(pre, own)]
        check(O, stats, Q, *rows, scale, f"prefix {prefix} {dqk}/{dv} {dtype}")
    else:  # a row without keys of its own sees the prefix alone
        for b, x in enumerate(lengths):
            k, v = ((np.concatenate((p, per[b]), axis=1)) for p, per in zip(pre, own))
            qb, sb, ob = Q[b: b + 1], stats[b: b + 1], O[b: b + 1]
            if x >= n:
                check(ob, sb, qb, [k], [v], scale, f"prefix, sequence {b}")
            else:
                assert n == 1 and x == 0
                check(ob, sb, qb, [pre[0]], [pre[1]], scale, f"prefix alone, sequence {b}")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_prefix_equals_long_lists(A, dtype):
    # the same keys, once as a shared prefix and once in every sequence's own list
    page, prefix, B = 32, 640, 6
    lengths = [37, 1, 64, 90, 33, 10]
    c = make(A, 30, 20 + 6 * 3, 2, page, 128, 128, dtype)
    ptab = torch.randperm(20, generator=torch.Generator().manual_seed(31)).to(torch.int32)
    t = (20 + torch.arange(18).view(6, 3)).to(torch.int32)
    Q, L = queries(32, B, 8, 1, 128), torch.tensor(lengths, dtype=torch.int32).cuda()
    s1, s2 = torch.empty(B, 8, 1, device="cuda"), torch.empty(B, 8, 1, device="cuda")
    a = A.attention_cached(Q, c, t.cuda(), L, scale=0.0884, prefix_table=ptab.cuda(), prefix_length=prefix, stats=s1)
    whole = torch.cat((ptab.expand(6, 20), t), 1).contiguous().cuda()
    b = A.attention_cached(Q, c, whole, L + prefix, scale=0.0884, stats=s2)
    # both are within 2^-8 sum p |v| of the same result, sum p |v| <= 1.1 here
    assert (a - b).abs().max() <= 2 * 1.1 * 2.0 ** -8 and (s1 - s2).abs().max() <= 1e-4


def test_same_bits_twice_and_strided_output(A):
    lengths, page = [3000, 100, 1700], 64
    c = make(A, 40, 80, 2, page, 128, 128, "e4m3")
    t, L = tables_for(41, 80, lengths, page, 47).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    Q = queries(42, 3, 16, 2, 128)
    buf = torch.full((3, 2, 20, 136), 5.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :, 2:18, 8:136].transpose(1, 2)
    A.attention_cached(Q, c, t, L, scale=0.0884, out=out)
    first = out.clone()
    assert (buf[:, :, :2] == 5).all() and (buf[:, :, 18:] == 5).all() and (buf[..., :8] == 5).all()
    for _ in range(3):
        again = A.attention_cached(Q, c, t, L, scale=0.0884, out_dtype=torch.bfloat16)
        assert torch.equal(again, first)


def test_replayed_graphs_with_growing_lengths(A):
    # two graphs of one plan, replayed in turn while the lengths on the device grow; eager calls of another plan in between
    page, width = 16, 40
    c = make(A, 50, 4 * width, 2, page, 128, 128, "bf16")
    t = torch.randperm(4 * width, generator=torch.Generator().manual_seed(51)).view(4, width).to(torch.int32).cuda()
    L = torch.tensor([1, 100, 37, 500], dtype=torch.int32).cuda()
    Q = queries(52, 4, 8, 1, 128)
    outs = [torch.empty(4, 8, 1, 128, device="cuda") for _ in range(2)]
    plan = A.CachedAttentionPlan(c, Q, outs[0], max_length=width * page, table_width=width, scale=0.0884, chunk=128)
    plan.forward(Q, t, L, outs[0])
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            plan.forward(Q, t, L, o)
        graphs.append(g)
    for step in range(5):
        for g, o in zip(graphs, outs):
            L += 7
            g.replay()
            eager = A.attention_cached(Q, c, t, L, scale=0.0884, chunk=128)
            torch.cuda.synchronize()
            assert torch.equal(o, eager), step


def test_another_stream(A):
    lengths, page = [900, 1300], 32
    c = make(A, 60, 72, 4, page, 64, 64, "e4m3")
    t, L = tables_for(61, 72, lengths, page, 41).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    Q = queries(62, 2, 8, 1, 64)
    ref = A.attention_cached(Q, c, t, L, scale=0.125)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = A.attention_cached(Q, c, t, L, scale=0.125, stream=s)
    s.synchronize()
    assert torch.equal(got, ref)


def test_cache_past_32_bits(A):
    # pages whose byte offsets pass 2^32, a long list, few rows
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    n_pages, page = 42000, 256  # x 2 heads x 128 x 2 bytes = 5.5 GB each of K and V
    c = A.PagedCache.empty(n_pages, 2, page, 128, 128)
    length = 70001
    t = torch.randperm(n_pages, generator=torch.Generator().manual_seed(70))[:274].to(torch.int32).view(1, 274)
    t[0, 0], t[0, 1] = n_pages - 1, 33333
    t[0, 2:] = torch.where((t[0, 2:] == n_pages - 1) | (t[0, 2:] == 33333), torch.tensor(0, dtype=torch.int32), t[0, 2:])
    g = torch.Generator(device="cuda").manual_seed(71)
    k, v = (torch.randn(1, 2, length, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    j = torch.arange(length)
    slots = (t[0, j // page].long() * page + j % page).to(torch.int32).cuda()
    c.append(k, v, slots[None])
    Q = queries(72, 1, 4, 1, 128)
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor([length], dtype=torch.int32).cuda(), scale=0.0884)
    check(O, None, Q, [k[0].cpu().double().numpy()], [v[0].cpu().double().numpy()], 0.0884, "past 2^32")


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,H_q,H_kv,n,page,prefix,chunk,bad", [
    (50, 32, 8, 1, 16, 5, 0, []),          # 200 rows a k/v head, less than a tile of keys
    (64, 32, 8, 1, 64, 700, 0, []),        # 256: one workgroup's rows
    (65, 8, 2, 1, 32, 1024, 256, [3, 9]),  # 260: the last wavefronts have four rows; two pages are no pages
    (40, 16, 1, 2, 16, 333, 128, [0, 20]), # 1280 rows, the last page among the bad ones, three ranges
    (300, 1, 1, 1, 256, 2000, 0, []),
    (23, 64, 4, 3, 128, 130, 128, [1]),    # 1104 rows; the second range has bad keys only
])
def test_prefix_of_many_rows(A, dqk, dv, dtype, B, H_q, H_kv, n, page, prefix, chunk, bad):
    pp, own = -(-prefix // page), 20
    n_pages = pp + 2 + B * 2
    c = make(A, 80, n_pages, H_kv, page, dqk, dv, dtype)
    order = torch.randperm(n_pages - 1, generator=torch.Generator().manual_seed(81)).to(torch.int32) + 1  # (page 0 holds NaN)
    ptab = order[:pp].clone()
    for i in bad:
        ptab[i] = -1 if i % 2 else n_pages
    width = -(-own // page)
    t = order[pp: pp + B * width].view(B, width).clone()
    lengths = [n + (7 * b) % (own - n) for b in range(B)]
    spoil_behind(c, list(t) + [ptab], lengths + [prefix])
    Q = queries(82, B, H_q, n, dqk)
    stats = torch.empty(B, H_q, n, device="cuda")
    scale = dqk ** -0.5
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=scale, prefix_table=ptab.cuda(), prefix_length=prefix,
                           stats=stats, chunk=chunk, out_dtype=torch.bfloat16 if B == 64 else torch.float32)
    kv = values(c)
    live = [j for j in range(prefix) if 0 <= int(ptab[j // page]) < n_pages]
    pre = [np.stack([x[int(ptab[j // page]), :, j % page] for j in live], axis=1) if live else np.zeros((H_kv, 0, x.shape[3])) for x in kv]
    some = sorted({0, 1, B // 2, B - 2, B - 1})  # (the definition in 64 bits takes its time)
    rows = [[np.concatenate((p, listed(x, t[b].tolist(), lengths[b])), axis=1) for b in some] for p, x in zip(pre, kv)]
    check(O[some], stats[some], Q[some], *rows, scale, f"{B} x {H_q}/{H_kv} x {n} behind {prefix}, {dqk}/{dv} {dtype}")
    # the others against the walk of few rows: the same keys as every sequence's own list
    whole = torch.cat((ptab.expand(B, pp), t), 1).contiguous().cuda() if prefix % page == 0 else None
    if whole is not None:
        s2 = torch.empty_like(stats)
        O2 = A.attention_cached(Q, c, whole, torch.tensor(lengths, dtype=torch.int32).cuda() + prefix, scale=scale, stats=s2)
        top = float(max(np.nanmax(np.abs(np.where(np.isfinite(x), x, np.nan))) for x in kv[1:]))
        assert (O.float() - O2).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -8) * top and (stats - s2).abs().max() <= 2e-4


def test_negative_scale_of_many_rows(A):
    c = make(A, 90, 12, 2, 64, 64, 64, "bf16")
    ptab, t = torch.arange(8, dtype=torch.int32), torch.full((200, 1), 9, dtype=torch.int32)
    Q = queries(91, 200, 4, 1, 64)
    O = A.attention_cached(Q, c, t.cuda(), torch.full((200,), 3, dtype=torch.int32).cuda(), scale=-0.3, prefix_table=ptab.cuda(), prefix_length=500)
    some = [0, 99, 199]
    rows = [[np.concatenate((listed(x, ptab.tolist(), 500), listed(x, [9], 3)), axis=1) for _ in some] for x in values(c)]
    check(O[some], None, Q[some], *rows, -0.3, "negative scale")


@pytest.mark.parametrize("dqk,dv,dtype", [(64, 64, "e4m3"), (128, 128, "bf16"), (192, 128, "bf16")])
@pytest.mark.parametrize("B,n,prefix,chunk", [(188, 1, 400, 128), (100, 2, 1290, 256), (300, 4, 700, 128)])
def test_few_ranges_of_many_row_tiles(A, dqk, dv, dtype, B, n, prefix, chunk):
    # one k/v head: fewer ranges of the prefix than XCDs, with many row tiles each, in the own keys' launch and in one of its own
    H_q, page = 8, 64
    pp = -(-prefix // page)
    n_pages = pp + B + 1
    c = make(A, 100, n_pages, 1, page, dqk, dv, dtype)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(101)).to(torch.int32)
    ptab, t = order[:pp], order[pp: pp + B].view(B, 1)
    lengths = [n + (5 * b) % (page - n) for b in range(B)]
    spoil_behind(c, list(t) + [ptab], lengths + [prefix])
    Q = queries(102, B, H_q, n, dqk)
    stats = torch.empty(B, H_q, n, device="cuda")
    L = torch.tensor(lengths, dtype=torch.int32).cuda()
    O = A.attention_cached(Q, c, t.cuda(), L, scale=dqk ** -0.5, prefix_table=ptab.cuda(), prefix_length=prefix, stats=stats, chunk=chunk)
    kv = values(c)
    some = sorted({0, 1, 31, 32, B // 2, B - 2, B - 1})
    rows = [[np.concatenate((listed(x, ptab.tolist(), prefix), listed(x, t[b].tolist(), lengths[b])), axis=1) for b in some] for x in kv]
    check(O[some], stats[some], Q[some], *rows, dqk ** -0.5, f"{B} x 8/1 x {n} behind {prefix}, {dqk}/{dv} {dtype}")
    # every row was written, and the layout that the library chooses gives the same within both sides' roundings
    O2 = A.attention_cached(Q, c, t.cuda(), L, scale=dqk ** -0.5, prefix_table=ptab.cuda(), prefix_length=prefix)
    top = float(max(np.nanmax(np.abs(np.where(np.isfinite(x), x, np.nan))) for x in kv[1:]))
    assert (O - O2).abs().max() <= 2 * (2.0 ** -8 + 4e-5) * top


def test_one_handle_on_two_streams_at_once(A):
    # handles are immutable: calls that share one, with a workspace each, may overlap
    lengths, page = [3000, 2000, 2500], 64
    c = make(A, 110, 128, 4, page, 128, 128, "bf16")
    t, L = tables_for(111, 128, lengths, page, 47).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    Q = [queries(112 + i, 3, 16, 2, 128).contiguous() for i in range(2)]
    h = A.ae_cached_create(c.handle, B=3, H_q=16, n_new=2, table_width=47, max_length=3000, scale=0.09)
    size = A.ae_cached_workspace_bytes(h)
    assert size > 0
    ws, O = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)], [torch.empty(3, 16, 2, 128, device="cuda") for _ in range(2)]
    ref = [A.attention_cached(q, c, t, L, scale=0.09, max_length=3000) for q in Q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for w, s in zip(ws, streams):
        A.ae_cached_init_workspace(h, w.data_ptr(), size, s.cuda_stream)
    for _ in range(20):
        for q, w, o, s in zip(Q, ws, O, streams):
            A.ae_cached_forward(h, q.data_ptr(), *c.pointers(), t.data_ptr(), L.data_ptr(), 0, o.data_ptr(), 0, w.data_ptr(), size, s.cuda_stream)
    torch.cuda.synchronize()
    A.ae_cached_destroy(h)
    for o, r in zip(O, ref):
        assert torch.equal(o, r)


@pytest.mark.parametrize("B,n,prefix,launches", [(3, 2, 0, 1), (3, 2, 70, 1), (2, 17, 70, 2)])
def test_one_row_of_queries_for_all(A, B, n, prefix, launches):
    page, width = 16, 4
    c = make(A, 120, B * width + 5, 2, page, 64, 64, "bf16")
    t = torch.arange(B * width, dtype=torch.int32).view(B, width).cuda()
    L = torch.tensor([60, 33, 47][:B], dtype=torch.int32).cuda()
    kw = dict(prefix_length=prefix) if prefix else {}
    tables = dict(prefix_table=(B * width + torch.arange(5, dtype=torch.int32)).cuda()) if prefix else {}
    Q = queries(121, 1, 1, 1, 64).view(64).expand(B, 4, n, 64)
    out = torch.empty(B, 4, n, 64, device="cuda")
    plan = A.CachedAttentionPlan(c, Q, out, max_length=64, table_width=width, scale=0.125, **kw)
    assert A.ae_cached_query(plan.handle)["launches"] == launches
    plan.forward(Q, t, L, out, **tables)
    assert torch.equal(out, A.attention_cached(Q.contiguous(), c, t, L, scale=0.125, **kw, **tables))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,n,length,chunk,prefix", [(1, 1, 600, 0, 0), (1, 1, 600, 128, 0), (2, 3, 50, 128, 0), (2, 3, 600, 128, 0), (1, 1, 20, 128, 300),
                                                     (2, 3, 200, 128, 300), (3, 17, 40, 0, 300), (3, 17, 40, 128, 300), (3, 17, 200, 128, 300)])
def test_bad_queries_and_keys_give_nan(A, dtype, B, n, length, chunk, prefix):
    # NaN and infinite queries, and a NaN key that every row sees, make their rows NaN and no others, however the keys are cut
    page, width = 16, 40
    c = make(A, 130, B * width + 20, 2, page, 64, 64, dtype)
    t, ptab = torch.arange(B * width, dtype=torch.int32).view(B, width).cuda(), torch.arange(B * width, B * width + 20, dtype=torch.int32).cuda()
    L = torch.full((B,), length, dtype=torch.int32, device="cuda")
    kw = dict(scale=0.125, chunk=chunk, **(dict(prefix_table=ptab[: -(-prefix // page)].contiguous(), prefix_length=prefix) if prefix else {}))
    Q, stats = queries(131, B, 4, n, 64), torch.empty(B, 4, n, device="cuda")
    clean = A.attention_cached(Q, c, t, L, **kw)
    bad = torch.zeros(B, 4, n, dtype=torch.bool, device="cuda")
    for b, h, i, x in ((0, 1, 0, "nan"), (B - 1, 2, n - 1, "inf"), (B - 1, 0, n // 2, "-inf")):
        Q[b, h, i, 7] = float(x)
        bad[b, h, i] = True
    O = A.attention_cached(Q, c, t, L, stats=stats, **kw)
    assert torch.isnan(O[bad]).all() and torch.isnan(stats[bad]).all()
    assert torch.equal(O[~bad], clean[~bad]) and torch.isfinite(stats[~bad]).all()
    # a key of the last sequence's first page, second k/v head: heads 2 and 3
    (c.k if dtype == "bf16" else c.k.view(torch.uint8))[(B - 1) * width, 1, 3, 5] = float("nan") if dtype == "bf16" else 0x7f
    bad[B - 1, 2:] = True
    O = A.attention_cached(Q, c, t, L, stats=stats, **kw)
    assert torch.isnan(O[bad]).all() and torch.isnan(stats[bad]).all()
    assert torch.equal(O[~bad], clean[~bad]) and torch.isfinite(stats[~bad]).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [1024, 128])
@pytest.mark.parametrize("H_q", [2, 16, 32])  # (how many threads add up a row's partial results)
def test_bad_values_of_vanishing_weight(A, dtype, chunk, H_q):
    # a NaN value whose weight is too small for 32 bits (e^-256 of the others) makes its column NaN, in the same range of keys and in another
    page, width = 16, 32
    c = make(A, 140, width, 1, page, 64, 64, dtype)
    k = torch.zeros(1, 1, 512, 64, dtype=torch.bfloat16, device="cuda")
    k[:, :, :64] = 4.0
    c.append(k, torch.randn(1, 1, 512, 64, generator=torch.Generator().manual_seed(141)).to(torch.bfloat16).cuda(), torch.arange(512, dtype=torch.int32).cuda())
    t, L = torch.arange(width, dtype=torch.int32).view(1, width).cuda(), torch.tensor([500], dtype=torch.int32).cuda()
    Q = torch.ones(1, H_q, 1, 64, dtype=torch.bfloat16, device="cuda")
    clean = A.attention_cached(Q, c, t, L, scale=1.0, chunk=chunk)
    (c.v if dtype == "bf16" else c.v.view(torch.uint8))[20, 0, 3, 9] = float("nan") if dtype == "bf16" else 0x7f  # key 323
    O = A.attention_cached(Q, c, t, L, scale=1.0, chunk=chunk)
    others = [d for d in range(64) if d != 9]
    assert torch.isnan(O[..., 9]).all() and torch.equal(O[..., others], clean[..., others]) and torch.isfinite(clean).all()


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("B,H_q,H_kv,n,page,prefix,chunk,bad,scale", [
    (7, 16, 2, 5, 16, 333, 0, [0, 3, 20], 0.1),      # pages that are no pages in the first tile of 64 keys, two of its four, and the last page
    (7, 16, 2, 5, 32, 1000, 256, [1, 8, 31], -0.1),  # in the first tile, in front of the second range, the last page; a negative scale
    (5, 12, 1, 3, 16, 64, 0, [], 0.1),               # one whole tile
    (3, 40, 1, 1, 16, 65, 0, [4], 0.1),              # the second tile's only key is hidden
    (9, 40, 1, 1, 32, 129, 128, [4], -0.1),          # the second range has no other key
    (9, 40, 1, 1, 16, 400, 128, [0, 1, 2, 3, 12, 13, 14, 15], 0.1),  # whole tiles, the first one of a range among them
    (260, 8, 1, 1, 16, 200, 0, [5], 0.1),            # 2080 rows
    (4, 64, 8, 6, 64, 700, 0, [0], -0.1),
    (2, 34, 2, 2, 16, 5, 0, [], 0.1),                # a few keys
    (2, 34, 2, 2, 32, 70, 0, [0, 1, 2], 0.1),        # no key at all
])
def test_prefix_in_a_launch_of_its_own(A, dqk, dv, dtype, B, H_q, H_kv, n, page, prefix, chunk, bad, scale):
    pp, own = -(-prefix // page), n + 30
    width = -(-own // page)
    n_pages = pp + 1 + B * width
    c = make(A, 150, n_pages, H_kv, page, dqk, dv, dtype)
    order = torch.randperm(n_pages - 1, generator=torch.Generator().manual_seed(151)).to(torch.int32) + 1  # (page 0 holds NaN)
    ptab, t = order[:pp].clone(), order[pp: pp + B * width].view(B, width).clone()
    for i in bad:
        ptab[i] = -1 if i % 2 else n_pages
    lengths = [n + (7 * b) % (own - n) for b in range(B)]
    spoil_behind(c, list(t) + [ptab], lengths + [prefix])
    Q, stats, out = queries(152, B, H_q, n, dqk), torch.empty(B, H_q, n, device="cuda"), torch.empty(B, H_q, n, dv, device="cuda")
    plan = A.CachedAttentionPlan(c, Q, out, max_length=max(lengths), table_width=width, scale=scale, prefix_length=prefix, chunk=chunk)
    assert A.ae_cached_query(plan.handle)["launches"] == 2
    plan.forward(Q, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), out, stats=stats, prefix_table=ptab.cuda())
    kv = values(c)
    live = [j for j in range(prefix) if 0 <= int(ptab[j // page]) < n_pages]
    pre = [np.stack([x[int(ptab[j // page]), :, j % page] for j in live], axis=1) if live else np.zeros((H_kv, 0, x.shape[3])) for x in kv]
    some = sorted({0, 1, B // 2, B - 2, B - 1})
    rows = [[np.concatenate((p, listed(x, t[b].tolist(), lengths[b])), axis=1) for b in some] for p, x in zip(pre, kv)]
    check(out[some], stats[some], Q[some], *rows, scale, f"{B} x {H_q}/{H_kv} x {n} behind {prefix}, page {page}, {dqk}/{dv} {dtype}")


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,n,page,chunk,prefix", [(4, 4, 40, 16, 0, 0), (6, 2, 130, 32, 128, 0), (3, 1, 700, 64, 256, 0), (2, 1, 33, 16, 0, 90)])
def test_many_new_tokens(A, dqk, dv, dtype, H_q, H_kv, n, page, chunk, prefix):
    # a prompt's piece: tokens whose visible keys end in different tiles; a sequence that has no more keys than those, and one that has fewer
    lengths = [n, n + 77, 2 * n + 301] + ([] if prefix else [n // 2])
    B, width, pp = len(lengths), -(-max(lengths) // page), -(-prefix // page)
    n_pages = pp + sum(-(-x // page) for x in lengths) + 1
    c = make(A, 160, n_pages, H_kv, page, dqk, dv, dtype)
    t, ptab = tables_for(161, n_pages, lengths, page, width, first=pp), torch.arange(pp, dtype=torch.int32)
    spoil_behind(c, list(t) + [ptab], lengths + [prefix])
    Q, stats = queries(162, B, H_q, n, dqk), torch.empty(B, H_q, n, device="cuda")
    kw = dict(prefix_table=ptab.cuda(), prefix_length=prefix) if prefix else {}
    O = A.attention_cached(Q, c, t.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), scale=dqk ** -0.5, chunk=chunk, stats=stats, **kw)
    kv = values(c)
    rows = [[np.concatenate((listed(x, ptab.tolist(), prefix), listed(x, t[b].tolist(), lengths[b])), axis=1) for b in range(B)] for x in kv]
    check(O, stats, Q, *rows, dqk ** -0.5, f"{n} new tokens, {dqk}/{dv} {dtype} {H_q}/{H_kv} page {page} chunk {chunk} prefix {prefix}")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,length,chunk", [(40, 40, 0), (40, 95, 128), (130, 300, 128), (130, 300, 0), (700, 900, 0)])
def test_special_values_among_many_new_tokens(A, dtype, n, length, chunk):
    # NaN in values and keys of new tokens in different tiles of keys: rows that do not see them keep their bits
    page = 16
    c = make(A, 170, -(-length // page) + 1, 2, page, 64, 64, dtype)
    t = torch.randperm(c.n_pages - 1, generator=torch.Generator().manual_seed(171)).to(torch.int32).view(1, -1) + 1
    Q, L = queries(172, 1, 4, n, 64), torch.tensor([length], dtype=torch.int32).cuda()
    run = lambda: A.attention_cached(Q, c, t.cuda(), L, scale=0.125, chunk=chunk)
    clean = run()
    nan = float("nan") if dtype == "bf16" else 0x7f
    K, V = (x if dtype == "bf16" else x.view(torch.uint8) for x in (c.k, c.v))
    first = length - n  # key of the first new token
    seen = torch.zeros(4, n, 64, dtype=torch.bool)
    for i, head, d in ((1, 0, 5), (n // 2, 1, 9), (n // 2 + 1, 0, 33), (n - 2, 0, 60)):
        V[int(t[0, (first + i) // page]), head, (first + i) % page, d] = nan
        seen[2 * head: 2 * head + 2, i:, d] = True
    i = n - 5
    K[int(t[0, (first + i) // page]), 1, (first + i) % page, 0] = nan
    seen[2:, i:] = True
    O = run()[0].cpu()
    assert torch.isnan(O[seen]).all() and torch.equal(O[~seen], clean[0].cpu()[~seen])


@pytest.mark.parametrize("dqk,dv,dtype", [(64, 64, "bf16"), (128, 128, "e4m3")])
@pytest.mark.parametrize("B,H_q,H_kv", [(16, 8, 2), (40, 2, 2), (16, 6, 2), (10, 12, 2), (6, 24, 2)])
def test_same_bits_whoever_is_last(A, dqk, dv, dtype, B, H_q, H_kv):
    # in the launch that walks the prefix too, a workgroup of either kind may be the last of a sequence, which joins the partial results: with
    # a page of own keys those of the prefix are, with thousands of hidden ones behind it those of the own list (their ranges come
    # later and outnumber the places)
    page, prefix, long = 16, 8192, 40000
    pp, width = prefix // page, long // page
    c = make(A, 180, pp + B, H_kv, page, dqk, dv, dtype)
    order = torch.randperm(pp + B, generator=torch.Generator().manual_seed(181)).to(torch.int32).cuda()
    ptab, t = order[:pp].contiguous(), torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    t[:, 0] = order[pp:]
    Q, out, stats = queries(182, B, H_q, 1, dqk), torch.empty(B, H_q, 1, dv, device="cuda"), torch.empty(B, H_q, 1, device="cuda")
    plan = A.CachedAttentionPlan(c, Q, out, max_length=long, table_width=width, scale=dqk ** -0.5, prefix_length=prefix, chunk=1024)
    assert A.ae_cached_query(plan.handle)["launches"] == 1
    got = []
    for n in (page, long, page, long, page, long):
        plan.forward(Q, t, torch.full((B,), n, dtype=torch.int32, device="cuda"), out, stats=stats, prefix_table=ptab)
        got.append((out.clone(), stats.clone()))
    for o, s in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(s, got[0][1])
