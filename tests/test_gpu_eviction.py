"""GPU parity of the weights that cached entries receive (ae_weigh_forward) and of their eviction (ae_evict_forward), and a serving loop that uses both.

Bounds.  What an entry receives is a sum over at most R rows of exp(s - stat), s off by e (D 2^-24 |scale| sum |q k|, 4e-7 of the cap or of the largest
score), the exponent, formed in powers of two, by 2^-22 of |s| + |stat|, its power by 2^-22 of itself; the sum of R + 1 terms adds (R + 1) 2^-24.  An
eviction rounds nothing: whole lists, rows and weights are equal."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import dequantise, kept_entries, received
from oracle.span_oracle import span_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bits(t):
    return t if t.dtype in (torch.uint8, torch.bfloat16) else t.view(torch.uint8)


def setup(A, seed, H_kv, page, lengths, dqk, dv, dtype, spoil=True):
    """A cache of N(0, 1) rows, shuffled page lists (with room for a page more), NaN behind their ends."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(n, 0) // page) for n in lengths]
    width, n_pages = max(need) + 1, sum(need) + len(need) + 1
    c = A.PagedCache.empty(n_pages, H_kv, page, dqk, dv, dtype=dtype)
    k, v = (torch.randn(1, H_kv, n_pages * page, d, generator=g).to(torch.bfloat16).cuda() for d in (dqk, dv))
    c.append(k, v, torch.arange(n_pages * page, dtype=torch.int32).cuda()[None])
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table, at = torch.full((len(lengths), width), -9, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, : n + 1] = order[at: at + n + 1]
        at += n + 1
    if spoil:
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lengths):
            for j in range(n):
                used[table[b, j // page], j % page] = True
        rest = ~used.cuda()
        for t in (c.k, c.v):
            (t if dtype == "bf16" else t.view(torch.uint8)).transpose(1, 2)[rest] = float("nan") if dtype == "bf16" else 0x7f
    return c, table


def values(pages, exps):
    return pages.cpu().double().numpy() if exps is None else dequantise(pages.view(torch.uint8).cpu().numpy(), exps.cpu().numpy())


def rows_of(pages, table, length):
    """[H, length, D] of a page list; zeros on a page outside the cache."""
    page = pages.shape[2]
    out = np.zeros((pages.shape[1], length, pages.shape[3]))
    for j in range(length):
        if 0 <= table[j // page] < pages.shape[0]:
            out[:, j] = pages[table[j // page], :, j % page]
    return out


def queries(seed, B, H, n, D):
    return (1.5 * torch.randn(B, n, H, D, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda().transpose(1, 2)


def check_received(got, was, Q, keys, stats, n, scale, cap):
    """got, was: [B, H_kv, capacity] of the call; entries behind the list keep what was there."""
    for b in range(Q.shape[0]):
        L, R = keys[b].shape[1], Q.shape[1] * n // keys[b].shape[0]
        assert torch.equal(got[b, :, L:], was[1][b, :, L:]), "an entry behind the list"
        if L == 0:
            continue
        q, s = Q[b].cpu().double().numpy(), stats[b].cpu().double().numpy()
        ref = received(q, keys[b], s, scale, cap)
        old = was[0][b, :, :L].cpu().double().numpy().copy()
        old[:, max(0, L - n):] = 0.0
        most = abs(scale) * float(np.abs(q).max((0, 1)) @ np.nan_to_num(np.abs(keys[b])).max((0, 1)))
        e = q.shape[2] * 2.0 ** -24 * most + 4e-7 * min(cap, most) + 2.0 ** -22 * (most + np.abs(s[np.isfinite(s)]).max(initial=0.0)) + 2.0 ** -21
        bound = 2 * e * ref + (R + 1) * 2.0 ** -24 * (ref + np.abs(old))
        off = np.abs(got[b, :, :L].cpu().double().numpy() - (ref + old))
        assert np.all(off <= bound + 1e-30), (b, float(np.nanmax(off - bound)), int(np.isnan(off).sum()))


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("cap", [0.0, 6.0])
@pytest.mark.parametrize("H_q,H_kv,n,page,lengths", [
    (1, 1, 1, 16, [1]),
    (32, 8, 1, 64, [777, 300, 64, 1, 0]),
    (6, 2, 3, 16, [3, 2, 50, 33, 160]),
    (8, 8, 37, 32, [400, 37, 30, 129]),
    (16, 1, 9, 128, [257, 9]),
    (4, 2, 130, 16, [130, 290]),
])
def test_weights_match_definition(A, dqk, dv, dtype, cap, H_q, H_kv, n, page, lengths):
    """One token and many, more new tokens than keys, lists that end inside a tile, garbage behind them."""
    c, t = setup(A, 1, H_kv, page, lengths, dqk, dv, dtype)
    Q, B, scale, room = queries(2, len(lengths), H_q, n, dqk), len(lengths), dqk ** -0.5, max(lengths) + 5
    stats = torch.empty(B, H_q, n, device="cuda")
    A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=scale, cap=cap, stats=stats)
    W = torch.rand(B, H_kv, room, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) * 4
    for b, L in enumerate(lengths):
        W[b, :, max(0, L - n): L] = float("nan")  # what new entries held does not matter
    P = torch.full((B, H_kv, room), -5, dtype=torch.int32, device="cuda")
    new = ints(100 * np.arange(B)[:, None] + np.arange(n))
    was, out = W.clone(), torch.full_like(W, 7.0)
    A.cache_weights(Q, c, t.cuda(), ints(lengths), stats, W, P, new, scale=scale, cap=cap, max_length=max(lengths), out=out)
    assert torch.equal(W.nan_to_num(-1), was.nan_to_num(-1))
    keys = [rows_of(values(c.k, c.k_exp), t[b].tolist(), lengths[b]) for b in range(B)]
    check_received(out, (was, torch.full_like(W, 7.0)), Q, keys, stats, n, scale, cap)
    for b, L in enumerate(lengths):
        want = np.full(room, -5)
        for j in range(max(0, L - n), L):
            want[j] = 100 * b + j - (L - n)
        assert (P[b].cpu().numpy() == want).all()
    got = A.cache_weights(Q, c, t.cuda(), ints(lengths), stats, W, scale=scale, cap=cap)  # in place, without positions, up to the room
    assert got is W
    for b, L in enumerate(lengths):
        assert torch.equal(W[b, :, :L], out[b, :, :L])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_weights_of_pages_outside_and_rows_that_give_nothing(A, dtype):
    lengths, page, n = [100, 70, 40], 16, 2
    c, t = setup(A, 4, 2, page, lengths, 64, 64, dtype)
    t[0, 2], t[0, 6], t[1, 0], t[1, 3] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    t[2, :] = -1
    Q, stats = queries(5, 3, 4, n, 64), torch.empty(3, 4, n, device="cuda")
    A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=-0.125, stats=stats)
    assert torch.isneginf(stats[2]).all()
    stats[0, 1] = stats[1, 0, 1] = float("-inf")
    W = torch.rand(3, 2, 112, device="cuda")
    was = W.clone()
    A.cache_weights(Q, c, t.cuda(), ints(lengths), stats, W, scale=-0.125)
    keys = [rows_of(values(c.k, c.k_exp), t[b].tolist(), lengths[b]) for b in range(3)]
    for b in range(3):  # hidden keys: a score of 0 in the definition, which is not what they get
        for j in range(lengths[b]):
            if not 0 <= int(t[b, j // page]) < c.n_pages:
                old = 0.0 if j >= lengths[b] - n else was[b, :, j]
                assert (W[b, :, j] == old).all()
                W[b, :, j] = torch.tensor(received(Q[b].cpu().double().numpy(), keys[b], stats[b].cpu().numpy(), -0.125)[:, j], device="cuda").float() + old
    check_received(W, (was, was), Q, keys, stats, n, -0.125, 0.0)


def test_weights_and_special_values(A):
    """A NaN key has a NaN weight and no other one has; a row with the statistic -inf gives nothing even to that; a query of NaN reaches its k/v head."""
    c, t = setup(A, 6, 2, 16, [60], 64, 64, "bf16")
    Q, stats = queries(7, 1, 4, 1, 64), torch.empty(1, 4, 1, device="cuda")
    A.attention_cached(Q, c, t.cuda(), ints([60]), scale=0.1, stats=stats)
    W = lambda: torch.zeros(1, 2, 60, device="cuda")
    clean = A.cache_weights(Q, c, t.cuda(), ints([60]), stats, W(), scale=0.1)
    c.k[int(t[0, 1]), 0, 4, 9] = float("nan")
    got = A.cache_weights(Q, c, t.cuda(), ints([60]), stats, W(), scale=0.1)
    assert torch.isnan(got[0, 0, 20])
    got[0, 0, 20] = clean[0, 0, 20]
    assert torch.equal(got, clean)
    none = torch.full_like(stats, float("-inf"))
    assert (A.cache_weights(Q, c, t.cuda(), ints([60]), none, W(), scale=0.1) == 0).all()
    Q2 = Q.clone()
    Q2[0, 3, 0, 0] = float("nan")
    got = A.cache_weights(Q2, c, t.cuda(), ints([60]), stats, W(), scale=0.1)
    assert torch.isnan(got[0, 1]).all() and torch.isnan(got[0, 0]).sum() == 1


def test_weights_behind_a_prefix(A):
    """The prefix takes its part of every row; the entries' own weights and what is missing add up."""
    page, lengths = 32, [90, 200]
    c, t = setup(A, 8, 2, page, lengths + [64], 128, 128, "bf16")
    pre, t = t[2, :2].cuda(), t[:2].contiguous()
    Q, stats = queries(9, 2, 8, 1, 128), torch.empty(2, 8, 1, device="cuda")
    A.attention_cached(Q, c, t.cuda(), ints(lengths), scale=0.09, stats=stats, prefix_table=pre, prefix_length=64)
    W = torch.zeros(2, 2, 224, device="cuda")
    A.cache_weights(Q, c, t.cuda(), ints(lengths), stats, W, scale=0.09)
    keys = [rows_of(values(c.k, None), t[b].tolist(), lengths[b]) for b in range(2)]
    check_received(W, (torch.zeros_like(W),) * 2, Q, keys, stats, 1, 0.09, 0.0)
    assert (W.sum(-1) < 4).all() and (W.sum(-1) > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_weights_strides_expanded_rows_and_shared_positions(A, dtype):
    c, t = setup(A, 10, 2, 32, [70, 40], 64, 64, dtype)
    L = ints([70, 40])
    one = (torch.randn(64, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16).cuda().expand(2, 4, 3, 64)
    stats = torch.empty(2, 4, 3, device="cuda")
    A.attention_cached(one, c, t.cuda(), L, scale=0.1, stats=stats)
    W, P = torch.zeros(2, 2, 96, device="cuda"), torch.zeros(2, 2, 96, dtype=torch.int32, device="cuda")
    A.cache_weights(one, c, t.cuda(), L, stats, W, P, ints([5, 6, 7]), scale=0.1)
    W2 = A.cache_weights(one.contiguous(), c, t.cuda(), L, stats, torch.zeros_like(W), scale=0.1)
    assert torch.equal(W, W2) and P[0, 1, 67:70].tolist() == [5, 6, 7] and P[1, 0, 37:40].tolist() == [5, 6, 7] and (P > 0).sum() == 12


def make_lists(seed, B, H_kv, room, levels=0):
    """Weights (with `levels`: only so many different ones) and distinct positions in any order."""
    g = np.random.RandomState(seed)
    W = g.rand(B, H_kv, room).astype(np.float32) ** 3 * 9
    if levels:
        W = np.floor(W / 9 * levels).astype(np.float32)
    P = np.stack([[g.permutation(2 * room)[:room] for _ in range(H_kv)] for _ in range(B)]).astype(np.int32)
    return W, P


def check_eviction(A, c, t, lengths, W, P, keep, recent, sinks, max_length=None, in_place=False):
    B, H_kv, room = W.shape
    max_length = max_length or room
    real = [min(max(n, 0), max_length) for n in lengths]
    w, p, page = torch.tensor(W, device="cuda"), ints(P), c.page_size
    want = [bits(x).clone() if x is not None else None for x in (c.k, c.v, c.k_exp, c.v_exp)]
    wo, po = (w, p) if in_place else (torch.full_like(w, -3.0), torch.full_like(p, -3))
    ww, wp = wo.cpu().numpy().copy(), po.cpu().numpy().copy()
    src, dst, heads = [], [], []
    for b in range(B):
        for h in range(H_kv):
            holds = kept_entries(W[b, h, : real[b]], P[b, h, : real[b]], keep, recent, sinks)
            ww[b, h, : len(holds)], wp[b, h, : len(holds)] = W[b, h, holds], P[b, h, holds]
            for i, j in enumerate(holds):
                if i != j:
                    a, z = int(t[b, j // page]), int(t[b, i // page])
                    if 0 <= a < c.n_pages and 0 <= z < c.n_pages:
                        src.append((a, j % page)), dst.append((z, i % page)), heads.append(h)
    if src:
        s, d, h = np.array(src), np.array(dst), np.array(heads)
        for x in want:
            if x is not None:
                x[d[:, 0], h, d[:, 1]] = x[s[:, 0], h, s[:, 1]]
    out = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    plan = A.CacheEvictionPlan(c, w, keep=keep, recent=recent, sinks=sinks, max_length=max_length, table_width=t.shape[1])
    plan.forward(t.cuda(), ints(lengths), w, p, out, weights_out=wo, positions_out=po)
    assert out.tolist() == [min(n, keep) for n in real]
    assert np.array_equal(wo.cpu().numpy().view(np.uint32), ww.view(np.uint32)) and np.array_equal(po.cpu().numpy(), wp)
    for got, x in zip((c.k, c.v, c.k_exp, c.v_exp), want):
        if x is not None:
            got = bits(got)
            same = got == x if x.dtype == torch.uint8 else got.view(torch.int16) == x.view(torch.int16)
            assert same.all(), int((~same).sum())


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,lengths,keep,recent,sinks,levels", [
    (16, [1], 1, 0, 0, 0),
    (64, [300, 100, 101, 0, 99], 100, 25, 4, 0),
    (32, [500, 33, 400], 65, 0, 0, 5),
    (16, [200, 190], 17, 17, 0, 0),
    (128, [700, 650], 512, 600, 3, 3),
    (256, [900, 1], 1, 0, 1, 1),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_eviction_matches_definition(A, dqk, dv, dtype, page, lengths, keep, recent, sinks, levels, in_place):
    """Nothing to do, half a list, most of it; ties; protected entries alone, more of them than stay; a page border inside."""
    c, t = setup(A, 20, 2, page, lengths, dqk, dv, dtype)
    W, P = make_lists(21, len(lengths), 2, max(lengths) + 3, levels)
    check_eviction(A, c, t, lengths, W, P, keep, recent, sinks, max_length=max(lengths), in_place=in_place)


@pytest.mark.parametrize("L,keep", [(4095, 1000), (4097, 4000), (8000, 100), (16384, 8192), (16385, 2048), (33000, 30000), (65536, 512), (65537, 40000), (150001, 7)])
def test_eviction_of_long_lists(A, L, keep):
    """Every variant of the selection, with ties over the whole list."""
    lengths = [L, L - 1000]
    c, t = setup(A, 22, 1, 256, lengths, 64, 64, "e4m3", spoil=False)
    W, P = make_lists(23, 2, 1, L, levels=L // 3)
    check_eviction(A, c, t, lengths, W, P, keep, keep // 4, 4, in_place=L % 2 == 0)


def test_eviction_of_special_weights(A):
    """NaN below all, infinities, both zeros alike, subnormal numbers in order, negative ones; positions at both ends of their range."""
    L = 1200
    c, t = setup(A, 24, 2, 32, [L, 800], 64, 64, "bf16")
    g = np.random.RandomState(25)
    W = g.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, 3e-45, 1e-39, -1e-40, -2.0, 7.0, 3e38], dtype=np.float32), (2, 2, L))
    W[0, 0, 5] = np.array([0xffc00001], dtype=np.uint32).view(np.float32)[0]
    P = g.randint(-2 ** 31, 2 ** 31, (2, 2, L)).astype(np.int32)
    P[:, :, 3], P[:, :, 9] = -2 ** 31, 2 ** 31 - 1
    for keep, recent, sinks in ((L - 1, 0, 0), (600, 1, 0), (300, 0, 0), (90, 2 ** 31 - 1, 0), (50, 0, 2 ** 31 - 1)):
        check_eviction(A, c, t, [L, 800], W, P, keep, recent, sinks)


def test_eviction_with_lengths_and_pages_outside(A):
    """Lengths below zero and beyond the most; rows that would come from or go to a page outside the cache are not copied."""
    c, t = setup(A, 26, 2, 16, [160, 160, 160], 64, 64, "e4m3")
    t[0, 0], t[0, 9], t[1, 3], t[1, 7] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    W, P = make_lists(27, 3, 2, 170)
    check_eviction(A, c, t, [160, 160, -4], W, P, 70, 10, 2, max_length=160)
    check_eviction(A, c, t, [160, 5000, 0], W, P, 150, 0, 0, max_length=160)
    check_eviction(A, c, t, [160, 3, 100], W, P, 500, 0, 0, max_length=160)


def test_eviction_gives_the_same_bits_on_two_streams(A):
    """Two plans at once on lists of their own."""
    made = []
    for seed in (30, 31):
        c, t = setup(A, seed, 2, 64, [2000, 1500], 128, 128, "bf16")
        W, P = make_lists(seed, 2, 2, 2000, levels=300)
        made.append((c, t.cuda(), ints([2000, 1500]), torch.tensor(W, device="cuda"), ints(P)))
    want = []
    for c, t, L, W, P in made:
        k, v, w, p = c.k.clone(), c.v.clone(), W.clone(), P.clone()
        n = A.cache_evict(A.PagedCache(k, v), t, L, w, p, keep=900, recent=100, sinks=2)
        want.append((k, v, w, p, n))
    torch.cuda.synchronize()
    got = []
    for c, t, L, W, P in made:
        s = torch.cuda.Stream()
        got.append((c.k, c.v, W, P, A.cache_evict(c, t, L, W, P, keep=900, recent=100, sinks=2, stream=s)))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert torch.equal(x.nan_to_num(-1.0) if x.is_floating_point() else x, y.nan_to_num(-1.0) if y.is_floating_point() else y)


class Model:
    """What the loop below should do, in 64 bits: a list of entries per k/v head."""

    def __init__(self, H_kv):
        self.e = [[] for _ in range(H_kv)]  # [key, value, weight, position]

    def append(self, k, v, positions):
        for h, e in enumerate(self.e):
            e.extend([k[h, i], v[h, i], 0.0, positions[i]] for i in range(len(positions)))

    def attend(self, q, scale, cap):
        H_q, n, _ = q.shape
        g, out, lse = H_q // len(self.e), np.zeros((H_q, n, len(self.e[0][0][1]))), np.zeros((H_q, n))
        for h in range(H_q):
            e = self.e[h // g]
            k, v = np.array([x[0] for x in e])[None, None], np.array([x[1] for x in e])[None, None]
            L = len(e)
            end = (L - n + 1 + np.arange(n))[None]
            o, s, _ = span_attention(q[None, h: h + 1], k, v, 0 * end, end, scale=scale, cap=cap)
            out[h], lse[h] = o[0, 0], s[0, 0]
        return out, lse

    def weigh(self, q, lse, scale, cap):
        got = received(q, np.array([[x[0] for x in e] for e in self.e]), lse, scale, cap)
        for h, e in enumerate(self.e):
            for x, w in zip(e, got[h]):
                x[2] += w

    def evict(self, keep, recent, sinks):
        for h, e in enumerate(self.e):
            self.e[h] = [e[i] for i in kept_entries([x[2] for x in e], [x[3] for x in e], keep, recent, sinks)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_a_serving_loop_that_evicts(A, dtype, cap):
    """A prompt in pieces, then single tokens: append, attend, weigh, evict once the list has grown over its room; every output, the entries that stay and
    their weights against the same loop in 64 bits.  The single steps run from a captured graph as well."""
    H_q, H_kv, D, page, keep, room, scale = 4, 2, 64, 16, 40, 64, 0.125
    c = A.PagedCache.empty(2 * room // page + 1, H_kv, page, D, D, dtype=dtype)
    table = ints([[3, 0, 7, 5], [1, 8, 2, 6]])
    W, P = torch.zeros(2, H_kv, room, device="cuda"), torch.zeros(2, H_kv, room, dtype=torch.int32, device="cuda")
    L = ints([0, 0])
    models = [Model(H_kv) for _ in range(2)]
    g = torch.Generator().manual_seed(40)
    seen = 0

    def tokens(n):
        q, k, v = (torch.randn(2, H, n, D, generator=g).to(torch.bfloat16) for H in (H_q, H_kv, H_kv))
        if dtype == "e4m3":  # on the grid of the cache: nothing is rounded on the way
            k, v = (x.float().to(torch.float8_e4m3fn).to(torch.bfloat16) for x in (k, v))
        return q, k, v

    plans = {}

    def step(q, k, v, pos, out, stats):
        n = q.shape[2]
        if n not in plans:
            plans[n] = (A.CachedAttentionPlan(c, q, out, max_length=room, table_width=4, scale=scale, cap=cap),
                        A.CacheWeightsPlan(c, q, W, max_length=room, table_width=4, scale=scale, cap=cap),
                        A.CacheEvictionPlan(c, W, keep=keep, recent=8, sinks=2, max_length=room, table_width=4))
        attention, weigh, evict = plans[n]
        at = L.view(2, 1) + torch.arange(n, device="cuda", dtype=torch.int32)
        c.append(k, v, torch.gather(table, 1, (at // page).long()) * page + at % page)
        L.add_(n)
        attention.forward(q, table, L, out, stats=stats)
        weigh.forward(q, table, L, stats, W, P, pos)
        new = torch.empty_like(L)
        evict.forward(table, L, W, P, new)
        L.copy_(new)

    def check(q, k, v, pos, out, stats):
        n = q.shape[2]
        for b, m in enumerate(models):
            m.append(k[b].double().numpy(), v[b].double().numpy(), pos)
            o, lse = m.attend(q[b].double().numpy(), scale, cap)
            # weights rounded to bf16, 2^-8 of values up to 5; the scores' errors are below 1e-5
            assert np.abs(out[b].cpu().double().numpy() - o).max() <= (2.0 ** -8 + 1e-4) * 5 and np.abs(stats[b].cpu().numpy() - lse).max() <= 1e-4
            m.weigh(q[b].double().numpy(), lse, scale, cap)
            m.evict(keep, 8, 2)
            size = len(m.e[0])
            assert int(L[b]) == size
            for h in range(H_kv):
                assert P[b, h, :size].tolist() == [x[3] for x in m.e[h]], "the entries that stay"
                want = np.array([x[2] for x in m.e[h]])
                assert np.abs(W[b, h, :size].cpu().numpy() - want).max() <= 1e-4 * (1 + want.max())

    for n in (30, 20, 7):
        q, k, v = tokens(n)
        pos = list(range(seen, seen + n))
        out, stats = torch.empty(2, H_q, n, D, device="cuda"), torch.empty(2, H_q, n, device="cuda")
        step(q.cuda(), k.cuda(), v.cuda(), ints(pos), out, stats)
        check(q, k, v, pos, out, stats)
        seen += n
    q1, k1, v1 = (x.cuda() for x in tokens(1))
    pos1, out, stats = ints([0]), torch.empty(2, H_q, 1, D, device="cuda"), torch.empty(2, H_q, 1, device="cuda")
    graph = None
    for i in range(12):
        q, k, v = tokens(1)
        for a, x in ((q1, q), (k1, k), (v1, v)):
            a.copy_(x)
        pos1.fill_(seen)
        if i % 4 == 3:
            if graph is None:
                torch.cuda.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step(q1, k1, v1, pos1, out, stats)
            graph.replay()
        else:
            step(q1, k1, v1, pos1, out, stats)
        check(q, k, v, [seen], out, stats)
        seen += 1


def test_refusals_of_the_binding(A):
    c, t = setup(A, 50, 2, 16, [40], 64, 64, "bf16")
    Q, L, td = queries(51, 1, 4, 1, 64), ints([40]), t.cuda()
    W, P, S = torch.zeros(1, 2, 48, device="cuda"), torch.zeros(1, 2, 48, dtype=torch.int32, device="cuda"), torch.zeros(1, 4, 1, device="cuda")
    ok = dict(scale=0.1)
    for args in ((Q.float(), c, td, L, S, W), (Q, c, td, L, S[:, :2], W), (Q, c, td, L, S, W.double()), (Q, c, td, L, S, W[:, :1]), (Q, c, td, L.long(), S, W),
                 (Q, c, td, L, S, W, P), (Q, c, td, L, S, W, P.long(), ints([1])), (Q, c, td, L, S, W, P, ints([1, 2])), (Q, c, td, L, S, W[..., ::2]),
                 (Q, c, td.cpu(), L, S, W)):
        with pytest.raises(ValueError):
            A.cache_weights(*args, **ok)
    with pytest.raises(A.AeAttnError):
        A.cache_weights(Q, c, td, L, S, W, scale=0.1, max_length=49)
    with pytest.raises(A.AeAttnError):
        A.cache_weights(Q, c, td, L, S, W, scale=0.0)
    for args in ((c, td, L, W.double(), P), (c, td, L, W, P.float()), (c, td, L.long(), W, P), (c, td.cpu(), L, W, P), (c, td, L, W, P[..., :40])):
        with pytest.raises(ValueError):
            A.cache_evict(*args, keep=8)
    with pytest.raises(A.AeAttnError):
        A.cache_evict(c, td, L, W, P, keep=0)
    with pytest.raises(A.AeAttnError):
        A.cache_evict(c, td, L, W, P, keep=8, lengths_out=L)
