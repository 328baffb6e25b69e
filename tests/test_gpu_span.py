"""GPU parity of span attention (ae_span_forward, ae_span_backward) against its 64-bit definition.

Bounds.  Products of bf16 values are exact in fp32, a score's sum of D of them is off by at most D 2^-24 sum |q k|; a capped score adds 4e-7 of the
cap or of the largest score, whichever is less (series: 2e-7 of the score; else, beyond 0.6 of the cap, an exponential and a reciprocal, an ulp each, times
twice the cap), a distance 2^-22 of the term.
e_s, their sum over the case, is the exponents' absolute error and the weights' relative one; of a normalised weight 2 e_s.  A weight is rounded once
to bf16: half a step, 2^-8 of it.  So |O - ref| <= (2^-8 + 2 e_s + 2^-20) sum_j p_j |v_j|, a bf16 result adds 2^-8 of itself, the statistic is within
e_s + 2^-20 (1 + |stat|).  Gradients: the oracle forms what these errors, the rounding of dS to bf16, and those of dP (D_v 2^-24 sum |dO v|) and
delta (D_v 2^-24 sum |dO O|, O being the definition's in fp32, so 2^-24 |O| more) amount to, element by element; sums over L add L 2^-24 of it."""
import numpy as np
import pytest
import torch

from oracle.span_oracle import document_spans, span_attention, span_attention_backward, spans_of

pytestmark = pytest.mark.gpu
DIMS = [(64, 64), (128, 128), (192, 128)]
SCORES = [dict(), dict(cap=12.0), dict(slopes=True), dict(cap=5.0, slopes=True)]


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def rows(seed, B, H, L, D, by=1.0, order="blhd"):
    g = torch.Generator().manual_seed(seed)
    if order == "blhd":
        return (torch.randn(B, L, H, D, generator=g) * by).to(torch.bfloat16).cuda().transpose(1, 2)
    return (torch.randn(B, H, L, D, generator=g) * by).to(torch.bfloat16).cuda()


def slopes_of(H):
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


def score_error(Q, K, scale, cap, slopes, L):
    q, k = Q.float().abs().amax(), K.float().abs()
    most = float((Q.float().abs().amax(dim=(0, 1, 2)) @ k.amax(dim=(0, 1, 2))))
    return Q.shape[3] * 2.0 ** -24 * abs(scale) * most + 4e-7 * min(cap, abs(scale) * most) + (2.0 ** -22 * max(map(abs, slopes)) * L if slopes else 0.0) + 2.0 ** -21


def host(t):
    return t.detach().float().cpu().double().numpy()


def spans_tensor(begin, end):
    return tuple(torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda") for x in (begin, end))


def run_forward(A, Q, K, V, begin, end, out_dtype=torch.bfloat16, mask="spans", spans=None, window=0, **kw):
    B, H_q, L_q, _ = Q.shape
    slopes = slopes_of(H_q) if kw.get("slopes") is True else kw.get("slopes")
    kw = dict(kw, slopes=slopes, scale=kw.get("scale", Q.shape[3] ** -0.5))
    out = torch.full((B, L_q, H_q, V.shape[3]), float("nan"), dtype=out_dtype, device="cuda").transpose(1, 2)
    stats = torch.full((B, H_q, L_q), float("nan"), device="cuda")
    if mask == "spans" and spans is None:
        spans = spans_tensor(begin, end)
    A.span_attention_forward(Q, K, V, mask=mask, spans=spans, window=window, out=out, stats=stats, **kw)
    ref, lse, mag = span_attention(host(Q), host(K), host(V), begin, end, scale=kw["scale"], cap=kw.get("cap", 0.0), slopes=slopes)
    e = score_error(Q, K, kw["scale"], kw.get("cap", 0.0), slopes, Q.shape[2] + K.shape[2])
    bound = (2.0 ** -8 + 2 * e + 2.0 ** -20) * mag
    if out_dtype == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    off = np.abs(host(out) - ref)
    assert np.all(off <= bound + 1e-30), f"output: {np.nanmax(off - bound):.3e} beyond its bound, nan {np.isnan(off).sum()}"
    got = host(stats)
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got), empty)
    off = np.abs(got[~empty] - lse[~empty])
    assert np.all(off <= e + 2.0 ** -20 * (1 + np.abs(lse[~empty]))), f"statistic: {off.max():.3e}"
    return out, stats


def run_backward(A, Q, K, V, dO, begin, end, o_dtype=torch.float32, grad_dtype=torch.bfloat16, mask="spans", spans=None, window=0, **kw):
    H_q = Q.shape[1]
    slopes = slopes_of(H_q) if kw.get("slopes") is True else kw.get("slopes")
    kw = dict(kw, slopes=slopes, scale=kw.get("scale", Q.shape[3] ** -0.5))
    cap = kw.get("cap", 0.0)
    ref, lse, _ = span_attention(host(Q), host(K), host(V), begin, end, scale=kw["scale"], cap=cap, slopes=slopes)
    O, stats = torch.tensor(ref, device="cuda").to(o_dtype), torch.tensor(lse, dtype=torch.float32, device="cuda")
    if mask == "spans" and spans is None:
        spans = spans_tensor(begin, end)
    got = A.span_attention_backward(Q, K, V, O, dO, stats, mask=mask, spans=spans, window=window, grad_dtype=grad_dtype, **kw)
    e = score_error(Q, K, kw["scale"], cap, slopes, Q.shape[2] + K.shape[2]) + 2.0 ** -23 * float(np.abs(lse[np.isfinite(lse)]).max(initial=0.0))
    do, d_v = np.abs(host(dO)), V.shape[3]
    half_o = 2.0 ** -24 if o_dtype == torch.float32 else 2.0 ** -8
    e_dp = d_v * 2.0 ** -24 * float((do.max((0, 1, 2)) @ np.abs(host(V)).max((0, 1, 2)))) + (d_v * 2.0 ** -24 + half_o) * float((do * np.abs(ref)).sum(-1).max())
    want, bounds = span_attention_backward(host(Q), host(K), host(V), host(dO), begin, end, scale=kw["scale"], cap=cap, slopes=slopes, e_p=e, e_dp=e_dp)
    L = max(Q.shape[2] * H_q // K.shape[1], K.shape[2])
    for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bounds):
        bound = b * (1 + 2.0 ** -7 + L * 2.0 ** -24) + (L * 2.0 ** -24 * 256 * b if L else 0)
        if grad_dtype == torch.bfloat16:
            bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(w)
        off = np.abs(host(g) - w)
        assert np.all(off <= bound + 1e-30), f"{name}: {np.nanmax(off - bound):.3e} beyond its bound, nan {np.isnan(off).sum()}"
    return got


def documents(seed, B, L, most, padding=0):
    """Offsets [B, n + 1] of documents of 1 to `most` tokens, the rows padded with empty ones."""
    g = np.random.RandomState(seed)
    out = []
    for _ in range(B):
        at = [0]
        while at[-1] < L - padding:
            at.append(min(L - padding, at[-1] + g.randint(1, most + 1)))
        out.append(at)
    n = max(map(len, out))
    return np.array([a + [a[-1]] * (n - len(a)) for a in out])


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("mask", ["none", "causal", "sliding_window", "documents", "prefix"])
def test_forward_and_backward(A, dims, score, mask):
    """Every kernel of the operator; several tiles, odd lengths, shared heads."""
    B, H_q, H_kv, L = 2, 4, 2, 333
    Q, K, V, dO = rows(1, B, H_q, L, dims[0], 2.0), rows(2, B, H_kv, L, dims[0]), rows(3, B, H_kv, L, dims[1]), rows(4, B, H_q, L, dims[1])
    kw = dict(score)
    if mask in ("documents", "prefix"):
        at = documents(5, B, L, 150, padding=9)
        prefix = np.random.RandomState(6).randint(0, 100, (B, at.shape[1] - 1)) if mask == "prefix" else None
        begin, end = document_spans(at, L, prefix=prefix)
    else:
        kw.update(mask=mask, window=70 if mask == "sliding_window" else 0)
        begin, end = spans_of(mask, B, L, L, kw["window"])
    run_forward(A, Q, K, V, begin, end, **kw)
    run_backward(A, Q, K, V, dO, begin, end, **kw)


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("L_q,L_k", [(1, 1), (1, 700), (2, 65), (31, 33), (257, 64), (64, 300), (300, 64), (513, 512)])
@pytest.mark.parametrize("mask", ["none", "causal", "sliding_window"])
def test_lengths(A, dims, L_q, L_k, mask):
    """One row, tiles' borders, more queries than keys (causal: the first rows see nothing) and fewer."""
    Q, K, V, dO = rows(1, 1, 3, L_q, dims[0], 2.0), rows(2, 1, 1, L_k, dims[0]), rows(3, 1, 1, L_k, dims[1]), rows(4, 1, 3, L_q, dims[1])
    window = 17 if mask == "sliding_window" else 0
    begin, end = spans_of(mask, 1, L_q, L_k, window)
    kw = dict(mask=mask, window=window, cap=9.0, slopes=True)
    run_forward(A, Q, K, V, begin, end, out_dtype=torch.float32, **kw)
    run_backward(A, Q, K, V, dO, begin, end, grad_dtype=torch.float32, **kw)


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("kind", ["unsorted", "outside", "some_empty", "all_empty", "one_key", "falling"])
def test_any_spans(A, dims, kind):
    """Spans in any order: overlapping, empty, beyond both ends of the keys; per batch entry and shared by the batch."""
    B, H, L_q, L_k = 2, 2, 290, 410
    g = np.random.RandomState(7)
    Q, K, V, dO = rows(1, B, H, L_q, dims[0]), rows(2, B, H, L_k, dims[0]), rows(3, B, H, L_k, dims[1]), rows(4, B, H, L_q, dims[1])
    begin = g.randint(0, L_k, (B, L_q))
    end = begin + g.randint(1, 200, (B, L_q))
    if kind == "outside":
        begin, end = begin - 300, end + 100
    elif kind == "some_empty":
        end = np.where(g.rand(B, L_q) < 0.4, begin - g.randint(0, 5, (B, L_q)), end)
        begin[:, 64:160] = end[:, 64:160] = 50
    elif kind == "all_empty":
        end = begin.copy()
    elif kind == "one_key":
        end = begin + 1
    elif kind == "falling":
        begin = np.tile(np.maximum(L_k - 1 - 2 * np.arange(L_q), 0), (B, 1))
        end = begin + 40
    given = spans_tensor(begin, end)
    cut = np.clip(begin, 0, L_k), np.clip(end, 0, L_k)
    run_forward(A, Q, K, V, *cut, spans=given)
    run_backward(A, Q, K, V, dO, *cut, spans=given)
    one = tuple(t[1] for t in given)  # one row for the batch
    shared = tuple(np.tile(x[1], (B, 1)) for x in cut)
    run_forward(A, Q, K, V, *shared, spans=one)
    run_backward(A, Q, K, V, dO, *shared, spans=one)


@pytest.mark.parametrize("scale", [0.3, -0.3])
@pytest.mark.parametrize("cap", [0.5, 20.0, 1000.0, 1e6])
def test_caps(A, scale, cap):
    """Scores far beyond the cap, around it and far below; both signs of the scale."""
    Q, K, V, dO = rows(1, 1, 2, 200, 64, 3.0), rows(2, 1, 2, 200, 64), rows(3, 1, 2, 200, 64), rows(4, 1, 2, 200, 64)
    begin, end = spans_of("causal", 1, 200, 200)
    kw = dict(mask="causal", scale=scale, cap=cap)
    run_forward(A, Q, K, V, begin, end, **kw)
    run_backward(A, Q, K, V, dO, begin, end, **kw)


def test_large_caps_change_nothing(A):
    """Far below the cap the capped score is the score: relative error 2e-7 of it, where 1 - 2 / (1 + e^2y) alone would lose 1e-7 of the cap."""
    Q, K, V = rows(1, 1, 2, 300, 128, 2.0), rows(2, 1, 2, 300, 128), rows(3, 1, 2, 300, 128)
    stats = [torch.empty(1, 2, 300, device="cuda") for _ in range(2)]
    for cap, s in zip((0.0, 1e6), stats):
        A.span_attention_forward(Q, K, V, scale=0.1, cap=cap, stats=s)
    # scores up to 25: 2e-7 * 25, the cubic term 25^3 / 3e12, and two roundings of the statistic
    assert (stats[0] - stats[1]).abs().max() <= 25 * 2e-7 + 1e-8 + 2.0 ** -20 * 8


@pytest.mark.parametrize("slopes", [[0.0, 0.0], [-0.01, 0.02], [4.0, 0.5]])
def test_slopes(A, slopes):
    Q, K, V, dO = rows(1, 1, 2, 200, 64), rows(2, 1, 1, 260, 64), rows(3, 1, 1, 260, 64), rows(4, 1, 2, 200, 64)
    begin, end = spans_of("none", 1, 200, 260)
    run_forward(A, Q, K, V, begin, end, mask="none", slopes=slopes)
    run_backward(A, Q, K, V, dO, begin, end, mask="none", slopes=slopes)


@pytest.mark.parametrize("mask,prefix", [("none", False), ("causal", False), ("causal", True), ("sliding_window", False)])
@pytest.mark.parametrize("B,L", [(1, 1), (1, 300), (3, 1000)])
def test_document_spans(A, mask, prefix, B, L):
    at = documents(3, B, L, max(1, L // 4), padding=min(7, L - 1))
    at = np.concatenate([at, at[:, -1:], at[:, -1:]], 1)  # empty documents
    pre = np.random.RandomState(1).randint(-3, L, (B, at.shape[1] - 1)) if prefix else None
    begin, end = document_spans(at, L, mask, 13, pre)
    got = A.document_spans(torch.tensor(at, dtype=torch.int32, device="cuda"), L, mask=mask, window=13 if mask == "sliding_window" else 0,
                           prefix=None if pre is None else torch.tensor(pre, dtype=torch.int32, device="cuda"))
    g0, g1 = (t.cpu().numpy() for t in got)
    empty = begin >= end
    assert np.array_equal(g0 >= g1, empty)
    assert np.array_equal(g0[~empty], begin[~empty]) and np.array_equal(g1[~empty], end[~empty])


def test_documents_equal_separate_calls(A):
    """Packed documents give what each gives on its own."""
    L, at = 600, [0, 1, 90, 91, 347, 600]
    Q, K, V = rows(1, 1, 4, L, 128), rows(2, 1, 2, L, 128), rows(3, 1, 2, L, 128)
    spans = A.document_spans(torch.tensor(at, dtype=torch.int32, device="cuda"), L)
    stats = torch.empty(1, 4, L, device="cuda")
    O = A.span_attention_forward(Q, K, V, scale=0.1, mask="spans", spans=spans, stats=stats)
    for a, b in zip(at, at[1:]):
        s = torch.empty(1, 4, b - a, device="cuda")
        q, k, v = (t[:, :, a:b].contiguous() for t in (Q, K, V))
        o = A.span_attention_forward(q, k, v, scale=0.1, stats=s)
        mag = A.span_attention_forward(q, k, v.abs(), scale=0.1)
        assert ((O[:, :, a:b] - o).abs() <= (2 * 2.0 ** -8 + 1e-4) * mag + 1e-6).all()  # (weights rounded on other references: half a step each)
        assert (stats[:, :, a:b] - s).abs().max() <= 2e-5


def test_strides_and_layouts(A):
    """Views of a fused projection, heads of keys expanded from one, an output with gaps that stay as they were."""
    B, H, L = 2, 3, 130
    fused = torch.randn(B, L, H, 3 * 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda().transpose(1, 2)
    Q, K, V = fused[..., :64], fused[..., 64:128], fused[..., 128:]
    begin, end = spans_of("causal", B, L, L)
    run_forward(A, Q, K, V, begin, end, mask="causal")
    run_backward(A, Q, K, V, rows(4, B, H, L, 64, order="bhld"), begin, end, mask="causal", o_dtype=torch.bfloat16)
    K1, V1 = K[:, :1].expand(B, H, L, 64), V[:, :1].expand(B, H, L, 64)
    run_forward(A, Q, K1, V1, begin, end, mask="causal")
    wide = torch.full((B, H, L, 96), 7.0, device="cuda")
    A.span_attention_forward(Q, K, V, scale=0.125, out=wide[..., :64])
    assert (wide[..., 64:] == 7).all() and not (wide[..., :64] == 7).any()


def test_gradients_against_differences(A):
    """The gradients are those of the forward pass itself: central differences of sum(O dO) in one direction for each input."""
    B, H_q, H_kv, L, D = 1, 4, 2, 150, 64
    Q, K, V, dO = rows(1, B, H_q, L, D), rows(2, B, H_kv, L, D), rows(3, B, H_kv, L, D), rows(4, B, H_q, L, D)
    at = documents(2, B, L, 60)
    begin, end = document_spans(at, L)
    kw = dict(scale=0.2, cap=4.0, slopes=slopes_of(H_q))
    spans = spans_tensor(begin, end)
    stats = torch.empty(B, H_q, L, device="cuda")
    O = A.span_attention_forward(Q, K, V, mask="spans", spans=spans, stats=stats, **kw)
    grads = A.span_attention_backward(Q, K, V, O, dO, stats, mask="spans", spans=spans, **kw)
    for n in range(3):
        d = np.random.RandomState(n).randn(*grads[n].shape)
        x = [host(t) for t in (Q, K, V)]
        f = []
        for sign in (1, -1):
            y = list(x)
            y[n] = x[n] + sign * 1e-4 * d
            f.append((span_attention(*y, begin, end, scale=kw["scale"], cap=kw["cap"], slopes=kw["slopes"])[0] * host(dO)).sum())
        want, got = (f[0] - f[1]) / 2e-4, (host(grads[n]) * d).sum()
        # (rounding errors of 2^-8 of each weight and score gradient, independent: far below 2^-6 of the sum's deviation, |grad| |d|)
        assert abs(got - want) <= 2.0 ** -6 * np.sqrt((host(grads[n]) ** 2).sum())


def test_same_bits_again(A):
    """No order of workgroups changes a bit."""
    Q, K, V, dO = rows(1, 2, 8, 500, 128), rows(2, 2, 2, 500, 128), rows(3, 2, 2, 500, 128), rows(4, 2, 8, 500, 128)
    stats = torch.empty(2, 8, 500, device="cuda")
    first = None
    for _ in range(4):
        O = A.span_attention_forward(Q, K, V, scale=0.09, cap=30.0, stats=stats)
        now = [O, stats.clone(), *A.span_attention_backward(Q, K, V, O, dO, stats, scale=0.09, cap=30.0)]
        if first is None:
            first = now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_graph_and_streams(A):
    """A captured training step, replayed on new inputs between eager work; two streams at once on one plan."""
    B, H_q, H_kv, L = 1, 4, 2, 400
    make = lambda s: (rows(s, B, H_q, L, 128), rows(s + 1, B, H_kv, L, 128), rows(s + 2, B, H_kv, L, 128), rows(s + 3, B, H_q, L, 128))
    Q, K, V, dO = (t.contiguous() for t in make(10))
    out, stats = torch.empty(B, H_q, L, 128, device="cuda"), torch.empty(B, H_q, L, device="cuda")
    grads = [torch.empty(t.shape, device="cuda") for t in (Q, K, V)]
    at = torch.tensor([0, 100, 101, 300], dtype=torch.int32, device="cuda")
    plan = A.SpanAttentionPlan(Q, K, V, out, scale=0.1, cap=20.0, mask="spans")

    def step():
        spans = A.document_spans(at, L)
        plan.forward(Q, K, V, out, spans=spans, stats=stats)
        plan.backward(Q, K, V, out, dO, stats, *grads, spans=spans)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        for t, x in zip((Q, K, V, dO), make(20 + 10 * n)):
            t.copy_(x)
        at[2] = 102 + 50 * n
        step()
        want = [t.clone() for t in (out, stats, *grads)]
        for t in (out, stats, *grads):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, stats, *grads)))
    spans = A.document_spans(at, L)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for s in streams:
        o, st = torch.empty_like(out), torch.empty_like(stats)
        g = [torch.empty_like(x) for x in grads]
        torch.cuda.synchronize()
        plan.forward(Q, K, V, o, spans=spans, stats=st, stream=s)
        plan.backward(Q, K, V, o, dO, st, *g, spans=spans, stream=s)
        results.append((o, st, *g))
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(want, r))


def test_refusals_of_the_binding(A):
    Q, K, V = rows(1, 1, 2, 40, 64), rows(2, 1, 2, 40, 64), rows(3, 1, 2, 40, 64)
    spans = spans_tensor(*spans_of("causal", 1, 40, 40))
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K, V, scale=1.0, mask="spans")
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K, V, scale=1.0, mask="causal", spans=spans)
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K, V, scale=1.0, mask="spans", spans=tuple(t.long() for t in spans))
    with pytest.raises(ValueError):
        A.span_attention_forward(Q.float(), K, V, scale=1.0)
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K[:, :, :30], V, scale=1.0)
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K, V, scale=1.0, slopes=[1.0])
    with pytest.raises(ValueError):
        A.span_attention_forward(Q, K, V, scale=1.0, out=torch.empty(1, 1, 40, 64, device="cuda").expand(1, 2, 40, 64))
    O, stats = A.span_attention_forward(Q, K, V, scale=1.0), torch.zeros(1, 2, 40, device="cuda")
    with pytest.raises(ValueError):
        A.span_attention_backward(Q, K, V, O, torch.ones((), device="cuda").to(torch.bfloat16).expand(O.shape), stats, scale=1.0)
    with pytest.raises(ValueError):
        A.span_attention_backward(Q, K, V, O, Q, stats[:, :, :30], scale=1.0)
    with pytest.raises(A.AeAttnError):
        A.span_attention_forward(Q, K, V, scale=1.0, cap=-1.0)


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("mask", ["none", "causal", "sliding_window", "unsorted"])
@pytest.mark.parametrize("kv_splits", [2, 5, 256])
def test_keys_in_ranges(A, dims, score, mask, kv_splits):
    """Ranges with keys of some rows, of none, of all; more ranges than tiles; rows that see nothing."""
    B, H_q, H_kv, L_q, L_k = 2, 4, 2, 70, 460
    Q, K, V = rows(1, B, H_q, L_q, dims[0], 2.0), rows(2, B, H_kv, L_k, dims[0]), rows(3, B, H_kv, L_k, dims[1])
    kw = dict(score, kv_splits=kv_splits)
    if mask == "unsorted":
        g = np.random.RandomState(7)
        begin = g.randint(0, L_k, (B, L_q))
        end = np.where(g.rand(B, L_q) < 0.2, begin, np.minimum(begin + g.randint(1, 300, (B, L_q)), L_k))
    else:
        kw.update(mask=mask, window=100 if mask == "sliding_window" else 0)
        begin, end = spans_of(mask, B, L_q, L_k, kw["window"])
    run_forward(A, Q, K, V, begin, end, out_dtype=torch.bfloat16 if kv_splits == 5 else torch.float32, **kw)


def test_ranges_are_chosen_where_there_are_few_rows(A):
    Q, K, V = rows(1, 1, 8, 3, 128, 2.0), rows(2, 1, 2, 5000, 128), rows(3, 1, 2, 5000, 128)
    plan = A.SpanAttentionPlan(Q, K, V, torch.empty(1, 8, 3, 128, device="cuda"), scale=0.1)
    assert plan.split_bytes > 0
    begin, end = spans_of("causal", 1, 3, 5000)
    a = run_forward(A, Q, K, V, begin, end, out_dtype=torch.float32, mask="causal", slopes=True)
    b = run_forward(A, Q, K, V, begin, end, out_dtype=torch.float32, mask="causal", slopes=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    whole = A.SpanAttentionPlan(Q, K, V, torch.empty(1, 8, 3, 128, device="cuda"), scale=0.1, kv_splits=1)
    assert whole.split_bytes == 0


def test_ranges_on_two_streams_and_in_a_graph(A):
    """Every call has partial results of its own."""
    Q, K, V = rows(1, 1, 8, 40, 64, 2.0), rows(2, 1, 2, 3000, 64), rows(3, 1, 2, 3000, 64)
    out = torch.empty(1, 8, 40, 64, device="cuda")
    plan = A.SpanAttentionPlan(Q, K, V, out, scale=0.1, kv_splits=6)
    want = plan.forward(Q, K, V, out).clone()
    torch.cuda.synchronize()
    results = []
    for _ in range(2):
        s, o = torch.cuda.Stream(), torch.empty_like(out)
        torch.cuda.synchronize()
        results.append(plan.forward(Q, K, V, o, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for r in results)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.forward(Q, K, V, out)
    for n in range(3):
        Q.copy_(rows(10 + n, 1, 8, 40, 64))
        eager = plan.forward(Q, K, V, torch.empty_like(out))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("dims,B,H_q,H_kv,L", [((64, 64), 4, 16, 16, 600), ((128, 128), 4, 16, 16, 300), ((192, 128), 3, 24, 12, 515)])
@pytest.mark.parametrize("kind", ["documents", "unsorted", "some_empty"])
def test_many_workgroups_with_walks_of_unequal_length(A, dims, B, H_q, H_kv, L, kind):
    """Backward calls whose tiles are put in an order, another one for each batch entry."""
    Q, K, V, dO = rows(91, B, H_q, L, dims[0]), rows(92, B, H_kv, L, dims[0]), rows(93, B, H_kv, L, dims[1]), rows(94, B, H_q, L, dims[1])
    if kind == "documents":
        begin, end = document_spans(documents(95, B, L, 400, padding=7), L)
    else:
        g = np.random.RandomState(96)
        begin = g.randint(0, L, (B, L))
        end = begin + g.randint(0, 80, (B, L))
        if kind == "some_empty":
            end[:, 100:400] = begin[:, 100:400]
    run_forward(A, Q, K, V, begin, end)
    run_backward(A, Q, K, V, dO, begin, end)


@pytest.mark.parametrize("B,H_q,H_kv,L_q,L_k", [(2, 32, 8, 1500, 1500), (1, 64, 16, 700, 2000), (1, 16, 16, 2000, 700), (1, 4, 2, 16385, 16385), (1, 16, 16, 16384, 300)])
def test_an_order_of_tiles_changes_nothing(A, B, H_q, H_kv, L_q, L_k):
    """Given spans that are the causal mask, whose own order needs no other, at sizes on both sides of the largest order."""
    Q, K, V, dO = rows(97, B, H_q, L_q, 128), rows(98, B, H_kv, L_k, 128), rows(99, B, H_kv, L_k, 128), rows(100, B, H_q, L_q, 128)
    stats = torch.empty(B, H_q, L_q, device="cuda")
    O = A.span_attention_forward(Q, K, V, scale=0.09, stats=stats)
    end = (torch.arange(L_q, device="cuda", dtype=torch.int32) + (L_k - L_q + 1)).clamp(min=0)
    spans = torch.zeros_like(end), end
    want = A.span_attention_backward(Q, K, V, O, dO, stats, scale=0.09)
    got = A.span_attention_backward(Q, K, V, O, dO, stats, scale=0.09, mask="spans", spans=spans)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("cap", [1e-20, 1e-6, 1e-3, 3e3, 1e5, 1e9, 1e14, 1e30])
def test_caps_whose_series_is_cut_or_left_out(A, cap):
    Q, K, V, dO = rows(1, 1, 2, 100, 64, 3.0), rows(2, 1, 2, 100, 64), rows(3, 1, 2, 100, 64), rows(4, 1, 2, 100, 64)
    begin, end = spans_of("causal", 1, 100, 100)
    run_forward(A, Q, K, V, begin, end, mask="causal", scale=0.3, cap=cap)
    run_backward(A, Q, K, V, dO, begin, end, mask="causal", scale=0.3, cap=cap)


@pytest.mark.parametrize("cap", [30.0, 50.0, 51.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_rows_whose_scores_are_all_at_the_cap(A, cap, sign):
    """Every score far beyond the cap on one side, or, in the later rows, on both."""
    Q, V, dO = rows(1, 1, 2, 150, 64).abs() + 0.5, rows(3, 1, 2, 150, 64), rows(4, 1, 2, 150, 64)
    K = sign * (rows(2, 1, 2, 150, 64).abs() + 0.5)
    K[:, :, 100::3] *= -1
    begin, end = spans_of("causal", 1, 150, 150)
    run_forward(A, Q, K, V * 2.0 ** -20, begin, end, mask="causal", scale=30.0, cap=cap)
    run_forward(A, Q, K, V * 2.0 ** 20, begin, end, mask="causal", scale=30.0, cap=cap)
    run_backward(A, Q, K, V, dO, begin, end, mask="causal", scale=30.0, cap=cap)


@pytest.mark.parametrize("cap", [2e36, 1e37, 2e38])
def test_the_largest_caps_leave_the_scores(A, cap):
    """Scale / cap next to the smallest 32-bit number with all its bits: the series is its first term."""
    Q, K, V, dO = rows(1, 1, 2, 100, 64, 3.0), rows(2, 1, 2, 100, 64), rows(3, 1, 2, 100, 64), rows(4, 1, 2, 100, 64)
    begin, end = spans_of("causal", 1, 100, 100)
    scale = 0.3 if cap < 1e38 else 3.0
    run_forward(A, Q, K, V, begin, end, mask="causal", scale=scale, cap=cap)
    run_forward(A, Q, K, V, begin, end, mask="causal", scale=-scale, cap=cap, slopes=True)
    run_backward(A, Q, K, V, dO, begin, end, mask="causal", scale=scale, cap=cap)


def test_strides_of_spans_that_do_not_matter(A):
    """Rows of one batch entry, or of one query, have no distance: any stride will do, and two different ones."""
    Q, K, V, dO = rows(1, 1, 2, 40, 64), rows(2, 1, 2, 40, 64), rows(3, 1, 2, 40, 64), rows(4, 1, 2, 40, 64)
    begin, end = spans_tensor(*spans_of("causal", 1, 40, 40))
    odd = torch.stack([end[0], end[0]])[1:].as_strided((1, 40), (7, 1))
    want = A.span_attention_forward(Q, K, V, scale=0.1, mask="spans", spans=(begin, end))
    assert torch.equal(A.span_attention_forward(Q, K, V, scale=0.1, mask="spans", spans=(begin, odd)), want)
    one = torch.stack([end[0, 20:22], end[0, 20:22]], 1)[:1, :1].as_strided((1, 1), (1, 2))
    got = A.span_attention_forward(Q[:, :, 20:21], K, V, scale=0.1, mask="spans", spans=(begin[:, :1], one))
    assert got.shape == (1, 2, 1, 64) and torch.isfinite(got).all()
    two = spans_tensor(*spans_of("causal", 2, 40, 40))
    with pytest.raises(ValueError):  # where they matter they have to be the same
        A.span_attention_forward(*(t.expand(2, -1, -1, -1) for t in (Q, K, V)), scale=0.1, mask="spans", spans=(two[0], two[1][:1].expand(2, 40)))


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("L_q,L_k", [(300, 300), (90, 333)])
def test_the_steepest_slopes(A, dims, cap, L_q, L_k):
    """Every row sees its own key, which (and the nearest ones) has the weight: the statistic is off by 2^-22 of the slope times 128 at most, and of
    slope times distance, 40 for the keys that weigh more than e^-40 with the scores' own differences."""
    slopes = [128.0, 31.0, 4.0, 0.5]
    Q, K, V, dO = rows(1, 1, 4, L_q, dims[0]), rows(2, 1, 2, L_k, dims[0]), rows(3, 1, 2, L_k, dims[1]), rows(4, 1, 4, L_q, dims[1])
    for mask in ("causal", "none"):
        begin, end = spans_of(mask, 1, L_q, L_k)
        _, stats = run_forward(A, Q, K, V, begin, end, mask=mask, cap=cap, slopes=slopes, out_dtype=torch.float32)
        _, lse, _ = span_attention(host(Q), host(K), host(V), begin, end, scale=dims[0] ** -0.5, cap=cap, slopes=slopes)
        e = score_error(Q, K, dims[0] ** -0.5, cap, None, 0) + 2.0 ** -22 * (128 * np.array(slopes) + 40)
        assert np.all(np.abs(host(stats) - lse) <= (e[:, None] + 2.0 ** -20 * (1 + np.abs(lse))))
        run_backward(A, Q, K, V, dO, begin, end, mask=mask, cap=cap, slopes=slopes)


@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("score", [dict(), dict(cap=12.0)])
def test_rows_that_see_far_keys_alone(A, dims, score):
    """Spans 65536 keys away, next to each other and not, under slopes: errors of 2^-22 slope (L_q + L_k) of a score, as the bounds above have it."""
    L_q, L_k = 70, 66000
    Q, K, V, dO = rows(1, 1, 2, L_q, dims[0]), rows(2, 1, 1, L_k, dims[0]), rows(3, 1, 1, L_k, dims[1]), rows(4, 1, 2, L_q, dims[1])
    begin = np.where(np.arange(L_q) % 2, 100, 20)[None]
    end = begin + 1 + 3 * np.arange(L_q)
    kw = dict(score, slopes=[1.0, -0.25])
    run_forward(A, Q, K, V, begin, end, out_dtype=torch.float32, **kw)
    run_backward(A, Q, K, V, dO, begin, end, **kw)
