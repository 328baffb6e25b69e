"""The operators of a serving loop as they are used together: rotary positions, append, attention over the cache, for prompts and
token by token, eager and from a captured graph; and the rotary positions' gradient behind the attention's."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import attend, dequantise, quantise, rotary as oracle_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


class Layer:
    """A cache of one layer, its page lists, and what has been written to it (64 bits, in order)."""

    def __init__(self, A, B, H_kv, D, page, width, dtype, seed):
        self.A, self.page, self.B = A, page, B
        self.cache = A.PagedCache.empty(B * width + 2, H_kv, page, D, D, dtype=dtype)
        order = torch.randperm(B * width + 2, generator=torch.Generator().manual_seed(seed))
        self.table = order[: B * width].view(B, width).to(torch.int32).to(DEV)
        self.rows = [[np.zeros((H_kv, 0, D)) for _ in range(B)] for _ in range(2)]

    def slots(self, positions):
        """positions [B, L] int64, -1: nothing."""
        p = positions.clamp(min=0)
        s = torch.gather(self.table.long(), 1, p // self.page) * self.page + p % self.page
        return torch.where(positions >= 0, s, -1).to(torch.int32)

    def note(self, K, V, positions):
        for rows, x in zip(self.rows, (K, V)):
            v = x.cpu().double().numpy()
            if self.cache.k_exp is not None:
                v = dequantise(*quantise(v))
            for b in range(self.B):
                live = (positions[b] >= 0).cpu().numpy()
                rows[b] = np.concatenate((rows[b], v[b][:, live]), axis=1)

    def check(self, O, Q, scale, what):
        for b in range(self.B):
            q = Q[b].cpu().double().numpy()
            ref, _ = attend(q, self.rows[0][b], self.rows[1][b], scale)
            mag, _ = attend(q, self.rows[0][b], np.abs(self.rows[1][b]), scale)
            # weights are rounded to bf16 (2^-8 of each at most), all else is in 32 bits
            err, bound = np.abs(O[b].cpu().double().numpy() - ref), (2.0 ** -8 + 4e-5) * mag + 1e-30
            assert (err <= bound).all(), (what, b, float((err / bound).max()))


def projected(seed, B, L, H_q, H_kv, D):
    """Q, K, V as a fused projection leaves them: views of [B, L, (H_q + 2 H_kv) D]."""
    x = torch.randn(B, L, (H_q + 2 * H_kv) * D, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)
    q, k, v = x.split([H_q * D, H_kv * D, H_kv * D], dim=-1)
    return [t.unflatten(-1, (-1, D)).transpose(1, 2) for t in (q, k, v)]


@pytest.mark.parametrize("dtype,H_q,H_kv,D,page", [("bf16", 8, 2, 128, 16), ("e4m3", 8, 8, 64, 32), ("e4m3", 16, 2, 128, 64)])
def test_prompt_then_tokens(A, dtype, H_q, H_kv, D, page):
    lengths, B, width = [37, 100, 1], 3, 8
    f, amp = A.rotary_frequencies(D, scaling="by_parts", factor=4.0)
    layer = Layer(A, B, H_kv, D, page, width, dtype, 1)
    scale = D ** -0.5
    # prompts, padded to the longest
    L = max(lengths)
    pos = torch.arange(L, device=DEV).repeat(B, 1)
    pos = torch.where(pos < torch.tensor(lengths, device=DEV)[:, None], pos, -1)
    q, k, v = projected(2, B, L, H_q, H_kv, D)
    qr, kr = A.rotary_forward(q, k, pos.to(torch.int32), freqs=f, amplitude=amp)
    # a bf16 output is off by half a step of it at most, and 6e-7 of its two terms
    ref = oracle_rotary(k.cpu().double().numpy(), pos.cpu().numpy(), f, amp)
    assert (np.abs(kr.cpu().double().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-5).all()
    layer.cache.append(kr, v, layer.slots(pos))
    layer.note(kr, v, pos)
    # what is read back for the prompts' attention is what was written
    kb, vb = layer.cache.read(layer.slots(pos))
    for b, n in enumerate(lengths):
        assert np.array_equal(kb[b, :, :n].cpu().double().numpy(), layer.rows[0][b]) and (kb[b, :, n:] == 0).all() and (vb[b, :, n:] == 0).all()
        O = A.attention_forward(qr[b: b + 1, :, :n], kb[b: b + 1, :, :n], vb[b: b + 1, :, :n], scale=scale, mask="causal")
        last = A.attention_cached(qr[b: b + 1, :, n - 1: n], layer.cache, layer.table[b: b + 1].contiguous(),
                                  torch.tensor([n], dtype=torch.int32, device=DEV), scale=scale)
        # the prompt's last row, once as part of the prompt and once as its newest token (the first has its own bound of 1e-2)
        assert (O[:, :, n - 1:] - last).abs().max() <= 1e-2 + 2.0 ** -7 * float(last.abs().max())
    # tokens: two sequences take one at a time, the third pauses every other step; drafts of three at the end
    now = torch.tensor(lengths, device=DEV)
    for step in range(7):
        n = 1 if step < 5 else 3
        p = now[:, None] + torch.arange(n, device=DEV)
        q, k, v = projected(10 + step, B, n, H_q, H_kv, D)
        qr, kr = A.rotary_forward(q, k, p.to(torch.int32), freqs=f, amplitude=amp)
        if n == 1 and step % 2:
            p[2] = -1
        layer.cache.append(kr, v, layer.slots(p))
        layer.note(kr, v, p)
        now = now + (p >= 0).sum(1)
        O = A.attention_cached(qr, layer.cache, layer.table, now.to(torch.int32), scale=scale)
        layer.check(O, qr, scale, step)


def test_step_from_a_captured_graph(A):
    # two layers' rotary, append and attention in one graph; positions, slots and lengths change on the device between replays
    B, H_q, H_kv, D, page, width = 4, 8, 2, 64, 16, 12
    f, _ = A.rotary_frequencies(D)
    layers = [Layer(A, B, H_kv, D, page, width, t, 3 + i) for i, t in enumerate(("bf16", "e4m3"))]
    q, k, v = [x.contiguous() for x in projected(5, B, 1, H_q, H_kv, D)]
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    outs = [torch.empty(B, H_q, 1, D, device=DEV) for _ in layers]
    pos = torch.zeros(B, 1, dtype=torch.int32, device=DEV)
    slots = [torch.full((B, 1), -1, dtype=torch.int32, device=DEV) for _ in layers]
    lengths = torch.ones(B, dtype=torch.int32, device=DEV)
    rot = A.RotaryPlan(q, k, pos, qr, kr, freqs=f)
    plans = [A.CachedAttentionPlan(l.cache, qr, o, max_length=width * page, table_width=width, scale=0.125, chunk=128) for l, o in zip(layers, outs)]

    def step():
        rot.forward(q, k, pos, qr, kr)
        for l, s, p, o in zip(layers, slots, plans, outs):
            l.cache.append(kr, v, s)
            p.forward(qr, l.table, lengths, o)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(40):
        for dst, src in zip((q, k, v), projected(100 + i, B, 1, H_q, H_kv, D)):
            dst.copy_(src)
        at = torch.full((B, 1), i, device=DEV)
        pos.copy_(at)
        lengths.fill_(i + 1)
        for l, s in zip(layers, slots):
            s.copy_(l.slots(at))
        g.replay()
        torch.cuda.synchronize()
        for l, o in zip(layers, outs):
            l.note(kr, v, at)
            if i % 6 == 5:
                l.check(o, qr, 0.125, i)


def test_two_plans_side_by_side(A):
    # calls of different plans on two streams at once, each with ranges that are joined
    B, H, D, page, width = 2, 4, 128, 32, 60
    g = torch.Generator().manual_seed(6)
    made = []
    for i in range(2):
        c = A.PagedCache.empty(B * width, H, page, D, D)
        k, w = (torch.randn(1, H, B * width * page, D, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
        c.append(k, w, torch.arange(B * width * page, dtype=torch.int32, device=DEV)[None])
        t = torch.randperm(B * width, generator=g).view(B, width).to(torch.int32).to(DEV)
        Q = torch.randn(B, H, 1, D, generator=g).to(torch.bfloat16).to(DEV)
        out = torch.empty(B, H, 1, D, device=DEV)
        plan = A.CachedAttentionPlan(c, Q, out, max_length=width * page, table_width=width, scale=0.088, chunk=128)
        made.append((plan, Q, t, torch.tensor([1900 - i, 700], dtype=torch.int32, device=DEV), out))
    expect = [p.forward(Q, t, L, o).clone() for p, Q, t, L, o in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(30):
        for s, (p, Q, t, L, o) in zip(streams, made):
            p.forward(Q, t, L, o, stream=s)
    torch.cuda.synchronize()
    for e, m in zip(expect, made):
        assert torch.equal(e, m[-1])


def test_gradient_through_rotary_and_attention(A):
    from oracle import attention_backward
    B, H_q, H_kv, L, D = 1, 4, 2, 96, 64
    f, amp = A.rotary_frequencies(32)
    q, k, v = [x.contiguous() for x in projected(7, B, L, H_q, H_kv, D)]
    pos = torch.arange(L, dtype=torch.int32, device=DEV) + 11
    qr, kr = A.rotary_forward(q, k, pos, freqs=f, amplitude=amp, layout="interleaved")
    stats = torch.empty(B, H_q, L, device=DEV)
    O = A.attention_forward(qr, kr, v, scale=0.125, mask="causal", stats=stats)
    dO = torch.randn(O.shape, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    dqr, dkr, _ = A.attention_backward(qr, kr, v, O, dO, stats, scale=0.125, mask="causal")
    dq, dk = A.rotary_backward(dqr, dkr, pos, freqs=f, amplitude=amp, layout="interleaved")
    ref = attention_backward(qr.float().cpu(), kr.float().cpu(), v.float().cpu(), dO.float().cpu(), scale=0.125, norm="softmax", mask="causal")
    for got, r in ((dq, ref[0]), (dk, ref[1])):
        want = oracle_rotary(r, pos.cpu().numpy(), f, amp, "interleaved", backward=True)
        err = np.abs(got.cpu().double().numpy() - want) / np.maximum(np.abs(want).max(axis=-1, keepdims=True), 1.0)
        # the attention's own bound, turned: two elements of a pair at most add up to sqrt(2) of it
        assert err.max() <= 1.5e-2 and err.mean() <= 1.5e-3, (err.max(), err.mean())


def test_memory_of_outputs_on_another_stream(A):
    # an output is allocated where it is written: given back, its memory serves that stream, not the one the caller was on
    B, H, L, D = 2, 4, 50, 64
    f, _ = A.rotary_frequencies(D)
    x = torch.randn(B, H, L, D, generator=torch.Generator().manual_seed(20)).to(torch.bfloat16).to(DEV)
    pos = torch.arange(L, dtype=torch.int32, device=DEV)
    c = A.PagedCache.empty(8, H, 16, D, D)
    slots = torch.arange(B * L, dtype=torch.int32, device=DEV).view(B, L)
    c.append(x, x.clone(), slots)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for call in (lambda: A.rotary_forward(x, x, pos, freqs=f, stream=s), lambda: A.rotary_backward(x, x, pos, freqs=f, stream=s),
                 lambda: c.read(slots, stream=s)):
        got = call()
        s.synchronize()
        assert torch.equal(*got)
        at = {t.data_ptr() for t in got}
        del got
        here = [torch.empty_like(x) for _ in range(8)]
        assert not at & {t.data_ptr() for t in here}


def test_plan_dropped_while_another_stream_uses_its_workspace(A):
    B, H, D, page, width = 2, 4, 128, 32, 60
    g = torch.Generator().manual_seed(21)
    c = A.PagedCache.empty(B * width, H, page, D, D)
    k, v = (torch.randn(1, H, B * width * page, D, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    c.append(k, v, torch.arange(B * width * page, dtype=torch.int32, device=DEV)[None])
    t = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
    L = torch.tensor([1900, 700], dtype=torch.int32, device=DEV)
    Q, out = torch.randn(B, H, 1, D, generator=g).to(torch.bfloat16).to(DEV), torch.empty(B, H, 1, D, device=DEV)
    ref = A.attention_cached(Q, c, t, L, scale=0.088, chunk=128)
    s = torch.cuda.Stream()
    for _ in range(3):
        plan = A.CachedAttentionPlan(c, Q, out, max_length=width * page, table_width=width, scale=0.088, chunk=128)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)  # (some milliseconds in front of the call)
        plan.forward(Q, t, L, out, stream=s)
        at, size = plan.workspace.data_ptr(), plan.workspace_bytes
        del plan
        taken = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
        assert at not in {x.data_ptr() for x in taken}
        s.synchronize()
        assert torch.equal(out, ref)
        out.fill_(7.0)
