"""CPU-only checks of the operators around a key/value cache: symbols, refusals, frequencies, the definitions in 64 bits."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_15349_amd", "libae_attn.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libae_attn.so not built (run __graft_entry__.build())")


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def refused(A, status, call, *a, **kw):
    with pytest.raises(A.AeAttnError) as ei:
        call(*a, **kw)
    assert ei.value.status == status, str(ei.value)


def test_library_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "ae_serving.h")).read()
    names = set(re.findall(r"\b(ae_[a-z]+_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)))
    assert {"ae_rotary_create", "ae_rotary_backward", "ae_cache_append", "ae_cache_read"} <= names
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), f"{n} declared in the header but not exported"


ROT = dict(B=2, H_q=4, H_k=2, L=10, D=64, frequencies=[1.0] * 16)


@pytest.mark.parametrize("patch,status", [
    (dict(B=0), 1), (dict(H_q=0), 1), (dict(H_k=-1), 1), (dict(L=0), 1), (dict(D=0), 1), (dict(frequencies=[]), 1), (dict(frequencies=[1.0] * 33), 1),
    (dict(D=512, frequencies=[1.0] * 129), 1), (dict(frequencies=[float("nan")]), 1), (dict(frequencies=[float("inf")]), 1), (dict(frequencies=[6.5]), 1),
    (dict(amplitude=float("nan")), 1), (dict(layout=2), 1), (dict(dtype=3), 1), (dict(q_stride=(-1, 64, 64)), 1), (dict(position_stride=-1), 1),
    (dict(D=2048), 2), (dict(H_q=70000), 2), (dict(B=1 << 20, L=1 << 20), 2),
])
def test_rotary_refusals(A, patch, status):
    refused(A, status, A.ae_rotary_create, **{**ROT, **patch})


def test_rotary_call_refusals(A):
    h = A.ae_rotary_create(**ROT)
    p = 1 << 20
    for a in ((0, p, p, p, p), (p, 0, p, 2 * p, 3 * p), (p, 2 * p, 0, 3 * p, 4 * p), (p, 2 * p, 3 * p, 0, 4 * p), (p, 2 * p, 3 * p, 4 * p, 0),
              (p + 1, 2 * p, 3 * p, 4 * p, 5 * p), (p, 2 * p, 3 * p + 2, 4 * p, 5 * p), (p, 2 * p, 3 * p, 2 * p, 5 * p), (p, 2 * p, 3 * p, 4 * p, p),
              (p, 2 * p, 3 * p, 4 * p, 4 * p), (p, 2 * p, 3 * p, 3 * p, 5 * p)):
        refused(A, 1, A.ae_rotary_forward, h, *a)
        refused(A, 1, A.ae_rotary_backward, h, *a)
    A.ae_rotary_destroy(h)
    A.ae_rotary_destroy(None)
    refused(A, 1, A.ae_rotary_forward, None, p, 2 * p, 3 * p, 4 * p, 5 * p)
    # in place with other strides
    h = A.ae_rotary_create(**{**ROT, "H_k": 0}, q_out_stride=(4 * 640, 64, 256))
    refused(A, 1, A.ae_rotary_forward, h, p, 0, 2 * p, p, 0)
    A.ae_rotary_destroy(h)


CACHE = dict(n_pages=4, page_size=32, H_kv=2, D_qk=128, D_v=128)


@pytest.mark.parametrize("patch,status", [
    (dict(n_pages=0), 1), (dict(H_kv=0), 1), (dict(page_size=0), 1), (dict(page_size=8), 1), (dict(page_size=48), 1), (dict(page_size=512), 1),
    (dict(dtype=2), 1), (dict(D_qk=64), 2), (dict(D_v=96), 2), (dict(n_pages=1 << 27), 2),
])
def test_cache_refusals(A, patch, status):
    refused(A, status, A.ae_cache_create, **{**CACHE, **patch})


def test_cache_call_refusals(A):
    p = 1 << 20
    for dtype in ("bf16", "e4m3"):
        h = A.ae_cache_create(**CACHE, dtype=dtype)
        e = (6 * p, 7 * p) if dtype == "e4m3" else (0, 0)
        ok = dict(K=p, k_stride=(0, 0, 0), V=2 * p, v_stride=(0, 0, 0), B=1, L=4, slots=3 * p, slot_stride=0, K_pages=4 * p, V_pages=5 * p,
                  K_exp=e[0], V_exp=e[1])
        for patch in (dict(K=0), dict(V=0), dict(slots=0), dict(K_pages=0), dict(V_pages=0), dict(K=p + 8), dict(slots=3 * p + 2), dict(B=0), dict(L=0),
                      dict(slot_stride=-1), dict(k_stride=(512, 128, 4)), dict(v_stride=(-8, 8, 8)), dict(V=p), dict(V_pages=4 * p), dict(K=4 * p),
                      dict(K_exp=0 if e[0] else 6 * p), dict(V_exp=0 if e[0] else 6 * p)):
            a = {**ok, **patch}
            refused(A, 1, A.ae_cache_append, h, *a.values())
            refused(A, 1, A.ae_cache_read, h, a["K_pages"], a["V_pages"], a["K_exp"], a["V_exp"], a["B"], a["L"], a["slots"], a["slot_stride"],
                    a["K"], a["k_stride"], a["V"], a["v_stride"])
        A.ae_cache_destroy(h)
    A.ae_cache_destroy(None)


CACHED = dict(B=2, H_q=8, n_new=1, table_width=4, max_length=100, scale=0.1)


@pytest.mark.parametrize("patch,status", [
    (dict(B=0), 1), (dict(H_q=0), 1), (dict(n_new=0), 1), (dict(table_width=0), 1), (dict(H_q=7), 1), (dict(max_length=0), 1), (dict(max_length=129), 1),
    (dict(prefix_length=-1), 1), (dict(chunk=-128), 1), (dict(chunk=100), 1), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(out_dtype=2), 1), (dict(q_stride=(1024, 128, 4)), 1), (dict(o_stride=(-8, 128, 128)), 1), (dict(B=1 << 22), 2),
    (dict(prefix_length=(1 << 30) + 1), 2), (dict(B=1 << 20, prefix_length=1 << 20, chunk=128), 2),
])
def test_cached_refusals(A, patch, status):
    c = A.ae_cache_create(**CACHE)
    refused(A, status, A.ae_cached_create, c, **{**CACHED, **patch})
    A.ae_cache_destroy(c)


def test_cached_call_refusals(A):
    refused(A, 1, A.ae_cached_create, None, **CACHED)
    p = 1 << 20
    for dtype, prefix, chunk in (("bf16", 0, 0), ("e4m3", 0, 0), ("bf16", 50, 0), ("e4m3", 50, 128)):
        c = A.ae_cache_create(**CACHE, dtype=dtype)
        h = A.ae_cached_create(c, **CACHED, prefix_length=prefix, chunk=chunk)
        A.ae_cache_destroy(c)  # (the handle keeps what it needs of it)
        ws = A.ae_cached_workspace_bytes(h)
        assert (ws > 0) == (prefix > 0)
        e = (6 * p, 7 * p) if dtype == "e4m3" else (0, 0)
        ok = dict(Q=p, K_pages=2 * p, V_pages=3 * p, K_exp=e[0], V_exp=e[1], table=4 * p, lengths=5 * p, prefix_table=8 * p if prefix else 0, O=9 * p,
                  stats=10 * p, workspace=11 * p if ws else 0, workspace_bytes=ws)
        bad = [dict(Q=0), dict(K_pages=0), dict(V_pages=0), dict(table=0), dict(lengths=0), dict(O=0), dict(Q=p + 8), dict(O=9 * p + 8), dict(table=4 * p + 2),
               dict(stats=10 * p + 1), dict(O=p), dict(O=2 * p), dict(stats=9 * p), dict(stats=5 * p), dict(prefix_table=0 if prefix else 8 * p),
               dict(K_exp=0 if e[0] else 6 * p), dict(V_exp=0 if e[1] else 7 * p)]
        if ws:
            bad += [dict(workspace=0), dict(workspace=11 * p + 16), dict(workspace_bytes=ws - 1), dict(workspace=9 * p), dict(workspace=4 * p)]
            refused(A, 1, A.ae_cached_init_workspace, h, 0, ws)
            refused(A, 1, A.ae_cached_init_workspace, h, 11 * p, ws - 1)
        for patch in bad:
            refused(A, 1, A.ae_cached_forward, h, *{**ok, **patch}.values())
        A.ae_cached_destroy(h)
    A.ae_cached_destroy(None)
    for call in (A.ae_cached_workspace_bytes, A.ae_cached_query):
        refused(A, 1, call, None)
    refused(A, 1, A.ae_cached_init_workspace, None, p, 0)
    refused(A, 1, A.ae_cached_forward, None, *[p] * 12)


def test_cached_layout(A):
    c = A.ae_cache_create(n_pages=1 << 16, page_size=64, H_kv=8, D_qk=128, D_v=128)
    try:
        def layout(**kw):
            h = A.ae_cached_create(c, **{**CACHED, "H_q": 32, "table_width": 1 << 14, **kw})
            q, ws = A.ae_cached_query(h), A.ae_cached_workspace_bytes(h)
            A.ae_cached_destroy(h)
            return q, ws
        # one long sequence is cut, many short ones are not; a caller's ranges are taken
        q, ws = layout(B=1, max_length=100000)
        assert q["own_chunk"] % 128 == 0 and q["own_chunk"] < 100000 and q["launches"] == 1 and ws > 0
        q, ws = layout(B=256, max_length=300)
        assert q["own_chunk"] >= 300 and ws == 0
        assert layout(B=4, max_length=5000, chunk=640)[0]["own_chunk"] == 640
        # rows of few sequences share the launch, those of many walk the prefix in one of their own
        assert layout(B=4, max_length=300, prefix_length=2000)[0]["launches"] == 1
        q, _ = layout(B=256, H_q=64, max_length=300, prefix_length=32768)
        assert q["launches"] == 2 and q["prefix_chunk"] % 128 == 0
        assert layout(B=4, n_new=16, max_length=300, prefix_length=2000)[0]["launches"] == 2  # (64 rows a sequence)
        for B in (1, 7, 63, 200):  # no size is left without a layout
            for n in (1, 3, 8, 40):
                for L in (n, 77, 4097, 900000):
                    q, _ = layout(B=B, n_new=n, max_length=max(n, L))
                    assert q["waves"] in (4, 8) and q["own_chunk"] % 128 == 0
    finally:
        A.ae_cache_destroy(c)


def test_frequencies(A):
    plain, one = A.rotary_frequencies(64)
    assert one == 1.0 and plain[0] == 1.0 and math.isclose(plain[-1], 10000.0 ** (-62 / 64))
    lin, _ = A.rotary_frequencies(64, scaling="linear", factor=4.0)
    assert all(math.isclose(a, b / 4) for a, b in zip(lin, plain))
    ntk, _ = A.rotary_frequencies(64, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and math.isclose(ntk[-1], plain[-1] / 4)
    parts, amp = A.rotary_frequencies(64, scaling="by_parts", factor=4.0)
    assert math.isclose(amp, 0.1 * math.log(4) + 1) and parts[0] == plain[0] and math.isclose(parts[-1], plain[-1] / 4)
    assert all(b / 4 <= a * (1 + 1e-12) and a <= b * (1 + 1e-12) for a, b in zip(parts, plain))
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=64, base=0.0), dict(rot_dim=64, factor=0.5), dict(rot_dim=64, scaling="else"),
                dict(rot_dim=2, scaling="ntk", factor=2.0), dict(rot_dim=64, scaling="by_parts", fast_turns=1.0)):
        with pytest.raises(ValueError):
            A.rotary_frequencies(**bad)


def test_host_tensors_are_refused(A):
    import torch
    q = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        A.rotary_forward(q, None, torch.arange(3, dtype=torch.int32), freqs=[1.0] * 32)
    with pytest.raises(ValueError):
        A.PagedCache.empty(2, 2, 16, 64, 64, device="cpu")
    with pytest.raises(ValueError):
        A.PagedCache(*[torch.zeros(2, 2, 16, 64, dtype=torch.float16)] * 2)


def test_definition_of_the_quantised_rows():
    from oracle.serving_oracle import E4M3, dequantise, quantise
    assert E4M3[126] == 448 and E4M3[1] == 2.0 ** -9 and E4M3[8] == 2.0 ** -6 and np.isnan(E4M3[127]) and E4M3[128 + 56] == -1.0
    g = np.random.default_rng(1)
    x = g.standard_normal((50, 64)) * np.exp(4 * g.standard_normal((50, 1)))
    q, e = quantise(x)
    top, k = np.abs(x).max(-1), e.astype(int) - 127
    assert (top <= 448 * np.ldexp(1.0, k)).all() and (top > 448 * np.ldexp(1.0, k - 1)).all()
    near = np.abs(x[..., None] - E4M3[:127] * np.ldexp(1.0, k)[:, None, None]).min(-1)
    assert np.allclose(np.minimum(np.abs(dequantise(q, e) - x), np.abs(dequantise(q, e) - x)), np.minimum(near, np.abs(x[..., None] + E4M3[:127] * np.ldexp(1.0, k)[:, None, None]).min(-1)))
    import torch  # the 8-bit type's own rounding says the same
    t = torch.from_numpy(x * np.ldexp(1.0, -k)[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(t, quantise(torch.from_numpy(x * np.ldexp(1.0, -k)[:, None]).float().double().numpy() * np.ldexp(1.0, k)[:, None])[0])


@pytest.mark.parametrize("patch,status", [(dict(scale=3e38), 1), (dict(B=64, prefix_length=1 << 28, chunk=128), 2)])
def test_cached_limits(A, patch, status):
    # a scale whose product with log2(e) is infinite; partial results of 2^21 ranges of 512 rows
    c = A.ae_cache_create(**CACHE)
    refused(A, status, A.ae_cached_create, c, **{**CACHED, **patch})
    A.ae_cache_destroy(c)


class OnDevice:
    """A host tensor that says it is on the device: the checks and the strides of a plan can be looked at without one."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def offsets(strides, shape):
    """Element offset of every row of [B, H, L, D]."""
    B, H, L, _ = shape
    return [b * strides[0] + h * strides[1] + l * strides[2] for b in range(B) for h in range(H) for l in range(L)]


def offsets_in_c(strides, shape):
    """The same as the C ABI takes the strides."""
    s, (_, H, L, D) = [int(x) for x in strides], shape
    return offsets([H * L * D, L * D, D] if s == [0, 0, 0] else [0, 0, 0] if s == [-2 ** 63, 0, 0] else s, shape)


def expanded_rows(D, dtype):
    """Tensors with every combination of expanded dimensions, sizes of one among them."""
    import itertools

    import torch
    for B, H, L in ((2, 4, 10), (1, 4, 10), (2, 1, 10), (2, 4, 1), (1, 1, 10), (1, 1, 1)):
        for kept in itertools.product((False, True), repeat=3):
            yield torch.zeros(*[n if k else 1 for n, k in zip((B, H, L), kept)], D, dtype=dtype).expand(B, H, L, D)
        yield torch.zeros(D, dtype=dtype).expand(3, 5, 11, D)[:B, :H, :L]  # (sizes of one with a stride of zero)


def test_rows_are_where_the_tensor_has_them(A, monkeypatch):
    import torch
    calls = []

    def note(name, keep):
        real = getattr(A, name)

        def call(*a, **kw):
            calls.append(keep(a, kw))
            return real(*a, **kw)

        monkeypatch.setattr(A, name, call)

    note("ae_rotary_create", lambda a, kw: (kw["q_stride"], kw["k_stride"]))
    note("ae_cached_create", lambda a, kw: (kw["q_stride"],))
    pos = OnDevice(torch.zeros(10, dtype=torch.int32))
    for t in expanded_rows(64, torch.bfloat16):
        want, (B, H, L, D) = offsets(t.stride(), t.shape), t.shape
        x, out = OnDevice(t), OnDevice(torch.zeros(t.shape, dtype=t.dtype))
        A.RotaryPlan(x, x, OnDevice(pos.t[:L]), out, out, freqs=[1.0] * 32)
        for s in calls.pop():
            assert offsets_in_c(s, t.shape) == want, (t.shape, t.stride())
        # (a plan whose call needs no workspace, hence no device: one range of keys)
        cache = A.PagedCache(OnDevice(torch.zeros(4, H, 16, 64, dtype=torch.bfloat16)), OnDevice(torch.zeros(4, H, 16, 64, dtype=torch.bfloat16)))
        A.CachedAttentionPlan(cache, x, out, max_length=64, table_width=4, scale=1.0)
        assert offsets_in_c(calls.pop()[0], t.shape) == want, (t.shape, t.stride())
        assert all(offsets_in_c(s, t.shape) == want for s in cache._rows(t, t, B, L)), (t.shape, t.stride())
    assert not calls


def test_one_row_for_all_is_read_only(A):
    one, p = (A.ONE_ROW, 0, 0), 1 << 20
    for bad in ((A.ONE_ROW, 64, 0), (A.ONE_ROW, 0, 64), (0, A.ONE_ROW, 0), (64, 0, A.ONE_ROW)):
        refused(A, 1, A.ae_rotary_create, **ROT, q_stride=bad)
        refused(A, 1, A.ae_rotary_create, **ROT, k_out_stride=bad)
    for name, forward in (("q_stride", True), ("k_stride", True), ("q_out_stride", False), ("k_out_stride", False)):
        h = A.ae_rotary_create(**ROT, **{name: one})
        refused(A, 1, A.ae_rotary_backward if forward else A.ae_rotary_forward, h, p, 2 * p, 3 * p, 4 * p, 5 * p)
        A.ae_rotary_destroy(h)
    h = A.ae_cache_create(**CACHE)
    refused(A, 1, A.ae_cache_read, h, 4 * p, 5 * p, 0, 0, 1, 4, 3 * p, 0, p, one, 2 * p, (0, 0, 0))
    refused(A, 1, A.ae_cache_read, h, 4 * p, 5 * p, 0, 0, 1, 4, 3 * p, 0, p, (0, 0, 0), 2 * p, one)
    refused(A, 1, A.ae_cache_append, h, p, (A.ONE_ROW, 8, 8), 2 * p, one, 1, 4, 3 * p, 0, 4 * p, 5 * p)
    A.ae_cached_destroy(A.ae_cached_create(h, **CACHED, q_stride=one))
    refused(A, 1, A.ae_cached_create, h, **CACHED, o_stride=one)
    refused(A, 1, A.ae_cached_create, h, **CACHED, q_stride=(A.ONE_ROW, 128, 128))
    A.ae_cache_destroy(h)


def allocations(monkeypatch):
    """Records, for every torch.empty, the stream that the allocating thread had entered (None: the current one)."""
    import contextlib

    import torch
    seen, inside, real = [], [None], torch.empty

    @contextlib.contextmanager
    def entered(stream):
        inside.append(stream)
        yield
        inside.pop()

    def empty(*a, **kw):
        seen.append(inside[-1])
        return real(*a, **kw)

    monkeypatch.setattr(torch.cuda, "stream", entered)
    monkeypatch.setattr(torch, "empty", empty)
    return seen


@pytest.mark.parametrize("stream", [None, "another"])
def test_outputs_belong_to_the_stream_that_writes_them(A, monkeypatch, stream):
    import torch
    seen = allocations(monkeypatch)

    class Plan:
        def __init__(self, *a, **kw):
            pass

        def forward(self, *a, stream=None):
            return stream

        backward = forward

    monkeypatch.setattr(A, "RotaryPlan", Plan)
    x = torch.zeros(1, 2, 3, 64)
    for call in (A.rotary_forward, A.rotary_backward):
        call(x, x, torch.zeros(3, dtype=torch.int32), freqs=[1.0] * 32, stream=stream)
        assert seen == [stream, stream]
        seen.clear()
    cache = A.PagedCache.__new__(A.PagedCache)
    cache.handle, cache.device, cache._bf16, cache._int, cache.H_kv, cache.D_qk, cache.D_v = None, torch.device("cpu"), torch.bfloat16, torch.int32, 2, 64, 64
    cache.k = cache.v = x
    cache.k_exp = cache.v_exp = None
    monkeypatch.setattr(A, "_enqueue", lambda *a: None)
    cache.read(torch.zeros(3, dtype=torch.int32), stream=stream)
    assert seen == [stream, stream]


def test_workspace_is_held_for_the_streams_that_use_it(A, monkeypatch):
    import types

    import torch
    current, calls, held = [types.SimpleNamespace(cuda_stream=5)], [], []
    monkeypatch.setattr(A, "_raw_stream", lambda index: current[0].cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: current[0])
    monkeypatch.setattr(A, "_enqueue", lambda call, device, stream, *a: calls.append(stream))
    x, table, L = OnDevice(torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16)), torch.zeros(2, 70, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    cache = A.PagedCache(*[OnDevice(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))] * 2)
    for chunk, some in ((128, True), (1152, False)):  # ranges that are joined; one range, no workspace
        current[0] = types.SimpleNamespace(cuda_stream=5)
        plan = A.CachedAttentionPlan(cache, x, x, max_length=1100, table_width=70, scale=1.0, chunk=chunk)
        assert (plan.workspace is not None) == some
        if some:
            ws, plan.workspace = plan.workspace, types.SimpleNamespace(data_ptr=lambda: 0, record_stream=held.append)
        other, third = types.SimpleNamespace(cuda_stream=8), types.SimpleNamespace(cuda_stream=9)
        calls.clear()
        for s in (None, current[0], other, other, None):
            plan.forward(x, table, L, x, stream=s)
        current[0] = third
        plan.forward(x, table, L, x)
        plan.forward(x, table, L, x, stream=other)
        assert len(calls) == 7 and held == ([other, third] if some else [])
        held.clear()
