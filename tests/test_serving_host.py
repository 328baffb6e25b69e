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
