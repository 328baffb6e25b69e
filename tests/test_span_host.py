"""CPU-only checks of span attention: symbols, refusals, the definition in 64 bits."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from oracle.span_oracle import document_spans, span_attention, span_attention_backward, spans_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_15349_amd", "libae_attn.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libae_attn.so not built (run __graft_entry__.build())")


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def refused(A, status, call, *a, **kw):
    with pytest.raises(A.AeAttnError) as ei:
        call(*a, **kw)
    assert ei.value.status == status, str(ei.value)


@built
def test_library_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "ae_span.h")).read()
    names = set(re.findall(r"\b(ae_span_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)))
    assert {"ae_span_create", "ae_span_forward", "ae_span_backward", "ae_span_documents"} <= names
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), f"{n} declared in the header but not exported"


SPAN = dict(B=2, H_q=4, H_kv=2, L_q=10, L_k=20, D_qk=64, D_v=64, scale=0.1)


@built
@pytest.mark.parametrize("patch,status", [
    (dict(B=0), 1), (dict(H_q=0), 1), (dict(H_kv=0), 1), (dict(L_q=0), 1), (dict(L_k=0), 1), (dict(H_kv=3), 1), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=3e38), 1), (dict(cap=-1.0), 1), (dict(cap=float("inf")), 1), (dict(cap=float("nan")), 1), (dict(cap=1e-44), 1),
    (dict(scale=1e-30, cap=1e30), 1), (dict(mask=4), 1), (dict(mask="sliding_window"), 1), (dict(mask="sliding_window", window=-1), 1),
    (dict(out_dtype=2), 1), (dict(slopes=[0.0, 0.0, float("nan"), 0.0]), 1), (dict(slopes=[1e35] * 4), 1), (dict(q_stride=(640, 64, 60)), 1),
    (dict(k_stride=(-64, 64, 64)), 1), (dict(v_stride=(0, 0, 32)), 1), (dict(o_stride=(640, 64, 66)), 1), (dict(D_qk=128), 2), (dict(D_qk=96, D_v=96), 2),
    (dict(B=1 << 24, H_q=2), 2), (dict(L_q=1 << 29), 2), (dict(H_q=258, slopes=[0.0] * 258), 2), (dict(L_k=1 << 24, slopes=[0.0] * 4), 2),
    (dict(L_k=1 << 26), 2), (dict(B=1 << 20, L_q=1 << 19), 2),
])
def test_create_refusals(A, patch, status):
    refused(A, status, A.ae_span_create, **{**SPAN, **patch})


@built
def test_call_refusals(A):
    p = 1 << 20
    h = A.ae_span_create(**SPAN, mask="spans")
    good = [p, 2 * p, 3 * p, 4 * p, 5 * p, 10, 6 * p, 7 * p]  # Q, K, V, begin, end, stride, O, stats
    for n, bad in [(0, 0), (1, 0), (2, 0), (6, 0), (0, p + 8), (6, 6 * p + 4), (7, 7 * p + 2), (3, 0), (4, 0), (3, 4 * p + 1), (5, -1), (6, p), (6, 5 * p),
                   (7, 2 * p), (7, 6 * p)]:
        a = list(good)
        a[n] = bad
        refused(A, 1, A.ae_span_forward, h, *a)
    refused(A, 1, A.ae_span_forward, None, *good)
    need = A.ae_span_backward_workspace_bytes(h)
    assert need >= 2 * 4 * 10 * 4 + 2 * 2 * 10 * 4
    #       Q  K      V      begin  end    stride O      dO     strides    stats  dQ      dK      dV      type  ws      bytes
    good = [p, 2 * p, 3 * p, 4 * p, 5 * p, 10, 6 * p, 7 * p, (0, 0, 0), 8 * p, 9 * p, 10 * p, 11 * p, "bf16", 12 * p, need]
    for n, bad in [(0, 0), (6, 0), (7, 0), (9, 0), (10, 0), (12, 0), (14, 0), (7, 7 * p + 8), (14, 12 * p + 8), (9, 8 * p + 1), (13, 2), (3, 0), (15, need - 1),
                   (8, (0, 64, 32)), (8, (-8, 64, 64)), (8, (640, 64, 68)), (10, 6 * p), (11, 10 * p + 8), (12, 10 * p), (14, 8 * p)]:
        a = list(good)
        a[n] = bad
        refused(A, 1, A.ae_span_backward, h, *a)
    refused(A, 1, A.ae_span_backward, None, *good)
    A.ae_span_destroy(h)
    A.ae_span_destroy(None)
    h = A.ae_span_create(**SPAN)
    refused(A, 1, A.ae_span_forward, h, p, 2 * p, 3 * p, 4 * p, 5 * p, 0, 6 * p, 0)  # spans that no one asked for
    A.ae_span_destroy(h)


@built
def test_documents_refusals(A):
    p = 1 << 20
    good = [2, 100, 3, p, 4, 2 * p, 3, "causal", 0, 3 * p, 4 * p]
    for n, bad in [(0, 0), (1, 0), (2, 0), (3, 0), (9, 0), (10, 0), (3, p + 2), (4, -1), (6, -1), (7, "spans"), (7, 9), (7, "sliding_window"), (9, p), (10, 3 * p)]:
        a = list(good)
        a[n] = bad
        refused(A, 1, A.ae_span_documents, *a)
    good[1] = (1 << 28) + 1
    refused(A, 2, A.ae_span_documents, *good)


@built
def test_host_tensors_are_refused(A):
    import torch

    x = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        A.span_attention_forward(x, x, x, scale=1.0, out=torch.zeros(1, 2, 8, 64))
    with pytest.raises(ValueError):
        A.document_spans(torch.zeros(3, dtype=torch.int32), 8)


def test_definition_by_hand():
    """Two keys, one score ln 3 above the other: weights 3/4 and 1/4; a cap and a distance that give the same."""
    V = np.array([[[[1.0], [5.0]]]])
    Q, K = np.array([[[[1.0]]]]), np.array([[[[np.log(3.0)], [0.0]]]])
    O, lse, mag = span_attention(Q, K, V, np.array([[0]]), np.array([[2]]), scale=1.0)
    assert np.allclose(O, 2.0) and np.allclose(lse, np.log(4.0)) and np.allclose(mag, 2.0)
    O, _, _ = span_attention(Q, K, V, np.array([[1]]), np.array([[2]]), scale=1.0)
    assert np.allclose(O, 5.0)
    O, lse, _ = span_attention(Q, K, V, np.array([[2]]), np.array([[2]]), scale=1.0)
    assert O.item() == 0.0 and np.isneginf(lse).all()
    # one query on the second of two keys: the first is a distance of one away
    O, _, _ = span_attention(Q, 0 * K, V, np.array([[0]]), np.array([[2]]), scale=1.0, slopes=[np.log(3.0)])
    assert np.allclose(O, (1 + 3 * 5) / 4)
    cap = np.log(3.0) / np.tanh(1.0)  # a score of `cap` is bent to ln 3
    O, _, _ = span_attention(Q * cap / np.log(3.0), K, V, np.array([[0]]), np.array([[2]]), scale=1.0, cap=cap)
    assert np.allclose(O, 2.0)


def test_spans_by_hand():
    assert [x[0].tolist() for x in spans_of("causal", 1, 3, 2)] == [[0, 0, 0], [0, 1, 2]]
    assert [x[0].tolist() for x in spans_of("sliding_window", 1, 2, 4, 2)] == [[1, 2], [3, 4]]
    begin, end = document_spans([0, 2, 2, 5], 6, "causal", prefix=[0, 9, 2])
    assert begin[0].tolist() == [0, 0, 2, 2, 2, 0] and end[0].tolist() == [1, 2, 4, 4, 5, 0]


@pytest.mark.parametrize("kw", [dict(), dict(cap=2.0), dict(slopes=[0.3, 0.1]), dict(cap=1.0, slopes=[0.2, -0.1])])
def test_gradients_are_differences(kw):
    """Central differences of step 1e-5 in 64 bits: their error is about 1e-10 of the third derivative and 1e-11 of rounding."""
    g = np.random.RandomState(0)
    Q, K, V, dO = g.randn(1, 2, 5, 3), g.randn(1, 1, 6, 3), g.randn(1, 1, 6, 4), g.randn(1, 2, 5, 4)
    begin, end = np.array([[0, 1, 2, 3, 0]]), np.array([[6, 4, 2, 6, 1]])
    got, _ = span_attention_backward(Q, K, V, dO, begin, end, scale=0.7, **kw)
    for n in range(3):
        want = np.zeros_like(got[n])
        for at in np.ndindex(want.shape):
            f = []
            for step in (1e-5, -1e-5):
                x = [Q.copy(), K.copy(), V.copy()]
                x[n][at] += step
                f.append((span_attention(*x, begin, end, scale=0.7, **kw)[0] * dO).sum())
            want[at] = (f[0] - f[1]) / 2e-5
        assert np.abs(got[n] - want).max() < 1e-7


@built
def test_split_refusals(A):
    for kw in (dict(kv_splits=-1), dict(kv_splits=257)):
        refused(A, 1, A.ae_span_create, **{**SPAN, **kw})
    refused(A, 2, A.ae_span_create, **{**SPAN, "L_q": 1 << 20, "H_q": 1 << 10, "kv_splits": 256})
    p = 1 << 20
    good = [p, 2 * p, 3 * p, 0, 0, 0, 6 * p, 7 * p]
    h = A.ae_span_create(**SPAN, kv_splits=3)
    need = A.ae_span_workspace_bytes(h)
    assert need == 3 * 2 * 4 * 10 * 65 * 4
    for ws, size in ((0, need), (8 * p, need - 1), (8 * p + 8, need), (6 * p, need), (p, need)):
        refused(A, 1, A.ae_span_forward_split, h, *good, ws, size)
    for n, bad in [(0, 0), (6, 0), (6, 2 * p), (7, 7 * p + 2)]:
        a = list(good)
        a[n] = bad
        refused(A, 1, A.ae_span_forward_split, h, *a, 8 * p, need)
    refused(A, 1, A.ae_span_forward_split, None, *good, 8 * p, need)
    refused(A, 1, A.ae_span_workspace_bytes, None)
    A.ae_span_destroy(h)


@built
def test_ranges_that_are_chosen(A):
    """Few rows over many keys are cut, many rows are not."""
    def ranges(**kw):
        d = {**SPAN, "D_qk": 128, "D_v": 128, **kw}
        h = A.ae_span_create(**d)
        n = A.ae_span_workspace_bytes(h) / (d["B"] * d["H_q"] * d["L_q"] * 129 * 4)
        A.ae_span_destroy(h)
        return int(n)

    assert ranges(B=1, H_q=16, H_kv=16, L_q=17, L_k=8192) >= 8
    assert 4 <= ranges(B=1, H_q=16, H_kv=16, L_q=512, L_k=4096) <= 8
    assert ranges(B=4, H_q=32, H_kv=8, L_q=64, L_k=4096) == 2
    for kw in (dict(B=2, H_q=12, H_kv=12, L_q=1023, L_k=1023), dict(B=1, H_q=32, H_kv=8, L_q=8192, L_k=8192), dict(B=1, H_q=4, H_kv=4, L_q=10, L_k=100),
               dict(B=1, H_q=16, H_kv=16, L_q=17, L_k=8192, mask="sliding_window", window=100), dict(B=1, H_q=16, H_kv=16, L_q=17, L_k=8192, kv_splits=1)):
        assert ranges(**kw) == 0


@built
def test_slopes_far_above_the_scale_are_refused(A):
    for slopes in ([0.0, 1e2, 0.0, 0.0], [-1e2] * 4):
        refused(A, 1, A.ae_span_create, **{**SPAN, "scale": 1e-29, "slopes": slopes})
    A.ae_span_destroy(A.ae_span_create(**{**SPAN, "scale": 1e-27, "slopes": [1e2] * 4}))


CAP_PARAMS = """
#include <stdio.h>
#include <stdlib.h>
#include "%s"
int main(int n, char** a) {
  for (int i = 1; i + 1 < n; i += 2) {
    const float scale = strtof(a[i], nullptr), cap = strtof(a[i + 1], nullptr);
    const ae::CapParams c = ae::cap_params(scale, cap);
    printf("%%d %%.9g %%.9g %%.9g", (int)ae::cap_ok(scale, cap), c.limit, c.unit, c.e);
    for (float x : c.poly) printf(" %%.9g", x);
    for (float x : c.tanh) printf(" %%.9g", x);
    printf("\\n");
  }
}
"""


def test_constants_of_accepted_caps(tmp_path):
    """Over all accepted magnitudes of cap and scale the capped score that the kernels' constants stand for, evaluated in 64 bits: where the series holds, the
    definition's to 3e-7 of itself, a term of it that is left out included; where it does not, the exact form's constants are there."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not there")
    src, out = tmp_path / "cap.hip", str(tmp_path / "cap")
    src.write_text(CAP_PARAMS % os.path.join(ROOT, "paper_2502_15349_amd", "csrc", "span.hpp"))
    subprocess.run([hipcc, "--offload-host-only", "-O1", "-std=c++17", str(src), "-o", out], check=True, capture_output=True)
    pairs = [(s, c) for s in (0.125, -0.125, 1.0, 1e-3, 1e3, 1e-30, 1e-37, 1e30) for c in [10.0 ** n for n in range(-37, 38)] + [50.0, 2e36, 1.5e38]]
    got = subprocess.run([out, *[repr(x) for p in pairs for x in p]], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    assert len(got) == len(pairs)
    accepted = 0
    for (scale, cap), line in zip(pairs, got):
        ok, limit, unit, e, *rest = (float(x) for x in line.split())
        scale, cap = float(np.float32(scale)), float(np.float32(cap))
        if not ok:
            continue
        accepted += 1
        poly, tanh, k = np.array(rest[:5]), np.array(rest[5:]), scale / cap
        # (constants below 2^-126 have fewer bits; unit log2(e) rounded twice)
        assert abs(unit - cap / np.log(2)) <= 2e-7 * unit and abs(e - 2 * k / np.log(2)) <= 2e-7 * abs(e) + 1e-44
        if limit < 0:
            assert (poly == 0).all() and (tanh == 0).all()
            continue
        assert abs(tanh[0] - k) <= 2e-7 * abs(k) and abs(poly[0] - scale / np.log(2)) <= 2e-7 * abs(scale) + 1e-44, (scale, cap)
        s = limit * np.array([1.0, 0.99, 0.5, 1e-2, 1e-6])
        y = k * s
        for c, want in ((tanh, np.tanh(y)), (poly, cap / np.log(2) * np.tanh(y))):
            value = s * sum(x * (s * s) ** n for n, x in enumerate(c))
            assert np.all(np.abs(value - want) <= 3e-7 * np.abs(want) + 1e-44 * s), (scale, cap)
    assert accepted > 400


@built
def test_steep_slopes_are_refused(A):
    for slopes in ([0.0, 128.5, 0.0, 0.0], [-1e3] * 4, [0.0, 0.0, 0.0, 1e20]):
        refused(A, 2, A.ae_span_create, **{**SPAN, "slopes": slopes})
    A.ae_span_destroy(A.ae_span_create(**{**SPAN, "slopes": [128.0, -128.0, 0.0, 1.0]}))
