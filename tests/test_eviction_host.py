"""CPU-only checks of capped and biased scores over the cache, of the weights of cached entries and of their eviction: refusals, definitions."""
import os

import numpy as np
import pytest

from oracle.serving_oracle import attend, kept_entries, received

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2502_15349_amd", "libae_attn.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libae_attn.so not built (run __graft_entry__.build())")
CACHE = dict(n_pages=4, page_size=32, H_kv=2, D_qk=128, D_v=128)
CACHED = dict(B=2, H_q=8, n_new=1, table_width=4, max_length=100, scale=0.1)
WEIGH = dict(B=2, H_q=8, n_new=3, table_width=4, max_length=100, capacity=128, scale=0.1)
EVICT = dict(B=2, table_width=4, max_length=100, capacity=128, keep=50)


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


@pytest.fixture(params=["bf16", "e4m3"])
def cache(A, request):
    h = A.ae_cache_create(**CACHE, dtype=request.param)
    yield h, request.param == "e4m3"
    A.ae_cache_destroy(h)


def refused(A, status, call, *a, **kw):
    with pytest.raises(A.AeAttnError) as ei:
        call(*a, **kw)
    assert ei.value.status == status, str(ei.value)


@built
@pytest.mark.parametrize("patch,status", [
    (dict(cap=-1.0), 1), (dict(cap=float("nan")), 1), (dict(cap=float("inf")), 1), (dict(cap=1e-44), 1), (dict(cap=1e30, scale=1e-30), 1),
    (dict(slopes=[0.0] * 7 + [float("nan")]), 1), (dict(slopes=[1e35] * 8), 1), (dict(cap=5.0, H_q=7), 1), (dict(cap=5.0, scale=0.0), 1),
    (dict(cap=5.0, scale=float("nan")), 1), (dict(cap=5.0, max_length=129), 1), (dict(H_q=258, slopes=[0.0] * 258), 2),
    (dict(table_width=1 << 20, max_length=(1 << 24) + 1, slopes=[0.0] * 8), 2), (dict(prefix_length=1 << 24, slopes=[0.0] * 8), 2),
    (dict(cap=5.0, n_new=9, prefix_length=64), 2), (dict(cap=5.0, B=1025, prefix_length=64), 2),
])
def test_scored_refusals(A, cache, patch, status):
    refused(A, status, A.ae_cached_create, cache[0], **{**CACHED, "cap": 0.0, **patch})


@built
def test_scored_handles(A, cache):
    refused(A, 1, A.ae_cached_create, None, **CACHED, cap=1.0)
    with pytest.raises(ValueError):
        A.ae_cached_create(cache[0], **CACHED, slopes=[1.0])
    for kw in (dict(cap=3.0), dict(slopes=[0.5] * 8), dict(cap=3.0, scale=-0.1), dict(cap=3.0, n_new=8, prefix_length=64), dict(cap=3.0, B=256, prefix_length=64)):
        h = A.ae_cached_create(cache[0], **{**CACHED, **kw})
        assert A.ae_cached_query(h)["launches"] == 1
        A.ae_cached_destroy(h)


@built
@pytest.mark.parametrize("patch,status", [
    (dict(B=0), 1), (dict(H_q=0), 1), (dict(H_q=7), 1), (dict(n_new=0), 1), (dict(table_width=0), 1), (dict(max_length=0), 1), (dict(max_length=129), 1),
    (dict(capacity=99), 1), (dict(scale=0.0), 1), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(cap=-1.0), 1), (dict(cap=float("nan")), 1),
    (dict(q_stride=(1024, 128, 4)), 1), (dict(q_stride=(-8, 8, 8)), 1), (dict(B=1 << 22), 2), (dict(B=1 << 23, H_q=2, n_new=2), 2),
    (dict(table_width=1 << 26, max_length=(1 << 30) + 1, capacity=1 << 31), 2), (dict(B=1, H_q=1 << 14, n_new=1 << 11), 2),
])
def test_weigh_refusals(A, cache, patch, status):
    refused(A, status, A.ae_weigh_create, cache[0], **{**WEIGH, **patch})
    refused(A, 1, A.ae_weigh_create, None, **WEIGH)


@built
def test_weigh_call_refusals(A, cache):
    p = 1 << 20
    h = A.ae_weigh_create(cache[0], **WEIGH)
    #     Q  K      Ke                        table  lengths stats  weights out    positions new    stride
    ok = [p, 2 * p, 3 * p if cache[1] else 0, 4 * p, 5 * p, 6 * p, 7 * p, 8 * p, 9 * p, 10 * p, 3]
    bytes_ = 4 * 2 * 2 * 128
    for n, bad in [(0, 0), (1, 0), (2, 0 if cache[1] else 3 * p), (3, 0), (4, 0), (5, 0), (6, 0), (7, 0), (8, 0), (9, 0), (0, p + 8), (1, 2 * p + 8), (3, 4 * p + 2),
                   (4, 5 * p + 1), (5, 6 * p + 2), (6, 7 * p + 2), (7, 8 * p + 2), (8, 9 * p + 2), (9, 10 * p + 2), (10, -1), (7, p), (7, 2 * p), (7, 4 * p), (7, 5 * p),
                   (7, 6 * p), (7, 9 * p), (7, 10 * p), (8, 7 * p), (8, 5 * p), (8, 10 * p), (7, 7 * p + 4), (6, 8 * p + bytes_ - 4), (8, 8 * p + 4), (8, 7 * p - 4)]:
        a = list(ok)
        a[n] = bad
        refused(A, 1, A.ae_weigh_forward, h, *a)
    refused(A, 1, A.ae_weigh_forward, None, *ok)
    A.ae_weigh_destroy(h)
    A.ae_weigh_destroy(None)


@built
@pytest.mark.parametrize("patch,status", [
    (dict(B=0), 1), (dict(table_width=0), 1), (dict(max_length=0), 1), (dict(max_length=129), 1), (dict(capacity=99), 1), (dict(keep=0), 1), (dict(recent=-1), 1),
    (dict(sinks=-1), 1), (dict(B=1 << 24), 2), (dict(table_width=1 << 26, max_length=(1 << 30) + 1, capacity=1 << 31), 2),
])
def test_evict_refusals(A, cache, patch, status):
    refused(A, status, A.ae_evict_create, cache[0], **{**EVICT, **patch})
    refused(A, 1, A.ae_evict_create, None, **EVICT)


@built
def test_evict_call_refusals(A, cache):
    p = 1 << 20
    h = A.ae_evict_create(cache[0], **EVICT)
    need = A.ae_evict_workspace_bytes(h)
    #     K  V      Ke, Ve                                          table  lengths weights pos   w out  p out   l out   ws      bytes
    ok = [p, 2 * p, *((3 * p, 4 * p) if cache[1] else (0, 0)), 5 * p, 6 * p, 7 * p, 8 * p, 9 * p, 10 * p, 11 * p, 12 * p, need]
    for n, bad in [(0, 0), (1, 0), (4, 0), (5, 0), (6, 0), (7, 0), (8, 0), (9, 0), (10, 0), (11, 0), (12, need - 1), (2, 0 if cache[1] else 3 * p),
                   (3, 0 if cache[1] else 4 * p), (0, p + 8), (1, 2 * p + 8), (4, 5 * p + 2), (6, 7 * p + 1), (9, 10 * p + 2), (11, 12 * p + 2), (1, p), (8, 8 * p),
                   (9, 7 * p), (10, 6 * p), (10, 5 * p), (8, 5 * p), (11, 7 * p), (9, 9 * p), (8, 7 * p + 4), (9, 8 * p - 4), (9, 9 * p + 4), (8, 8 * p + 8)]:
        a = list(ok)
        a[n] = bad
        refused(A, 1, A.ae_evict_forward, h, *a)
    refused(A, 1, A.ae_evict_forward, None, *ok)
    refused(A, 1, A.ae_evict_workspace_bytes, None)
    A.ae_evict_destroy(h)
    A.ae_evict_destroy(None)


@built
def test_host_tensors_are_refused(A):
    import torch

    class Fake:
        handle, device, H_kv, D_qk, page_size = None, torch.device("cuda:0"), 2, 64, 16

    with pytest.raises(ValueError):
        A.CacheWeightsPlan(Fake, torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16), max_length=16, table_width=1, scale=1.0)
    with pytest.raises(ValueError):
        A.CacheEvictionPlan(Fake, torch.zeros(1, 2, 16), keep=4, max_length=16, table_width=1)


def test_received_sums_to_the_rows():
    """With the attention's own statistic a row gives one in all."""
    g = np.random.RandomState(0)
    q, k = g.randn(4, 3, 8), g.randn(2, 7, 8)
    _, lse = attend(q, k, k, 0.3)
    assert np.allclose(received(q, k, lse, 0.3).sum(1), 2 * 3)
    _, lse = attend(g.randn(2, 1, 8), k[:, :0], k[:, :0], 0.3)
    assert received(q[:, :1], k[:, :0], np.full((4, 1), -np.inf), 0.3).shape == (2, 0)


def test_kept_entries_by_hand():
    w, p = [5.0, 1.0, 3.0, 2.0, 4.0], [0, 1, 2, 3, 4]
    assert kept_entries(w, p, 9) == [0, 1, 2, 3, 4]
    assert kept_entries(w, p, 3) == [0, 4, 2]
    assert kept_entries(w, p, 2, recent=2) == [3, 4]
    assert kept_entries(w, p, 3, recent=1, sinks=2) == [0, 1, 4]
    assert kept_entries([1.0] * 5, p, 2) == [0, 1]
    assert kept_entries([np.nan, -1.0, -np.inf, 0.0], [3, 2, 1, 0], 3) == [3, 1, 2]
