"""Span attention, capped and biased scores over the cache, cache weights and eviction where elements lie beyond 2^31 of their tensor's start: the same
rows in a small tensor give the same bits, as the same instance of a kernel walks the same tiles in the same order."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def test_span_attention_of_large_tensors(A):
    """2 x 72 heads x 131072 rows of 128: 2.4e9 elements; the last 16 heads again by themselves."""
    B, H, L, D, few = 2, 72, 131072, 128, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    Q, K, V, dO = (torch.randn(B, H, L, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    kw = dict(scale=0.09, cap=20.0, mask="sliding_window", window=64)

    def both(q, k, v, do):
        stats = torch.empty(q.shape[:3], device="cuda")
        O = A.span_attention_forward(q, k, v, stats=stats, out_dtype=torch.bfloat16, kv_splits=1, **kw)
        return O, stats, *A.span_attention_backward(q, k, v, O, do, stats, grad_dtype=torch.bfloat16, **kw)

    want = both(*(t[1:, H - few:].clone() for t in (Q, K, V, dO)))
    got = both(Q, K, V, dO)
    for a, b in zip(want, got):
        assert torch.equal(a, b[1:, H - few:])


@pytest.mark.parametrize("dtype,n_pages", [("bf16", 36000), ("e4m3", 72000)])
def test_pages_far_into_the_cache(A, dtype, n_pages):
    """Lists on the last of so many pages of 8 x 64 rows of 128 (4.7e9 bytes), against a cache that holds just these."""
    H_kv, page, D, lengths, n = 8, 64, 128, [300, 129], 2
    g = torch.Generator(device="cuda").manual_seed(2)
    width = 5
    used = 2 * width
    k, v = (torch.randn(1, H_kv, used * page, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(2, 32, n, D, generator=g, device="cuda").to(torch.bfloat16)
    weights = torch.rand(2, H_kv, width * page, generator=g, device="cuda")
    L = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    results = []
    for pages in (used, n_pages):
        cache = A.PagedCache.empty(pages, H_kv, page, D, D, dtype=dtype)
        slots = torch.arange(used * page, dtype=torch.int32, device="cuda")[None] + (pages - used) * page
        cache.append(k, v, slots)
        table = (pages - 1 - torch.arange(used, dtype=torch.int32, device="cuda")).view(2, width).contiguous()
        stats = torch.empty(2, 32, n, device="cuda")
        O = A.attention_cached(Q, cache, table, L, scale=0.09, cap=20.0, slopes=[2.0 ** (-h / 4) for h in range(32)])
        A.attention_cached(Q, cache, table, L, scale=0.09, cap=20.0, stats=stats)
        w, p = weights.clone(), torch.arange(width * page, dtype=torch.int32, device="cuda").expand(2, H_kv, -1).contiguous()
        new = torch.tensor([900, 901], dtype=torch.int32, device="cuda")
        A.cache_weights(Q, cache, table, L, stats, w, p, new, scale=0.09, cap=20.0)
        kept = A.cache_evict(cache, table, L, w, p, keep=100, recent=20, sinks=2)
        rows = cache.read(slots)
        results.append((O, stats, w, p, kept, *rows))
        del cache
    for a, b in zip(*results):
        assert torch.equal(a, b)
