"""GPU tests of the paged cache (ae_cache_append / ae_cache_read): 8-bit values and exponents are equal, bit for bit, to the
definition in 64 bits (the division by a power of two is exact, so there is one rounding and no tolerance)."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import dequantise, quantise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def rows(seed, B, H, L, D, order="bhld", spread=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, H, L, D), generator=g) * torch.exp(spread * torch.randn((B, H, L, 1), generator=g))
    x = x.to(torch.bfloat16)
    return x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if order == "blhd" else x.cuda()


def some_slots(seed, n_slots, B, L):
    return torch.randperm(n_slots, generator=torch.Generator().manual_seed(seed))[: B * L].view(B, L).to(torch.int32).cuda()


def filled(A, n_pages, H, page, dqk, dv, dtype):
    """A cache whose buffers hold a known pattern."""
    c = A.PagedCache.empty(n_pages, H, page, dqk, dv, dtype=dtype)
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(0x35)
    return c


def at_slots(pages, slots):
    """[B, H, L, ...] of the pages' rows at the slots."""
    page = pages.shape[2]
    p, i = slots.long() // page, slots.long() % page
    return pages[p, :, i].transpose(1, 2)


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("B,H,L,page,order,spread", [(1, 1, 1, 16, "bhld", 0.0), (3, 2, 5, 32, "blhd", 3.0), (2, 3, 131, 64, "bhld", 8.0),
                                                    (7, 8, 1, 256, "blhd", 0.0), (2, 12, 77, 128, "blhd", 20.0)])
def test_e4m3_rows(A, dqk, dv, B, H, L, page, order, spread):
    n_pages = -(-B * L // page) + 2
    c = filled(A, n_pages, H, page, dqk, dv, "e4m3")
    k, v, slots = rows(1, B, H, L, dqk, order, spread), rows(2, B, H, L, dv, order, spread), some_slots(3, n_pages * page, B, L)
    c.append(k, v, slots)
    ko, vo = c.read(slots)
    torch.cuda.synchronize()
    for x, pages, exps, back in ((k, c.k, c.k_exp, ko), (v, c.v, c.v_exp, vo)):
        q, e = quantise(x.cpu().double().numpy())
        assert np.array_equal(at_slots(exps, slots).cpu().numpy(), e)
        assert np.array_equal(at_slots(pages.view(torch.uint8), slots).cpu().numpy(), q)
        ref = torch.from_numpy(dequantise(q, e)).to(torch.bfloat16)
        assert torch.equal(back.cpu(), ref)
        # half a step of e4m3: 2^-4 of the value, or of the smallest normal number 2^-6 times the row's power of two
        x64 = x.cpu().double().numpy()
        step = 2.0 ** -4 * np.maximum(np.abs(x64), 2.0 ** -6 * np.ldexp(1.0, e.astype(int) - 127)[..., None])
        assert (np.abs(dequantise(q, e) - x64) <= step).all()
        # nothing else was written
        other = torch.ones(n_pages, page, dtype=torch.bool)
        other[slots.cpu().long() // page, slots.cpu().long() % page] = False
        assert (pages.view(torch.uint8).cpu().transpose(1, 2)[other] == 0x35).all() and (exps.cpu().transpose(1, 2)[other] == 0x35).all()


@pytest.mark.parametrize("dqk,dv", [(64, 64), (128, 128), (192, 128)])
def test_bf16_rows(A, dqk, dv):
    c = filled(A, 9, 3, 32, dqk, dv, "bf16")
    k, v, slots = rows(4, 2, 3, 61, dqk, "blhd"), rows(5, 2, 3, 61, dv), some_slots(6, 9 * 32, 2, 61)
    c.append(k, v, slots)
    ko, vo = c.read(slots)
    assert torch.equal(ko, k) and torch.equal(vo, v)
    assert torch.equal(at_slots(c.k, slots), k) and torch.equal(at_slots(c.v, slots), v)


def test_magnitudes_at_the_edges(A):
    # rows of zeros, of the smallest and the largest numbers, of 448 and just above it; infinities and NaN beside finite elements
    D = 64
    r = torch.zeros(1, 1, 12, D)
    r[0, 0, 1, 0] = 448.0
    r[0, 0, 2, :2] = torch.tensor([450.0, -1.0])
    r[0, 0, 3] = 3.3e38
    r[0, 0, 4, ::2] = 1e-39
    r[0, 0, 5, 3] = 9.2e-41
    r[0, 0, 6, :4] = torch.tensor([float("inf"), 1.0, -2.5, float("nan")])
    r[0, 0, 7, :2] = float("-inf")
    r[0, 0, 8, :3] = torch.tensor([-447.0, 1.0625, 0.001])
    r[0, 0, 9] = torch.linspace(-1, 1, D) * 2.0 ** -120
    r[0, 0, 10, 5] = -1.1754944e-38
    r[0, 0, 11] = float("nan")
    x = r.to(torch.bfloat16).cuda()
    c = filled(A, 2, 1, 16, D, D, "e4m3")
    slots = torch.arange(12, dtype=torch.int32).cuda() + 3
    c.append(x, x.clone(), slots)
    back, _ = c.read(slots)
    q, e = quantise(x.cpu().double().numpy())
    assert np.array_equal(at_slots(c.k_exp, slots[None]).cpu().numpy(), e)
    stored = at_slots(c.k.view(torch.uint8), slots[None]).cpu().numpy()
    nan = (stored & 127) == 127
    assert np.array_equal(nan, ~np.isfinite(x.cpu().double().numpy()))
    assert np.array_equal(stored[~nan], q[~nan])
    ref = torch.from_numpy(dequantise(q, e)).to(torch.bfloat16)
    assert torch.equal(torch.isnan(back.cpu()), torch.isnan(ref))
    assert torch.equal(back.cpu()[~torch.isnan(ref)], ref[~torch.isnan(ref)])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_slots_outside_the_cache(A, dtype):
    # padded rows: skipped when written, zeros when read; the same slot may be read twice
    c = filled(A, 2, 2, 16, 128, 128, dtype)
    k, v = rows(7, 1, 2, 6, 128), rows(8, 1, 2, 6, 128)
    slots = torch.tensor([5, -1, 31, 32, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32).cuda()
    c.append(k, v, slots)
    ko, vo = c.read(torch.tensor([5, 31, 5, -1, 32, 2 ** 31 - 1], dtype=torch.int32).cuda())
    assert torch.equal(ko[:, :, 0], ko[:, :, 2]) and (ko[:, :, 3:] == 0).all() and (vo[:, :, 3:] == 0).all()
    if dtype == "bf16":
        assert torch.equal(ko[:, :, :2], k[:, :, [0, 2]]) and torch.equal(vo[:, :, :2], v[:, :, [0, 2]])
    other = [i for i in range(32) if i not in (5, 31)]
    for t in (c.k, c.v):
        b = t.view(torch.uint8).transpose(1, 2).reshape(32, -1)
        assert (b[other] == 0x35).all()


def test_large_cache(A):
    # byte offsets past 2^32
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    n_pages = 42000  # x 2 heads x 256 x 128 x 2 bytes = 5.5 GB
    c = A.PagedCache.empty(n_pages, 2, 256, 128, 128)
    k, v = rows(9, 1, 2, 4, 128), rows(10, 1, 2, 4, 128)
    slots = torch.tensor([n_pages * 256 - 1, 33000 * 256, 0, 17000 * 256 + 7], dtype=torch.int32).cuda()
    c.append(k, v, slots)
    ko, vo = c.read(slots)
    assert torch.equal(ko, k) and torch.equal(vo, v)
    assert torch.equal(c.k[n_pages - 1, :, 255], k[0, :, 0]) and torch.equal(c.v[33000, :, 0], v[0, :, 1])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_one_row_for_all_slots(A, dtype):
    # a vector expanded over batch, heads and rows, as slots are cleared
    c = filled(A, 5, 3, 16, 192, 128, dtype)
    slots = some_slots(16, 5 * 16, 2, 21)
    k, v = rows(17, 1, 1, 1, 192).view(192).expand(2, 3, 21, 192), torch.zeros(128, dtype=torch.bfloat16).cuda().expand(2, 3, 21, 128)
    c.append(k, v, slots)
    ko, vo = c.read(slots)
    assert (vo == 0).all() and torch.equal(ko, ko[:1, :1, :1].expand_as(ko).contiguous())
    step = 0.0 if dtype == "bf16" else 2.0 ** -4  # of the value, or of the smallest normal number, below 2^-13 of the row's largest
    assert ((ko.float() - k.float()).abs() <= step * k.float().abs().clamp(min=2.0 ** -13 * float(k.float().abs().max()))).all()
    other = torch.ones(5 * 16, dtype=torch.bool)
    other[slots.cpu().long().flatten()] = False
    for t in (c.k, c.v):
        assert (t.view(torch.uint8).transpose(1, 2).reshape(80, -1).cpu()[other] == 0x35).all()
