"""GPU parity of rotary positions (ae_rotary_forward / _backward) against the 64-bit definition.

Bounds.  An output is two products and a sum of them in 32 bits, with sines and cosines good to 2e-7: |error| <= 6e-7 * a (|x1| + |x2|)
before the output is rounded to its type, at most half a step (2^-9 of the value for bf16's 8 bits, 2^-24 for fp32)."""
import numpy as np
import pytest
import torch

from oracle.serving_oracle import rotary as oracle_rotary

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def A():
    from paper_2502_15349_amd import ae_attn
    return ae_attn


def heads(seed, B, H, L, D, dtype, order):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, H, D) if order == "blhd" else (B, H, L, D), generator=g).to(dtype).cuda()
    return x.transpose(1, 2) if order == "blhd" else x


def check(got, x, pos, f, amp, layout, backward=False):
    ref = oracle_rotary(x.cpu().double().numpy(), pos.cpu().numpy(), f, amp, layout, backward)
    n = len(f)
    mag = np.zeros(ref.shape)
    a = np.abs(x.cpu().double().numpy())
    i1 = np.arange(n) if layout == "half" else 2 * np.arange(n)
    i2 = i1 + (n if layout == "half" else 1)
    mag[..., i1] = mag[..., i2] = a[..., i1] + a[..., i2]
    err = np.abs(got.cpu().double().numpy() - ref)
    bound = 6e-7 * abs(amp) * mag * (1 + HALF_STEP[got.dtype]) + HALF_STEP[got.dtype] * np.abs(ref)
    print(f"{tuple(x.shape)} rot {2 * n} {layout}: max {err.max():.3e}, of the bound {np.max(err / np.maximum(bound, 1e-300)):.3f}", flush=True)
    assert (err <= bound).all()
    assert torch.equal(got[..., 2 * n:], x[..., 2 * n:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,H_q,H_k,L,D,rot,order", [
    (1, 1, 0, 1, 64, 64, "bhld"), (1, 32, 8, 1, 128, 128, "bhld"), (2, 12, 3, 37, 64, 32, "blhd"), (3, 5, 5, 129, 192, 64, "bhld"),
    (2, 3, 1, 33, 80, 20, "blhd"), (1, 2, 2, 70, 7, 6, "bhld"), (1, 17, 4, 300, 256, 256, "blhd"), (64, 8, 1, 2, 128, 96, "bhld"),
])
def test_forward_and_backward(A, dtype, layout, B, H_q, H_k, L, D, rot, order):
    f, amp = A.rotary_frequencies(rot, scaling="by_parts" if rot > 2 else "none", factor=8.0)
    q = heads(1, B, H_q, L, D, dtype, order)
    k = heads(2, B, H_k, L, D, dtype, order) if H_k else None
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(0, 200000, (B, L), generator=g).to(torch.int32).cuda()
    got = A.rotary_forward(q, k, pos, freqs=f, amplitude=amp, layout=layout)
    back = A.rotary_backward(q, k, pos, freqs=f, amplitude=amp, layout=layout)
    for x, y, z in zip((q, k), got, back):
        if x is not None:
            check(y, x, pos, f, amp, layout)
            check(z, x, pos, f, amp, layout, backward=True)
        else:
            assert y is None and z is None


@pytest.mark.parametrize("where", [0, 10 ** 6, 2 ** 31 - 40, -5, -2 ** 31])
def test_far_positions(A, where):
    # angles of up to 2^31 radians, modulo a turn; positions shared by the batch
    f, _ = A.rotary_frequencies(128)
    f[5], f[6] = 5.99, -1.5
    q = heads(4, 2, 2, 40, 128, torch.float32, "bhld")
    pos = (torch.arange(40, dtype=torch.int64) + where).to(torch.int32).cuda()
    got, _ = A.rotary_forward(q, None, pos, freqs=f)
    check(got, q, pos, f, 1.0, "half")


def test_known_turns(A):
    # a quarter, a half and three quarters of a turn: the identities that a wrong quadrant would break
    q = heads(5, 1, 1, 4, 16, torch.float32, "bhld")
    f = [np.pi / 2] * 8
    y, _ = A.rotary_forward(q, None, torch.arange(4, dtype=torch.int32).cuda(), freqs=f)
    a, b = q[..., :8], q[..., 8:]
    for l, (u, v) in enumerate([(a, b), (-b, a), (-a, -b), (b, -a)]):
        assert torch.allclose(y[0, 0, l, :8], u[0, 0, l], atol=1e-6) and torch.allclose(y[0, 0, l, 8:], v[0, 0, l], atol=1e-6)


def test_gradient_is_that_of_the_forward_pass(A):
    # <y, R x> = <R^T y, x> for every pair of inputs, and the map is linear: the backward pass is the forward's transpose
    f, amp = A.rotary_frequencies(64, scaling="by_parts", factor=4.0)
    x, y = heads(6, 2, 3, 50, 128, torch.float32, "bhld"), heads(7, 2, 3, 50, 128, torch.float32, "bhld")
    pos = torch.arange(50, dtype=torch.int32).cuda()
    for layout in ("half", "interleaved"):
        rx, _ = A.rotary_forward(x, None, pos, freqs=f, amplitude=amp, layout=layout)
        ry, _ = A.rotary_backward(y, None, pos, freqs=f, amplitude=amp, layout=layout)
        left, right = (y.double() * rx.double()).sum(), (ry.double() * x.double()).sum()
        # each of the 2 * 2 * 3 * 50 * 128 products is off by at most 1e-6 of its factors, of magnitude about 1
        assert abs(left - right) <= 1e-6 * (y.double().abs() * (x.double().abs() + 1) * 2).sum()


def test_in_place_offset_strides_and_unwritten_rows(A):
    # rows of a larger buffer (a fused projection's q and k side by side), in place; what lies between and behind stays
    f, amp = A.rotary_frequencies(128)
    buf = torch.randn(2, 60, 12 * 128 + 8, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    before = buf.clone()
    q = buf[:, :50, : 8 * 128].view(2, 50, 8, 128).transpose(1, 2)
    k = buf[:, :50, 8 * 128: 12 * 128].view(2, 50, 4, 128).transpose(1, 2)
    pos = torch.arange(50, dtype=torch.int32).cuda() + 77
    q0, k0 = q.clone(), k.clone()
    r = A.rotary_forward(q, k, pos, freqs=f, out=(q, k))
    assert r[0].data_ptr() == q.data_ptr()
    check(q, q0, pos, f, 1.0, "half")
    check(k, k0, pos, f, 1.0, "half")
    assert torch.equal(buf[:, 50:], before[:, 50:]) and torch.equal(buf[..., 12 * 128:], before[..., 12 * 128:])


def test_narrow_alignment_gives_the_same(A):
    # rows that start at an odd element take the kernel of single elements
    f, amp = A.rotary_frequencies(64)
    x = torch.randn(1, 3, 20, 65, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()[..., 1:]
    pos = torch.arange(20, dtype=torch.int32).cuda()
    y, _ = A.rotary_forward(x, None, pos, freqs=f)
    z, _ = A.rotary_forward(x.contiguous(), None, pos, freqs=f)
    assert torch.equal(y, z)


def test_many_rows_and_another_stream(A):
    f, amp = A.rotary_frequencies(64)
    q = heads(10, 3, 40, 3001, 64, torch.bfloat16, "blhd")
    k = heads(11, 3, 8, 3001, 64, torch.bfloat16, "blhd")
    pos = torch.randint(0, 9000, (3, 3001), generator=torch.Generator().manual_seed(12)).to(torch.int32).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = A.rotary_forward(q, k, pos, freqs=f, stream=s)
    s.synchronize()
    b = A.rotary_forward(q, k, pos, freqs=f)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(b[0][:, ::13, ::100], q[:, ::13, ::100], pos[:, ::100], f, 1.0, "half")


def test_replayed_graph(A):
    f, amp = A.rotary_frequencies(128)
    q, k = heads(13, 4, 8, 1, 128, torch.bfloat16, "blhd"), heads(14, 4, 2, 1, 128, torch.bfloat16, "blhd")
    pos = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    plan = A.RotaryPlan(q, k, pos, qo, ko, freqs=f)
    plan.forward(q, k, pos, qo, ko)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan.forward(q, k, pos, qo, ko)
    for step in range(3):
        pos.fill_(1000 * step + 3)
        g.replay()
        torch.cuda.synchronize()
        got = qo.clone()
        eager, _ = A.rotary_forward(q, k, pos, freqs=f)
        assert torch.equal(got, eager)


def test_expanded_tensors_are_read_and_not_written(A):
    # a gradient that is the same for every head, as a sum over heads leaves it; and heads that share their input
    f, amp = A.rotary_frequencies(64, scaling="by_parts", factor=4.0)
    pos = torch.arange(33, dtype=torch.int32).cuda()
    one = heads(11, 2, 1, 33, 64, torch.bfloat16, "bhld")
    many = one.expand(2, 5, 33, 64)
    for call in (A.rotary_forward, A.rotary_backward):
        got, _ = call(many, None, pos, freqs=f, amplitude=amp)
        ref, _ = call(many.contiguous(), None, pos, freqs=f, amplitude=amp)
        assert torch.equal(got, ref)
        with pytest.raises(ValueError, match="expanded"):
            call(many.contiguous(), None, pos, freqs=f, amplitude=amp, out=(many, None))
    plan = A.RotaryPlan(many, None, pos, torch.empty_like(got), None, freqs=f, amplitude=amp)
    with pytest.raises(ValueError, match="expanded"):
        plan.backward(got, None, pos, many, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_row_for_all(A, dtype):
    # a vector expanded over batch, heads and rows: a gradient that is the same everywhere, as a sum over all rows leaves it
    f, amp = A.rotary_frequencies(64, scaling="by_parts", factor=4.0)
    pos = torch.arange(33, dtype=torch.int32).cuda() + 5
    row = torch.randn(80, generator=torch.Generator().manual_seed(15)).to(dtype).cuda()
    many, other = row.expand(2, 5, 33, 80), (row + 1).expand(3, 3, 33, 80)[:2, :1]  # (a size of one with a stride of zero)
    for call, backward in ((A.rotary_forward, False), (A.rotary_backward, True)):
        got = call(many, other, pos, freqs=f, amplitude=amp)
        ref = call(many.contiguous(), other.contiguous(), pos, freqs=f, amplitude=amp)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
        check(got[0], many, pos, f, amp, "half", backward)
        with pytest.raises(ValueError, match="expanded"):
            call(many.contiguous(), None, pos, freqs=f, amplitude=amp, out=(many, None))
