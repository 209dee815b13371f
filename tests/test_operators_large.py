"""The operators past 32-bit offsets, in values and in bytes: what lies at the end of large tensors against the same work on a small one, or in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def cp():
    import paper_2207_01260_b200 as m
    m.lib()
    return m


def test_group_norm_gradients(cp):
    """2.4 billion values, of which the last images alone are not zero."""
    N, hw, C, G = 2900, 112, 64, 8
    g = torch.Generator(device="cuda").manual_seed(51)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy, res = (torch.zeros((N, hw, hw, C), dtype=BF16, device="cuda") for _ in range(3))
    for t in (x, dy, res):
        t[-2:] = r(2, hw, hw, C).to(BF16)
    gamma, beta = 1 + 0.3 * r(C), 0.3 * r(C)
    last = [t[-2:].clone() for t in (x, dy, res)]
    _, stats = cp.cprune_group_norm(x, C, G, gamma, beta, 1e-5, "silu", res)
    dx, dgamma, dbeta, dres = cp.cprune_group_norm_backward(dy, x, C, G, stats, gamma, beta, "silu", res, dx=dy, dresidual=x)
    want = cp.cprune_group_norm_backward(last[1], last[0], C, G, stats[-2:].contiguous(), gamma, beta, "silu", last[2])
    # (how an image is shared out, and with it the order of its float32 sums, depends on the batch)
    for got, w in ((dx[-2:], want[0]), (dres[-2:], want[3])):
        assert torch.all((got.double() - w.double()).abs() <= 2 * 2.0 ** -8 * w.double().abs() + 1e-5)
    for got, w in ((dgamma, want[1]), (dbeta, want[2])):
        assert torch.all((got - w).abs() <= 1e-5 * hw * hw)
    assert not dx[:2].any() and not dres[:2].any()


def test_clipping(cp):
    """A tensor of 1.2 billion float32 values at an odd address, behind a bf16 one."""
    n = 1_200_000_001
    room = torch.zeros(n + 9, device="cuda")
    a = room[1:n + 1]
    a[::1_000_003] = 3.0
    a[-1] = 4.0
    b = torch.full((33,), 0.5, device="cuda", dtype=BF16)
    total = float(9.0 * (n // 1_000_003 + 1) + 16.0 + 33 * 0.25) ** 0.5
    norm = cp.cprune_clip_gradients([b, a], 1.0)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    f = 1.0 / (total + 1e-6)
    assert abs(float(a[-1]) / f - 4.0) <= 1e-6 and torch.all((a[::1_000_003][:-1] / f - 3.0).abs() <= 1e-6) and float(room[0]) == 0 and not room[n + 1:].any()
    assert int((a != 0).sum()) == n // 1_000_003 + 2 and torch.all((b.float() / f / 0.5 - 1).abs() <= 2.0 ** -8)


def test_rounding_and_back(cp):
    """2.3 billion values in memory."""
    rows, C, tail = 20_500_000, 108, 1000
    x = torch.zeros((rows, 112), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(52)
    x[-tail:, :C] = torch.randn((tail, C), generator=g, device="cuda").to(BF16)
    last = x[-tail:].clone()
    codes, scales, values = cp.cprune_mx_quantize(x, C, values=x)
    assert values is x
    c, s, v = cp.cprune_mx_quantize(last, C, values=True)
    assert torch.equal(codes[-tail:], c) and torch.equal(x[-tail:], v) and not x[:1000].any()
    del x, values
    back = cp.cprune_mx_dequantize(codes, scales, C, BF16)
    assert torch.equal(back[-tail:], v) and not back[:1000].any()


@pytest.mark.parametrize("out,f32", [(24, False), (24, True), (400, False)])
def test_product(cp, out, f32):
    """Rows of 2.3 billion values in memory.  Weights that add up a block of 32 channels each: such sums are exact."""
    rows, C, tail = 20_500_000 if out == 24 else 6_000_000, 108 if out == 24 else 360, 1000
    x = torch.zeros((rows, cp.cprune_padded_channels(C)), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(53)
    x[-tail:, :C] = torch.randn((tail, C), generator=g, device="cuda").to(BF16)
    w = torch.zeros((out, C), device="cuda")
    w[torch.arange(C) // 32, torch.arange(C)] = 1.0
    y = cp.cprune_mx_fc(x, C, *cp.cprune_mx_pack(w), out, out_f32=f32)
    cp.cprune_poll_device_status()
    v = torch.zeros((tail, -(-C // 32) * 32), dtype=torch.float64, device="cuda")
    v[:, :C] = cp.cprune_mx_quantize(x[-tail:].clone(), C, values=True)[2][:, :C].double()
    want = v.view(tail, -1, 32).sum(2)
    got = y[-tail:]
    assert torch.equal(got[:, :want.shape[1]], want.to(got.dtype)) and not got[:, want.shape[1]:].any() and not y[:1000].any()
