"""Group norm with an activation, and its gradients, against the definition in 64 bits; what the calls refuse."""
import ctypes

import pytest
import torch

EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# Half a step of the stored type, relative to the value.
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# Roundings to float32 on the way to a value: sums are trees over at most a few dozen sequential additions per thread, so 64 units of
# 2^-24 of the terms' magnitudes cover every one of them (z has six, the combination of the partial means and deviations the rest; the
# exponential of silu is good to 2^-21 of a value that enters with at most |z| / 4).
UNITS = 64 * 2.0 ** -24


@pytest.fixture(scope="module")
def cp():
    from paper_2207_01260_b200 import build
    build.build()
    import paper_2207_01260_b200 as m
    m.lib()
    return m


def lanes(cp, C, dtype):
    return cp.cprune_padded_channels(C) if dtype == "bf16" else C


def activation(cp, seed, N, H, W, C, dtype, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros((N, H, W, lanes(cp, C, dtype)), dtype=TYPES[dtype])
    x[..., :C] = (torch.randn((N, H, W, C), generator=g, dtype=torch.float64) * scale + shift).to(TYPES[dtype])
    return x


def affine(seed, C):
    g = torch.Generator().manual_seed(seed)
    return 1.0 + 0.3 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g)


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "relu6": lambda: z.clamp(0, 6), "silu": lambda: z * torch.sigmoid(z)}[act]()


def slope64(z, act):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "relu6": lambda: ((z > 0) & (z < 6)).double(),
            "silu": lambda: s * (1 + z * (1 - s))}[act]()


def reference(x, C, G, gamma, beta, act, res, stats=None):
    """(y, mean, rstd, z, xhat, magnitude of the terms of z), in 64 bits, of logical channels."""
    N, H, W, _ = x.shape
    v = x[..., :C].double().reshape(N, H * W, G, C // G)
    if stats is None:
        mean = v.mean((1, 3), keepdim=True)
        rstd = 1 / (((v - mean) ** 2).mean((1, 3), keepdim=True) + EPS).sqrt()
    else:
        mean, rstd = (stats.double()[..., k].reshape(N, 1, G, 1) for k in (0, 1))
    xhat = ((v - mean) * rstd).reshape(N, H, W, C)
    z = xhat * gamma.double() + beta.double()
    size = xhat.abs() * gamma.double().abs() + beta.double().abs()
    # an error of the mean, relative to the values it is taken of, reaches z through rstd and gamma
    size = size + gamma.double().abs() * ((mean.abs() + 1 / rstd) * rstd).expand_as(v).reshape(N, H, W, C)
    if res is not None:
        z = z + res[..., :C].double()
        size = size + res[..., :C].double().abs()
    return act64(z, act), mean.reshape(N, G), rstd.reshape(N, G), z, xhat, size


CASES = [
    # N, H, W, C, groups, type, activation, shortcut
    (1, 1, 1, 1, 1, "bf16", "none", False),            # one value: the variance is 0
    (2, 1, 1, 8, 8, "f32", "relu", True),              # one value per group
    (1, 1, 1, 16, 2, "bf16", "silu", False),
    (3, 5, 5, 12, 12, "bf16", "relu", False),          # a group per channel
    (1, 7, 7, 352, 32, "bf16", "relu", True),          # groups of 11 channels
    (2, 14, 14, 180, 12, "bf16", "relu6", False),
    (2, 9, 13, 91, 7, "f32", "silu", True),            # rows that are no multiple of 16 bytes
    (1, 8, 8, 20, 1, "f32", "relu6", True),
    (2, 28, 28, 44, 4, "bf16", "silu", True),
    (1, 56, 56, 108, 12, "bf16", "none", False),
    (1, 3, 4, 601, 1, "f32", "none", False),           # more columns than a block has threads
    (2, 3, 3, 2200, 11, "bf16", "relu", False),
    (1, 2, 3, 4104, 8, "bf16", "relu", True),
    (5, 1, 3, 136, 17, "bf16", "silu", False),         # pad lanes that fill a vector
    (1, 61, 67, 24, 3, "f32", "relu", False),
    (70, 4, 4, 32, 4, "bf16", "relu", True),
    (1, 112, 112, 36, 4, "bf16", "relu6", True),       # a large image
    (2, 160, 150, 40, 2, "f32", "silu", False),
    (2, 120, 100, 44, 4, "bf16", "silu", True),
    (300, 5, 7, 72, 9, "bf16", "relu6", False),        # more images than blocks run at a time
    (1, 3, 500, 2056, 4, "bf16", "relu", True),        # slices of the channels that groups straddle
    (1, 31, 33, 16382, 2, "f32", "none", False),       # the widest groups, nearly
]


def close(name, got, want, bound):
    off = (got.double() - want).abs()
    worst = (off / bound.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, (name, worst)


@pytest.mark.gpu
@pytest.mark.parametrize("N,H,W,C,G,dtype,act,with_res", CASES)
def test_forward(cp, N, H, W, C, G, dtype, act, with_res):
    x = activation(cp, 1, N, H, W, C, dtype, 1.7, 0.6)
    res = activation(cp, 2, N, H, W, C, dtype) if with_res else None
    gamma, beta = affine(3, C)
    y, stats = cp.cprune_group_norm(x.cuda(), C, G, gamma.cuda(), beta.cuda(), EPS, act, res.cuda() if with_res else None)
    y, stats = y.cpu(), stats.cpu()
    want, mean, rstd, _, _, size = reference(x, C, G, gamma, beta, act, res)
    assert y.dtype == TYPES[dtype] and y.shape == x.shape
    assert torch.all(y[..., C:] == 0)
    close("mean", stats[..., 0], mean, UNITS * (mean.abs() + 1 / rstd))
    # an error of the variance counts with its share of variance + eps
    close("rstd", stats[..., 1], rstd, UNITS * rstd)
    close("y", y[..., :C], want, STEP[dtype] * want.abs() + 1.1 * UNITS * size)


@pytest.mark.gpu
@pytest.mark.parametrize("N,H,W,C,G,dtype,act,with_res", CASES)
def test_gradients(cp, N, H, W, C, G, dtype, act, with_res):
    x = activation(cp, 4, N, H, W, C, dtype, 1.7, 0.6)
    dy = activation(cp, 5, N, H, W, C, dtype)
    res = activation(cp, 6, N, H, W, C, dtype) if with_res else None
    gamma, beta = affine(7, C)
    _, mean, rstd, _, _, _ = reference(x, C, G, gamma, beta, act, res)
    stats = torch.stack([mean, rstd], -1).float()
    dx, dgamma, dbeta, dres = (None if t is None else t.cpu() for t in cp.cprune_group_norm_backward(
        dy.cuda(), x.cuda(), C, G, stats.cuda(), gamma.cuda(), beta.cuda(), act, res.cuda() if with_res else None))
    _, _, rstd, z, xhat, size = reference(x, C, G, gamma, beta, act, res, stats)
    rstd = rstd.reshape(N, 1, 1, G, 1)
    dz = dy[..., :C].double() * slope64(z, act)
    # an error of z changes silu's slope by at most half as much
    dz_off = UNITS * dy[..., :C].double().abs() * (1.1 + (0.5 * size if act == "silu" else 0))
    grouped = lambda v: v.reshape(N, H, W, G, C // G)  # noqa: E731
    t = grouped(dz * gamma.double())
    t_off = grouped(dz_off * gamma.double().abs() + UNITS * (dz * gamma.double()).abs())
    h = grouped(xhat)
    h_off = UNITS * grouped(size / gamma.double().abs().clamp(min=1e-9)).clamp(max=1e6)
    mean_of = lambda v: v.mean((1, 2, 4), keepdim=True)  # noqa: E731
    m1, m2 = mean_of(t), mean_of(t * h)
    m1_off = mean_of(t_off + UNITS * t.abs())
    m2_off = mean_of(t_off * h.abs() + t.abs() * h_off + UNITS * (t * h).abs())
    want = rstd * (t - m1 - h * m2)
    off = rstd * (t_off + m1_off + h.abs() * m2_off + h_off * m2.abs() + UNITS * (t.abs() + m1.abs() + (h * m2).abs()))
    close("dx", grouped(dx[..., :C]), want, STEP[dtype] * want.abs() + off)
    assert torch.all(dx[..., C:] == 0)
    close("dbeta", dbeta, dz.sum((0, 1, 2)), (dz_off + UNITS * dz.abs()).sum((0, 1, 2)))
    h_off = h_off.reshape(N, H, W, C)
    close("dgamma", dgamma, (dz * xhat).sum((0, 1, 2)), (dz_off * xhat.abs() + dz.abs() * h_off + UNITS * (dz * xhat).abs()).sum((0, 1, 2)))
    if with_res:
        close("dresidual", dres[..., :C], dz, STEP[dtype] * dz.abs() + dz_off)
        assert torch.all(dres[..., C:] == 0)
    else:
        assert dres is None


@pytest.mark.gpu
@pytest.mark.parametrize("act,with_res", [("silu", False), ("none", True), ("relu", False)])
def test_gradients_against_differences(cp, act, with_res):
    """dL/dx, dL/dgamma and dL/dbeta of L = sum(y dy) against central differences of the definition in 64 bits."""
    N, H, W, C, G = 1, 3, 2, 6, 2
    x, dy = activation(cp, 8, N, H, W, C, "f32"), activation(cp, 9, N, H, W, C, "f32")
    res = activation(cp, 10, N, H, W, C, "f32") if with_res else None
    gamma, beta = affine(11, C)
    z = reference(x, C, G, gamma, beta, act, res)[3]
    assert act != "relu" or z.abs().min() > 1e-3            # no value next to the border, where there is no difference quotient
    _, stats = cp.cprune_group_norm(x.cuda(), C, G, gamma.cuda(), beta.cuda(), EPS, act, None if res is None else res.cuda())
    dx, dgamma, dbeta, _ = cp.cprune_group_norm_backward(dy.cuda(), x.cuda(), C, G, stats, gamma.cuda(), beta.cuda(), act, None if res is None else res.cuda())
    loss = lambda a, b, c: (reference(a, C, G, b, c, act, res)[0] * dy.double()).sum()  # noqa: E731
    args = [x.double(), gamma.double(), beta.double()]
    for k, got in enumerate((dx, dgamma, dbeta)):
        h, flat = 1e-5, got.cpu().double().reshape(-1)
        for i in range(flat.numel()):
            up, down = [a.clone() for a in args], [a.clone() for a in args]
            up[k].view(-1)[i] += h
            down[k].view(-1)[i] -= h
            d = (loss(*up) - loss(*down)) / (2 * h)
            # third derivatives of order 100 times h^2, and the float32 of the kernel
            assert abs(d - flat[i]) <= 1e-5 * (1 + abs(d)), (k, i, d, flat[i])


@pytest.mark.gpu
def test_mean_far_from_the_spread(cp):
    """A mean of 1000 spreads: squares minus the squared mean would leave nothing of the variance."""
    x = activation(cp, 12, 2, 23, 19, 30, "f32", 0.01, 10.0)
    gamma, beta = torch.ones(30), torch.zeros(30)
    y, stats = cp.cprune_group_norm(x.cuda(), 30, 3, eps=EPS)
    want, mean, rstd, _, _, size = reference(x, 30, 3, gamma, beta, "none", None)
    close("rstd", stats.cpu()[..., 1], rstd, UNITS * rstd)
    close("y", y.cpu(), want, STEP["f32"] * want.abs() + UNITS * size)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("W", [5, 6000])                    # on chip, in two passes
def test_values_that_are_no_numbers_stay_in_their_group(cp, dtype, bad, W):
    x = activation(cp, 13, 2, 6, W, 24, dtype)
    clean = cp.cprune_group_norm(x.cuda(), 24, 4, activation="relu")[0].cpu()
    x[1, 3, 2, 7] = bad                                     # image 1, group 1
    y = cp.cprune_group_norm(x.cuda(), 24, 4, activation="relu")[0].cpu()
    assert torch.isnan(y[1, ..., 6:12]).all()
    y[1, ..., 6:12] = clean[1, ..., 6:12]
    assert torch.equal(y, clean)


@pytest.mark.gpu
@pytest.mark.parametrize("C, G, dtype", [(1030, 103, "f32"), (4120, 10, "bf16")])
def test_groups_of_two_slices_have_one_mean(cp, C, G, dtype):
    """Blocks of both slices work such a group out: what is written and what is used does not depend on their timing."""
    x = activation(cp, 21, 1, 40, 40, C, dtype).cuda()
    first = cp.cprune_group_norm(x, C, G)
    for _ in range(30):
        again = cp.cprune_group_norm(x, C, G)
        assert torch.equal(again[1], first[1]) and torch.equal(again[0], first[0])


@pytest.mark.gpu
@pytest.mark.parametrize("hw", [6, 60, 190])
def test_in_place_and_other_streams_and_graphs(cp, hw):
    """The same bits in place, on another stream, captured and replayed, and twice in a row."""
    C, G = 40, 5
    x = activation(cp, 14, 3, hw, hw, C, "bf16").cuda()
    dy = activation(cp, 15, 3, hw, hw, C, "bf16").cuda()
    res = activation(cp, 16, 3, hw, hw, C, "bf16").cuda()
    gamma, beta = (t.cuda() for t in affine(17, C))
    y, stats = cp.cprune_group_norm(x, C, G, gamma, beta, EPS, "relu", res)
    grads = cp.cprune_group_norm_backward(dy, x, C, G, stats, gamma, beta, "relu", res)
    z = x.clone()
    assert torch.equal(cp.cprune_group_norm(z, C, G, gamma, beta, EPS, "relu", res, y=z)[0], y)
    z = res.clone()
    assert torch.equal(cp.cprune_group_norm(x, C, G, gamma, beta, EPS, "relu", z, y=z)[0], y)
    a, b = dy.clone(), x.clone()
    got = cp.cprune_group_norm_backward(a, b, C, G, stats, gamma, beta, "relu", res, dx=a, dresidual=b)
    assert all(torch.equal(u, v) for u, v in zip(got, grads))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = cp.cprune_group_norm(x, C, G, gamma, beta, EPS, "relu", res, stream=side)
    more = cp.cprune_group_norm_backward(dy, x, C, G, other[1], gamma, beta, "relu", res, stream=side)
    side.synchronize()
    assert torch.equal(other[0], y) and torch.equal(other[1], stats) and all(torch.equal(u, v) for u, v in zip(more, grads))
    graph = torch.cuda.CUDAGraph()
    xin = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        yg, sg = cp.cprune_group_norm(xin, C, G, gamma, beta, EPS, "relu", res)
        gg = cp.cprune_group_norm_backward(dy, xin, C, G, sg, gamma, beta, "relu", res)
    for _ in range(2):
        xin.copy_(x)
        graph.replay()
        assert torch.equal(yg, y) and all(torch.equal(u, v) for u, v in zip(gg, grads))


@pytest.mark.gpu
def test_more_than_32_bits_of_bytes(cp):
    """2.4 billion values: the last images of a batch lie past 32-bit offsets, in values and in bytes."""
    N, hw, C = 2900, 112, 64
    x = torch.zeros((N, hw, hw, C), dtype=torch.bfloat16, device="cuda")
    one = activation(cp, 18, 2, hw, hw, C, "bf16").cuda()
    x[-2:] = one
    y, stats = cp.cprune_group_norm(x, C, 8, activation="relu", y=x)
    # (how an image is shared out, and with it the order of its sums, may depend on the batch: the bounds are those against the definition)
    want, mean, rstd, _, _, size = reference(one.cpu(), C, 8, torch.ones(C), torch.zeros(C), "relu", None)
    close("rstd", stats[-2:, :, 1].cpu(), rstd, UNITS * rstd)
    close("y", y[-2:].cpu(), want, STEP["bf16"] * want.abs() + UNITS * size)
    assert not y[:2].any()


def test_refusals(cp):
    L, vp = cp.lib(), ctypes.c_void_p
    ws = cp.lib().cprune_group_norm_workspace_bytes
    assert ws(0, 2, 7, 7, 24, 3, 1) > 0 and ws(0, 64, 112, 112, 24, 3, 0) > 0 and ws(0, 2, 7, 7, 24, 3, 0) == 0      # (a small forward pass stays on chip)
    assert ws(0, 2, 7, 7, 24, 5, 0) == 0 and ws(2, 2, 7, 7, 24, 3, 0) == 0 and ws(0, 0, 7, 7, 24, 3, 0) == 0

    def forward(x=0x1000, type=0, N=64, H=112, W=112, C=24, G=3, gamma=0x2000, beta=0x2000, eps=1e-5, act=1, res=None, y=0x3000, stats=0x4000, work=0x5000, size=1 << 20):
        return L.cprune_group_norm(vp(x), type, N, H, W, C, G, vp(gamma), vp(beta), eps, act, vp(res), vp(y), vp(stats), vp(work), size, vp(0))

    def backward(dy=0x1000, x=0x1000, type=0, N=2, C=24, G=3, stats=0x4000, act=1, res=None, dx=0x3000, dres=None, work=0x5000, size=1 << 20):
        return L.cprune_group_norm_backward(vp(dy), vp(x), type, N, 7, 7, C, G, vp(stats), vp(0x2000), vp(0x2000), act, vp(res), vp(dx), vp(0x2000), vp(0x2000), vp(dres),
                                            vp(work), size, vp(0))

    for call in (forward, backward):
        assert call(x=None) == 1 and call(stats=None) == 1 and call(N=0) == 1 and call(C=0) == 1 and call(G=0) == 1 and call(G=5) == 1
        assert call(type=2) == 1 and call(type=-1) == 1 and call(act=4) == 1 and call(act=-1) == 1
        assert call(x=0x1008) == 1 and call(res=0x1002) == 1 and call(stats=0x4004) == 1 and call(work=0x5004) == 1
        assert call(type=1, x=0x1002) == 1
        assert call(size=16) == 3 and call(work=None) == 3
        assert call(N=70000) == 2 and call(C=16400, G=2) == 2 and call(C=(1 << 20) + 8, G=1 << 17 | 1) == 2
    assert forward(y=None) == 1 and forward(eps=0.0) == 1 and forward(eps=-1.0) == 1 and forward(eps=float("nan")) == 1 and forward(eps=float("inf")) == 1
    assert forward(H=0) == 1 and forward(H=1 << 15, W=1 << 12) == 2
    assert backward(dy=None) == 1 and backward(dx=None) == 1 and backward(dres=0x6000) == 1
    # the activation that the group norm alone has
    assert L.cprune_fc(vp(0x1000), 1, 8, vp(0x1000), vp(0x1000), 8, 3, 0, vp(0x1000), vp(0)) == 1
    assert "silu" in cp.NORM_ACT and "silu" not in cp.binding.ACT


def test_python_refusals(cp):
    x = torch.zeros((1, 2, 2, 16), dtype=torch.bfloat16)
    for bad in (dict(x=x.half(), C=16), dict(x=x[0], C=16), dict(x=x, C=17), dict(x=x, C=8), dict(x=x, C=0), dict(x=x, C=16, activation="gelu"),
                dict(x=x.transpose(1, 3).contiguous().transpose(1, 3), C=16), dict(x=x, C=16)):      # (the last: not on the device)
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_group_norm(bad.pop("x"), bad.pop("C"), 2, **bad)
        assert e.value.status == 1


@pytest.mark.gpu
def test_python_refusals_on_the_device(cp):
    x = torch.zeros((1, 2, 2, 16), dtype=torch.bfloat16, device="cuda")
    g = torch.ones(16, device="cuda")
    for bad in (dict(gamma=g.double()), dict(gamma=g[:8]), dict(gamma=torch.ones(32, device="cuda")[::2]), dict(beta=torch.ones(16)), dict(residual=x[:, :1]),
                dict(y=x.float()), dict(stats=torch.zeros(1, 2, 2)), dict(residual=x.float())):
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_group_norm(x, 16, 2, **bad)
        assert e.value.status == 1
    with pytest.raises(cp.CpruneError) as e:
        cp.cprune_group_norm(x, 16, 3)
    assert e.value.status == 1
    with pytest.raises(cp.CpruneError) as e:
        cp.cprune_group_norm_backward(x, x, 16, 2, torch.zeros((1, 2, 2), device="cuda"), workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")[:16])
    assert e.value.status == 3


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["first pixel", "top row", "steps", "normal"])
@pytest.mark.parametrize("H,W,C,G,dtype", [
    (112, 112, 512, 512, "bf16"), (112, 112, 512, 32, "bf16"), (224, 224, 256, 256, "bf16"), (112, 112, 1280, 1280, "bf16"), (112, 112, 1280, 32, "bf16"),
    (112, 112, 512, 512, "f32"), (113, 111, 129, 129, "f32"), (112, 112, 44, 4, "bf16"), (56, 56, 12, 12, "f32"), (25, 25, 16, 16, "bf16")])
def test_variance_of_images_with_a_border(cp, H, W, C, G, dtype, kind):
    """Flat images but for their first pixel or row, as behind a convolution with padding, and steps: what is far from the rest is what a thread sees first, or many
    times over.  At most 2^-24 a rounding: a thread's squares in runs of up to 40, of which up to half count in the mean and twice in what they add to the
    deviations, 44 runs, half of them in the mean, 16 levels of sums of threads and chunks, 8 for the differences themselves: 94 units of the variance, 47 of rstd."""
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.zeros((2, H, W, lanes(cp, C, dtype)), dtype=TYPES[dtype], device="cuda")
    v = x[..., :C]
    if kind == "normal":
        v.copy_(torch.randn((2, H, W, C), generator=g, device="cuda") * 1.7 + 0.6)
    else:
        v.copy_(0.25 + torch.rand(C, generator=g, device="cuda"))
        if kind == "first pixel":
            v[0, 0, 0], v[1, -1, -1] = 40.0, -70.0
        elif kind == "top row":
            v[0, 0], v[1, :, 0] = 40.0, -70.0
        else:
            v[0, H // 2:], v[1, ::2] = 7.7, -0.3
    for image in (x, x[:1]):
        stats = cp.cprune_group_norm(image.contiguous(), C, G)[1]
        w = image[..., :C].double().reshape(-1, H * W, G, C // G)
        mean = w.mean((1, 3), keepdim=True)
        rstd = 1 / (((w - mean) ** 2).mean((1, 3)) + EPS).sqrt()
        mean = mean.reshape(rstd.shape)
        close("mean", stats[..., 0], mean, UNITS * (mean.abs() + 1 / rstd))
        close("rstd", stats[..., 1], rstd, UNITS * rstd)


@pytest.mark.gpu
@pytest.mark.parametrize("N,H,W", [(2, 1, 1), (2, 5, 5), (2, 6, 6000), (40, 60, 60)])      # on chip, fewer blocks than an image can have; in two passes
def test_means_whose_square_leaves_float32(cp, N, H, W):
    """4e19, 1000 spreads: the deviations' squares are numbers."""
    x = activation(cp, 32, N, H, W, 24, "f32", 4e16, 4e19)
    y, stats = cp.cprune_group_norm(x.cuda(), 24, 24)
    want, mean, rstd, _, _, size = reference(x, 24, 24, torch.ones(24), torch.zeros(24), "none", None)
    close("mean", stats.cpu()[..., 0], mean, UNITS * (mean.abs() + 1 / rstd))
    # (of a single value the variance is 0 in 64 bits; here its mean is rounded, which leaves it as it is)
    close("rstd", stats.cpu()[..., 1], rstd, UNITS * rstd)
    close("y", y.cpu(), want, STEP["f32"] * want.abs() + UNITS * size)


@pytest.mark.gpu
@pytest.mark.parametrize("H,W,C,G,dtype,act,with_res", [
    (112, 112, 512, 32, "f32", "none", False), (113, 111, 129, 3, "f32", "relu", True), (112, 112, 1280, 1280, "bf16", "silu", False), (112, 112, 512, 512, "bf16", "relu6", True),
    (40, 40, 44, 4, "f32", "silu", True), (97, 101, 24, 24, "f32", "none", True)])
def test_gradients_of_one_sign(cp, H, W, C, G, dtype, act, with_res):
    """The same dy everywhere, as of a mean: every addition of a thread rounds the same way.  Half of the additions of a run (64 at most, or 40 and 40 runs) count in the
    mean of the partial sums, 13 for the sums over threads, 12 for chunks and channels: 65 roundings at most, some of them the other way."""
    g = torch.Generator(device="cuda").manual_seed(33)
    x, res, dy = (torch.zeros((1, H, W, lanes(cp, C, dtype)), dtype=TYPES[dtype], device="cuda") for _ in range(3))
    x[..., :C] = torch.randn((1, H, W, C), generator=g, device="cuda")
    res[..., :C] = torch.randn((1, H, W, C), generator=g, device="cuda")
    dy[..., :C] = 0.1
    gamma, beta = torch.rand(C, generator=g, device="cuda") + 0.5, torch.randn(C, generator=g, device="cuda")
    if not with_res:
        res = None
    stats = torch.empty((1, G, 2), device="cuda")
    _, mean, rstd, _, _, _ = reference(x, C, G, gamma, beta, act, res)
    stats[..., 0], stats[..., 1] = mean, rstd
    dx, dgamma, dbeta, _ = cp.cprune_group_norm_backward(dy, x, C, G, stats, gamma, beta, act, res)
    _, _, rstd, z, xhat, size = reference(x, C, G, gamma, beta, act, res, stats)
    dz = dy[..., :C].double() * slope64(z, act)
    dz_off = UNITS * dy[..., :C].double() * (1.1 + 0.5 * size) if act == "silu" else torch.zeros_like(dz)
    close("dbeta", dbeta, dz.sum((0, 1, 2)), (dz_off + UNITS * dz.abs()).sum((0, 1, 2)))
    h_off = UNITS * (size / gamma.double())
    close("dgamma", dgamma, (dz * xhat).sum((0, 1, 2)), (dz_off * xhat.abs() + dz.abs() * h_off + UNITS * (dz * xhat).abs()).sum((0, 1, 2)))
    t, t_off, h, h_off = ((v.reshape(H * W, G, C // G)) for v in (dz * gamma.double(), (dz_off + UNITS * dz.abs()) * gamma.double(), xhat, h_off))
    m1, m2 = t.mean((0, 2), keepdim=True), (t * h).mean((0, 2), keepdim=True)
    m1_off, m2_off = t_off.mean((0, 2), keepdim=True) + UNITS * t.abs().mean((0, 2), keepdim=True), (t_off * h.abs() + t.abs() * h_off + UNITS * (t * h).abs()).mean((0, 2), keepdim=True)
    r = rstd.reshape(1, G, 1)
    want = r * (t - m1 - h * m2)
    off = r * (t_off + m1_off + h.abs() * m2_off + h_off * m2.abs() + UNITS * (t.abs() + m1.abs() + (h * m2).abs()))
    close("dx", dx[..., :C].reshape(want.shape), want, STEP[dtype] * want.abs() + off)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,W,C,G", [(3, 5, 7, 20, 10), (1, 9, 9, 756, 3), (30, 25, 155, 300, 150), (2, 40, 40, 96, 48), (64, 33, 35, 48, 16), (1, 1, 3, 34, 17), (2, 3, 500, 2056, 4)])
def test_flat_channels(cp, N, H, W, C, G, dtype):
    """A value per channel, those of a group 1 % apart or less; groups whose channels are equal.  The deviations are those of a few numbers around a mean that is as good
    as float32 can be: half a unit of the mean is 0.5 * 2^-23 / 0.01 = 6e-6 of such a deviation, and counts with its square; equal numbers have no deviations."""
    g = torch.Generator(device="cuda").manual_seed(34)
    base = torch.rand((G, 1), generator=g, device="cuda") * 300 + 1
    step = torch.randint(-2, 3, (G, C // G), generator=g, device="cuda") * (2.0 ** -6 if dtype == "bf16" else 2.0 ** -9)
    step[::3] = 0.0
    x = torch.zeros((N, H, W, lanes(cp, C, dtype)), dtype=TYPES[dtype], device="cuda")
    x[..., :C] = (base * (1 + step)).reshape(C)
    y, stats = cp.cprune_group_norm(x, C, G)
    v = x[0, 0, 0, :C].double().reshape(G, C // G)
    mean, var = v.mean(1), v.var(1, correction=0)
    rstd = 1 / (var + EPS).sqrt()
    close("mean", stats[..., 0], mean.expand(N, G), 2.0 ** -23 * mean)
    # what the variance is off by: its own roundings, 24 of 2^-24, and the square of what the mean is off by
    off = (24 * 2.0 ** -24 * var + (2.0 ** -23 * mean) ** 2) / (var + EPS) / 2 + 2.0 ** -23
    close("rstd", stats[..., 1], rstd.expand(N, G), off * rstd)
    flat = (v == v[:, :1]).all(1).repeat_interleave(C // G)
    assert flat.any() and not y[..., :C][..., flat].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H,W,C,G", [(1, 31, 33, 16382, 2), (2, 3, 3, 2200, 2), (3, 40, 40, 600, 3), (64, 33, 35, 96, 2), (1, 1, 1, 4104, 1)])
def test_a_channel_far_from_the_others(cp, N, H, W, C, G, dtype):
    """The first or the last channel of a group: its distance is rounded to 2^-24 of it, the deviations are that distance over the root of the group's channels."""
    g = torch.Generator(device="cuda").manual_seed(35)
    for at in (0, C // G - 1):
        x = torch.zeros((N, H, W, lanes(cp, C, dtype)), dtype=TYPES[dtype], device="cuda")
        v = x[..., :C].view(N, H, W, G, C // G)
        v.copy_(0.25 + torch.rand((N, H, W, G, C // G), generator=g, device="cuda") * 1e-3)
        v[..., at] = 700.0
        stats = cp.cprune_group_norm(x, C, G)[1]
        w = v.double()
        mean = w.mean((1, 2, 4))
        rstd = 1 / (w.var((1, 2, 4), correction=0) + EPS).sqrt()
        close("mean", stats[..., 0], mean, UNITS * (mean.abs() + 1 / rstd))
        close("rstd", stats[..., 1], rstd, UNITS * rstd)
