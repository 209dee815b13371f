"""MXFP4: rounding (bit for bit against the format's definition), back, and the product with packed weights against 64 bits; refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def cp():
    from paper_2207_01260_b200 import build
    build.build()
    import paper_2207_01260_b200 as m
    m.lib()
    return m


def rounded(x):
    """(codes, scale exponents + 127, values in 64 bits) of rows, by search among the format's values."""
    rows, C = x.shape
    blocks = -(-C // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :C] = x
    v = v.reshape(rows, blocks, 32)
    top = np.abs(v).max(-1)
    bad = ~np.isfinite(top)
    e = np.where(top > 0, np.frexp(np.where(bad, 1.0, top))[1] - 3, -127).clip(min=-127)
    with np.errstate(invalid="ignore"):
        a = np.where(bad[..., None], 0.0, np.abs(v) / np.exp2(e.astype(np.float64))[..., None])
    d = np.abs(a[..., None] - GRID)
    m = d.argmin(-1)
    tie = (m + 1 < 8) & (np.take_along_axis(d, np.minimum(m + 1, 7)[..., None], -1)[..., 0] == d.min(-1)) & (m % 2 == 1)
    m = m + tie
    codes = m | (np.signbit(v) & ~bad[..., None]).astype(np.int64) << 3
    values = np.where(bad[..., None], np.nan, np.where(np.signbit(v), -1, 1) * GRID[m] * np.exp2(e.astype(np.float64))[..., None])
    return codes.reshape(rows, -1), np.where(bad, 255, e + 127), values.reshape(rows, -1)[:, :C]


def packed_bytes(codes, scales):
    rows, blocks = scales.shape
    c = codes.reshape(rows, -1, 2)
    tiles = np.zeros((-(-rows // 128) * 128, -(-blocks // 4) * 4), dtype=np.uint8)
    tiles[:rows, :blocks] = scales
    return (c[..., 0] | c[..., 1] << 4).astype(np.uint8), tiles.reshape(-1, 4, 32, tiles.shape[1] // 4, 4).transpose(0, 3, 2, 1, 4)


def matrix(seed, rows, C, kind):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, C), generator=g)
    if kind == "ties":           # multiples of a quarter up to 8, in blocks scaled by any power of two: every tie and every saturation
        x = torch.randint(-32, 33, (rows, C), generator=g).float() / 4 * torch.exp2(torch.randint(-20, 20, (rows, -(-C // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :C]
    elif kind == "range":        # from subnormal to the largest numbers
        x = x * torch.exp2(torch.randint(-148, 120, (rows, -(-C // 32)), generator=g).double()).repeat_interleave(32, 1)[:, :C]
        x = x.float()
    elif kind == "zeros":
        x = torch.where(torch.rand((rows, C), generator=g) < 0.97, -0.0, x)
    elif kind == "bad":
        for i in range(rows):
            x[i, (7 * i) % C] = (math.nan, math.inf, -math.inf, 1.0)[i % 4]
    return x


def in_memory(cp, x, dtype):
    x = x.to(TYPES[dtype])
    if dtype == "f32":
        return x
    y = torch.zeros((x.shape[0], cp.cprune_padded_channels(x.shape[1])), dtype=torch.bfloat16)
    y[:, :x.shape[1]] = x
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["normal", "ties", "range", "zeros", "bad"])
@pytest.mark.parametrize("rows,C", [(1, 1), (1, 32), (3, 33), (130, 108), (5, 129), (257, 31), (2, 1280), (33, 250), (1000, 44)])
def test_rounding(cp, rows, C, kind, dtype):
    x = in_memory(cp, matrix(1, rows, C, kind), dtype)
    codes, scales, values = cp.cprune_mx_quantize(x.cuda(), C, values=True)
    c, s, v = rounded(x[:, :C].double().numpy())
    want_codes, want_scales = packed_bytes(c, s)
    got_scales = scales.cpu().numpy().copy()
    flat = got_scales.transpose(0, 3, 2, 1, 4).reshape(-1, got_scales.shape[1] * 4)       # rows behind the last are left as they were
    assert np.array_equal(flat[:rows], want_scales.transpose(0, 3, 2, 1, 4).reshape(-1, got_scales.shape[1] * 4)[:rows])
    good = s != 255                                   # a block without a value has any codes
    gc = codes.cpu().numpy().reshape(rows, -1, 16)
    assert np.array_equal(gc[good], want_codes.reshape(rows, -1, 16)[good])
    back = cp.cprune_mx_dequantize(codes, scales, C, TYPES[dtype])
    for got in (values, back):
        assert got.shape == x.shape and got.dtype == TYPES[dtype]
        assert np.array_equal(got.cpu()[:, :C].double().numpy(), v, equal_nan=True)       # exact: the values are numbers of either type
        assert not got[:, C:].any()
    y = x.cuda()
    assert torch.equal(cp.cprune_mx_quantize(y, C, values=y)[2].nan_to_num(9.0), values.nan_to_num(9.0))


@pytest.mark.gpu
def test_rounding_leaves_the_rows_behind_the_last(cp):
    x = in_memory(cp, matrix(2, 40, 70, "normal"), "bf16").cuda()
    scales = torch.full((1, 1, 32, 4, 4), 99, dtype=torch.uint8, device="cuda")
    cp.cprune_mx_quantize(x, 70, scales=scales)
    rows = scales.cpu().permute(0, 3, 2, 1, 4).reshape(128, 4)
    assert torch.all(rows[40:] == 99) and torch.all(rows[:40, 3] == 0) and torch.all(rows[:40, :3] > 100)


def product(cp, seed, rows, inn, out, act="none", with_res=False, out_f32=False, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = in_memory(cp, matrix(seed, rows, inn, kind), "bf16")
    w, b = torch.randn((out, inn), generator=g) / math.sqrt(inn), torch.randn(out, generator=g)
    res = in_memory(cp, torch.randn((rows, out), generator=g), "bf16") if with_res else None
    codes, scales, bias = cp.cprune_mx_pack(w.cuda(), b.cuda())
    y = cp.cprune_mx_fc(x.cuda(), inn, codes, scales, bias, out, act, None if res is None else res.cuda(), out_f32)
    cp.cprune_poll_device_status()
    qx, qw = (torch.from_numpy(rounded(t.double().numpy())[2]) for t in (x[:, :inn], w))
    z = qx @ qw.t() + b.double()
    size = qx.abs() @ qw.abs().t() + b.double().abs()
    if res is not None:
        z, size = z + res[:, :out].double(), size + res[:, :out].double().abs()
    want = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "relu6": lambda: z.clamp(0, 6)}[act]()
    y = y.cpu()
    assert y.dtype == (torch.float32 if out_f32 else torch.bfloat16) and y.shape == (rows, out if out_f32 else cp.cprune_padded_channels(out))
    assert not y[:, out:].any()
    return y[:, :out].double(), want, size


def check_product(got, want, size, inn, out_f32):
    # Products are exact.  A sum of n terms by additions that truncate is off by at most n 2^-23 of the terms' magnitudes; the partial sums here
    # have at most 128 such additions in a row (128 channels, or the steps of a chain), the rest is rounded: 2^-24 each, a few more
    units = (min(inn, 128) + 16) * 2.0 ** -23
    bound = (2.0 ** -24 if out_f32 else 2.0 ** -8) * want.abs() + units * size
    off = (got - want).abs()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    worst = (off[~nan] / bound[~nan].clamp(min=1e-300)).max().item() if (~nan).any() else 0.0
    assert worst <= 1.0, worst


PRODUCTS = [
    # rows, in, out
    (1, 1, 1), (1, 1280, 1000), (2, 512, 10), (16, 33, 24), (17, 100, 129), (5, 4096, 33), (40, 72, 300), (127, 256, 128), (128, 32, 8), (129, 257, 136),
    (300, 960, 320), (64, 1280, 1000), (784, 24, 144), (1000, 144, 24), (513, 512, 512), (200, 31, 257), (2048, 130, 40), (260, 2100, 260), (3000, 64, 1100), (19000, 24, 144), (9600, 1, 40), (10000, 500, 384), (19100, 33, 320), (200, 8192, 500),
    (33, 700, 1000), (100, 5000, 200), (128, 64, 130), (128, 257, 1000), (100, 64, 1000), (17, 2100, 24), (4700, 40, 8), (16, 16384, 100),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,inn,out", PRODUCTS)
def test_product(cp, rows, inn, out):
    got, want, size = product(cp, 3, rows, inn, out)
    check_product(got, want, size, inn, False)
    got, want, size = product(cp, 4, rows, inn, out, "relu", True)
    check_product(got, want, size, inn, False)
    got, want, size = product(cp, 5, rows, inn, out, "relu6", rows % 2 == 0, True)
    check_product(got, want, size, inn, True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 200, 700])
def test_product_of_values_that_are_no_numbers(cp, rows):
    """A NaN or an infinity makes its row NaN and no other, through the activation too."""
    got, want, size = product(cp, 6, rows, 96, 200, "relu", kind="bad")
    assert torch.isnan(want).any() and not torch.isnan(want).all()
    check_product(got, want, size, 96, False)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [4, 300])
def test_product_of_large_and_small_scales(cp, rows):
    """Scales of weights above 2 and far below 1, of activations the other way round."""
    g = torch.Generator().manual_seed(7)
    inn, out = 160, 136
    up = torch.exp2(torch.randint(-30, 31, (inn // 32,), generator=g).float()).repeat_interleave(32)
    x = in_memory(cp, torch.randn((rows, inn), generator=g) * up, "bf16")
    w = torch.randn((out, inn), generator=g) / up * torch.exp2(torch.randint(-6, 7, (out, 1), generator=g).float())
    codes, scales, bias = cp.cprune_mx_pack(w.cuda())
    got = cp.cprune_mx_fc(x.cuda(), inn, codes, scales, bias, out, out_f32=True).cpu().double()
    qx, qw = (torch.from_numpy(rounded(t.double().numpy())[2]) for t in (x[:, :inn], w))
    check_product(got, qx @ qw.t(), qx.abs() @ qw.abs().t(), inn, True)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 1000])
def test_shapes_streams_graphs_and_in_place(cp, rows):
    inn, out = 200, 150
    g = torch.Generator().manual_seed(8)
    x = in_memory(cp, torch.randn((rows * 4, inn), generator=g), "bf16").cuda().view(rows, 2, 2, -1)
    res = in_memory(cp, torch.randn((rows * 4, out), generator=g), "bf16").cuda().view(rows, 2, 2, -1)
    codes, scales, bias = cp.cprune_mx_pack((torch.randn((out, inn, 1, 1), generator=g) / 14).cuda(), torch.ones(out).cuda())
    y = cp.cprune_mx_fc(x, inn, codes, scales, bias, out, "relu", res)
    assert y.shape == res.shape
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = cp.cprune_mx_fc(x, inn, codes, scales, bias, out, "relu", res, stream=side)
    side.synchronize()
    assert torch.equal(other, y)
    z = res.clone()
    assert torch.equal(cp.cprune_mx_fc(x, inn, codes, scales, bias, out, "relu", z, y=z), y)
    graph = torch.cuda.CUDAGraph()
    xin = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        yg = cp.cprune_mx_fc(xin, inn, codes, scales, bias, out, "relu", res)
    for _ in range(2):
        xin.copy_(x)
        graph.replay()
        assert torch.equal(yg, y)
    cp.cprune_poll_device_status()


def test_refusals(cp):
    L, vp = cp.lib(), ctypes.c_void_p
    assert [L.cprune_mx_blocks(c) for c in (0, 1, 32, 33)] == [0, 1, 1, 2]
    assert [L.cprune_mx_scale_bytes(*a) for a in ((1, 1), (128, 128), (129, 129), (0, 5), (5, 0))] == [512, 512, 2048, 0, 0]

    def quantize(x=0x1000, type=0, rows=2, C=40, codes=0x2000, scales=0x3000, values=0x4000):
        return L.cprune_mx_quantize(vp(x), type, rows, C, vp(codes), vp(scales), vp(values), vp(0))

    def dequantize(codes=0x2000, scales=0x3000, rows=2, C=40, type=0, x=0x1000):
        return L.cprune_mx_dequantize(vp(codes), vp(scales), rows, C, type, vp(x), vp(0))

    for call in (quantize, dequantize):
        assert call(x=None) == 1 and call(type=2) == 1 and call(type=-1) == 1 and call(rows=0) == 1 and call(C=0) == 1
        assert call(codes=None) == 1 and call(scales=None) == 1 and call(codes=0x2008) == 1 and call(scales=0x3004) == 1 and call(x=0x1002) == 1
        assert call(type=1, x=0x1002) == 1 and call(rows=1 << 40) == 2 and call(C=(1 << 22) + 1) == 2
    assert quantize(codes=None, scales=None, values=None) == 1 and quantize(values=0x4004) == 1 and dequantize(codes=None, scales=None) == 1
    assert L.cprune_mx_pack(vp(0x1000), vp(0), 4, 8, vp(0), vp(0), vp(0x4000), vp(0)) == 1
    assert L.cprune_mx_pack(vp(0), vp(0), 4, 8, vp(0x2000), vp(0x3000), vp(0x4000), vp(0)) == 1
    assert L.cprune_mx_pack(vp(0x1000), vp(2), 4, 8, vp(0x2000), vp(0x3000), vp(0x4000), vp(0)) == 1
    assert L.cprune_mx_pack(vp(0x1000), vp(0), 0, 8, vp(0x2000), vp(0x3000), vp(0x4000), vp(0)) == 1

    def fc(x=0x1000, rows=2, inn=40, codes=0x2000, scales=0x3000, b=0x4000, out=24, act=0, res=None, f32=0, y=0x5000, work=0x6000, size=1 << 30):
        return L.cprune_mx_fc(vp(x), rows, inn, vp(codes), vp(scales), vp(b), out, act, vp(res), f32, vp(y), vp(work), size, vp(0))

    assert fc(x=None) == 1 and fc(codes=None) == 1 and fc(scales=None) == 1 and fc(b=None) == 1 and fc(y=None) == 1
    assert fc(rows=0) == 1 and fc(inn=0) == 1 and fc(out=0) == 1 and fc(act=3) == 1 and fc(act=-1) == 1
    assert fc(x=0x1008) == 1 and fc(codes=0x2008) == 1 and fc(scales=0x3008) == 1 and fc(res=0x7008) == 1 and fc(y=0x5008) == 1 and fc(f32=1, y=0x5002) == 1
    assert fc(b=0x4002) == 1 and fc(work=0x6008) == 1
    assert fc(work=None) == 3 and fc(size=8) == 3
    assert fc(rows=1 << 31) == 2 and fc(inn=(1 << 22) + 1) == 2 and fc(out=(1 << 24) + 1) == 2


def test_python_refusals(cp):
    x = torch.zeros((4, 40), dtype=torch.bfloat16)
    codes, scales, bias = torch.zeros((24, 32), dtype=torch.uint8), torch.zeros((1, 1, 32, 4, 4), dtype=torch.uint8), torch.zeros(24)
    for f in (lambda: cp.cprune_mx_quantize(x, 41), lambda: cp.cprune_mx_quantize(x.half(), 40), lambda: cp.cprune_mx_quantize(x, 0), lambda: cp.cprune_mx_quantize(x, 40),
              lambda: cp.cprune_mx_dequantize(codes, scales, 40), lambda: cp.cprune_mx_dequantize(codes, scales, 40, torch.float16),
              lambda: cp.cprune_mx_pack(torch.zeros(4, 8)), lambda: cp.cprune_mx_pack(torch.zeros(4, 8, 3, 3)),
              lambda: cp.cprune_mx_fc(x.float(), 40, codes, scales, bias, 24), lambda: cp.cprune_mx_fc(x, 40, codes, scales, bias, 24, "silu"),
              lambda: cp.cprune_mx_fc(x, 40, codes, scales, bias, 0), lambda: cp.cprune_mx_fc(x, 40, codes, scales, bias, 24)):
        with pytest.raises(cp.CpruneError) as e:
            f()
        assert e.value.status == 1


@pytest.mark.gpu
def test_python_refusals_on_the_device(cp):
    x = torch.zeros((4, 40), dtype=torch.bfloat16, device="cuda")
    codes, scales, bias = cp.cprune_mx_pack(torch.zeros((24, 40), device="cuda"))
    ok = dict(x=x, in_features=40, codes=codes, scales=scales, b_packed=bias, out_features=24)
    cp.cprune_mx_fc(**ok)
    for bad in (dict(codes=codes[:23]), dict(scales=scales[:, :0]), dict(b_packed=bias[:23]), dict(out_features=25), dict(residual=x), dict(y=x), dict(residual=x[:, :24]),
                dict(codes=codes.int()), dict(workspace=torch.zeros(64, device="cuda"))):
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_mx_fc(**{**ok, **bad})
        assert e.value.status == 1
    with pytest.raises(cp.CpruneError) as e:
        cp.cprune_mx_fc(**ok, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


@pytest.mark.gpu
@pytest.mark.parametrize("rows, inn, out", [(28636, 667, 25), (28636, 512, 25), (45922, 261, 31), (27735, 471, 292), (22063, 706, 66), (38000, 320, 384), (12544, 960, 320)])
def test_rows_are_read_before_their_place_is_filled_again(cp, rows, inn, out):
    """Weights that add up one block of 32 channels each.  The values of a block are multiples of half its scale, at most 6 of it: their sums are exact in
    float32, and every bit counts.  Repeated, with the rows in the cache: the faster they come, the sooner their places are filled again."""
    x = torch.zeros(rows, cp.cprune_padded_channels(inn), device="cuda", dtype=torch.bfloat16)
    x[:, :inn] = torch.randn(rows, inn, generator=torch.Generator("cuda").manual_seed(31), device="cuda")
    w = torch.zeros(out, inn, device="cuda")
    w[torch.arange(inn) // 32 % out, torch.arange(inn)] = 1.0
    packed = cp.cprune_mx_pack(w)
    values = torch.zeros(rows, -(-inn // 32) * 32, device="cuda", dtype=torch.float64)
    values[:, :inn] = cp.cprune_mx_quantize(x, inn, values=True)[2][:, :inn]
    want = values.view(rows, -1, 32).sum(2)
    assert want.shape[1] <= out
    for _ in range(10):
        y = cp.cprune_mx_fc(x, inn, *packed, out, out_f32=True)
        assert torch.equal(y[:, :want.shape[1]].double(), want) and not y[:, want.shape[1]:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,inn,out", [(129, 25088, 10), (300, 16384, 64), (129, 65536, 24), (200, 131072, 400), (129, 1 << 20, 8), (20, 1 << 20, 8), (8, 25088, 4096)])
def test_product_of_many_channels_of_one_sign(cp, rows, inn, out):
    """Values and weights that are positive, in blocks of any scale: every addition to the accumulator truncates the same way, at most 2^-23 of the sum so far; a step takes 64 channels, so that n
    steps are off by n 2^-24 of the sum in the mean of their partial sums.  What a step itself cuts off (64 products, each exact) and the rest count 16 such units."""
    g = torch.Generator(device="cuda").manual_seed(41)
    x = torch.zeros((rows, cp.cprune_padded_channels(inn)), dtype=torch.bfloat16, device="cuda")
    by = lambda n: torch.exp2(torch.randint(-8, 1, (n, inn // 32), generator=g, device="cuda").float()).repeat_interleave(32, 1)  # noqa: E731
    x[:, :inn] = (torch.rand((rows, inn), generator=g, device="cuda") + 0.1) * by(rows)
    w = (torch.rand((out, inn), generator=g, device="cuda") + 0.1) * by(out)
    codes, scales, bias = cp.cprune_mx_pack(w)
    got = cp.cprune_mx_fc(x, inn, codes, scales, bias, out, out_f32=True).double()
    cp.cprune_poll_device_status()
    want = torch.zeros((rows, out), dtype=torch.float64, device="cuda")
    qw = cp.cprune_mx_dequantize(codes, scales, inn)
    qx = cp.cprune_mx_quantize(x, inn, values=True)[2]
    for c in range(0, inn, 16384):
        want += qx[:, c:min(c + 16384, inn)].double() @ qw[:, c:c + 16384].double().t()
    off = ((got - want).abs() / want).max().item()
    steps = -(-inn // 64)
    assert off <= (steps / 2 + 16) * 2.0 ** -23
