"""Results that share memory with an input, or with one another, in a way that the interface does not allow are refused before anything is launched."""
import ctypes

import pytest
import torch

# (the addresses are none: a call that is not refused would fail for want of a device here, and must not find one)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")
vp = ctypes.c_void_p
X, Y, Z, U, G, B, S, T, W = (0x10000000 * k for k in range(1, 10))


@pytest.fixture(scope="module")
def L():
    from paper_2207_01260_b200 import build
    build.build()
    import paper_2207_01260_b200 as m
    return m.lib()


@pytest.mark.parametrize("type,half", [(0, 2), (1, 4)])
def test_group_norm(L, type, half):
    N, H, C, groups = 64, 112, 24, 3
    size = N * H * H * C * half

    def call(x=X, res=Z, y=Y, gamma=G, beta=B, stats=S, work=W):
        return L.cprune_group_norm(vp(x), type, N, H, H, C, groups, vp(gamma), vp(beta), 1e-5, 1, vp(res), vp(y), vp(stats), vp(work), 1 << 24, vp(0))

    assert size < 0x10000000
    for bad in (dict(y=X + 16), dict(y=X + size - 16), dict(x=Y + size - 16), dict(y=Z + 32), dict(res=Y + 16), dict(y=G), dict(beta=Y + 64), dict(stats=X + 8), dict(stats=Y + size - 8),
                dict(stats=G), dict(work=X), dict(work=S), dict(work=Y + 256), dict(work=Z - 16)):
        assert call(**bad) == 1, bad
    # the same place, and neighbours, are something else: these fail later, at the device that is not there
    for good in (dict(), dict(y=X), dict(y=Z), dict(y=X + size), dict(x=Y + size), dict(res=None, gamma=None, beta=None)):
        assert call(**good) != 1, good


def test_group_norm_gradients(L):
    N, H, C, groups = 64, 56, 24, 3
    size = N * H * H * C * 2
    D, E = 0xa0000000, 0xb0000000

    def call(dy=Y, x=X, res=Z, dx=U, dres=T, gamma=G, beta=B, stats=S, dgamma=D, dbeta=E, work=W):
        return L.cprune_group_norm_backward(vp(dy), vp(x), 0, N, H, H, C, groups, vp(stats), vp(gamma), vp(beta), 1, vp(res), vp(dx), vp(dgamma), vp(dbeta), vp(dres),
                                            vp(work), 1 << 24, vp(0))

    for bad in (dict(dx=T), dict(dx=T + 16), dict(dx=Y, dres=Y), dict(dx=X + 16), dict(dres=X + size - 16), dict(dx=Y + 16), dict(dres=Z + 16), dict(dgamma=E), dict(dgamma=E + 4),
                dict(dgamma=G), dict(dbeta=B), dict(dgamma=B), dict(dbeta=X), dict(dgamma=U + 8), dict(dbeta=S), dict(dx=S), dict(dres=G), dict(work=D), dict(work=X + 16), dict(work=U)):
        assert call(**bad) == 1, bad
    for good in (dict(), dict(dx=Y), dict(dx=X, dres=Y), dict(dx=Z), dict(dx=T + size), dict(res=None, dres=None), dict(dgamma=None, dbeta=None)):
        assert call(**good) != 1, good


def test_mx(L):
    rows, C = 1000, 100
    size, codes = rows * 104 * 2, rows * 4 * 16

    def quantize(x=X, c=Y, s=S, v=Z):
        return L.cprune_mx_quantize(vp(x), 0, rows, C, vp(c), vp(s), vp(v), vp(0))

    for bad in (dict(v=X + 16), dict(x=Z + size - 16), dict(c=X), dict(c=Z + 16), dict(s=Y), dict(s=Y + codes - 16), dict(s=X + 16), dict(s=Z)):
        assert quantize(**bad) == 1, bad
    for good in (dict(), dict(v=X), dict(v=None), dict(c=None, s=None), dict(s=Y + codes), dict(c=X + size)):
        assert quantize(**good) != 1, good
    assert L.cprune_mx_dequantize(vp(X), vp(S), rows, C, 0, vp(X), vp(0)) == 1 and L.cprune_mx_dequantize(vp(X), vp(S), rows, C, 0, vp(S - size + 16), vp(0)) == 1
    assert L.cprune_mx_dequantize(vp(X), vp(S), rows, C, 0, vp(S - size), vp(0)) != 1

    def pack(w=X, b=B, c=Y, s=S, p=G):
        return L.cprune_mx_pack(vp(w), vp(b), 1000, 100, vp(c), vp(s), vp(p), vp(0))

    for bad in (dict(c=X), dict(s=Y), dict(p=X + 16), dict(p=B), dict(p=Y), dict(p=S), dict(c=B), dict(s=B)):
        assert pack(**bad) == 1, bad
    for good in (dict(), dict(b=None)):
        assert pack(**good) != 1, good


@pytest.mark.parametrize("rows", [8, 1000, 20000])
@pytest.mark.parametrize("f32", [0, 1])
def test_mx_product(L, rows, f32):
    inn, out = 200, 72
    size = rows * 72 * (4 if f32 else 2)

    def call(x=X, c=Y, s=S, b=B, res=Z, y=U, work=W):
        return L.cprune_mx_fc(vp(x), rows, inn, vp(c), vp(s), vp(b), out, 1, vp(res), f32, vp(y), vp(work), 1 << 27, vp(0))

    for bad in (dict(y=X), dict(y=X + 16), dict(y=Z + 16), dict(res=U + size - 16), dict(y=Y), dict(y=S), dict(y=B), *([dict(y=Z)] if f32 else [])):
        assert call(**bad) == 1, bad
    if L.cprune_mx_fc_workspace_bytes(rows, inn, out):
        for bad in (dict(work=X), dict(work=U), dict(work=Z), dict(work=Y), dict(work=S), dict(work=B)):
            assert call(**bad) == 1, bad
    for good in (dict(), dict(res=None), *([] if f32 else [dict(y=Z)]), dict(y=Z + rows * 72 * 2)):
        assert call(**good) != 1, good
