"""Global gradient norm and clipping against 64 bits: lists of tensors of both types at any address; what the calls refuse."""
import ctypes
import math

import pytest
import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def cp():
    from paper_2207_01260_b200 import build
    build.build()
    import paper_2207_01260_b200 as m
    m.lib()
    return m


def tensors(seed, sizes, dtypes, offset=0, scale=0.1):
    """Views of one buffer per tensor that begin `offset` values after a 16-byte boundary, between guards."""
    g = torch.Generator().manual_seed(seed)
    got = []
    for i, n in enumerate(sizes):
        dtype = TYPES[dtypes[i % len(dtypes)]]
        room = torch.full((n + offset + 24,), 77.0, dtype=dtype)
        room[offset + 8:offset + 8 + n] = (scale * torch.randn(n, generator=g)).to(dtype)
        got.append(room.cuda()[offset + 8:offset + 8 + n])
    return got


def expected(grads, max_norm):
    norm = math.sqrt(sum(float(t.cpu().double().square().sum()) for t in grads))
    factor = min(1.0, max_norm / (norm + 1e-6))
    return norm, [t.cpu().double() * factor for t in grads]


def check(grads, norm, results, want_norm, want):
    assert norm.shape == (1,) and norm.dtype == torch.float32
    # float64 sums; one rounding
    assert abs(float(norm) - want_norm) <= (2.0 ** -24 + 1e-12) * want_norm
    for t, r, w in zip(grads, results, want):
        # the factor and the product are rounded to float32, the result to its type; below the smallest normal number to a multiple of 2^-149
        step = STEP["bf16" if t.dtype == torch.bfloat16 else "f32"]
        off = (r.cpu().double() - w).abs()
        assert torch.all(off <= (step + 2.0 ** -22) * w.abs() + 2.0 ** -148)


SIZES = [
    [1], [7], [0, 5, 0], [4096], [4095, 4097, 1, 16385], [64 * 3 * 49, 64, 64, 64 * 64 * 9, 10, 512 * 358 * 9],
    [(7 * i) % 91 for i in range(70)], [3 + i % 5 for i in range(1030)], [3_000_001],
]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("dtypes,offset", [(["f32"], 0), (["f32"], 1), (["bf16"], 0), (["bf16"], 3), (["bf16", "f32"], 2)])
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clip(cp, sizes, dtypes, offset, max_norm):
    grads = tensors(1, sizes, dtypes, offset)
    want_norm, want = expected(grads, max_norm)
    before = [t.clone() for t in grads]
    # into other tensors, whose vectors lie elsewhere
    into = tensors(2, sizes, dtypes, (offset + 1) % 8)
    norm = cp.cprune_clip_gradients(grads, max_norm, out=into)
    check(grads, norm, into, want_norm, want)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    assert torch.equal(cp.cprune_gradient_norm(grads), norm)
    # in place: the same bits
    again = cp.cprune_clip_gradients(grads, max_norm)
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(grads, into))
    for t in (*grads, *into):           # nothing beside the tensors was written
        room = t._base if t._base is not None else t
        n, at = t.numel(), t.storage_offset()
        assert torch.all(room[:at] == 77) and torch.all(room[at + n:] == 77)


@pytest.mark.gpu
def test_values_whose_squares_leave_float32(cp):
    for scale in (1e-30, 1e25):
        grads = tensors(3, [1000, 33], ["f32"], 0, scale)
        want_norm, want = expected(grads, 1e20)
        norm = cp.cprune_clip_gradients(grads, 1e20)
        check(grads, norm, grads, want_norm, want)


@pytest.mark.gpu
def test_values_that_are_no_numbers(cp):
    grads = tensors(4, [100, 5000], ["f32", "bf16"])
    grads[1][77] = float("inf")
    into = [torch.empty_like(t) for t in grads]
    norm = cp.cprune_clip_gradients(grads, 1.0, out=into)
    assert torch.isinf(norm).all() and torch.isnan(into[1][77]) and not into[0].any() and into[1].isnan().sum() == 1
    grads[0][3] = float("nan")
    norm = cp.cprune_clip_gradients(grads, 1.0)
    assert torch.isnan(norm).all() and all(torch.isnan(t).all() for t in grads)


@pytest.mark.gpu
def test_the_list_may_be_any_iterable(cp):
    grads = tensors(6, [100, 5000], ["f32", "bf16"])
    norm = cp.cprune_gradient_norm(grads)
    into = [torch.empty_like(t) for t in grads]
    for lists in ((grads, into), (tuple(grads), tuple(into)), (iter(grads), (t for t in into))):
        assert torch.equal(cp.cprune_clip_gradients(lists[0], 1.0, out=lists[1]), norm)
    assert torch.equal(cp.cprune_gradient_norm(iter(grads)), norm)
    want = [t.clone() for t in into]
    cp.cprune_clip_gradients((t for t in grads), 1.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))


@pytest.mark.gpu
def test_no_gradients(cp):
    assert float(cp.cprune_clip_gradients([], 1.0)) == 0.0 and float(cp.cprune_gradient_norm([torch.zeros(0, device="cuda")])) == 0.0


@pytest.mark.gpu
def test_streams_and_graphs(cp):
    grads = tensors(5, [100_000, 513, 64 * 64 * 9], ["f32", "bf16", "f32"])
    into = [torch.empty_like(t) for t in grads]
    norm = cp.cprune_clip_gradients(grads, 1.0, out=into)
    want = [t.clone() for t in into]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = cp.cprune_clip_gradients(grads, 1.0, out=into, stream=side)
    side.synchronize()
    assert torch.equal(other, norm) and all(torch.equal(a, b) for a, b in zip(into, want))
    start = [t.clone() for t in grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n1 = cp.cprune_clip_gradients(grads, 1.0)
    for _ in range(2):                      # the captured list outlives the call's arrays
        for t, s in zip(grads, start):
            t.copy_(s)
        graph.replay()
        assert torch.equal(n1, norm) and all(torch.equal(a, b) for a, b in zip(grads, want))


def test_refusals(cp):
    L, vp = cp.lib(), ctypes.c_void_p
    assert L.cprune_gradient_workspace_bytes(-1) == 0 and 0 < L.cprune_gradient_workspace_bytes(0) < L.cprune_gradient_workspace_bytes(5000)

    def call(addresses=(0x1000, 0x2000), counts=(5, 6), types=(0, 1), n=2, max_norm=1.0, out=None, norm=0x3000, work=0x4000, size=1 << 20):
        a = (vp * 2)(*addresses)
        c = (ctypes.c_ulonglong * 2)(*counts)
        t = (ctypes.c_int * 2)(*types)
        o = None if out is None else (vp * 2)(*out)
        got = L.cprune_clip_gradients(a, c, t, n, max_norm, o, vp(norm), vp(work), size, vp(0))
        if out is None and max_norm == 1.0:
            assert L.cprune_gradient_norm(a, c, t, n, vp(norm), vp(work), size, vp(0)) == got
        return got

    assert call(n=-1) == 1 and call(norm=None) == 1 and call(norm=0x3002) == 1 and call(work=0x4008) == 1
    assert call(addresses=(0x1001, 0x2000)) == 1 and call(addresses=(0x1000, 0x2002)) == 1 and call(addresses=(None, 0x2000)) == 1
    assert call(types=(0, 2)) == 1 and call(types=(-1, 1)) == 1
    assert call(out=(0x1000, 0x2002)) == 1 and call(out=(None, 0x2000)) == 1
    assert call(max_norm=-1.0) == 1 and call(max_norm=float("nan")) == 1
    assert call(counts=(1 << 44, 1)) == 2
    assert call(work=None) == 3 and call(size=100) == 3
    assert L.cprune_clip_gradients(None, None, None, 2, 1.0, None, vp(0x3000), vp(0x4000), 1 << 20, vp(0)) == 1


def test_python_refusals(cp, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = torch.zeros(8)
    for grads, out in (([t.half()], None), ([torch.zeros(4, 4).t()], None), ([t], None)):       # (the last: not on the device)
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_clip_gradients(grads, 1.0, out=out)
        assert e.value.status == 1


@pytest.mark.gpu
def test_python_refusals_on_the_device(cp):
    t, u = torch.zeros(8, device="cuda"), torch.zeros(9, device="cuda")
    for grads, kw in (([t, t], {}), ([t], {"out": [u]}), ([t], {"out": [t.bfloat16()]}), ([t, u], {"out": [t]}), ([t], {"norm": torch.zeros(1)}),
                      ([t], {"norm": torch.zeros(1, device="cuda", dtype=torch.float64)}), ([t, torch.zeros(3)], {})):
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_clip_gradients(grads, 1.0, **kw)
        assert e.value.status == 1


@pytest.mark.gpu
def test_tensors_that_overlap_are_refused(cp):
    flat = torch.ones(64, device="cuda")
    a, b, c, d = flat[:16], flat[15:32], flat[32:48], flat[48:]
    for grads, kw in (([a, b], {}), ([c, b, a], {}), ([a, c], {"out": [a, b]}), ([a, c], {"out": [flat[1:17], c]}), ([a, c], {"out": [c, a]}),
                      ([a, c], {"out": [d, d]}), ([a, c[:0], b], {"norm": torch.zeros(1, device="cuda")})):
        with pytest.raises(cp.CpruneError) as e:
            cp.cprune_clip_gradients(grads, 1.0, **kw)
        assert e.value.status == 1 and (flat == 1).all()
    cp.cprune_clip_gradients([a, c, c[:0]], 1.0, out=[a, d, d[:0]])
    assert (c == 1).all() and torch.equal(a, d) and (a < 1).all()


def test_overlap_by_the_steps_in_python(cp):
    refuse = cp.binding._refuse_overlap
    refuse("f", [100, 164, 0], [16, 3, 0], [1, 0, 1])
    refuse("f", [100, 164], [16, 3], [1, 0], [100, 170])
    for a, c, t, o in (([100, 160], [16, 3], [1, 0], None), ([164, 100], [3, 17], [0, 1], None), ([100, 164], [16, 3], [1, 0], [100, 166]), ([100, 200], [4, 4], [1, 1], [200, 300])):
        with pytest.raises(cp.CpruneError):
            refuse("f", a, c, t, o)


@pytest.mark.gpu
@pytest.mark.parametrize("dtypes", [["f32"], ["bf16"], ["f32", "bf16"]])
def test_factors_below_the_smallest_normal_number(cp, dtypes):
    """2e37 a value, clipped to 1e-2: a factor of 3e-43, results of 6e-6 (and one of 1e-12, results of some hundred times 2^-149)."""
    for scale, max_norm in ((2e37, 1e-2), (1e30, 1e-42), (1e-3, 1e-42)):
        grads = tensors(7, [2_000_000, 33, 1_000_001], dtypes, 1, scale)
        want_norm, want = expected(grads, max_norm)
        norm = cp.cprune_clip_gradients(grads, max_norm)
        assert torch.isinf(norm) if want_norm > 3.5e38 else abs(float(norm) - want_norm) <= 2.0 ** -23 * want_norm
        for t, w in zip(grads, want):
            step = STEP["bf16" if t.dtype == torch.bfloat16 else "f32"]
            # max_norm itself becomes a float32; below the smallest normal number a multiple of 2^-149, of 2^-133 as bf16, which is half a step off at most
            w = w * (ctypes.c_float(max_norm).value / max_norm)
            off = (t.cpu().double() - w).abs()
            assert torch.all(off <= (step + 2.0 ** -22) * w.abs() + (2.0 ** -134 + 2.0 ** -149 if t.dtype == torch.bfloat16 else 2.0 ** -149)), scale


def test_norm_and_workspace_apart_from_the_list(cp):
    refuse = cp.binding._refuse_overlap
    refuse("f", [100, 164], [16, 3], [1, 0], None, ((170, 4), (300, 1000)))
    for others in (((160, 4), (300, 1000)), ((172, 4), (60, 41)), ((300, 4), (300, 64))):
        with pytest.raises(cp.CpruneError):
            refuse("f", [100, 164], [16, 3], [1, 0], None, others)


@pytest.mark.gpu
def test_a_norm_in_the_list_is_refused(cp):
    flat = torch.ones(4096, device="cuda")
    for call in (lambda **k: cp.cprune_gradient_norm([flat[:1000]], **k), lambda **k: cp.cprune_clip_gradients([flat[:1000]], 1.0, **k),
                 lambda **k: cp.cprune_clip_gradients([flat[2000:3000]], 1.0, out=[flat[:1000]], **k)):
        for bad in (dict(norm=flat[999:1000]), dict(workspace=torch.empty(0, device="cuda", dtype=torch.uint8).set_(flat.untyped_storage()))):
            with pytest.raises(cp.CpruneError) as e:
                call(**bad)
            assert e.value.status in (1, 3) and (flat == 1).all()
        assert e.value.status == 1
    assert abs(float(cp.cprune_gradient_norm([flat[:1000]], norm=flat[1000:1001])) - 1000 ** 0.5) <= 1e-5
