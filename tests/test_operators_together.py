"""The operators around the convolutions in one run, as they are used: a pruned conv task, group norm and activation, a 1x1 layer and the classifier in 4-bit
weights; then the gradients of the norm's parameters, clipped together with others."""
import threading

import numpy as np
import pytest
import torch

import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cp():
    import paper_2207_01260_b200 as m
    m.lib()
    return m


class Candidate:
    """One pruned layer and what follows it.  64 filters of which 48 are kept, 6 groups, a 1x1 layer of 72 features with a shortcut, 10 classes."""

    def __init__(self, cp, batch):
        self.cp, self.batch = cp, batch
        m = wl.single_task()
        w, b = (torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in wl.model_weights(m)["conv"])
        _, w, b, _ = cp.cprune_select_filters(w, 48, b)
        self.plan = cp.cprune_task_plan(batch, 64, 32, 32, 48, 3, 3, 1, 1, activation="none")
        self.conv = cp.cprune_pack_weights(self.plan, w, b)
        g = torch.Generator(device="cuda").manual_seed(5)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.gamma, self.beta = 1 + 0.2 * r(48), 0.2 * r(48)
        self.w1, self.b1, self.w2, self.b2 = r(72, 48, 1, 1) / 7, 0.1 * r(72), r(10, 72) / 8, 0.1 * r(10)
        self.mx1, self.mx2 = cp.cprune_mx_pack(self.w1, self.b1), cp.cprune_mx_pack(self.w2, self.b2)
        self.shortcut = torch.zeros((batch, 32, 32, 72), dtype=torch.bfloat16, device="cuda")
        self.shortcut[..., :72] = r(batch, 32, 32, 72)

    def forward(self, x):
        cp = self.cp
        a = cp.cprune_task_run(self.plan, cp.cprune_cast_input(x), *self.conv)
        n, stats = cp.cprune_group_norm(a, 48, 6, self.gamma, self.beta, 1e-5, "silu")
        p = cp.cprune_mx_fc(n, 48, *self.mx1, 72, "relu", self.shortcut)
        q = cp.cprune_global_avgpool(p, 72)
        return a, n, stats, p, q, cp.cprune_mx_fc(q, 72, *self.mx2, 10, out_f32=True)


def values(cp, t, C):
    """What a tensor's rows, or weights, stand for after the rounding to 4 bits, in 64 bits."""
    c, s, _ = cp.cprune_mx_quantize(t, C)
    return cp.cprune_mx_dequantize(c, s, C).double()


@pytest.mark.parametrize("batch", [2, 16])
def test_a_run_of_them(cp, batch):
    net = Candidate(cp, batch)
    x = torch.from_numpy(wl.model_input(wl.single_task(), batch)).cuda()
    a, n, stats, p, q, logits = net.forward(x)
    cp.cprune_poll_device_status()
    # every step against 64 bits of its own input: half a step of the stored type, and float32 sums
    v = a[..., :48].double().reshape(batch, 1024, 6, 8)
    mean, var = v.mean((1, 3), keepdim=True), v.var((1, 3), correction=0, keepdim=True)
    z = ((v - mean) / (var + 1e-5).sqrt()).reshape(batch, 32, 32, 48) * net.gamma.double() + net.beta.double()
    want = z * torch.sigmoid(z)
    assert torch.all((n[..., :48].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * (1 + z.abs()))
    rows = values(cp, n, 48)
    w1, w2 = values(cp, net.w1.reshape(72, 48).contiguous(), 48), values(cp, net.w2, 72)
    z = (rows @ w1.t() + net.b1.double()).reshape(batch, 32, 32, 72) + net.shortcut[..., :72].double()
    size = (rows.abs() @ w1.abs().t() + net.b1.double().abs()).reshape(z.shape) + net.shortcut[..., :72].double().abs()
    want = z.clamp(min=0)
    assert torch.all((p[..., :72].double() - want).abs() <= 2.0 ** -8 * want.abs() + 64 * 2.0 ** -23 * size)
    want = p[..., :72].double().mean((1, 2))
    assert torch.all((q[:, :72].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5)
    rows = values(cp, q, 72)
    want, size = rows @ w2.t() + net.b2.double(), rows.abs() @ w2.abs().t() + net.b2.double().abs()
    assert torch.all((logits.double() - want).abs() <= 2.0 ** -24 * want.abs() + 100 * 2.0 ** -23 * size)
    # a short training's step behind it
    g = torch.Generator(device="cuda").manual_seed(6)
    dy = torch.randn(n.shape, generator=g, device="cuda").bfloat16()
    da, dgamma, dbeta, _ = cp.cprune_group_norm_backward(dy, a, 48, 6, stats, net.gamma, net.beta, "silu")
    dw = torch.randn((48, 64, 3, 3), generator=g, device="cuda").bfloat16()
    grads = [dgamma, dbeta, dw, da]
    total = float(torch.sqrt(sum(t.double().square().sum() for t in grads)))
    before = [t.double().clone() for t in grads]
    norm = cp.cprune_clip_gradients(grads, 2.0)
    assert abs(float(norm) - total) <= 2.0 ** -23 * total and total > 2.0
    for t, b in zip(grads, before):
        want = b * (2.0 / (total + 1e-6))
        assert torch.all((t.double() - want).abs() <= (2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24) * want.abs() + 2.0 ** -22 * want.abs())


def test_a_run_of_them_captured_and_replayed(cp):
    net = Candidate(cp, 8)
    m = wl.single_task()
    x = torch.from_numpy(wl.model_input(m, 8)).cuda()
    other = torch.from_numpy(wl.model_input(m, 9)[1:]).cuda()
    want = [net.forward(v)[5].clone() for v in (x, other)]
    given = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = net.forward(given)[5]
    for v, w in ((x, want[0]), (other, want[1]), (x, want[0])):
        given.copy_(v)
        graph.replay()
        assert torch.equal(logits, w)
    cp.cprune_poll_device_status()


def work_of(cp, seed):
    """A call of every kernel, at sizes that share an SM with other work: the results, and a function that makes them again."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy = (r(4, 56, 56, 56).bfloat16() for _ in range(2))
    small, gamma, beta = r(2, 14, 14, 30), r(56), r(56)
    rows, few = r(20000, 192).bfloat16(), r(8, 8192).bfloat16()
    wide, deep, mid = cp.cprune_mx_pack(r(40, 192)), cp.cprune_mx_pack(r(256, 8192)), cp.cprune_mx_pack(r(600, 192))
    grads = [r(3000), r(70000).bfloat16(), r(11)]

    def again():
        y, stats = cp.cprune_group_norm(x, 56, 7, gamma, beta, 1e-5, "relu", dy)
        got = [y, stats, *cp.cprune_group_norm_backward(dy, x, 56, 7, stats, gamma, beta, "relu", y), *cp.cprune_group_norm(small, 30, 5)]
        got += [cp.cprune_mx_fc(rows, 192, *wide, 40), cp.cprune_mx_fc(few, 8192, *deep, 256, "relu"), cp.cprune_mx_fc(rows, 192, *mid, 600, out_f32=True)]
        got += [cp.cprune_mx_fc(few[:, :192].contiguous(), 192, *wide, 40)]
        into = [torch.empty_like(t) for t in grads]
        return got + [cp.cprune_clip_gradients(grads, 1.0, out=into), *into]

    return again


def test_threads_and_graphs_side_by_side(cp):
    """Two threads on their own streams, then two graphs replayed on two streams at once: the bits of each alone."""
    jobs = [work_of(cp, s) for s in (1, 2)]
    want = [[t.clone() for t in j()] for j in jobs]
    torch.cuda.synchronize()
    wrong = [[], []]

    def run(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(15):
                wrong[k] += [i for i, (a, b) in enumerate(zip(jobs[k](), want[k])) if not torch.equal(a, b)]

    threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [[], []]
    graphs, got = [torch.cuda.CUDAGraph() for _ in jobs], []
    for graph, job in zip(graphs, jobs):
        with torch.cuda.graph(graph):
            got.append(job())
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for a, b in zip(got[k], want[k]))
    cp.cprune_poll_device_status()


def test_a_call_that_failed_on_the_way_is_not_made_again(cp, monkeypatch):
    """Functions that say that a launch failed, in the library's place: a clipping in place has perhaps scaled a part of the list by then."""
    import ctypes
    b, made = cp.binding, []

    class Failing:
        def __getattr__(self, name):
            real = getattr(b._lib, name)
            if name.endswith("_bytes") or name == "cprune_padded_channels":
                return real
            fake = ctypes.CFUNCTYPE(ctypes.c_int, *real.argtypes)(lambda *a: made.append(name) or 4)
            keep.append(fake)
            return fake

    keep = []
    x = torch.zeros((2, 5, 5, 16), dtype=torch.bfloat16, device="cuda")
    _, stats = cp.cprune_group_norm(x, 16, 2)
    packed = cp.cprune_mx_pack(torch.zeros((8, 16), device="cuda"))
    calls = {"cprune_group_norm": lambda: cp.cprune_group_norm(x, 16, 2), "cprune_group_norm_backward": lambda: cp.cprune_group_norm_backward(x, x, 16, 2, stats),
             "cprune_clip_gradients": lambda: cp.cprune_clip_gradients([x], 1.0), "cprune_mx_quantize": lambda: cp.cprune_mx_quantize(x, 16),
             "cprune_mx_fc": lambda: cp.cprune_mx_fc(x, 16, *packed, 8)}
    real, failing = b._lib, Failing()
    try:
        b._hand_over(b._calls, failing)
        for name, call in calls.items():
            # a second try, by the steps in Python, would reach the real function: count it there as well
            monkeypatch.setattr(real, name, lambda *a, name=name: made.append(name) or 4)
            made.clear()
            with pytest.raises(cp.CpruneError) as e:
                call()
            assert e.value.status == 4 and name in str(e.value) and made == [name]
            monkeypatch.undo()
    finally:
        b._hand_over(b._calls, real)
    for call in calls.values():
        call()
    torch.cuda.synchronize()


def test_threads_that_count(cp):
    """As above, and an exception in a thread ends the test, and every round is counted."""
    from concurrent.futures import ThreadPoolExecutor
    jobs = [work_of(cp, s) for s in (3, 4)]
    want = [[t.clone() for t in j()] for j in jobs]
    torch.cuda.synchronize()

    def run(k):
        equal = 0
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(15):
                got = jobs[k]()
                assert len(got) == len(want[k])
                equal += all(torch.equal(a, b) for a, b in zip(got, want[k]))
        return equal

    with ThreadPoolExecutor(2) as pool:
        assert [f.result(timeout=300) for f in [pool.submit(run, k) for k in range(2)]] == [15, 15]
    cp.cprune_poll_device_status()
