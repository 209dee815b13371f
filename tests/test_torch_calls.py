"""The operators' calls in compiled code are an accelerator: the library loads and answers without them, and they are built anew for another version of torch."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def cp():
    from paper_2207_01260_b200 import build
    build.build()
    import paper_2207_01260_b200 as m
    m.lib()
    return m


def test_the_library_loads_without_them(cp):
    code = """
import sys, warnings
sys.modules["paper_2207_01260_b200._torch_calls"] = None          # an import raises ImportError
import torch
import paper_2207_01260_b200 as cp
with warnings.catch_warnings(record=True) as told:
    warnings.simplefilter("always")
    L = cp.lib()
assert [w for w in told if "_torch_calls.so" in str(w.message)], told
assert cp.cprune_padded_channels(9) == 16 and cp.lib() is L
for call in (lambda: cp.cprune_group_norm(torch.zeros(1, 2, 2, 16), 17, 1), lambda: cp.cprune_mx_quantize(torch.zeros(4, 16).half(), 16)):
    try:
        call()
    except cp.CpruneError as e:
        assert e.status == 1
    else:
        raise AssertionError("not refused")
print("fine")
"""
    got = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and got.stdout.strip() == "fine", got.stderr


def test_they_are_built_anew_for_another_version_of_torch(cp, monkeypatch):
    from paper_2207_01260_b200 import build
    headers = [os.path.join(build.INCLUDE, "cprune.h")]
    assert not build._calls_stale(headers) and cp.binding._calls.built == build._calls_for()
    monkeypatch.setattr(build, "_calls_for", lambda: "for torch 0.0")
    assert build._calls_stale(headers)


def test_a_host_compiler_that_fails_leaves_the_library(cp, monkeypatch, tmp_path):
    from paper_2207_01260_b200 import build
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_torch_calls.so"))
    for compiler in ("false", str(tmp_path / "none")):
        monkeypatch.setenv("CXX", compiler)
        with pytest.warns(RuntimeWarning, match="_torch_calls.so is not built"):
            assert build.build() == build.LIB
    assert not os.path.exists(build.CALLS)


@pytest.mark.gpu
def test_the_same_bits_without_them(cp, monkeypatch):
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy, rows, w, grads = r(2, 9, 9, 32).bfloat16(), r(2, 9, 9, 32).bfloat16(), r(300, 64).bfloat16(), r(40, 64), [r(1000), r(77).bfloat16()]
    packed = cp.cprune_mx_pack(w)

    def run():
        y, stats = cp.cprune_group_norm(x, 32, 4, activation="silu")
        into = [torch.empty_like(t) for t in grads]
        return [y, stats, *cp.cprune_group_norm_backward(dy, x, 32, 4, stats, activation="silu")[:3], cp.cprune_clip_gradients(grads, 1.0, out=into), *into,
                *cp.cprune_mx_quantize(rows, 64, values=True), cp.cprune_mx_fc(rows, 64, *packed, 40)]

    want = run()
    assert cp.binding._calls.group_norm(x, 32, 4, None, None, 1e-5, 0, None) is not None
    monkeypatch.setattr(cp.binding, "_calls", cp.binding._NoCalls())
    for a, b in zip(run(), want):
        assert a.shape == b.shape and torch.equal(a.flatten()[:1000], b.flatten()[:1000]) if a.dtype is torch.uint8 and a.dim() == 5 else torch.equal(a, b)
