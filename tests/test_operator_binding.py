"""The binding of the operators around the experts, on the host: what it needs, what it refuses, how its extension module is built."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    from paper_2506_14435_b200 import build
    build.build()
    from paper_2506_14435_b200 import binding
    return binding


def test_only_the_calls_that_go_through_the_extension_module_need_it(b):
    """As with another torch than the one it was built for, or before it is built."""
    code = """
import importlib.abc, sys
class Block(importlib.abc.MetaPathFinder):
    def find_spec(self, name, path, target=None):
        if name == "paper_2506_14435_b200._calls":
            raise ImportError("undefined symbol")
sys.meta_path.insert(0, Block())
import torch
import paper_2506_14435_b200 as mote
assert mote.lib.mote_route_scored(None, None, 0, 0, None, None, None, None) == 1
assert mote.lib.mote_rms_norm(None, 0, 64, 1e-6, None, None) == 0
for name in mote.__all__:
    getattr(mote, name)
norm = mote.MoteBlockNorm(64)
for _ in range(2):
    try:
        mote.mote_block_norm(norm, torch.zeros(3, 64, dtype=torch.bfloat16))
    except ImportError as e:
        assert "_calls.so" in str(e) and "paper_2506_14435_b200.build" in str(e)
    else:
        raise AssertionError("no error")
print("done")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr


def test_the_extension_module_is_linked_again_for_another_torch(b, monkeypatch, tmp_path):
    """Objects of two torch versions lie side by side: going back to the first one links it again, although it is older than the library."""
    from paper_2506_14435_b200 import build
    linked, calls = [], tmp_path / "_calls.so"

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def run(cmd, **kw):
        linked.append([c for c in cmd if c.endswith(".o")])
        calls.write_text(str(linked[-1]))
        return Done

    monkeypatch.setattr(build, "CALLS", str(calls))
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libmote.so"))
    monkeypatch.setattr(build, "_sources", lambda: [])
    monkeypatch.setattr(build.subprocess, "run", run)
    (tmp_path / "libmote.so").write_text("")
    a, other = tmp_path / "torch_calls-A.o", tmp_path / "torch_calls-B.o"
    a.write_text("")
    other.write_text("")
    os.utime(a, (1000, 1000))
    os.utime(other, (2000, 2000))
    for obj in (a, a, other, other, a, a):
        monkeypatch.setattr(build, "_compile_calls", lambda obj=obj: str(obj))
        build.build()
        assert calls.read_text() == str([str(obj)])
    assert linked == [[str(a)], [str(other)], [str(a)]]
    os.utime(a, (3000, 3000))                              # compiled anew
    build.build()
    assert len(linked) == 4


def test_tensors_that_require_grad_are_refused_where_grad_is_recorded(b):
    """The operators have no backward pass: a gradient would be lost without a word."""
    x = torch.zeros(3, 64, dtype=torch.bfloat16, requires_grad=True)
    plain = torch.zeros(3, 64, dtype=torch.bfloat16)
    norm = b.MoteBlockNorm(64)

    class Router:                                                  # (nothing of them is read before the tensors)
        device, _address = -1, 0

    class Linear:
        device, _address, _ws_T, _ws_address, _ws_bytes = -1, 0, 3, 0, 0

    class Layer:
        d = 64

    calls = [lambda t: b.mote_block_norm(norm, t), lambda t: b.mote_route_scored(Router, t), lambda t: b.mote_linear(Linear, t),
             lambda t: b.mote_moe_forward_scored(Layer, Router, t), lambda t: b.mote_moe_forward_scored(Layer, Router, plain, residual=t)]
    for call in calls:
        with pytest.raises(ValueError, match="requires grad"):
            call(x)
        with torch.no_grad(), pytest.raises(Exception) as e:       # not on a GPU
            call(x)
        assert "requires grad" not in str(e.value)


def test_outputs_over_weights_and_workspaces_are_refused(b):
    """On the host, before anything is launched; the addresses are never dereferenced."""
    SHAPE, row = 2, 256 * 4

    def norm(res_out=0x300000, normed=0x400000, **kw):
        f = dict(d=256, eps=1e-6, scale=1.0, post_norm=1, post_gain=0x500000, pre_gain=0x600000, res_dtype=1, gate_cols=0, gate_dtype=0,
                 gate_sigmoid=0, gate_tokens=1)
        f.update(kw)
        n = C.byref(b.mote_block_norm_t(*[f[k] for k, _ in b.mote_block_norm_t._fields_]))
        return b.lib.mote_block_norm(n, 0x100000, 256, 0x200000, 256, None, 4, res_out, normed, None)

    for gain in (0x500000, 0x600000):                       # a gain of 1 KB, outputs of 2 KB
        for at in (gain, gain + row - 16, gain - 2 * row + 16):
            assert norm(res_out=at) == SHAPE and norm(normed=at) == SHAPE, hex(at)

    def linear(out, bits=8, **kw):
        f = dict(N=128, K=256, W=0x500000, bits=bits, w_scale=0x600000, bias=0x700000, act=0)
        f.update(kw)
        l = C.byref(b.mote_linear_t(*[f[k] for k, _ in b.mote_linear_t._fields_]))
        return b.lib.mote_linear(l, 0x200000, 256, 100, None, 0, out, 1, 0x800000, 1 << 20, None)

    for at in (0x500000, 0x500000 + 128 * 256 - 16, 0x600000, 0x700000 + 512 - 16, 0x800000, 0x800000 + 256 + 128 * 512 - 16, 0x800000 - 16):
        assert linear(at) == SHAPE, hex(at)
    assert linear(0x500000 + 128 * 256, bits=16) == SHAPE   # bf16 weights take twice as much


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=-3), dict(k=2 ** 31 - 1), dict(n_groups=3), dict(topk_groups=0), dict(scoring=7)])
def test_a_router_that_the_library_refuses_is_refused_before_outputs_are_made(b, bad):
    f = dict(d=64, E=16, k=2, scoring=1, n_groups=1, topk_groups=1, renorm=1, scale=1.0, Wr=0x100000, w_dtype=0, logit_bias=None, select_bias=None,
             packed=0x100000)
    f.update(bad)

    class Router:
        device, struct = 0, b.mote_router_t(*[f[n] for n, _ in b.mote_router_t._fields_])
        _address = C.addressof(struct)

    with pytest.raises(b.MoteError):
        b.mote_route_scored(Router, torch.zeros(3, 64, dtype=torch.bfloat16))
