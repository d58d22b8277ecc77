"""What the operators around the experts refuse: wrong sizes, types, pointers and overlaps, on the host, before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import mote_oracle as O

OK, NULL_, SHAPE, ALIGN, WORKSPACE, DTYPE = 0, 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def b():
    from paper_2506_14435_b200 import build
    build.build()
    from paper_2506_14435_b200 import binding
    return binding


FAKE, ODD = 0x100000, 0x100004                    # never dereferenced: the checks run first


def router(b, **kw):
    f = dict(d=256, E=16, k=2, scoring=1, n_groups=4, topk_groups=2, renorm=1, scale=1.0, Wr=FAKE, w_dtype=0, logit_bias=None,
             select_bias=None, packed=FAKE)
    f.update(kw)
    return C.byref(b.mote_router_t(*[f[n] for n, _ in b.mote_router_t._fields_]))


def route(b, r, x=FAKE, ldx=256, T=4, idx=FAKE, w=FAKE):
    return b.lib.mote_route_scored(r, x, ldx, T, idx, w, None, None)


def test_route_scored_refusals(b):
    assert route(b, None) == NULL_
    for bad in (dict(d=252), dict(d=0), dict(d=32776), dict(E=0), dict(E=65), dict(k=0), dict(k=17), dict(E=32, k=9, n_groups=1, topk_groups=1),
                dict(n_groups=3), dict(n_groups=0), dict(topk_groups=0), dict(topk_groups=5), dict(k=5, topk_groups=1), dict(scoring=2),
                dict(scoring=-1), dict(scale=float("nan"))):
        assert route(b, router(b, **bad)) == SHAPE, bad
    assert route(b, router(b, w_dtype=2)) == DTYPE
    assert route(b, router(b, Wr=None)) == NULL_ and route(b, router(b, packed=None)) == NULL_
    assert route(b, router(b, Wr=ODD)) == ALIGN and route(b, router(b, packed=FAKE + 16)) == ALIGN
    r = router(b)
    assert route(b, r, T=-1) == SHAPE and route(b, r, T=(1 << 24) + 1) == SHAPE and route(b, r, ldx=248) == SHAPE
    assert route(b, r, ldx=260) == ALIGN and route(b, r, x=ODD) == ALIGN
    assert route(b, r, x=None) == NULL_ and route(b, r, idx=None) == NULL_ and route(b, r, w=None) == NULL_
    assert route(b, r, T=0, x=None, idx=None, w=None) == OK


def test_router_pack_refusals(b):
    pb, pack = b.lib.mote_router_pack_bytes, b.lib.mote_router_pack
    assert pb(16, 256, 0) > 0 and pb(0, 256, 0) == 0 and pb(65, 256, 0) == 0 and pb(16, 252, 0) == 0 and pb(16, 256, 7) == 0
    assert pb(16, 32776, 0) == 0
    n = pb(16, 256, 0)
    assert pack(FAKE, 7, 16, 256, FAKE, n, None) == DTYPE and pack(FAKE, 0, 16, 252, FAKE, n, None) == SHAPE
    assert pack(None, 0, 16, 256, FAKE, n, None) == NULL_ and pack(FAKE, 0, 16, 256, None, n, None) == NULL_
    assert pack(ODD, 0, 16, 256, FAKE, n, None) == ALIGN and pack(FAKE, 0, 16, 256, FAKE + 16, n, None) == ALIGN
    assert pack(FAKE, 0, 16, 256, FAKE, n - 1, None) == WORKSPACE


def test_moe_forward_scored_refusals(b):
    L = b.mote_layer_t(256, 512, 16, 2, 1, 0)
    for name, ctype in b.mote_layer_t._fields_[6:]:
        if ctype is C.c_void_p:
            setattr(L, name, 0x2000)
    L.Wr = L.router_bias = None                   # not used

    def call(layer, r, ws_bytes=1 << 30):
        return b.lib.mote_moe_forward_scored(layer, r, FAKE, None, 4, 0x200000, None, 0x300000, ws_bytes, None)

    assert call(None, router(b)) == NULL_ and call(C.byref(L), None) == NULL_
    for bad in (dict(d=264), dict(E=8, k=2), dict(k=3)):
        assert call(C.byref(L), router(b, **bad)) == SHAPE, bad
    assert call(C.byref(L), router(b, n_groups=3)) == SHAPE
    assert call(C.byref(L), router(b), ws_bytes=16) == WORKSPACE
    L.gate_packed = None
    assert call(C.byref(L), router(b)) == NULL_


def norm(b, **kw):
    f = dict(d=256, eps=1e-6, scale=1.0, post_norm=1, post_gain=FAKE, pre_gain=FAKE, res_dtype=1, gate_cols=0, gate_dtype=0,
             gate_sigmoid=0, gate_tokens=1)
    f.update(kw)
    return C.byref(b.mote_block_norm_t(*[f[n] for n, _ in b.mote_block_norm_t._fields_]))


def run_norm(b, n, y=0x100000, ldy=256, res=0x200000, ldr=256, gate=None, T=4, res_out=0x300000, normed=0x400000):
    return b.lib.mote_block_norm(n, y, ldy, res, ldr, gate, T, res_out, normed, None)


def test_block_norm_refusals(b):
    assert run_norm(b, None) == NULL_
    for bad in (dict(d=252), dict(d=0), dict(d=32776), dict(eps=-1.0), dict(eps=float("nan")), dict(gate_cols=2), dict(gate_cols=-1),
                dict(gate_tokens=-1)):
        assert run_norm(b, norm(b, **bad)) == SHAPE, bad
    assert run_norm(b, norm(b, res_dtype=3)) == DTYPE and run_norm(b, norm(b, gate_cols=1, gate_dtype=3), gate=FAKE) == DTYPE
    n = norm(b)
    assert run_norm(b, n, T=-1) == SHAPE and run_norm(b, n, T=(1 << 24) + 1) == SHAPE
    assert run_norm(b, n, ldy=248) == SHAPE and run_norm(b, n, ldr=248) == SHAPE
    assert run_norm(b, n, ldy=260) == ALIGN and run_norm(b, n, ldr=260) == ALIGN
    assert run_norm(b, norm(b, res_dtype=0), ldr=258) == ALIGN
    assert run_norm(b, n, y=None) == NULL_ and run_norm(b, n, res_out=None, normed=None) == NULL_
    assert run_norm(b, norm(b, gate_cols=1)) == NULL_
    for bad in (dict(y=ODD), dict(res=ODD), dict(res_out=ODD), dict(normed=ODD)):
        assert run_norm(b, n, **bad) == ALIGN, bad
    assert run_norm(b, norm(b, post_gain=ODD)) == ALIGN and run_norm(b, norm(b, pre_gain=ODD)) == ALIGN
    assert run_norm(b, norm(b, gate_cols=256, gate_dtype=1), gate=ODD) == ALIGN
    assert run_norm(b, norm(b, gate_cols=1, gate_dtype=1), gate=FAKE + 1) == ALIGN
    assert run_norm(b, norm(b, gate_cols=1, gate_dtype=0), gate=FAKE + 2) == ALIGN
    assert run_norm(b, n, y=None, res=None, res_out=None, normed=None, T=0) == OK


def test_block_norm_refuses_overlaps(b):
    n, f = norm(b), norm(b, res_dtype=0)
    row = 256 * 2
    assert run_norm(b, n, res_out=0x200000 + row) == SHAPE              # shifted by a row
    assert run_norm(b, n, ldr=512, res_out=0x200000) == SHAPE           # another stride
    assert run_norm(b, n, normed=0x300000 + row) == SHAPE               # the two outputs
    assert run_norm(b, n, normed=0x300000) == SHAPE
    assert run_norm(b, f, res_out=0x100000) == SHAPE                    # fp32 over bf16
    assert run_norm(b, f, res_out=0x100000, T=1) == SHAPE
    assert run_norm(b, f, ldy=512, res_out=0x100000) == SHAPE
    assert run_norm(b, f, normed=0x200000) == SHAPE                     # bf16 over fp32
    g = norm(b, gate_cols=256, gate_dtype=1, gate_tokens=1)
    assert run_norm(b, g, gate=0x300000) == SHAPE and run_norm(b, g, gate=0x400000 + row) == SHAPE


def linear(b, **kw):
    f = dict(N=128, K=256, W=FAKE, bits=16, w_scale=None, bias=None, act=0)
    f.update(kw)
    return C.byref(b.mote_linear_t(*[f[n] for n, _ in b.mote_linear_t._fields_]))


def run_linear(b, l, x=0x200000, ldx=256, T=4, res=None, ldr=128, out=0x300000, out_dtype=1, ws=0x400000, ws_bytes=1 << 40):
    return b.lib.mote_linear(l, x, ldx, T, res, ldr, out, out_dtype, ws, ws_bytes, None)


def test_linear_refusals(b):
    assert run_linear(b, None) == NULL_
    for bad in (dict(N=0), dict(N=(1 << 24) + 1), dict(K=0), dict(K=252), dict(K=65544), dict(bits=5), dict(bits=8, K=264, w_scale=FAKE),
                dict(act=5), dict(act=-1)):
        assert run_linear(b, linear(b, **bad)) == SHAPE, bad
        assert b.lib.mote_linear_workspace_bytes(linear(b, **bad), 4) == 0, bad
    l = linear(b)
    assert b.lib.mote_linear_workspace_bytes(l, -1) == 0 and b.lib.mote_linear_workspace_bytes(None, 4) == 0
    need = b.lib.mote_linear_workspace_bytes(l, 4)
    assert need >= 256
    assert run_linear(b, l, ws_bytes=need - 1) == WORKSPACE
    assert run_linear(b, l, T=-1) == SHAPE and run_linear(b, l, T=(1 << 24) + 1) == SHAPE
    assert run_linear(b, l, out_dtype=2) == DTYPE
    assert run_linear(b, linear(b, W=None)) == NULL_ and run_linear(b, linear(b, bits=8)) == NULL_
    for bad in (dict(x=None), dict(out=None), dict(ws=None)):
        assert run_linear(b, l, **bad) == NULL_, bad
    assert run_linear(b, l, ldx=248) == SHAPE and run_linear(b, l, res=FAKE, ldr=120) == SHAPE
    assert run_linear(b, l, ldx=260) == ALIGN and run_linear(b, l, ws=0x400010) == ALIGN
    for bad in (dict(x=ODD), dict(out=ODD), dict(res=ODD)):
        assert run_linear(b, l, **bad) == ALIGN, bad
    assert run_linear(b, linear(b, W=ODD)) == ALIGN and run_linear(b, linear(b, bias=ODD)) == ALIGN
    assert run_linear(b, linear(b, bits=4, w_scale=ODD)) == ALIGN
    assert run_linear(b, l, out=0x200000) == SHAPE                      # over x
    assert run_linear(b, l, res=0x300000, out_dtype=0) == SHAPE         # fp32 over a bf16 residual
    assert run_linear(b, l, res=0x300000, ldr=256) == SHAPE
    assert run_linear(b, l, res=0x300000 + 256) == SHAPE
    assert run_linear(b, l, x=None, out=None, ws=None, T=0) == OK


def test_python_calls_refuse_tensors_that_are_not_on_a_gpu(b):
    with pytest.raises(ValueError):
        b.MoteRouter(torch.zeros(4, 64), 2)
    with pytest.raises(ValueError):
        b.MoteLinear(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.MoteBlockNorm(64, pre_gain=torch.zeros(64))
    with pytest.raises(ValueError):
        b.mote_block_norm(b.MoteBlockNorm(64), torch.zeros(3, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.mote_block_norm(b.MoteBlockNorm(64), [1.0])


# ------------------------------------------------------------------------------------------------ the statements themselves
def test_scored_router_statement_on_small_cases():
    x, W = np.eye(4), np.array([[3.0, 0, 0, 0], [1, 0, 0, 0], [2, 0, 0, 0], [2, 0, 0, 0]])
    r = O.route_scored(x[:1], W, 3, scoring="sigmoid")
    assert r["idx"].tolist() == [[0, 2, 3]] and abs(r["w"].sum() - 1.0) < 1e-12
    # a bias moves the choice, not the weights
    r2 = O.route_scored(x[:1], W, 2, scoring="sigmoid", select_bias=[0, 1.0, 0, 0], renorm=False)
    assert r2["idx"].tolist() == [[1, 0]] and np.allclose(r2["w"], 1 / (1 + np.exp(-np.array([[1.0, 3.0]]))))
    # groups: {3, 1} against {2, 2}: sigmoid(3) + sigmoid(1) < 2 sigmoid(2)
    r3 = O.route_scored(x[:1], W, 1, scoring="sigmoid", n_groups=2, topk_groups=1)
    assert r3["idx"].tolist() == [[2]]
    assert O.route_scored(x[1:2], W, 2)["idx"].tolist() == [[0, 1]]     # all equal: lower index


def test_block_norm_statement_on_small_cases():
    y = np.array([[3.0, 4.0], [0.0, 0.0]])
    assert np.allclose(O.block_norm(y, np.ones((2, 2)), eps=0.5, scale=2.0), 1 + 2 * y)
    p = O.block_norm(y[:1], None, eps=0.0, post_norm=True, gate=np.array([[0.0]]), gate_sigmoid=True)
    assert np.allclose(p, 0.5 * y[:1] / np.sqrt(12.5))
    g = O.block_norm(np.ones((5, 2)), None, eps=0.0, gate=np.arange(4.0).reshape(2, 2), gate_tokens=3)
    assert g.tolist() == [[0, 1]] * 3 + [[2, 3]] * 2


def test_linear_statement_on_small_cases():
    assert O.linear([[1.0, 2]], [[3.0, 4]], bias=[-12.0], act="relu", residual=[[1.0]]).tolist() == [[1.0]]
    z = np.linspace(-6, 6, 25)
    t = torch.from_numpy(z)
    for act, f in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu),
                   ("gelu_tanh", lambda v: torch.nn.functional.gelu(v, approximate="tanh"))):
        assert np.allclose(O.activation(z, act), f(t).numpy(), atol=1e-15), act
