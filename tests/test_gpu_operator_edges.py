"""Inputs on which the operators around the experts (mote_route_scored, mote_block_norm, mote_linear) go wrong if a bound, a barred
entry or a value that is not finite is not minded, against statements in 64 bits (oracle/mote_oracle.py) and sharp bounds."""
import numpy as np
import pytest
import torch

from oracle import mote_oracle as O
from parity_utils import REL_FRO_TOL, bf16_bits, bf16_tensor
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mote():
    import paper_2506_14435_b200 as m
    return m


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ scored router
# A token and two router rows, 0 and 1, whose logits differ by a little in favour of row 0.  Its logit is one product of 1 and many
# small ones, each lost to an adder that has the 1 already; row 1's is the product 1 + m 2^-23 alone.
def spike_rows(kind, d):
    small_x, small_w, first, last = {
        # products of 2^-30, one after the other: 512 of them are 2^-21, each below half of the last place of 1
        "chain": (2.0 ** -15, 2.0 ** -15, 0, d),
        # products just below 2^-25 beside the 1, in one step of the tensor cores
        "step": (1.9375 * 2.0 ** -13, 1.03125 * 2.0 ** -13, 0, 64),
        # both
        "all": (1.9375 * 2.0 ** -13, 1.03125 * 2.0 ** -13, 0, d),
    }[kind]
    x, a = np.zeros(d), np.zeros(d)
    x[first:last], a[first:last] = small_x, small_w
    x[0] = a[0] = 1.0
    return x, a


@pytest.mark.parametrize("tokens", [1, 20, 333, 9728])
@pytest.mark.parametrize("d", [128, 2048, 8192, 32768])
@pytest.mark.parametrize("kind", ["chain", "step", "all"])
@pytest.mark.parametrize("E", [2, 64])
def test_route_scored_small_products_beside_a_large_one(mote, kind, d, tokens, E):
    x, a = spike_rows(kind, d)
    gain = (x[1:] @ a[1:]) * 2.0 ** 23                    # what row 0 has over 1, in units of 2^-23
    xt = torch.tensor(x, device="cuda").bfloat16()
    assert np.array_equal(_f64(xt), x)
    for m in sorted({max(1, round(gain * q)) for q in (0.1, 0.3, 0.5, 0.6, 0.7, 0.8, 0.9, 0.97, 1.03, 1.2)}):
        Wr = torch.zeros(E, d, dtype=torch.float64)
        Wr[:, 0] = -1.0
        Wr[0] = torch.tensor(a)
        Wr[1] = 0.0
        Wr[1, 0] = 1.0 + m * 2.0 ** -23
        Wt = Wr.cuda().float()
        assert torch.equal(Wt.double().cpu(), Wr) and gain != m
        xs = xt.repeat(tokens, 1)
        xs[1::2] *= 4.0                                   # (an exact multiple: the same order)
        for scoring, k in (("softmax", 1), ("sigmoid", 2)):
            idx = mote.mote_route_scored(mote.MoteRouter(Wt, k, scoring=scoring), xs)[0]
            want = [0, 1][:k] if gain > m else [1, 0][:k]
            assert bool((idx.cpu() == torch.tensor(want, dtype=torch.int32)).all()), (m, gain, idx[:3].tolist())


@pytest.mark.parametrize("d,E,w_dtype", [(2048, 64, torch.float32), (8192, 16, torch.float32), (32768, 8, torch.bfloat16), (32768, 64, torch.float32)])
def test_route_scored_wide_tokens_get_the_same_experts_in_every_batch(mote, d, E, w_dtype):
    """Pairs of rows that differ in their last bits, tokens of one sign with a leading channel: alone, in middle and in long batches
    the choice of exact arithmetic."""
    T = 9728
    x = _randn(201, 64, d).abs()
    x[::2, 0] *= 1000.0
    x = x.bfloat16()
    Wr = (_randn(202, E // 2, d).abs() * 0.02).repeat_interleave(2, dim=0)
    Wr[1::2] += (torch.rand(E // 2, d, generator=torch.Generator("cuda").manual_seed(203), device="cuda") - 0.5) * (2.0 ** -27 if w_dtype == torch.float32 else 2.0 ** -16)
    Wr = Wr.to(w_dtype).contiguous()
    want = torch.from_numpy(O.route_scored(_f64(x), _f64(Wr), 4, scoring="sigmoid")["idx"])
    r = mote.MoteRouter(Wr, 4, scoring="sigmoid")
    long = mote.mote_route_scored(r, x.repeat(T // 64, 1))[0].cpu().view(-1, 64, 4)
    assert bool((long == want).all())
    assert torch.equal(mote.mote_route_scored(r, x)[0].cpu(), want)
    assert torch.equal(mote.mote_route_scored(r, x[5:6])[0].cpu(), want[5:6])


@pytest.mark.parametrize("tokens", [1, 40, 2600])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n_groups,topk_groups", [(1, 1), (4, 3), (8, 8)])
def test_route_scored_barred_logits_are_last_whatever_the_bias(mote, tokens, scoring, n_groups, topk_groups):
    """A logit_bias of -inf bars an expert that select_bias favours too; where all are barred, the lower indices and weights of 0."""
    E, d, k = 64, 512, 6
    x = _randn(211, tokens, d).bfloat16()
    x[-1] = 0.0
    Wr = _randn(212, E, d) * 0.02
    sb = _randn(213, E) * 0.02
    lb = torch.zeros(E, device="cuda")
    lb[1::3] = -float("inf")
    sb[1::3] = 0.9
    opt = dict(scoring=scoring, n_groups=n_groups, topk_groups=topk_groups)
    idx, w, logits = mote.mote_route_scored(mote.MoteRouter(Wr, k, logit_bias=lb, select_bias=sb, **opt), x, want_logits=True)
    assert bool((idx % 3 != 1).all()) and bool((w > 0.0).all())
    assert bool((logits[:, 1::3] == -float("inf")).all())
    ref = O.route_scored(_f64(x), _f64(Wr), k, logit_bias=_f64(lb), select_bias=_f64(sb), **opt)
    assert np.array_equal(idx.cpu().numpy(), ref["idx"])
    # four are left: the others follow, the lower index first, with weights of 0
    lb[:] = -float("inf")
    lb[[3, 17, 40, 63]] = 0.0
    four = mote.mote_route_scored(mote.MoteRouter(Wr, k, logit_bias=lb, select_bias=sb, scoring=scoring), x)
    assert bool((four[0][:, :4].sort(dim=1).values.cpu() == torch.tensor([3, 17, 40, 63])).all())
    assert bool((four[0][:, 4:].cpu() == torch.tensor([0, 1])).all()) and bool((four[1][:, 4:] == 0.0).all())
    # none is left
    lb[:] = -float("inf")
    for bias in (None, sb):
        for renorm in (True, False):
            idx, w, _ = mote.mote_route_scored(mote.MoteRouter(Wr, k, logit_bias=lb, select_bias=bias, renorm=renorm, **opt), x)
            ref = O.route_scored(_f64(x[:1]), _f64(Wr), k, logit_bias=_f64(lb), select_bias=_f64(bias), **opt)
            assert bool((idx.cpu() == torch.from_numpy(ref["idx"])).all()) and bool((w == 0.0).all())


@pytest.mark.parametrize("tokens", [9, 3000])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("spread", [0.5, 8.0, 25.0])
def test_route_scored_weights_of_exact_logits(mote, scoring, spread, renorm, tokens):
    """Tokens with one channel of 1: the logits are the router's entries, so the weights' own arithmetic is seen.  In units of 2^-24: e^x 4, its
    argument's rounding |x|, seven additions, reciprocals and products of 2 and 1 each, twice with renorm: 32 and |x| at most."""
    E, d, k = 16, 1024, 8
    x = torch.zeros(tokens, d, device="cuda")
    x[torch.arange(tokens), torch.arange(tokens) % d] = 1.0
    Wr = _randn(231, E, d) * spread
    idx, w, logits = mote.mote_route_scored(mote.MoteRouter(Wr, k, scoring=scoring, renorm=renorm, scale=2.5), x.bfloat16(), want_logits=True)
    l = Wr.T[torch.arange(tokens) % d]
    assert torch.equal(logits, l)
    ref = O.route_scored(_f64(x), _f64(Wr), k, scoring=scoring, renorm=renorm, scale=2.5)
    assert np.array_equal(idx.cpu().numpy(), ref["idx"])
    far = _f64(l.max(dim=1, keepdim=True).values - l.gather(1, idx.long())) if scoring == "softmax" else 0.0
    assert np.all(np.abs(_f64(w) - ref["w"]) <= (32.0 + far) * 2.0 ** -24 * ref["w"] + 1e-37)


@pytest.mark.parametrize("tokens,d,E", [(1, 2048, 64), (50, 896, 60), (700, 5000, 16), (1200, 2048, 64), (2003, 5000, 64), (300, 32768, 64)])
@pytest.mark.parametrize("kind", ["normal", "outliers", "positive"])
@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16])
def test_route_scored_logits_within_the_bound_the_choice_relies_on(mote, tokens, d, E, kind, w_dtype):
    """A logit: 27 units of 2^-24 |x| |w|, and a weight what that and 32 units of its own arithmetic make of it."""
    x, Wr = _randn(241, tokens, d), _randn(242, E, d) * 0.02
    if kind == "outliers":
        x[:, ::97] *= 20.0
    elif kind == "positive":
        x, Wr = x.abs(), Wr.abs()
    x, Wr = x.bfloat16(), Wr.to(w_dtype)
    lb = _randn(243, E)
    for scoring in ("softmax", "sigmoid"):
        idx, w, logits = mote.mote_route_scored(mote.MoteRouter(Wr, 4, scoring=scoring, logit_bias=lb), x, want_logits=True)
        ref = O.route_scored(_f64(x), _f64(Wr), 4, scoring=scoring, logit_bias=_f64(lb))
        norms = np.linalg.norm(_f64(x), axis=1)[:, None] * np.linalg.norm(_f64(Wr), axis=1)[None]
        err = 27.0 * 2.0 ** -24 * norms + 2.0 ** -23 * np.abs(_f64(lb))
        assert np.all(np.abs(_f64(logits) - ref["logits"]) <= err)
        assert np.array_equal(idx.cpu().numpy(), ref["idx"])
        # a score moves by its logit's error and its denominator's, a renormalised one by the others' too
        rel = np.expm1(2.0 * err.max(axis=1, keepdims=True)) + (32.0 + np.ptp(ref["logits"], axis=1, keepdims=True)) * 2.0 ** -24
        assert np.all(np.abs(_f64(w) - ref["w"]) <= rel * ref["w"])


@pytest.mark.parametrize("tokens", [4, 70, 1200])
@pytest.mark.parametrize("scoring,n_groups,topk_groups,bias", [("softmax", 1, 1, False), ("softmax", 8, 3, False), ("softmax", 16, 5, False),
                                                               ("softmax", 8, 3, True), ("sigmoid", 1, 1, True), ("sigmoid", 8, 3, False),
                                                               ("sigmoid", 16, 5, True)])
@pytest.mark.parametrize("size", [1e22, 1e-24, 1.0])
def test_route_scored_tokens_whose_squares_leave_fp32(mote, tokens, scoring, n_groups, topk_groups, bias, size):
    """Their norm is infinite or its square vanishes, their logits are ordinary (some far apart, so that scores vanish): nothing is known of the
    errors, everything is evaluated."""
    E, d = 64, 1024
    x = _randn(321, tokens, d) * size
    x[::2] *= 60.0
    sb = _randn(323, E) * 0.02 if bias else None
    Wr = _randn(322, E // 2, d).repeat(2, 1) * (0.05 / size)
    Wr[E // 2:] += (torch.rand(E // 2, d, generator=torch.Generator("cuda").manual_seed(324), device="cuda") - 0.5) * (2.0 ** -24 / size)
    opt = dict(scoring=scoring, n_groups=n_groups, topk_groups=topk_groups)
    idx, w, _ = mote.mote_route_scored(mote.MoteRouter(Wr, 4, select_bias=sb, **opt), x.bfloat16())
    ref = O.route_scored(_f64(x.bfloat16()), _f64(Wr), 4, select_bias=_f64(sb), **opt)
    assert np.array_equal(idx.cpu().numpy(), ref["idx"])
    assert np.all(np.isfinite(_f64(w)))


@pytest.mark.parametrize("tokens", [1, 33, 1200])
@pytest.mark.parametrize("alike", [2, 3, 5, 8, 16])
@pytest.mark.parametrize("scoring,bias", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
def test_route_scored_several_groups_alike(mote, tokens, alike, scoring, bias):
    """Groups whose sums differ in their last bits: any number of them at the border between those that stay and the rest."""
    E, d, G = 64, 512, 16
    x = _randn(331, tokens, d).bfloat16()
    Wr = _randn(332, G, E // G, d) * 0.05
    Wr[:alike] = Wr[:1]
    Wr[:alike] += (torch.rand(alike, E // G, d, generator=torch.Generator("cuda").manual_seed(333), device="cuda") - 0.5) * 2.0 ** -25
    Wr = Wr.view(E, d)[torch.randperm(G, generator=torch.Generator().manual_seed(334)).repeat_interleave(4).cuda() * 4 +
                       torch.arange(4, device="cuda").repeat(G)].contiguous()
    sb = (_randn(335, 4) * 0.05).repeat(G) if bias else None
    for topk_groups in (1, 4, 9):
        opt = dict(scoring=scoring, n_groups=G, topk_groups=topk_groups)
        idx = mote.mote_route_scored(mote.MoteRouter(Wr, 4, select_bias=sb, **opt), x)[0]
        ref = O.route_scored(_f64(x), _f64(Wr), 4, select_bias=_f64(sb), **opt)
        assert np.array_equal(idx.cpu().numpy(), ref["idx"])


# ------------------------------------------------------------------------------------------------ projections
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,N", [(1, 72), (9, 71), (40, 72), (200, 72), (300, 71), (1500, 264)])
@pytest.mark.parametrize("act", ACTS)
def test_linear_values_that_are_not_finite(mote, act, T, N, out_dtype):
    """NaN and infinities before the activation (from a bias, from a token, from a weight) come out as the formula gives them."""
    K, inf = 256, float("inf")
    x, W, b = _randn(221, T, K).bfloat16(), (_randn(222, N, K) * 0.05).bfloat16(), _randn(223, N)
    b[3], b[17], b[40] = inf, -inf, float("nan")
    got = mote.mote_linear(mote.MoteLinear(W, bias=b, act=act), x, out_dtype=out_dtype).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = O.activation(np.array([inf, -inf, np.nan]), act)
    assert np.array_equal(got[:, [3, 17, 40]], np.broadcast_to(want, (T, 3)), equal_nan=True), got[0, [3, 17, 40]]
    rest = np.delete(got, [3, 17, 40], axis=1)
    assert np.isfinite(rest).all()
    # a NaN of a token reaches its whole row and no other, one of a weight its column
    b = torch.zeros(N, device="cuda")
    x[T // 2, 7] = float("nan")
    W[5, 100] = float("nan")
    got = mote.mote_linear(mote.MoteLinear(W, bias=b, act=act), x, out_dtype=out_dtype).isnan()
    assert bool(got[T // 2].all()) and bool(got[:, 5].all()) and int(got.sum()) == N + T - 1


@pytest.mark.parametrize("T,bits", [(7, 16), (16, 8), (400, 16), (1000, 4)])
@pytest.mark.parametrize("act", ACTS)
def test_linear_activations_relative_to_their_own_size(mote, act, T, bits):
    """Every product but one is zero, so z is known exactly: the activation's error relative to its value, in the tails too.
    Special-function results are off by 2^-22, the fit of the GELU's tail by 2^-20.9; a rounding (2^-24, up to seven of them with those of z
    and the constants) of an exponent a moves e^a by its part of a: |z|, twice the tanh's argument, or z^2 / 2."""
    from math import erfc
    K = 16
    z = torch.linspace(-13.0, 13.0, T * K, dtype=torch.float64).view(T, K)
    z[0, :4] = torch.tensor([0.0, 1e-3, -1e-3, -1e-20])
    x = z.to("cuda").bfloat16()
    if bits == 16:
        lin = mote.MoteLinear(torch.eye(K, device="cuda").bfloat16(), act=act)
    else:
        lin = mote.MoteLinear.quantized(torch.eye(K, device="cuda"), bits, act=act)
    z = _f64(x) * (1.0 if bits == 16 else lin.tensors["scale"].double().cpu().numpy() * (127 if bits == 8 else 7))
    u = np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)
    if act == "gelu":
        want = z * 0.5 * np.vectorize(erfc)(-z / np.sqrt(2.0))
    elif act == "gelu_tanh":
        want = z / (1.0 + np.exp(-2.0 * u))
    else:
        want = O.activation(z, act)
    exponent = {"none": 0.0 * z, "relu": 0.0 * z, "silu": np.abs(z), "gelu": z * z / 2.0, "gelu_tanh": 2.0 * np.abs(u)}[act]
    got = _f64(mote.mote_linear(lin, x, out_dtype=torch.float32))
    seen = (np.abs(want) > 1e-35) | (want == 0.0)
    assert np.all(np.abs(got - want)[seen] <= ((2.0 ** -19 + exponent * 2.0 ** -21) * np.abs(want))[seen])
    assert np.all(np.abs(got - want)[~seen] <= 1e-35)


@pytest.mark.parametrize("T,N,K", [(1, 40, 4096), (8, 33, 11008), (16, 48, 2048), (24, 40, 4096), (64, 24, 2048), (130, 24, 2048), (40, 16, 11008)])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("sign", ["random", "one"])
def test_linear_sums_in_32_bits(mote, T, N, K, bits, sign):
    """fp32 outputs against a bound that a partial sum rounded to fewer bits breaks.  A tensor-core instruction cuts its 16 products and the
    sum so far off 25 bits below the largest, and the result to 24: 10.5 units of 2^-24 of the largest magnitude there is.  That is a
    partial sum (a difference of two prefixes) or what one step of up to 64 products comes to.  20 units for the meeting of parts."""
    x, W = _randn(251, T, K), _randn(252, N, K) * 0.05
    if sign == "one":
        x, W = x.abs(), W.abs()
    x, b = x.bfloat16(), _randn(253, N)
    lin = mote.MoteLinear(W.bfloat16(), bias=b) if bits == 16 else mote.MoteLinear.quantized(W, bits, bias=b)
    if bits == 16:
        Wd, scale = _f64(W.bfloat16()), np.ones(N)
    else:
        q, _ = O.rtn_quantize(W.cpu().numpy(), bits)
        Wd, scale = q.astype(np.float64), lin.tensors["scale"].double().cpu().numpy()
    got = _f64(mote.mote_linear(lin, x, out_dtype=torch.float32))
    p = torch.from_numpy(_f64(x)).cuda()[:, None, :] * torch.from_numpy(Wd).cuda()[None]                # [T, N, K]
    prefix = p.view(T, N, K // 16, 16).sum(dim=3).cumsum(dim=2).abs().amax(dim=2)
    step = p.abs().view(T, N, K // 64, 64).sum(dim=3).amax(dim=2)
    largest = (2.0 * prefix + step).cpu().numpy() * scale
    want = p.sum(dim=2).cpu().numpy() * scale + _f64(b)
    tol = (10.5 * K / 16 + 20.0) * 2.0 ** -24 * largest + 4.0 * 2.0 ** -24 * np.abs(want - _f64(b)) + 2.0 ** -24 * np.abs(want)
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())


# ------------------------------------------------------------------------------------------------ the layer with a scored router
SIMT, TENSOR, STREAM, AUTO = 1, 2, 3, 0


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("d,f,E,k,T,path,opt", [
    (64, 112, 5, 5, 33, SIMT, dict()),                               # k = E
    (256, 512, 4, 2, 300, SIMT, dict(renorm=False)),
    (128, 128, 2, 1, 1, TENSOR, dict(scoring="sigmoid")),
    (384, 640, 3, 3, 515, TENSOR, dict()),
    (128, 256, 64, 8, 200, TENSOR, dict(scoring="sigmoid", n_groups=8, topk_groups=4, scale=2.5, sb=True)),
    (256, 128, 16, 4, 1000, TENSOR, dict(n_groups=4, topk_groups=3, lb=True, w=torch.bfloat16)),
    (896, 4864, 4, 2, 160, TENSOR, dict(lb=True)),
    (256, 512, 4, 2, 900, TENSOR, dict(scoring="sigmoid", renorm=False)),
    (128, 192, 2, 1, 1, STREAM, dict()),
    (896, 4864, 4, 2, 2, STREAM, dict(scoring="sigmoid", sb=True)),
    (896, 4864, 4, 2, 17, STREAM, dict(lb=True, bar=1)),             # an expert without tokens
    (512, 1024, 8, 2, 13, STREAM, dict(n_groups=4, topk_groups=2, scale=0.5)),
    (128, 256, 64, 8, 37, STREAM, dict(scoring="sigmoid", n_groups=8, topk_groups=2, sb=True, w=torch.bfloat16)),
    (256, 512, 4, 2, 64, STREAM, dict(lb=True, bar=2)),
    (128, 256, 16, 2, 12800, AUTO, dict(scoring="sigmoid", n_groups=4, topk_groups=2, sb=True)),
])
def test_moe_forward_scored_over_shapes(mote, d, f, E, k, T, path, opt, bits):
    o = dict(opt)
    wl = synth.custom("scored", d, f, E, k, T, 9000 + d + f + T, w_std=0.08)
    master = synth.master_layer(wl)
    layer, layer_or = mote.MoteLayer.from_master(master, path=path), O.build_layer(master)
    if bits != 16:
        layer, layer_or = layer.quantize_shared(bits), O.quantize_shared(layer_or, bits)
    Wr = (_randn(261, E, d) * 0.1).to(o.pop("w", torch.float32))
    lb = _randn(262, E) * 0.3 if o.pop("lb", False) else None
    if "bar" in o:
        lb[o.pop("bar")] = -float("inf")
    sb = _randn(263, E) * 0.05 if o.pop("sb", False) else None
    router = mote.MoteRouter(Wr, k, logit_bias=lb, select_bias=sb, **o)
    x_bits = synth.tokens(wl)
    x, res = bf16_tensor(x_bits), _randn(264, T, d).bfloat16()
    taps = layer.alloc_taps(T)
    out = mote.mote_moe_forward_scored(layer, router, x, residual=res, taps=taps)
    assert mote.lib.mote_device_status(layer._ws.data_ptr(), None) == 0
    some = np.arange(T) if T <= 1000 else np.arange(0, T, 41)       # (the oracle's layer token by token)
    route = O.route_scored(_f64(x), _f64(Wr), k, logit_bias=_f64(lb), select_bias=_f64(sb), **o)
    assert np.array_equal(taps["topk_idx"].cpu().numpy(), route["idx"])
    part = dict(logits=route["logits"][some], idx=route["idx"][some], w=route["w"][some], near_tie=route["near_tie"][some])
    ref = O.moe_forward(layer_or, x_bits[some], residual_bf16=bf16_bits(res)[some], route=part)
    if T == len(some):
        for name in ("offsets", "perm", "qx", "beta_x", "acc_gate", "acc_up", "qh", "beta_h", "acc_down"):
            assert np.array_equal(taps[name].cpu().numpy(), ref[name]), name
    got = O.bf16_to_f32(bf16_bits(out)[some]).astype(np.float64)
    assert np.linalg.norm(got - ref["out"]) / np.linalg.norm(ref["out"]) <= REL_FRO_TOL
    # captured, for other tokens; out in the residual's place
    x2 = bf16_tensor(synth.tokens(wl, stream=1))
    want = mote.mote_moe_forward_scored(layer, router, x2, residual=res)
    graph = torch.cuda.CUDAGraph()
    place = res.clone()
    with torch.cuda.graph(graph):
        mote.mote_moe_forward_scored(layer, router, x, residual=place, out=place)
    x.copy_(x2)
    place.copy_(res)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(place, want)


def test_operators_on_tensors_that_require_grad(mote):
    d = 64
    x = _randn(271, 5, d).bfloat16().requires_grad_()
    res = _randn(272, 5, d).bfloat16().requires_grad_()
    gate = _randn(273, 5, 1).requires_grad_()
    lin, norm, router = mote.MoteLinear((_randn(274, d, d)).bfloat16()), mote.MoteBlockNorm(d), mote.MoteRouter(_randn(275, 8, d), 2)
    plain = x.detach()
    for call in (lambda: mote.mote_linear(lin, x), lambda: mote.mote_linear(lin, plain, residual=res), lambda: mote.mote_block_norm(norm, x),
                 lambda: mote.mote_block_norm(norm, plain, res), lambda: mote.mote_block_norm(norm, plain, gate=gate),
                 lambda: mote.mote_route_scored(router, x)):
        with pytest.raises(ValueError, match="requires grad"):
            call()
        with torch.no_grad():
            call()
        with torch.inference_mode():
            call()
    with torch.no_grad():
        assert torch.equal(mote.mote_linear(lin, x, residual=res), mote.mote_linear(lin, plain, residual=res.detach()))


def test_operators_on_outputs_next_to_what_they_read(mote):
    """Side by side in one buffer is no overlap."""
    d, T = 128, 6
    buf = torch.zeros(4 * d + 2 * T * d, device="cuda")
    buf[:2 * d] = 1.0 + 0.1 * _randn(281, 2 * d)
    y, res = _randn(282, T, d).bfloat16(), _randn(283, T, d)
    want = mote.mote_block_norm(mote.MoteBlockNorm(d, post_norm=True, post_gain=buf[:d].clone(), pre_gain=buf[d:2 * d].clone()), y, res)
    norm = mote.MoteBlockNorm(d, post_norm=True, post_gain=buf[:d], pre_gain=buf[d:2 * d])
    r = mote.mote_block_norm(norm, y, res, res_out=buf[2 * d:2 * d + T * d].view(T, d))
    assert torch.equal(r[0], want[0]) and torch.equal(r[1], want[1])
    with pytest.raises(mote.MoteError):
        mote.mote_block_norm(norm, y, res, res_out=buf[2 * d - 4:2 * d - 4 + T * d].view(T, d))
    W = _randn(284, d, d).bfloat16()
    want = mote.mote_linear(mote.MoteLinear(W, bias=buf[:d].clone()), y, out_dtype=torch.float32)
    lin = mote.MoteLinear(W, bias=buf[:d])
    got = mote.mote_linear(lin, y, out=buf[d:d + T * d].view(T, d))
    assert torch.equal(got, want)
    with pytest.raises(mote.MoteError):
        mote.mote_linear(lin, y, out=buf[d - 4:d - 4 + T * d].view(T, d))


@pytest.mark.parametrize("gate_tokens", [2 ** 63 - 1, 2 ** 40, 7])
@pytest.mark.parametrize("T", [1, 7, 1300])
def test_block_norm_a_gate_for_more_tokens_than_there_are(mote, T, gate_tokens):
    d = 256
    y, res = _randn(291, T, d).bfloat16(), _randn(292, T, d).bfloat16()
    rows = (T - 1) // gate_tokens + 1
    for cols in (1, d):
        gate = _randn(293, rows, cols)
        got = mote.mote_block_norm(mote.MoteBlockNorm(d, gate_tokens=gate_tokens), y, res, gate=gate)
        each = gate[torch.arange(T, device="cuda") // gate_tokens]
        want = mote.mote_block_norm(mote.MoteBlockNorm(d), y, res, gate=each)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_routers_that_are_refused(mote):
    Wr, x = _randn(301, 16, 64), _randn(302, 3, 64).bfloat16()
    with pytest.raises(ValueError, match="scoring"):
        mote.MoteRouter(Wr, 2, scoring="tanh")
    for bad in (dict(k=0), dict(k=-3), dict(k=2 ** 31 - 1), dict(k=2, n_groups=3), dict(k=2, n_groups=4, topk_groups=5), dict(k=2, scale=float("nan"))):
        with pytest.raises(mote.MoteError):
            mote.mote_route_scored(mote.MoteRouter(Wr, **bad), x)


@pytest.mark.parametrize("T", [3, 400])
def test_device_status_through_the_objects(mote, T):
    """The word that a wait that ran out raises is set by the library's own wait on nothing, with a limit of 1 ms."""
    x = _randn(311, T, 64).bfloat16()
    lin, router = mote.MoteLinear(_randn(312, 64, 64).bfloat16()), mote.MoteRouter(_randn(313, 8, 64), 2)
    lin.check_device_status()                                   # no workspace yet
    mote.mote_linear(lin, x)
    mote.mote_route_scored(router, x)
    lin.check_device_status()
    router.check_device_status()
    for obj, word in ((lin, lin._ws), (router, router.tensors["packed"])):
        assert mote.lib.mote_selftest_bounded_wait(word.data_ptr(), 1000000, None) == 0
        with pytest.raises(mote.MoteError) as e:
            obj.check_device_status()
        assert e.value.status == 7
        obj.check_device_status()
        assert mote.lib.mote_selftest_bounded_wait(word.data_ptr(), 1000000, None) == 0
    mote.mote_linear(lin, x)                                    # clears its own
    lin.check_device_status()
    mote.mote_route_scored(router, x)                           # stays until it is read
    with pytest.raises(mote.MoteError):
        router.check_device_status()


def test_flags_that_have_no_truth_value(mote):
    """Their own error comes through."""
    two = torch.tensor([1, 0])
    x = _randn(341, 3, 64).bfloat16()
    with pytest.raises(RuntimeError, match="ambiguous"):
        mote.mote_route_scored(mote.MoteRouter(_randn(342, 8, 64), 2), x, want_logits=two)
    for bad in (dict(want_residual=two), dict(want_normed=two)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            mote.mote_block_norm(mote.MoteBlockNorm(64), x, **bad)
    assert mote.mote_route_scored(mote.MoteRouter(_randn(342, 8, 64), 2), x, want_logits=0)[2] is None
