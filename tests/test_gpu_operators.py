"""The operators around the experts (mote_route_scored, mote_block_norm, mote_linear, mote_moe_forward_scored) against their
statements in 64 bits (oracle/mote_oracle.py).

Tolerances are bounds on what fp32 arithmetic with one final rounding can be off by:
  * a rounding to a type: half a step, finfo(t).eps / 2 relative to the value (bf16 2^-8, fp32 2^-24);
  * a sum of K exact products in fp32, in any order: K 2^-24 sum |a b|; two times that where the additions truncate;
  * sqrt, division, expf and the like: a few 2^-24 relative; 2^-20 is taken for a chain of them."""
import numpy as np
import pytest
import torch

from oracle import mote_oracle as O
from workloads import synth
from parity_utils import REL_FRO_TOL, bf16_bits, bf16_tensor

pytestmark = pytest.mark.gpu

CHAIN = 2.0 ** -20
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def mote():
    import paper_2506_14435_b200 as m
    return m


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(shape, generator=_gen(seed), device="cuda")


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ scored router
def check_route(mote, x, Wr, k, lb=None, sb=None, **opt):
    router = mote.MoteRouter(Wr, k, logit_bias=lb, select_bias=sb, **opt)
    idx, w, logits = mote.mote_route_scored(router, x, want_logits=True)
    torch.cuda.synchronize()
    xd, Wd = _f64(x), _f64(Wr)
    ref = O.route_scored(xd, Wd, k, logit_bias=_f64(lb), select_bias=_f64(sb), **opt)
    assert np.array_equal(idx.cpu().numpy(), ref["idx"])
    # a logit: d products; a weight: its logit's error through the score (relative slope at most 1, twice with a denominator)
    d = x.shape[1]
    err = d * 2.0 ** -23 * (np.abs(xd) @ np.abs(Wd).T) + 2.0 ** -23 * np.abs(ref["logits"])
    fine = np.isfinite(ref["logits"])
    assert np.all(np.abs(_f64(logits)[fine] - ref["logits"][fine]) <= (err + 1e-30)[fine])
    tol = 2.0 * np.where(fine, err, 0.0).max(axis=1, keepdims=True) + CHAIN
    assert np.all(np.abs(_f64(w) - ref["w"]) <= tol * np.abs(ref["w"]) + 1e-37)
    # without the logits the same choice
    idx2, w2, none = mote.mote_route_scored(router, x)
    assert none is None and torch.equal(idx2, idx) and torch.equal(w2, w)
    return idx, w, ref


ROUTES = [
    dict(E=4, k=2), dict(E=16, k=2, renorm=False), dict(E=64, k=8, scoring="sigmoid", scale=2.5),
    dict(E=64, k=6, scoring="sigmoid", n_groups=8, topk_groups=4, sb=True), dict(E=60, k=4, lb=True, renorm=False, outliers=True),
    dict(E=33, k=8, scoring="softmax", sb=True), dict(E=48, k=5, n_groups=6, topk_groups=2, scoring="softmax"),
    dict(E=64, k=3, n_groups=64, topk_groups=5, scoring="sigmoid"), dict(E=2, k=1), dict(E=1, k=1), dict(E=8, k=8, scoring="sigmoid"),
    dict(E=63, k=7, n_groups=21, topk_groups=3, sb=True, lb=True),
]


@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d", [(1, 2048), (2, 8), (16, 896), (17, 72), (130, 1544), (777, 256)])
@pytest.mark.parametrize("opt", ROUTES, ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_route_scored(mote, T, d, opt, w_dtype):
    o = dict(opt)
    E, k, seed = o.pop("E"), o.pop("k"), T * 131 + d
    x = _randn(seed, T, d)
    if o.pop("outliers", False):
        x[:, ::97] *= 20.0
    Wr = (_randn(seed + 1, E, d) * 0.02).to(w_dtype)
    lb = _randn(seed + 2, E) * 0.5 if o.pop("lb", False) else None
    sb = _randn(seed + 3, E) * 0.02 if o.pop("sb", False) else None
    check_route(mote, x.bfloat16(), Wr, k, lb, sb, **o)


@pytest.mark.parametrize("T", [40, 1200])
@pytest.mark.parametrize("scoring,n_groups,bias", [("softmax", 1, False), ("sigmoid", 1, True), ("sigmoid", 8, True), ("softmax", 8, True)])
def test_route_scored_close_scores_are_told_apart_in_64_bits(mote, T, scoring, n_groups, bias):
    """Pairs of router rows that differ in their last bits only: fp32 sums cannot tell their logits apart, the choice must be
    that of exact arithmetic all the same."""
    E, k, d = 32, 4, 1024
    x = _randn(5, T, d).bfloat16()
    Wr = _randn(6, E // 2, d) * 0.02
    Wr = Wr.repeat_interleave(2, dim=0).contiguous()
    bump = torch.zeros_like(Wr)
    bump[1::2] = (torch.rand(E // 2, d, generator=_gen(7), device="cuda") - 0.5) * 2.0 ** -26
    Wr = Wr + bump
    assert not torch.equal(Wr[0], Wr[1])
    sb = (_randn(8, E // 2) * 0.02).repeat_interleave(2).contiguous() if bias else None
    check_route(mote, x, Wr.contiguous(), k, None, sb, scoring=scoring, n_groups=n_groups, topk_groups=4 if n_groups > 1 else 1)


@pytest.mark.parametrize("T", [3, 600])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_scored_equal_scores_go_to_the_lower_index(mote, T, scoring):
    x = _randn(9, T, 512).bfloat16()
    Wr = (_randn(10, 1, 512) * 0.02).repeat(24, 1).contiguous()
    idx, w, _ = check_route(mote, x, Wr, 5, scoring=scoring, n_groups=1)
    assert torch.equal(idx.cpu(), torch.arange(5, dtype=torch.int32).repeat(T, 1))
    idx, w, _ = check_route(mote, x, Wr, 5, scoring=scoring, n_groups=6, topk_groups=2)
    assert torch.equal(idx.cpu(), torch.arange(5, dtype=torch.int32).repeat(T, 1))
    assert torch.equal(mote.mote_route_scored(mote.MoteRouter(Wr, 5, scoring=scoring), torch.zeros_like(x))[0], idx)


@pytest.mark.parametrize("T", [5, 700])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_scored_barred_experts(mote, T, scoring):
    """-inf in a bias bars an expert, which is then taken only where nothing else is left, the lower index first."""
    E, d = 16, 256
    x = _randn(11, T, d).bfloat16()
    Wr = _randn(12, E, d) * 0.02
    bar = torch.zeros(E, device="cuda")
    bar[2:13] = -float("inf")
    for n_groups, topk_groups in ((1, 1), (4, 2)):
        idx, w, _ = check_route(mote, x, Wr, 4, None, bar, scoring=scoring, n_groups=n_groups, topk_groups=topk_groups)
    idx, w, _ = check_route(mote, x, Wr, 4, bar, None, scoring=scoring)
    assert set(idx.flatten().tolist()) <= {0, 1, 13, 14, 15}
    idx, _, _ = check_route(mote, x, Wr, 8, None, bar, scoring=scoring)            # five are open, three of the others follow
    assert torch.equal(idx[:, 5:].cpu(), torch.tensor([2, 3, 4], dtype=torch.int32).repeat(T, 1))


@pytest.mark.parametrize("T", [4, 500])
def test_route_scored_takes_any_values_without_leaving_the_experts(mote, T):
    """NaN and infinities give undefined weights, but k different experts all the same."""
    x = _randn(13, T, 128).bfloat16()
    x[0] = float("nan")
    x[1, 5] = float("inf")
    x[2] = 3e38
    for scoring in ("softmax", "sigmoid"):
        for n_groups in (1, 4):
            r = mote.MoteRouter(_randn(14, 16, 128), 4, scoring=scoring, n_groups=n_groups, topk_groups=min(2, n_groups))
            idx, _, _ = mote.mote_route_scored(r, x)
            s = idx.sort(dim=1).values
            assert int(s.min()) >= 0 and int(s.max()) < 16 and bool((s[:, 1:] > s[:, :-1]).all())


@pytest.mark.parametrize("T", [3, 40, 2100])
@pytest.mark.parametrize("scoring,n_groups,lb,sb", [("softmax", 1, False, False), ("sigmoid", 8, False, True), ("sigmoid", 8, True, False), ("softmax", 4, True, True)])
def test_route_scored_padded_batches_and_tiny_tokens(mote, T, scoring, n_groups, lb, sb):
    """Tokens of zeros have the biases for logits; tokens whose squares underflow are still told apart exactly."""
    E, d = 64, 512
    x = _randn(81, T, d)
    x[1::3] = 0.0
    x[2::3] *= 1e-30
    bias = lambda seed: (_randn(seed, E // 2) * 0.01).repeat_interleave(2).contiguous()
    check_route(mote, x.bfloat16(), _randn(82, E, d) * 0.02, 6, bias(83) if lb else None, bias(84) if sb else None, scoring=scoring,
                n_groups=n_groups, topk_groups=max(1, n_groups // 2))


@pytest.mark.parametrize("T", [3, 500])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,n_groups,topk_groups,k", [(16, 4, 2, 4), (40, 40, 9, 7), (50, 50, 8, 8), (64, 2, 1, 8), (36, 12, 11, 8)])
def test_route_scored_groups_with_barred_logits(mote, T, scoring, E, n_groups, topk_groups, k):
    """A logit_bias of -inf gives a score of zero: whole groups of them tie at zero, and are chosen only where no others are left."""
    x = _randn(94, T, 128).bfloat16()
    lb = torch.zeros(E, device="cuda")
    lb[2:E - 5] = -float("inf")
    check_route(mote, x, _randn(95, E, 128) * 0.1, k, lb, None, scoring=scoring, n_groups=n_groups, topk_groups=topk_groups)
    check_route(mote, x, _randn(95, E, 128) * 0.1, k, lb, _randn(96, E) * 0.05, scoring=scoring, n_groups=n_groups, topk_groups=topk_groups)


@pytest.mark.parametrize("T", [5, 40, 1200])
@pytest.mark.parametrize("E,n_groups,topk_groups", [(32, 8, 3), (32, 4, 4), (40, 20, 7), (24, 2, 1)])
def test_route_scored_softmax_groups_of_close_and_of_vanishing_scores(mote, T, E, n_groups, topk_groups):
    """Without a bias only ratios of a softmax's scores count: pairs of experts, and with them pairs of groups, that differ in their last
    bits; and logits so far apart that most scores vanish in fp32."""
    d = 512
    x = _randn(85, T, d)
    x[1::2] *= 40.0
    Wr = (_randn(86, E // 2, d) * 0.1).repeat(2, 1).contiguous()          # an expert's twin is in another group
    Wr[E // 2:] += (torch.rand(E // 2, d, generator=_gen(87), device="cuda") - 0.5) * 2.0 ** -24
    check_route(mote, x.bfloat16(), Wr, 4, scoring="softmax", n_groups=n_groups, topk_groups=topk_groups)


@pytest.mark.parametrize("T", [3, 300, 1200])
@pytest.mark.parametrize("n_groups,topk_groups", [(1, 1), (8, 3), (2, 1)])
def test_route_scored_biased_softmax_scores_that_hang_on_the_denominator(mote, T, n_groups, topk_groups):
    """A bias that takes the scores of one token away but for its own rounding: every difference is far below what fp32 can tell."""
    E, d = 32, 512
    x = _randn(88, 1, d).bfloat16().repeat(T, 1).contiguous()
    Wr = _randn(89, E, d) * 0.05
    sb = (-torch.softmax(x[:1].double() @ Wr.double().T, dim=1)[0]).float()
    check_route(mote, x, Wr, 6, None, sb, scoring="softmax", n_groups=n_groups, topk_groups=topk_groups)


# The same where there is work enough for the tcgen05 kernel, on whole and partial tiles.
@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d", [(905, 1400), (2003, 5000), (1024, 4096)])
@pytest.mark.parametrize("opt", ROUTES, ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
def test_route_scored_long(mote, T, d, opt, w_dtype):
    test_route_scored(mote, T, d, opt, w_dtype)


@pytest.mark.parametrize("scoring,n_groups,bias", [("softmax", 1, False), ("sigmoid", 1, True), ("sigmoid", 8, True), ("softmax", 8, True), ("softmax", 8, False)])
def test_route_scored_long_close_scores(mote, scoring, n_groups, bias):
    test_route_scored_close_scores_are_told_apart_in_64_bits(mote, 2500, scoring, n_groups, bias)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_scored_long_equal_scores(mote, scoring):
    test_route_scored_equal_scores_go_to_the_lower_index(mote, 6600, scoring)


def test_route_scored_long_any_values(mote):
    test_route_scored_takes_any_values_without_leaving_the_experts(mote, 39100)


@pytest.mark.parametrize("scoring,n_groups,lb,sb", [("softmax", 1, False, False), ("sigmoid", 8, False, True), ("sigmoid", 8, True, False), ("softmax", 4, True, True)])
def test_route_scored_long_padded_batches(mote, scoring, n_groups, lb, sb):
    test_route_scored_padded_batches_and_tiny_tokens(mote, 2600, scoring, n_groups, lb, sb)


@pytest.mark.parametrize("E,n_groups,topk_groups", [(32, 8, 3), (32, 4, 4), (40, 20, 7)])
def test_route_scored_long_softmax_groups(mote, E, n_groups, topk_groups):
    test_route_scored_softmax_groups_of_close_and_of_vanishing_scores(mote, 4900, E, n_groups, topk_groups)


@pytest.mark.parametrize("n_groups,topk_groups", [(1, 1), (8, 3), (2, 1)])
def test_route_scored_long_biased_softmax(mote, n_groups, topk_groups):
    test_route_scored_biased_softmax_scores_that_hang_on_the_denominator(mote, 4900, n_groups, topk_groups)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_route_scored_long_barred(mote, scoring):
    test_route_scored_groups_with_barred_logits(mote, 9800, scoring, 64, 2, 1, 8)
    test_route_scored_barred_experts(mote, 19600, scoring)


def test_route_scored_strided_rows_and_empty_batches(mote):
    wide = _randn(15, 50, 640).bfloat16()
    Wr = _randn(16, 24, 320) * 0.02
    check_route(mote, wide[:, 320:], Wr, 3)
    check_route(mote, wide[::2, :320], Wr, 3, scoring="sigmoid")
    idx, w, logits = mote.mote_route_scored(mote.MoteRouter(Wr, 3), wide[:0, :320], want_logits=True)
    assert idx.shape == (0, 3) and w.shape == (0, 3) and logits.shape == (0, 24)


def test_route_scored_does_not_depend_on_the_batch(mote):
    """The same tokens alone, in a short and in a long batch: the same experts."""
    x = _randn(17, 3000, 768).bfloat16()
    r = mote.MoteRouter(_randn(18, 64, 768) * 0.02, 8, scoring="sigmoid", n_groups=8, topk_groups=4)
    whole = mote.mote_route_scored(r, x)[0]
    for a, b in ((0, 1), (5, 37), (100, 900)):
        assert torch.equal(mote.mote_route_scored(r, x[a:b])[0], whole[a:b])


# ------------------------------------------------------------------------------------------------ norms around a block
def check_norm(mote, y, residual, eps=1e-6, pre_gain=None, gate=None, **opt):
    norm = mote.MoteBlockNorm(y.shape[1], eps=eps, pre_gain=pre_gain, **opt)
    res, n = mote.mote_block_norm(norm, y, residual, gate=gate)
    torch.cuda.synchronize()
    o = {k: v if not isinstance(v, torch.Tensor) else _f64(v) for k, v in opt.items()}
    yd, rd = _f64(y), _f64(residual)
    want = O.block_norm(yd, rd, eps=eps, gate=_f64(gate), **o)
    added = np.abs(want - (0.0 if rd is None else rd))
    # p is a chain of fp32 operations on an exact value (its sum of squares has terms of one sign)
    tol = HALF_STEP[res.dtype] * np.abs(want) + (CHAIN + y.shape[1] * 2.0 ** -24) * added + 2.0 ** -23 * np.abs(want) + 1e-37
    assert np.all(np.abs(_f64(res) - want) <= tol)
    want_n = O.gained_rms_norm(_f64(res), _f64(pre_gain), eps)
    assert np.all(np.abs(_f64(n) - want_n) <= (2.0 ** -8 + CHAIN + y.shape[1] * 2.0 ** -24) * np.abs(want_n) + 1e-37)
    return norm, res, n


@pytest.mark.parametrize("res_dtype", [torch.bfloat16, torch.float32, None])
@pytest.mark.parametrize("T,d", [(1, 2048), (1, 8), (3, 32768), (5, 264), (257, 896), (300, 8200), (1100, 136), (1300, 2048), (1030, 20000)])
def test_block_norm(mote, T, d, res_dtype):
    y = (_randn(T + d, T, d) * 0.7).bfloat16()
    residual = None if res_dtype is None else (_randn(T + d + 1, T, d) * 4.0).to(res_dtype)
    post, pre = 1.0 + 0.1 * _randn(1, d), 1.0 + 0.1 * _randn(2, d)
    check_norm(mote, y, residual)
    check_norm(mote, y, residual, pre_gain=pre, post_norm=True, scale=0.25, eps=1e-5)
    check_norm(mote, y, residual, pre_gain=pre, post_norm=True, post_gain=post, gate=_randn(3, T, 1).bfloat16(), gate_sigmoid=True)
    check_norm(mote, y, residual, gate=_randn(4, 1, d), gate_tokens=0)
    check_norm(mote, y, residual, pre_gain=pre, gate=_randn(5, T, d).bfloat16(), gate_sigmoid=True, scale=-2.0)
    rows = -(-T // 7)
    check_norm(mote, y, residual, gate=_randn(6, rows, d).bfloat16(), gate_tokens=7, post_norm=True)
    check_norm(mote, y, residual, gate=_randn(7, rows, 1), gate_tokens=7)


def test_block_norm_zero_and_large_rows(mote):
    y = _randn(20, 40, 512).bfloat16()
    y[3] = 0
    y[7] *= 1e15
    y[8] *= 1e-20
    res = _randn(21, 40, 512).bfloat16()
    res[3] = 0
    _, r, n = check_norm(mote, y, res, post_norm=True)
    assert float(r[3].abs().max()) == 0.0 and float(n[3].abs().max()) == 0.0
    check_norm(mote, y, res)


def test_block_norm_matches_the_plain_norm_on_its_own_output(mote):
    y, res = _randn(22, 33, 1536).bfloat16(), _randn(23, 33, 1536).bfloat16()
    r, n = mote.mote_block_norm(mote.MoteBlockNorm(1536), y, res)
    want = mote.mote_rms_norm(r)
    # the same arithmetic but for the order of the sum of squares
    assert float((n.float() - want.float()).abs().max()) <= 2.0 ** -7 * float(want.float().abs().max())


def test_block_norm_in_place_strided_and_partial_outputs(mote):
    d = 640
    wide = _randn(24, 70, 2 * d).bfloat16()
    y, res = wide[:, :d], wide[::1, d:]
    norm, r, n = check_norm(mote, y, res, post_norm=True)
    check_norm(mote, wide[::3, d:], _randn(25, 24, 2 * d)[:, :d])
    # outputs in the place of their inputs
    yc, rc = y.contiguous(), res.contiguous()
    r2, n2 = mote.mote_block_norm(norm, yc, rc, res_out=rc, normed_out=yc)
    assert r2.data_ptr() == rc.data_ptr() and torch.equal(r2, r) and torch.equal(n2, n)
    # one output only
    only_r = mote.mote_block_norm(norm, y, res, want_normed=False)
    only_n = mote.mote_block_norm(norm, y, res, want_residual=False)
    assert only_r[1] is None and torch.equal(only_r[0], r) and only_n[0] is None and torch.equal(only_n[1], n)
    # rows do not depend on the batch
    one = mote.mote_block_norm(norm, y[5:6], res[5:6])
    assert torch.equal(one[0], mote.mote_block_norm(norm, y[5:7], res[5:7])[0][:1])
    empty = mote.mote_block_norm(norm, y[:0], res[:0])
    assert empty[0].shape == (0, d) and empty[1].shape == (0, d)


@pytest.mark.parametrize("d", [64, 896, 2048, 4096, 8192, 8200])
def test_block_norm_rows_do_not_depend_on_the_batch(mote, d):
    y, res, gate = _randn(26, 2500, d).bfloat16(), _randn(27, 2500, d).bfloat16(), _randn(28, 2500, d).bfloat16()
    norm = mote.MoteBlockNorm(d, post_norm=True, post_gain=1.0 + 0.1 * _randn(29, d), gate_sigmoid=True)
    whole = mote.mote_block_norm(norm, y, res, gate=gate)
    for a, b in ((0, 1), (3, 300), (1100, 2500)):
        part = mote.mote_block_norm(norm, y[a:b], res[a:b], gate=gate[a:b])
        assert torch.equal(part[0], whole[0][a:b]) and torch.equal(part[1], whole[1][a:b])
    # in the place of its inputs, with rows on the way
    r, n = mote.mote_block_norm(norm, y, res, gate=gate, res_out=res, normed_out=y)
    assert torch.equal(r, whole[0]) and torch.equal(n, whole[1])


# ------------------------------------------------------------------------------------------------ projections
def make_linear(mote, N, K, bits, bias, act, seed):
    W = (_randn(seed, N, K) * 0.05).bfloat16()
    b = _randn(seed + 1, N) * 0.5 if bias else None
    if bits == 16:
        return mote.MoteLinear(W, bias=b, act=act), _f64(W), b
    q, scale = O.rtn_quantize(W.float().cpu().numpy(), bits)
    lin = mote.MoteLinear.quantized(W, bits, bias=b, act=act)
    return lin, O.rtn_dequant(q, scale).astype(np.float64), b


def check_linear(mote, lin, Wd, b, x, act, residual=None, out_dtype=torch.bfloat16, out=None):
    got = mote.mote_linear(lin, x, residual=residual, out_dtype=out_dtype, out=out)
    torch.cuda.synchronize()
    assert mote.lib.mote_device_status(lin._ws.data_ptr(), None) == 0
    xd, rd = _f64(x), _f64(residual)
    z = xd @ Wd.T + (0.0 if b is None else _f64(b))
    want = O.linear(xd, Wd, bias=_f64(b), act=act, residual=rd)
    mag = np.abs(xd) @ np.abs(Wd).T
    # the sum, then a chain of operations; every activation's slope is below 1.2
    tol = 1.2 * (x.shape[1] * 2.0 ** -23 * mag + CHAIN * np.abs(z)) + CHAIN * np.abs(want) + HALF_STEP[got.dtype] * np.abs(want) + 1e-30
    # an activation's value next to its zero: 1 + erf and 1 + tanh lose 2^-24 of the argument there
    tol += 2.0 ** -22 * np.abs(z)
    if rd is not None:
        tol += 2.0 ** -23 * np.abs(rd)
    bad = np.abs(_f64(got) - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float((np.abs(_f64(got) - want) / tol).max()))
    return got


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("T", [1, 7, 8, 9, 16, 17, 33, 64, 130, 333])
@pytest.mark.parametrize("N,K", [(256, 512), (1, 16), (37, 48), (1001, 1552), (2560, 2048), (513, 128)])
def test_linear(mote, T, N, K, bits):
    act = ["none", "relu", "silu", "gelu", "gelu_tanh"][(T + N) % 5]
    lin, Wd, b = make_linear(mote, N, K, bits, (T + K) % 2 == 0, act, T + N + K)
    x = _randn(T + 3 * N + K, T, K).bfloat16()
    residual = (_randn(N, T, N) * 2.0).bfloat16()
    check_linear(mote, lin, Wd, b, x, act, residual)
    check_linear(mote, lin, Wd, b, x, act, None, torch.float32)


@pytest.mark.parametrize("T,N,K,bits", [
    (17, 3300, 2048, 16), (32, 4104, 2048, 16), (33, 2127, 2048, 16), (48, 2200, 2048, 16), (49, 129, 64, 16), (64, 40, 72, 16), (16, 5001, 2048, 16),
    (31, 9001, 1040, 8), (32, 5000, 4096, 4), (33, 7000, 2048, 8), (47, 7000, 2048, 4), (48, 1100, 2048, 8), (49, 6000, 2048, 8), (64, 6000, 2048, 4),
    (64, 515, 80, 8), (65, 130, 48, 8), (65, 515, 80, 4), (80, 40, 16, 8)])
def test_linear_where_the_forms_meet(mote, T, N, K, bits):
    """Numbers of tokens and sizes on either side of where the weight stream hands over to the tensor-core product; the rows behind the
    last token stay."""
    lin, Wd, b = make_linear(mote, N, K, bits, True, "silu", T + N)
    x, residual = _randn(T + K, T, K).bfloat16(), _randn(N, T, N).bfloat16()
    out = torch.full((T + 2, N), 5.0, device="cuda")
    check_linear(mote, lin, Wd, b, x, "silu", residual, torch.float32, out=out[:T])
    assert bool((out[T:] == 5.0).all())
    check_linear(mote, lin, Wd, b, x, "silu")


@pytest.mark.parametrize("T", [5, 200, 1500])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
def test_linear_activations_over_their_range(mote, T, act):
    lin, Wd, b = make_linear(mote, 192, 256, 16, True, act, 31)
    x = (_randn(32, T, 256) * torch.logspace(-3, 2, T, device="cuda")[:, None]).bfloat16()
    check_linear(mote, lin, Wd, b, x, act, None, torch.float32)
    check_linear(mote, lin, Wd, b, x, act)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("T", [6, 40, 300])
def test_linear_strided_rows_in_place_and_empty(mote, T, bits):
    N, K = 328, 320
    lin, Wd, b = make_linear(mote, N, K, bits, True, "silu", 41)
    wide = _randn(42, T, 3 * K).bfloat16()
    x = wide[:, K:2 * K]
    res_wide = _randn(43, T, 2 * N + 3).bfloat16()
    got = check_linear(mote, lin, Wd, b, x, "silu", res_wide[:, :N])
    buf = res_wide[:, :N].contiguous()
    assert mote.mote_linear(lin, x, residual=buf, out=buf) is buf and torch.equal(buf, got)
    assert mote.mote_linear(lin, x[:0]).shape == (0, N)
    # rows behind the last token stay as they were
    out = torch.full((T + 3, N), 7.0, dtype=torch.bfloat16, device="cuda")
    mote.mote_linear(lin, x, residual=res_wide[:, :N], out=out[:T])
    assert torch.equal(out[:T], got) and bool((out[T:] == 7.0).all())


# ------------------------------------------------------------------------------------------------ streams, graphs
def test_operators_on_a_side_stream_and_in_graphs(mote):
    d, E, T = 512, 16, 24
    router = mote.MoteRouter(_randn(51, E, d) * 0.02, 2, scoring="sigmoid")
    norm = mote.MoteBlockNorm(d, post_norm=True)
    lin, _, _ = make_linear(mote, 384, d, 16, True, "gelu", 52)
    big, _, _ = make_linear(mote, 384, d, 8, True, "gelu", 53)
    x, res = _randn(54, T, d).bfloat16(), _randn(55, T, d).bfloat16()
    xl = _randn(56, 700, d).bfloat16()

    def step():
        r, n = mote.mote_block_norm(norm, x, res)
        return [r, n, *mote.mote_route_scored(router, n)[:2], mote.mote_linear(lin, n), mote.mote_linear(lin, xl), mote.mote_linear(big, xl),
                *mote.mote_route_scored(router, xl)[:2]]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    x2, res2, xl2 = _randn(57, T, d).bfloat16(), _randn(58, T, d).bfloat16(), _randn(59, 700, d).bfloat16()
    for a, b, c in ((x2, res2, xl2), (x.clone(), res.clone(), xl.clone())):
        x.copy_(a); res.copy_(b); xl.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        now = step()
        assert all(torch.equal(p, q) for p, q in zip(got, now))


# ------------------------------------------------------------------------------------------------ the layer with a scored router
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("T,N,K", [(333, 1001, 512), (300, 515, 4096), (70, 37, 8192), (1500, 2051, 256), (4100, 130, 64), (129, 7, 1024)])
def test_linear_residual_on_any_boundary(mote, T, N, K, bits):
    lin, Wd, b = make_linear(mote, N, K, bits, True, "gelu_tanh", 101)
    x, wide = _randn(102, T, K).bfloat16(), (_randn(103, T, N + 3) * 2.0).bfloat16()
    rows = wide[:, :N]
    check_linear(mote, lin, Wd, b, x, "gelu_tanh", rows, torch.float32)
    want = check_linear(mote, lin, Wd, b, x, "gelu_tanh", rows)
    place = rows.contiguous()
    got = mote.mote_linear(lin, x, residual=place, out=place)
    assert got is place and torch.equal(got, want)


@pytest.mark.parametrize("bits", [8, 4])
def test_a_captured_projection_keeps_its_workspace_when_longer_batches_come(mote, bits):
    lin, Wd, b = make_linear(mote, 512, 256, bits, True, "silu", 91)
    x = _randn(92, 8, 256).bfloat16()
    want = check_linear(mote, lin, Wd, b, x, "silu")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mote.mote_linear(lin, x)
    check_linear(mote, lin, Wd, b, _randn(93, 200, 256).bfloat16(), "silu")      # needs a larger one
    others = [torch.ones(64, device="cuda") for _ in range(64)]                  # would take the place of the smaller one
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((t == 1.0).all()) for t in others)


@pytest.mark.parametrize("path", ["auto", "simt", "tensor", "stream"])
@pytest.mark.parametrize("T", [1, 24, 40, 700])
def test_moe_forward_scored_against_the_oracle(mote, T, path):
    if path == "stream" and T > 64:
        pytest.skip("the weight stream takes up to 64 tokens")
    wl = synth.custom("scored", 128, 256, 8, 2, T, 4300, w_std=0.08)
    master = synth.master_layer(wl)
    layer = mote.MoteLayer.from_master(master, path=getattr(mote, "PATH_" + path.upper()))
    opt = dict(scoring="sigmoid", n_groups=4, topk_groups=2, scale=2.5)
    Wr, sb = _randn(61, 8, 128) * 0.1, _randn(62, 8) * 0.05
    router = mote.MoteRouter(Wr, 2, select_bias=sb, **opt)
    x_bits = synth.tokens(wl)
    x, res = bf16_tensor(x_bits), _randn(63, T, 128).bfloat16()
    taps = layer.alloc_taps(T)
    out = mote.mote_moe_forward_scored(layer, router, x, residual=res, taps=taps)
    torch.cuda.synchronize()
    assert mote.lib.mote_device_status(layer._ws.data_ptr(), None) == 0
    route = O.route_scored(_f64(x), _f64(Wr), 2, select_bias=_f64(sb), **opt)
    ref = O.moe_forward(O.build_layer(master), x_bits, residual_bf16=bf16_bits(res), route=route)
    assert np.array_equal(taps["topk_idx"].cpu().numpy(), ref["topk_idx"])
    for name in ("offsets", "perm", "qx", "beta_x", "acc_gate", "acc_up", "qh", "beta_h", "acc_down"):
        assert np.array_equal(taps[name].cpu().numpy(), ref[name]), name
    got = O.bf16_to_f32(bf16_bits(out)).astype(np.float64)
    assert np.linalg.norm(got - ref["out"]) / np.linalg.norm(ref["out"]) <= REL_FRO_TOL
    idx, w, _ = mote.mote_route_scored(router, x)
    assert torch.equal(idx, taps["topk_idx"]) and torch.equal(w, taps["topk_w"])


def test_moe_forward_scored_refuses_other_shapes_and_takes_empty_batches(mote):
    wl = synth.custom("scored", 128, 256, 8, 2, 4, 4301, w_std=0.08)
    layer = mote.MoteLayer.from_master(synth.master_layer(wl))
    router = mote.MoteRouter(_randn(97, 8, 128) * 0.05, 2)
    x = _randn(98, 4, 128).bfloat16()
    for bad in (dict(x=x.float()), dict(x=x[:, :64].contiguous()), dict(x=x, residual=x[:3]), dict(x=x, out=torch.empty(4, 128, device="cuda")),
                dict(x=x.cpu()), dict(x=x[0])):
        with pytest.raises(ValueError):
            mote.mote_moe_forward_scored(layer, router, **bad)
    with pytest.raises(mote.MoteError):
        mote.mote_moe_forward_scored(layer, mote.MoteRouter(_randn(97, 4, 128) * 0.05, 2), x)
    assert mote.mote_moe_forward_scored(layer, router, x).shape == (4, 128)


def test_a_block_as_it_is_used(mote):
    """Projection onto the residual stream, norm, scored router and experts, norm after the block with its gate, next projection;
    decode steps follow a prompt on the same objects."""
    d, T = 128, 300
    wl = synth.custom("block", d, 256, 8, 2, T, 4400, w_std=0.08)
    master = synth.master_layer(wl)
    layer = mote.MoteLayer.from_master(master)
    Wr, sb = _randn(71, 8, d) * 0.1, _randn(72, 8) * 0.05
    router = mote.MoteRouter(Wr, 2, scoring="sigmoid", select_bias=sb, n_groups=4, topk_groups=2)
    proj, Wp, _ = make_linear(mote, d, 192, 16, False, "none", 73)
    qkv, Wq, bq = make_linear(mote, 2 * d + 8, d, 16, True, "none", 74)
    pre = mote.MoteBlockNorm(d, pre_gain=1.0 + 0.1 * _randn(75, d))
    post = mote.MoteBlockNorm(d, post_norm=True, post_gain=1.0 + 0.1 * _randn(76, d), gate_sigmoid=True)
    one = mote.MoteBlockNorm(d)
    for tokens in (T, 1, 9):
        a, stream = _randn(77, tokens, 192).bfloat16(), (_randn(78, tokens, d) * 4).bfloat16()
        gate = _randn(79, tokens, 1).bfloat16()
        h = mote.mote_linear(proj, a, residual=stream)
        zero = torch.zeros_like(h)
        _, n = mote.mote_block_norm(pre, zero, h)
        y = mote.mote_moe_forward_scored(layer, router, n)
        r, n2 = mote.mote_block_norm(post, y, h, gate=gate)
        q = mote.mote_linear(qkv, n2)
        torch.cuda.synchronize()
        # each step from the step before it, as the device left it
        check_linear(mote, proj, Wp, None, a, "none", stream)
        assert torch.equal(h, mote.mote_linear(proj, a, residual=stream))
        route = O.route_scored(_f64(n), _f64(Wr), 2, scoring="sigmoid", select_bias=_f64(sb), n_groups=4, topk_groups=2)
        ref = O.moe_forward(O.build_layer(master), bf16_bits(n), route=route)
        got = O.bf16_to_f32(bf16_bits(y)).astype(np.float64)
        assert np.linalg.norm(got - ref["out"]) / np.linalg.norm(ref["out"]) <= REL_FRO_TOL
        want_r = O.block_norm(_f64(y), _f64(h), eps=1e-6, post_norm=True, post_gain=_f64(post.tensors["post_gain"]), gate=_f64(gate),
                              gate_sigmoid=True)
        assert np.all(np.abs(_f64(r) - want_r) <= 2.0 ** -8 * np.abs(want_r) + CHAIN * (np.abs(want_r) + np.abs(_f64(h))))
        want_n = O.gained_rms_norm(_f64(r), None, 1e-6)
        assert np.all(np.abs(_f64(n2) - want_n) <= (2.0 ** -8 + 2 * CHAIN) * np.abs(want_n))
        assert torch.equal(q, check_linear(mote, qkv, Wq, bq, n2, "none"))
    assert one.device is None
