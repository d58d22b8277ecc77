"""The operators' statements in 64 bits (oracle/mote_oracle.py) on small cases that are worked out by hand."""
import numpy as np

from oracle import mote_oracle as O


def test_scored_router_statement_bars_logits_of_minus_infinity():
    x, W = np.ones((1, 1)), np.array([[1.0], [2.0], [3.0], [0.5]])
    bar = [0.0, -np.inf, -np.inf, 0.0]
    for scoring in ("softmax", "sigmoid"):
        r = O.route_scored(x, W, 3, scoring=scoring, logit_bias=bar, select_bias=[0.0, 5.0, 6.0, 0.1])
        assert r["idx"].tolist()[0][:2] in ([0, 3], [3, 0]) and r["idx"][0, 2] == 1 and r["w"][0, 2] == 0.0
        assert abs(r["w"].sum() - 1.0) < 1e-12
        none = O.route_scored(x, W, 2, scoring=scoring, logit_bias=[-np.inf] * 4, select_bias=[0.0, 1.0, 2.0, 3.0])
        assert none["idx"].tolist() == [[0, 1]] and none["w"].tolist() == [[0.0, 0.0]]
