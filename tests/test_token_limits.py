"""What the token losses' oracles and the binding do at the ends of their ranges.  Nothing is launched: no GPU needed."""
import math

import numpy as np
import pytest

import paper_2312_14227_b200 as et
from oracle import token_oracle as tok

INF = float("inf")


def _logits(rows, width=4):
    return np.zeros((rows, width))                       # log probability -log 4 of every token


def test_oracle_rejected_token_of_probability_zero():
    """x = inf: the sigmoid loss of the pair and its gradient are 0; with label smoothing the loss is infinite."""
    y = _logits(4)
    y[1, 2] = -INF                                       # the rejected answer of pair 0
    t = np.array([0, 2, 1, 1])
    stats, S, dY, coef = tok.preference(y, t, None, [0, 1, 2, 3, 4], None, 4, 1.0, 0, 0.5, 0.0)
    assert S[1] == -INF and math.isclose(stats[0], 0.5 * math.log(2), rel_tol=1e-15)      # pair 1: x = 0
    assert coef[0] == 0 and coef[1] == 0 and not dY[:2].any() and coef[2] == -0.125 and coef[3] == 0.125
    assert tok.preference(y, t, None, [0, 1, 2, 3, 4], None, 4, 1.0, 0, 0.5, 0.1)[0][0] == INF


@pytest.mark.parametrize("gap", [1e4, INF])
def test_oracle_divergence_that_is_reported_only(gap):
    """kl_coef = 0: a reference far above the policy, or a taken token of probability 0, leaves loss and gradient alone."""
    y = _logits(2)
    y[0, 1] = -gap
    t, w, adv = np.array([1, 2]), np.full(2, 0.5), np.array([1.0, 2.0])
    old, ref = np.full(2, -math.log(4)), np.full(2, -1.0)
    stats, lp, dY, coef = tok.policy(y, t, w, adv, old, ref, 4, 1.0, 0.2, 0.2, 0.0)
    assert coef[0] == 0 and not dY[0].any() and coef[1] == -1.0                  # r = 0, r = 1
    assert math.isclose(stats[0], -1.0, rel_tol=1e-15) and stats[1] == stats[0] and stats[2] == INF
