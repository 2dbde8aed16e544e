"""What the bound of tests/needles.py finds, on the CPU: mistakes planted in a plain form."""
import math

import pytest
import torch

from tests import needles as N
from tests import rows_ref as R

D = 128
L, K_ACT = 700, 64


def _case():
    K = N.rows(torch, 1, L, K_ACT, 1)[0]
    K = torch.where(K.abs() == 1, K, torch.zeros(())).double()
    V = torch.randn(L, D, generator=torch.Generator().manual_seed(2)).half().double()
    return K, V, K * N.sharpness(K_ACT)


def test_the_formula_is_well_within_it():
    K, V, q = _case()
    assert N.gap(torch, K) > 50
    o, _ = R.softmax_rows(q, K, V)
    assert N.misses(torch, o.float(), V, 0.0) < 0.2
    assert N.misses(torch, o.half(), V, R.HALF["f16"]) <= 1


@pytest.mark.parametrize("mistake", ["dropped key", "dropped value", "another's value", "twice",
                                     "16-bit weights"])
def test_a_mistake_at_any_token_is_found(mistake):
    """For each of 700 tokens (for weights of 16 bits: in one of the rows)."""
    K, V, q = _case()
    s = q @ K.T / math.sqrt(D)
    p = torch.exp(s - s.amax(1, keepdim=True))
    if mistake == "16-bit weights":  # divided by a sum that was not rounded alike
        got = (p * 100.3).half().double() @ V / (p * 100.3).sum(1, keepdim=True)
        assert N.misses(torch, got, V, 0.0) > 10
        return
    for t in range(L):
        pt, Vt = p[t].clone(), V
        if mistake == "dropped key":
            pt[t] = 0
        elif mistake == "dropped value":
            Vt = V.clone()
            Vt[t] = 0
        elif mistake == "another's value":
            Vt = V.clone()
            Vt[t] = V[t - 1]
        total = pt.sum()
        if mistake == "twice":
            total = total + pt[t]
        got = (pt / total) @ Vt
        assert N.misses(torch, got[None].half(), V[t:t + 1], R.HALF["f16"]) > 100, t


def test_queries_of_one_part_are_found():
    """The bound of test_gpu_needles' large scores, for queries rounded once to 16 bits."""
    P = R.rotations(1, 8, "cpu")[0].double()
    q = torch.zeros(3, D, dtype=torch.float64)
    q[torch.arange(3), torch.arange(3)] = 5000.0
    s = (q @ P) / math.sqrt(D)
    rounded = (q @ P).half().double() / math.sqrt(D)
    most = 5000.0 * P.abs().max().item() / math.sqrt(D)
    bound = most * 2.0 ** -21 + 2.0 ** -20 + s.logsumexp(1).abs() * 2.0 ** -22
    assert ((rounded.logsumexp(1) - s.logsumexp(1)).abs() > 10 * bound).any()
    whole = (q @ P).float().double() / math.sqrt(D)
    assert ((whole.logsumexp(1) - s.logsumexp(1)).abs() <= bound).all()
