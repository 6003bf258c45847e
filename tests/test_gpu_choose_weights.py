"""Weights of the choice and their gradients are as exact as 32-bit arithmetic makes them, however far apart the logits are. Logits are multiples of 1/16, so that their differences
are exact. In steps of 2^-23: an exponential is 2 off at most, a sum, a product or a quotient half of one.
  logistic, alone        1 / (1 + e): 2 + 1/2 + 1/2, and the factor: 3.5
  softmax, alone         e / sum: 2, and 2 + 7/2 for a sum of up to 8, quotient and factor: 8.5
  softmax, normalised    the same over the chosen: 8.5
  logistic, normalised   e^(l - m) / (1 + e^l): 2 + 1 + 1, both in the sum and above it, 7/2, quotient and factor: 12.5
  gradients              two of the weights, the quotient by 1 + e^l (3.5), and products: twice the above and 7, of the sizes of what is added"""
import pytest
import torch

import paper_2605_26845_b200 as ms

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23
STEPS = {("sigmoid", False): 3.5, ("softmax", False): 8.5, ("softmax", True): 8.5, ("sigmoid", True): 12.5}


def logits(T, E, low, high, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(16 * low, 16 * high + 1, (T, E), generator=g, device="cuda").float() / 16


def exact(l, experts, score, normalise, factor, dw):
    """Weights, gradients of the logits and the sizes of what these are sums of, in 64 bits."""
    l = l.double()
    p = torch.softmax(l, -1) if score == "softmax" else torch.special.expit(l)
    other = torch.special.expit(-l)                                         # 1 - p of the logistic function
    chosen = torch.zeros_like(l).scatter_(1, experts, 1.0)
    a = torch.zeros_like(l).scatter_(1, experts, factor * dw.double())
    if normalise:
        log = l if score == "softmax" else torch.nn.functional.logsigmoid(l)
        q = torch.softmax(log.masked_fill(chosen == 0, -1e9), -1) * chosen
        d, size = q * (a - (a * q).sum(-1, keepdim=True)), q * (a.abs() + (a.abs() * q).sum(-1, keepdim=True))
        if score == "sigmoid":
            d, size = d * other, size * other
        return factor * torch.gather(q, 1, experts), d, size
    if score == "softmax":
        return factor * torch.gather(p, 1, experts), p * (a - (a * p).sum(-1, keepdim=True)), p * (a.abs() + (a.abs() * p).sum(-1, keepdim=True))
    return factor * torch.gather(p, 1, experts), a * p * other, (a * p * other).abs()


@pytest.mark.parametrize("score,normalise", STEPS)
@pytest.mark.parametrize("T,E,k", [(2000, 2, 2), (2000, 2, 1), (500, 8, 8), (500, 8, 3), (7, 5, 2)])
@pytest.mark.parametrize("low,high", [(-2, 2), (-20, -20), (-21, 0), (-80, -1), (-40, 40), (5, 80)])
def test_weights_and_gradients_of_32_bits(T, E, k, low, high, score, normalise):
    l = logits(T, E, low, high, T + E + high)
    for bias in (None, torch.linspace(1, 0, E, device="cuda") * 4):         # (the first experts, whatever their logits)
        got = ms.route_choose(l, k, score=score, bias=bias, normalise=normalise, factor=1.25)
        experts = got["experts"].view(T, k).long()
        g = torch.Generator("cuda").manual_seed(3)
        dw = torch.randn((T, k), generator=g, device="cuda")
        w, d, size = exact(l, experts, score, normalise, 1.25, dw)
        steps, tiny = STEPS[score, normalise] * STEP, 2.0 ** -125            # (and numbers below the normal ones)
        off = (got["weights"].view(T, k).double() - w).abs() - (steps * w + tiny)
        assert (off <= 0).all(), ((got["weights"].view(T, k).double() - w).abs() / w / STEP).max()
        have = ms.route_choose_backward(dw.view(-1), l, got["experts"], score=score, normalise=normalise, factor=1.25).double()
        off = (have - d).abs() - ((2 * steps + 7 * STEP) * size + tiny)
        assert (off <= 0).all(), ((have - d).abs() / size / STEP).nan_to_num(0).max()


@pytest.mark.parametrize("score,normalise", STEPS)
@pytest.mark.parametrize("E", [60, 256, 1024])
def test_rows_of_many_experts(E, score, normalise):
    """As above with sums of up to 32 on a lane and over 32 lanes: 36 additions, 18 steps; of the eight chosen 7 / 2."""
    l = logits(300, E, -30, 10, E)
    got = ms.route_choose(l, 8, score=score, normalise=normalise, factor=1.25)
    experts = got["experts"].view(300, 8).long()
    g = torch.Generator("cuda").manual_seed(3)
    dw = torch.randn((300, 8), generator=g, device="cuda")
    w, d, size = exact(l, experts, score, normalise, 1.25, dw)
    steps = (STEPS[score, normalise] + (14.5 if score == "softmax" and not normalise else 0)) * STEP
    assert ((got["weights"].view(300, 8).double() - w).abs() <= steps * w + 2.0 ** -125).all()
    have = ms.route_choose_backward(dw.view(-1), l, got["experts"], score=score, normalise=normalise, factor=1.25).double()
    assert ((have - d).abs() <= (2 * steps + 7 * STEP) * size + 2.0 ** -125).all()
