"""Tokens whose softmax is none, since a logit is infinite or NaN, do not pass for padding: they choose, and their weights are NaN, with a bias or without."""
import pytest
import torch

import paper_2605_26845_b200 as ms

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
WAYS = [(score, normalise, biased) for score in ("softmax", "sigmoid") for normalise in (False, True) for biased in (False, True)]


@pytest.mark.parametrize("score,normalise,biased", WAYS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_an_infinite_logit_does_not_pass_for_padding(score, normalise, biased, dtype):
    """The softmax of infinity is NaN; the logistic function of it is 1."""
    for E, k in ((4, 4), (40, 5), (256, 8), (1000, 32)):
        g = torch.Generator("cuda").manual_seed(E)
        l = torch.randn((9, E), generator=g, device="cuda").to(dtype)
        l[2, 3], l[5, 1:3], l[7] = INF, INF, -INF
        l[8, 1:], l[8, 0] = -INF, INF
        bias = torch.linspace(-0.1, 0.1, E, device="cuda") if biased else None
        got = ms.route_choose(l, k, score=score, bias=bias, normalise=normalise)
        e, w = got["experts"].view(9, k), got["weights"].view(9, k)
        fine, broken = torch.tensor([0, 1, 3, 4, 6], device="cuda"), torch.tensor([2, 5, 8], device="cuda")
        assert torch.isfinite(w[fine]).all() and (e[fine] >= 0).all() and (e[7] == -1).all() and (w[7] == 0).all()
        assert (e[broken[:2]] >= 0).all() and e[8, 0] == 0 and (e[8, 1:] == -1).all()
        assert all(len(set(row.tolist())) == k for row in e[[0, 1, 2, 3, 4, 5, 6]])
        if score == "softmax":
            assert torch.isnan(w[broken]).all()
        else:
            assert torch.isfinite(w[broken]).all() and w[8, 0] == 1
        if score == "softmax" or not biased:                                # by the logits, whatever the bias
            assert e[2, 0] == 3 and e[5, :2].tolist() == [1, 2]
            order = torch.sort(l[2].float(), descending=True, stable=True).indices[:k]
            assert torch.equal(e[2].long(), order)
        d = ms.route_choose_backward(torch.ones(9 * k, device="cuda"), l, got["experts"], score=score, normalise=normalise)
        assert torch.isfinite(d[fine]).all() and (d[7] == 0).all()
        if score == "sigmoid":
            assert torch.isfinite(d).all()
        elif normalise:                                                     # of the chosen alone
            assert torch.isnan(d[2, 3]) and torch.isnan(d[5, 1:3]).all() and torch.isnan(d[8, 0])
        else:                                                               # (experts that are switched off have no gradient)
            assert torch.equal(torch.isnan(d[broken]), l[broken] > -INF) and (d[8, 1:] == 0).all()


@pytest.mark.parametrize("score,normalise,biased", WAYS)
def test_a_logit_that_is_none_does_not_pass_for_padding(score, normalise, biased):
    """It is not chosen itself, and neither is an expert that the bias closes."""
    for E, k in ((5, 3), (64, 6), (700, 9)):
        g = torch.Generator("cuda").manual_seed(E)
        l = torch.randn((4, E), generator=g, device="cuda")
        l[1, 2], l[2, 1], l[2, 4] = NAN, NAN, INF
        l[3] = 0.5                                                          # (more than 32 equal ones)
        l[3, 0] = NAN
        bias = torch.zeros(E, device="cuda") if biased else None
        if biased:
            bias[0] = -INF
        got = ms.route_choose(l, k, score=score, bias=bias, normalise=normalise)
        e, w = got["experts"].view(4, k), got["weights"].view(4, k)
        assert (e >= 0).all() and torch.isfinite(w[0]).all() and torch.isnan(w[1:]).all()
        assert not (e[1] == 2).any() and not (e[2] == 1).any() and e[2, 0] == 4 and e[3].tolist() == list(range(1, k + 1))
        if biased:
            assert not (e == 0).any()


def test_a_broken_token_shows_where_its_rows_come_back():
    l = torch.zeros((6, 16), device="cuda")
    l[2, 5] = INF
    c = ms.route_choose(l, 2, bias=torch.zeros(16, device="cuda"))
    slot = ms.route_demand(c["experts"].view(1, 1, -1), 16)["slot"].view(-1)
    x = torch.ones((6, 64), dtype=torch.bfloat16, device="cuda")
    y = ms.rows_to_tokens(ms.tokens_to_rows(x, slot), slot, 2, weights=c["weights"], add=x)
    assert torch.isnan(y[2]).all() and torch.isfinite(y[[0, 1, 3, 4, 5]]).all()
