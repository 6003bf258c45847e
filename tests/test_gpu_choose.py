"""The router's choice and its gradient against 64-bit arithmetic. Experts have to be equal. Bounds of the weights, in steps of 2^-23: an exponential is 2 off and
its argument, which is at most `span` in size, half a step of that; sums have 32 terms on a lane and 5 steps over the lanes, so a quotient of them is off by span + 60."""
import math

import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_expert import Rounded

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
STEP = 2.0 ** -23
WAYS = [(score, normalise) for score in ("softmax", "sigmoid") for normalise in (False, True)]


def reference(logits, k, score, bias, normalise, factor):
    """Experts, and weights as a function of the 64-bit logits (for autograd)."""
    l = logits.double().requires_grad_()
    off = logits.isnan() | (logits == -math.inf)
    rank = l.detach()
    if bias is not None:
        rank = (torch.softmax(l.detach().masked_fill(off, -math.inf), -1).nan_to_num(0) if score == "softmax" else torch.special.expit(l.detach())) + bias.double()
    rank = rank.masked_fill(off, -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True)
    there = best.values[:, :k] > -math.inf
    experts = best.indices[:, :k]
    safe = torch.where(off, -1e4, l)
    picked = torch.where(there, torch.gather(safe, 1, experts), -1e4)
    if score == "softmax":
        p = torch.softmax(picked, -1) if normalise else torch.gather(torch.softmax(safe, -1), 1, experts)
    elif normalise:
        p = torch.softmax(torch.nn.functional.logsigmoid(picked), -1)
    else:
        p = torch.special.expit(picked)
    weights = factor * torch.where(there, p, 0.0)
    return torch.where(there, experts, -1).int(), weights, l


def check(logits, k, score, normalise, bias=None, factor=1.0, dweights=None):
    T, E = logits.shape
    got = ms.route_choose(logits, k, score=score, bias=bias, normalise=normalise, factor=factor)
    experts, weights, l = reference(logits, k, score, bias, normalise, factor)
    assert torch.equal(got["experts"].view(T, k), experts), (got["experts"].view(T, k) != experts).nonzero()[:4]
    finite = logits.double().nan_to_num(0, 0, 0)
    span = 2 * finite.abs().amax(-1, keepdim=True)
    w = weights.detach()
    tiny = 1e-36 * max(1.0, abs(factor))                    # (numbers below the normal ones)
    off = (got["weights"].view(T, k).double() - w).abs() - (w.abs() * (span + 64) * STEP + tiny)
    assert (off <= 0).all(), off.max()
    g = torch.Generator("cuda").manual_seed(T * E + k)
    dw = torch.randn((T, k), generator=g, device="cuda") if dweights is None else dweights
    d = ms.route_choose_backward(dw.view(-1), logits, got["experts"], score=score, normalise=normalise, factor=factor)
    want, = torch.autograd.grad(weights, l, dw.double())
    # every term of the gradient is a weight times a dw, or a score times a weight times a dw; each counts the errors of both
    size = (w * dw.double()).abs()
    total = size.sum(-1, keepdim=True)
    dense = torch.softmax(finite.masked_fill(logits == -math.inf, -math.inf), -1).nan_to_num(0) * total if score == "softmax" and not normalise else torch.zeros_like(finite)
    own = torch.zeros_like(finite).scatter_add_(1, experts.clamp_min(0).long(), size + (w.abs() / max(abs(factor), 1e-30)) * total)
    err = 4 * (span + 64) * STEP * (dense + own) + tiny
    off = (d.double() - want).abs() - Rounded(logits.dtype)(want, err)
    assert (off <= 0).all(), off.max()
    assert torch.isfinite(d).all()
    return got


def logits_of(T, E, dtype, seed, scale=1.5):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn((T, E), generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 2), (3, 8, 1), (17, 31, 5), (9, 32, 32), (33, 33, 3), (50, 60, 6), (16, 256, 8), (7, 64, 8), (5, 128, 4), (11, 160, 7),
                                   (6, 257, 9), (4, 512, 32), (8, 1023, 10), (3, 1024, 32), (1000, 64, 2)])
def test_choices_weights_and_gradients(T, E, k, dtype):
    l = logits_of(T, E, TYPES[dtype], T + E)
    g = torch.Generator("cuda").manual_seed(E)
    bias = torch.randn(E, generator=g, device="cuda") * 0.1
    for score, normalise in WAYS:
        check(l, k, score, normalise, factor=2.5)
        check(l, k, score, normalise, bias=bias)


@pytest.mark.parametrize("score,normalise", WAYS)
def test_ties_go_to_the_lowest_expert(score, normalise):
    g = torch.Generator("cuda").manual_seed(3)
    for E in (10, 40, 256, 1000):
        few = torch.randint(-1, 2, (200, E), generator=g, device="cuda").float()
        few[few == 0] *= -1                                                       # -0 and 0 are equal
        few[::2][few[::2] == 0] = 0.0
        check(few, min(E, 12), score, normalise)
        check(few, min(E, 12), score, normalise, bias=torch.zeros(E, device="cuda"))
        check(torch.full((5, E), 0.75, device="cuda"), 7, score, normalise, bias=torch.full((E,), -0.25, device="cuda"))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_that_32_bits_do_not_tell_apart(score):
    """Logits a step apart, and biases that undo the difference of the scores up to less than a step: the order is that of 64 bits."""
    g = torch.Generator("cuda").manual_seed(4)
    for E in (8, 64, 300):
        l = 1.0 + torch.randint(0, 4, (400, E), generator=g, device="cuda").float() * 2.0 ** -23
        check(l, 6, score, True, bias=torch.zeros(E, device="cuda"))
        l = torch.randn((1, E), generator=g, device="cuda").expand(100, E) + torch.randint(0, 3, (100, E), generator=g, device="cuda") * 2.0 ** -22
        s = torch.softmax(l[0].double(), -1) if score == "softmax" else torch.special.expit(l[0].double())
        check(l.contiguous(), 6, score, False, bias=(0.5 - s).float())
    big = torch.linspace(20, 60, 40, device="cuda").expand(3, 40).contiguous()     # logistic functions that are all 1 in 32 bits
    check(big, 5, score, True)
    check(big, 5, score, True, bias=torch.zeros(40, device="cuda"))


@pytest.mark.parametrize("score,normalise", WAYS)
def test_experts_that_are_switched_off(score, normalise):
    for E, k in ((6, 4), (64, 8), (200, 8)):
        l = logits_of(60, E, torch.float32, E)
        l[0] = -math.inf                                                        # padding
        l[1, 1:] = -math.inf
        l[2, :-2] = -math.inf
        l[3] = torch.finfo(torch.float32).min                                   # a mask of the lowest number leaves all of them equal
        l[4, ::2] = torch.finfo(torch.float32).min
        l[5:20][torch.rand(15, E, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) < 0.9] = -math.inf
        rest = l.clone()
        rest[3:5] = 0
        for bias in (None, torch.linspace(-0.5, 0.5, E, device="cuda")):
            got = check(rest, k, score, normalise, bias=bias)
            assert (got["experts"][:k] == -1).all() and (got["weights"][:k] == 0).all()
            got = ms.route_choose(l, k, score=score, bias=bias, normalise=normalise)
            assert (got["experts"].view(60, k)[3:5] >= 0).all() and torch.isfinite(got["weights"]).all()
        got = ms.route_choose(l, k, score=score, normalise=normalise)
        assert got["experts"][3 * k:4 * k].tolist() == list(range(k))
        if score == "softmax":
            assert torch.allclose(got["weights"][3 * k:4 * k], torch.full((k,), 1 / (k if normalise else E), device="cuda"), rtol=1e-6)
        closed = torch.zeros(E, device="cuda")
        closed[1:] = -math.inf                                                  # a bias closes all experts but one
        got = ms.route_choose(rest, 2, score=score, bias=closed, normalise=normalise)
        assert (got["experts"].view(60, 2)[:, 1] == -1).all() and set(got["experts"].view(60, 2)[:, 0].tolist()) == {-1, 0}


def test_one_normalised_choice_has_the_factor_for_its_weight_and_no_gradient():
    for scale in (0.1, 3.0, 40.0):
        l = logits_of(300, 60, torch.float32, 5, scale)
        for score in ("softmax", "sigmoid"):
            got = ms.route_choose(l, 1, score=score, normalise=True, factor=2.5)
            assert (got["weights"] == 2.5).all()
            assert (ms.route_choose_backward(torch.randn(300, device="cuda"), l, got["experts"], score=score, normalise=True, factor=2.5) == 0).all()


def test_logits_that_are_no_numbers():
    l = logits_of(8, 40, torch.float32, 2)
    l[1, 7], l[2] = math.nan, math.nan
    for score, normalise in WAYS:
        for bias in (None, torch.zeros(40, device="cuda")):
            got = ms.route_choose(l, 5, score=score, bias=bias, normalise=normalise)
            e, w = got["experts"].view(8, 5), got["weights"].view(8, 5)
            assert torch.isnan(w[1:3]).all() and not (e[1] == 7).any()
            assert (e[1] >= 0).all() or (score == "softmax" and bias is not None)      # (scores are NaN then: nobody)
            assert (e[2] == -1).all() and torch.isfinite(w[0]).all() and torch.isfinite(w[3:]).all()
    l[1:3] = 0
    l[1, 7] = math.inf
    got = ms.route_choose(l, 5, score="sigmoid")
    assert got["experts"].view(8, 5)[1, 0] == 7 and got["weights"].view(8, 5)[1, 0] == 1
    got = ms.route_choose(l, 5)
    assert got["experts"].view(8, 5)[1, 0] == 7 and torch.isnan(got["weights"].view(8, 5)[1]).all()      # as the softmax of infinity is
    assert torch.isfinite(got["weights"].view(8, 5)[2:]).all()


@pytest.mark.parametrize("normalise", [False, True])
def test_logits_far_from_zero(normalise):
    for score in ("softmax", "sigmoid"):
        l = logits_of(50, 64, torch.float32, 7, scale=30.0)
        check(l, 8, score, normalise)
        check(l - 200, 8, score, normalise)
        check(l + 200, 8, score, normalise)
        low = torch.zeros(64, device="cuda")
        low[:8] = 2.0                                                           # the bias chooses experts far below the greatest
        l[:, :8] = l[:, :8] - 120
        check(l, 8, score, normalise, bias=low)


def test_layouts_streams_and_graphs():
    l = logits_of(24, 60, torch.float32, 9)
    flat = ms.route_choose(l, 3)
    deep = ms.route_choose(l.view(2, 3, 4, 60), 3)
    assert deep["experts"].shape == deep["weights"].shape == (2, 3, 12)
    assert torch.equal(deep["experts"].flatten(), flat["experts"]) and torch.equal(deep["weights"].flatten(), flat["weights"])
    into = {k: torch.full_like(v, 3) for k, v in flat.items()}
    assert ms.route_choose(l, 3, out=into)["experts"] is into["experts"] and torch.equal(into["weights"], flat["weights"])
    none = ms.route_choose(l[:0], 3)
    assert none["experts"].shape == (0,) and ms.route_choose_backward(none["weights"], l[:0], none["experts"]).shape == (0, 60)
    odd = torch.zeros(1 + 24 * 60, device="cuda", dtype=torch.bfloat16)[1:].view(24, 60)         # starts within a word
    odd.copy_(l)
    assert torch.equal(ms.route_choose(odd, 3)["experts"], ms.route_choose(odd.clone(), 3)["experts"])
    dw = torch.randn(72, device="cuda")
    want = ms.route_choose_backward(dw, l, flat["experts"])
    assert torch.equal(ms.route_choose_backward(dw.view(2, 3, 12), l.view(2, 3, 4, 60), flat["experts"].view(2, 3, 12)).view(24, 60), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = ms.route_choose(l, 3)
        got = ms.route_choose_backward(dw, l, res["experts"])
    graph.replay()
    assert torch.equal(res["experts"], flat["experts"]) and torch.equal(got, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ms.route_choose_backward(dw, l, ms.route_choose(l, 3)["experts"])
    side.synchronize()
    assert torch.equal(got, want)


def test_experts_that_nobody_chose_have_no_gradient():
    l = logits_of(4, 20, torch.float32, 1)
    experts = torch.tensor([3, -1, 25, 7, -1, -1, 0, 19], dtype=torch.int32, device="cuda")     # (25 is no expert)
    dw = torch.ones(8, device="cuda")
    for score in ("softmax", "sigmoid"):
        d = ms.route_choose_backward(dw, l, experts, score=score, normalise=score == "softmax")
        kept = torch.zeros((4, 20), dtype=torch.bool, device="cuda")
        kept[0, 3] = kept[1, 7] = kept[3, 0] = kept[3, 19] = True
        assert (d[~kept] == 0).all()
