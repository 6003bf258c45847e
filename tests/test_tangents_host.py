"""Tensors with a tangent of autograd's forward mode are refused by the calls that autograd does not know: the tangent would be lost without a sign. (Without a GPU: tensors
without one are refused for where they are.)"""
import pytest
import torch
from torch.autograd import forward_ad

import __graft_entry__ as entry
import paper_2605_26845_b200 as ms


@pytest.fixture(scope="module", autouse=True)
def lib():
    entry.build()
    return ms.load_library()


x, w, slot, f, r4 = torch.zeros((4, 8)), torch.zeros(8), torch.zeros(8, dtype=torch.int32), torch.zeros(8), torch.zeros(4)
off, wg = torch.zeros(2, dtype=torch.int32), torch.zeros((1, 8, 8), dtype=torch.bfloat16)
xb, w4, s4 = x.bfloat16(), torch.zeros((1, 8, 4), dtype=torch.uint8), torch.zeros((1, 8, 1), dtype=torch.bfloat16)
SAVED = dict(gate=x, up=x)
CALLS = {
    "norm": (lambda t: ms.rms_norm(t, w), x), "norm weight": (lambda t: ms.rms_norm(x, t), w), "norm residual": (lambda t: ms.rms_norm(x, w, residual=t), x),
    "norm gradients": (lambda t: ms.rms_norm_backward(t, x, w, r4), x), "choice": (lambda t: ms.route_choose(t, 2), x), "bias": (lambda t: ms.route_choose(x, 2, bias=t), f),
    "choice gradients": (lambda t: ms.route_choose_backward(t, x, slot), f), "send": (lambda t: ms.tokens_to_rows(t, slot), x),
    "back": (lambda t: ms.rows_to_tokens(t, slot[:4], 2), x), "back weights": (lambda t: ms.rows_to_tokens(x, slot[:4], 2, weights=t), r4),
    "back gradients": (lambda t: ms.rows_to_tokens_backward(t, torch.zeros((8, 8)), slot, f), x),
    "experts": (lambda t: ms.expert_ffn(t, wg, wg, wg, off), xb), "experts' weights": (lambda t: ms.expert_ffn(xb, t, wg, wg, off), wg),
    "experts' gradients": (lambda t: ms.expert_ffn_backward(t, xb, wg, wg, wg, off, SAVED), xb), "4 bits": (lambda t: ms.expert_matvec4(t, w4, s4, off), xb),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_tangent_is_refused(name):
    call, t = CALLS[name]
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(t, torch.ones_like(t))
        for mode in (torch.enable_grad, torch.no_grad):                     # (no_grad does not turn forward mode off)
            with mode(), pytest.raises(ms.MoeschedError, match="tangent"):
                call(dual)
        with pytest.raises(ms.MoeschedError, match="CUDA tensor"):
            call(forward_ad.unpack_dual(dual).primal)
        with pytest.raises(ms.MoeschedError, match="CUDA tensor"):          # one of its own level, but without a tangent
            call(t)
        with forward_ad._set_fwd_grad_enabled(False), pytest.raises(ms.MoeschedError, match="CUDA tensor"):       # as within an autograd function
            call(dual)
    with pytest.raises(ms.MoeschedError, match="CUDA tensor"):
        call(dual)                                                          # the level is over
