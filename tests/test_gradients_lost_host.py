"""Every tensor that a call reads or writes is looked at: one that wants a gradient, or has a tangent, is refused where it would be lost. (Without a GPU.)"""
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
q, one = torch.zeros((4, 8)).to(torch.float8_e4m3fn), torch.zeros((4, 1))
rows, off, wg = torch.zeros((8, 8)), torch.zeros(2, dtype=torch.int32), torch.zeros((1, 8, 8), dtype=torch.bfloat16)
CALLS = {
    "scales of rows widened": (lambda t: ms.rows_widen(q, t, 32), one), "rows widened": (lambda t: ms.rows_widen(q, one, 32, torch.float32, out=t), x),
    "scales sent": (lambda t: ms.tokens_to_rows(x, slot, scale=t), one), "scales' rows": (lambda t: ms.tokens_to_rows(x, slot, scale=one, out_scale=t), torch.zeros((8, 1))),
    "rstd": (lambda t: ms.rms_norm_backward(x, x, w, t), r4), "y": (lambda t: ms.rms_norm(x, w, out={"y": t}), x), "scale": (lambda t: ms.rms_norm(x, w, group=32, out={"scale": t}), one),
    "dx": (lambda t: ms.rms_norm_backward(x, x, w, r4, out={"dx": t}), x), "weights": (lambda t: ms.route_choose(x, 2, out={"weights": t}), f),
    "drows": (lambda t: ms.rows_to_tokens_backward(x, rows, slot, f, out={"drows": t}), rows), "dlogits": (lambda t: ms.route_choose_backward(f, x, slot, out=t), x),
    "experts' dx": (lambda t: ms.expert_ffn_backward(wg[0], wg[0], wg, wg, wg, off, dict(gate=rows, up=rows), out=dict(dx=t, dw_gate=wg, dw_up=wg, dw_down=wg)), wg[0].clone()),
}


@pytest.mark.parametrize("name", CALLS)
def test_nothing_that_wants_a_gradient_passes(name):
    call, t = CALLS[name]
    want = t.clone().requires_grad_()
    with pytest.raises(ms.MoeschedError, match="no_grad"):
        call(want)
    with torch.no_grad(), pytest.raises(ms.MoeschedError, match="CUDA tensor"):
        call(want)
    with forward_ad.dual_level(), pytest.raises(ms.MoeschedError, match="tangent"):
        call(forward_ad.make_dual(t, torch.ones_like(t)))
    with pytest.raises(ms.MoeschedError, match="CUDA tensor"):
        call(t)
