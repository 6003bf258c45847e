"""Products with 4-bit weights where a team of warps has several units of work, and where a warp has an output's whole contraction."""
import math

import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_expert import F32, SLOPE, TYPES, Rounded, act_of, close, gamma, offsets_of, quantised, spans

pytestmark = pytest.mark.gpu

WARPS = 16                          # of a CTA; one CTA an SM


def work_of(R, N, E, lengths, gated):
    """Warps that share an output, units of work and teams, by the rules that stand beside the kernel."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles, split = -(-N // (16 if gated else 32)), 1
    while split < WARPS and 2 * min(E, R) * tiles * split < WARPS * sms:
        split *= 2
    rows = [sum(lengths[e::E]) for e in range(E)]
    ctas = min(sms, -(-(R // 8 + min(E, R)) * tiles // (WARPS // split)))
    return split, sum(-(-n // 8) for n in rows) * tiles, ctas * (WARPS // split)


def expected(x, w, up, offsets, E, kind, rnd):
    for e, s in spans(offsets, E):
        v = x[s].double()
        want, err = v @ w[e].T, gamma(x.shape[1]) * (v.abs() @ w[e].abs().T)
        if kind:
            u, eu = v @ up[e].T, gamma(x.shape[1]) * (v.abs() @ up[e].abs().T)
            f, _ = act_of(want, kind)
            err = SLOPE * err * (u.abs() + eu) + f.abs() * eu + F32 * (f * u).abs() + F32 * want.abs() * u.abs()
            want = f * u
        yield s, want, rnd(want, err)


FEW = [1, 0, 3, 2, 0, 9, 1, 1, 4, 0, 2, 17, 1, 1, 0, 8, 1, 2, 3, 1, 0, 1, 25, 1, 2, 1, 1, 5, 0, 1, 4, 2]       # 100 rows of 32 experts


@pytest.mark.parametrize("gated", [None, "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("K,N,group,lengths,E,split", [
    (384, 2600, 128, FEW, 32, 1), (640, 2600, 128, FEW, 32, 1), (192, 2600, 64, FEW, 32, 1), (160, 2600, 32, FEW, 32, 1),      # 3 and 5 scales a row
    (640, 1024, 128, [3, 297], 2, 16), (384, 1024, 64, [290, 0, 3, 7], 2, 16), (416, 1601, 32, [60, 0, 1, 90, 3, 0, 0, 46], 8, 4)])
def test_several_units_for_a_team(K, N, group, lengths, E, split, dtype, gated):
    dtype, R = TYPES[dtype], sum(lengths)
    shared, units, teams = work_of(R, N, E, lengths, gated)
    if gated and split > 1:
        assert shared >= split // 2                           # (twice as many units as of the plain product)
    else:
        assert shared == split
    assert units > teams
    x = torch.randn((R, K), generator=torch.Generator("cuda").manual_seed(K), device="cuda").to(dtype)
    q, scale, w = quantised(E, N, K, group, dtype, N)
    up = quantised(E, N, K, group, dtype, N + 1) if gated else (None, None, None)
    offsets, status = offsets_of(lengths), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    y = ms.expert_matvec4(x, q, scale, offsets, up[0], up[1], act=gated or "silu", status=status)
    assert status.item() == 0
    for s, want, err in expected(x, w, up[2], offsets, E, gated, Rounded(dtype)):
        close(y[s], want, err, "y")


def test_4_bit_rows_beside_rows_that_are_not_finite():
    """Rows outside the groups hold NaN; those inside have their values all the same."""
    for R, first, lengths, K in ((30, 4, [6, 9], 256), (90, 11, [60, 1], 384)):
        n = sum(lengths)
        x = torch.full((R, K), math.nan, dtype=torch.bfloat16, device="cuda")
        x[first:first + n] = torch.randn((n, K), generator=torch.Generator("cuda").manual_seed(R), device="cuda").bfloat16()
        q, scale, w = quantised(2, 40, K, 64, torch.bfloat16, 3)
        offsets = offsets_of(lengths, first=first)
        y = ms.expert_matvec4(x, q, scale, offsets, out=torch.full((R, 40), 7.0, dtype=torch.bfloat16, device="cuda"))
        assert (y[:first] == 7).all() and (y[first + n:] == 7).all()
        for s, want, err in expected(x, w, None, offsets, 2, None, Rounded(torch.bfloat16)):
            close(y[s], want, err, "y")
