"""The norm's output in 8 bits, bit for bit: the scale is the greatest value of a group times 1/448 and every value is y over that scale, product and quotient as
32 bits have them, and then the nearest of e4m3. y in 32 bits is h times rstd times the weight, each product rounded once, as the kernel makes it."""
import pytest
import torch

import paper_2605_26845_b200 as ms

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def check(x, w, group, eps=1e-6, residual=None):
    res = ms.rms_norm(x, w, eps, residual=residual, group=group, save=True)
    h = res.get("sum", x).float()
    y = (h * res["rstd"][:, None]) * w.float()
    if x.dtype == torch.float32:
        assert torch.equal(y.nan_to_num(3), res["y"].nan_to_num(3))
    rows, D = y.shape
    P = -(-D // group)
    parts = torch.nn.functional.pad(y, (0, P * group - D)).view(rows, P, group)
    scale = (parts.abs().amax(-1) * torch.tensor(1 / 448, dtype=torch.float32)).clamp_min(2.0 ** -126)
    assert torch.equal(torch.isnan(scale), torch.isnan(res["scale"]))
    assert torch.equal(scale.nan_to_num(3), res["scale"].nan_to_num(3)), (scale != res["scale"]).sum()
    q = (parts / scale[..., None]).view(rows, P * group)[:, :D]
    want = q.clamp(-448, 448).to(torch.float8_e4m3fn)                       # (NaN stays)
    assert torch.equal(want.float().nan_to_num(3), res["q"].float().nan_to_num(3)), (want.float() != res["q"].float()).sum()
    signs = ~torch.isnan(want.float())                                      # (a NaN has none)
    assert torch.equal((want.view(torch.uint8) >> 7)[signs], (res["q"].view(torch.uint8) >> 7)[signs])
    return y, scale


def inputs(rows, D, dtype, seed, std=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x, r = ((torch.randn(rows, D, generator=g, device="cuda") * s).to(dtype) for s in (std, 2 * std))
    return x, r, (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,D,group", [(1, 7168, 128), (40, 1000, 32), (3000, 7168, 128), (9001, 264, 64), (30000, 72, 32), (201, 32776, 128)])
def test_scales_and_values_are_quotients_of_32_bits(rows, D, group, dtype):
    x, r, w = inputs(rows, D, TYPES[dtype], rows + D)
    check(x, w, group)
    check(x, w, group, residual=r)


def test_every_size_of_number():
    """Weights in 32 bits take y from the smallest numbers to infinity: groups of the smallest scale, of scales that are not normal times 448, and of the largest."""
    for rows in (5, 500):
        for exponent in (-149, -140, -133, -127, -126, -125, -120, -118, -117, -116, -100, -30, 0, 60, 110, 118, 119, 120, 126):
            x, _, w = inputs(rows, 520, torch.float32, exponent + 200)
            w = (w.double() * 2.0 ** exponent).float()
            check(x, w, 32)
        x, _, w = inputs(rows, 520, torch.float32, 3)
        w = (w * torch.exp2(torch.linspace(-148, 126, 520, device="cuda"))).float()
        y, scale = check(x, w, 64)
        assert (scale < 2.0 ** -115).any() and (scale > 2.0 ** 100).any()   # (the first 64 weights end at 2^-114)


def test_infinite_and_missing_values():
    x, _, w = inputs(300, 264, torch.float32, 5)
    w[::7] = 3e38
    x[:, ::7] *= 4
    y, scale = check(x, w, 32)
    assert torch.isinf(y).any() and torch.isinf(scale).any()
    w[0], x[3, 5], x[9] = float("inf"), float("nan"), 0.0
    x[11, ::2] = -0.0
    w[33] = -0.0
    check(x, w, 64)
    check(x[:9].contiguous(), w, 64)


def test_values_in_the_middle_of_two():
    """A group with 448 times a power of two in it has that power for its scale: middles of neighbouring e4m3 numbers, and 32-bit numbers next to them, are all met."""
    every = torch.arange(127, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    middle = ((every[1:] + every[:-1]) / 2).float()
    near = torch.cat([middle, torch.nextafter(middle, torch.full_like(middle, 1e9)), torch.nextafter(middle, torch.zeros_like(middle)), every.float()])
    near = torch.cat([near, -near])                                         # 1010 values
    w = torch.zeros(34 * 32, device="cuda")
    for group in range(34):
        part = near[group * 31:(group + 1) * 31]
        w[group * 32:group * 32 + part.numel()] = part
        w[group * 32 + 31] = 448
    for power in (1.0, 2.0 ** -3, 2.0 ** 40, 2.0 ** -100):
        x = torch.ones((7, 34 * 32), device="cuda")                         # of equal values: rstd is 1 with eps = 0
        y, scale = check(x, w * power, 32, eps=0.0)
        assert (scale == power).all() and torch.equal(y[0], w * power)
