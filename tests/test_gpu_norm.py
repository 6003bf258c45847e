"""Norm of tokens and its gradients against 64-bit arithmetic. Bounds, in half steps of 32 bits (2^-24): the sum of a row is made of at most 128 products on a
thread, 5 steps over the lanes and 32 over the warps, so its root is off by 83 at most; with the quotient, the root's own 4 and two products, 95.
Then half a step of the type."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_expert import Rounded

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = 2.0 ** -24
ROOT = 95 * U


def near(got, want, err, what):
    off = (got.double() - want).abs() - err
    assert torch.isfinite(got).all(), what
    assert (off <= 0).all(), (what, off.max().item(), (got.double() - want).abs().max().item())


def inputs(rows, D, dtype, seed, scale=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x, r, dy, dsum = ((torch.randn(rows, D, generator=g, device="cuda") * s).to(dtype) for s in (scale, 2 * scale, 1, 0.5))
    return x, r, (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype), dy, dsum


def check(rows, D, dtype, residual, group, seed=0, scale=1.0, eps=1e-6):
    x, r, w, dy, dsum = inputs(rows, D, dtype, seed, scale)
    rnd = Rounded(dtype)
    res = ms.rms_norm(x, w, eps, residual=r if residual else None, group=group, save=True)
    h = x
    if residual:
        h = res["sum"]
        near(h, x.double() + r.double(), rnd(x.double() + r.double(), U * (x.double() + r.double()).abs()), "sum")
    h64, w64 = h.double().requires_grad_(), w.double().requires_grad_()
    c = torch.rsqrt((h64 * h64).mean(-1, keepdim=True) + eps)
    y = h64 * c * w64
    near(res["rstd"], c[:, 0].detach(), ROOT * c[:, 0].detach(), "rstd")
    yd = y.detach()
    near(res["y"], yd, rnd(yd, ROOT * yd.abs()), "y")
    if group:
        check_bits(res["q"], res["scale"], yd, group)
        less = ms.rms_norm(x, w, eps, residual=r if residual else None, group=group, want_y=False)
        assert "y" not in less and torch.equal(less["q"].view(torch.uint8), res["q"].view(torch.uint8)) and torch.equal(less["scale"], res["scale"])
    for extra in (None, dsum):
        got = ms.rms_norm_backward(dy, h, w, res["rstd"], dsum=extra)
        dx, dw = torch.autograd.grad(y, (h64, w64), dy.double(), retain_graph=True)
        dx = dx if extra is None else dx + extra.double()
        g, cd, hd = (dy.double() * w.double()).abs(), c.detach(), h.double().abs()
        dot = (g * hd).sum(-1, keepdim=True) / D * cd * cd
        # c counts three times, and the sum of g h has the length of that of the squares
        err = 4 * ROOT * cd * (g + 2 * dot * hd) + 2 * U * dx.abs()
        near(got["dx"], dx, rnd(dx, err), "dx")
        size = (dy.double() * h.double() * cd).abs().sum(0)
        near(got["dweight"], dw, rnd(dw, (rows * U + 2 * ROOT) * size), "dweight")
        again = ms.rms_norm_backward(dy, h, w, res["rstd"], dsum=extra)
        assert all(torch.equal(got[k], again[k]) for k in got)


def check_bits(q, scale, y, group):
    """The scale is that of the greatest value, and every value is the nearest to what it stands for, up to the error of y."""
    rows, D = y.shape
    P = -(-D // group)
    most = torch.nn.functional.pad(y.abs(), (0, P * group - D)).view(rows, P, group).amax(-1)
    want = (most / 448).clamp_min(2.0 ** -126)
    near(scale, want, (ROOT + 2 * U) * want, "scale")
    v = y / scale.double().repeat_interleave(group, 1)[:, :D]
    lo, hi = ((v * (1 + d)).clamp(-448, 448).float().to(torch.float8_e4m3fn).float() for d in (-2 * ROOT, 2 * ROOT))
    got = q.float()
    assert ((torch.minimum(lo, hi) <= got) & (got <= torch.maximum(lo, hi))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,D", [(1, 8), (3, 16), (1, 7168), (37, 72), (300, 256), (129, 1000), (777, 1032), (40, 4096), (5, 8192), (700, 2056)])
def test_norm_and_gradients(rows, D, dtype):
    for residual in (False, True):
        for group in (None, 32, 64, 128):
            check(rows, D, TYPES[dtype], residual, group, seed=rows + D)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [16384, 16392, 32768, 32776, 65528, 65536])
def test_wide_rows(D, dtype):
    check(3, D, TYPES[dtype], True, 128, seed=D)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [295, 296, 297, 593, 5000])
def test_many_rows(rows, dtype):
    check(rows, 264, TYPES[dtype], True, 64, seed=rows)


def test_small_and_large_values():
    for scale in (1e-3, 100.0):
        check(20, 512, torch.float16, True, 128, seed=1, scale=scale)
    for scale in (1e-12, 1e8):
        check(20, 512, torch.float32, True, 128, seed=2, scale=scale, eps=0.0)
        check(20, 512, torch.bfloat16, False, 32, seed=3, scale=scale)


def test_rows_of_zeros():
    """y is 0, its groups have the smallest scale, and nothing is NaN; with eps = 0 the row is 0 times infinity."""
    for dtype in TYPES.values():
        x, w = torch.zeros((3, 136), dtype=dtype, device="cuda"), torch.ones(136, dtype=dtype, device="cuda")
        x[1] = 2.0
        res = ms.rms_norm(x, w, 1e-6, group=64, save=True)
        assert (res["y"][::2] == 0).all() and (res["q"].float()[::2] == 0).all() and (res["scale"][::2] == 2.0 ** -126).all()
        grads = ms.rms_norm_backward(torch.ones_like(x), x, w, res["rstd"])
        assert torch.isfinite(grads["dx"]).all() and torch.isfinite(grads["dweight"]).all()
        res = ms.rms_norm(x, w, 0.0, group=64)
        assert torch.isnan(res["y"][::2]).all() and torch.isfinite(res["y"][1]).all()
        assert torch.isnan(res["q"].float()[::2]).all() and torch.isnan(res["scale"][::2]).all() and torch.isfinite(res["scale"][1]).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_value_that_is_no_number_stays_in_its_row(value):
    for dtype in TYPES.values():
        x, r, w, dy, _ = inputs(9, 264, dtype, 5)
        x[4, 100] = value
        good, bad = torch.arange(9, device="cuda") != 4, 4
        res = ms.rms_norm(x, w, residual=r, group=32, save=True)
        y = res["y"].double()
        assert torch.isfinite(y[good]).all()
        wide = ms.rows_widen(res["q"], res["scale"], 32, torch.float32)
        assert torch.isfinite(wide[good]).all()
        if value != value:
            assert torch.isnan(y[bad]).all() and torch.isnan(wide[bad]).all()
        else:                                               # 1 / sqrt(inf) = 0, and 0 times infinity
            assert torch.isnan(y[bad, 100]) and torch.isnan(wide[bad, 96:128]).all() and (y[bad, :100] == 0).all()


def test_outputs_in_place_of_inputs_and_of_an_earlier_call():
    for dtype in TYPES.values():
        for D in (72, 1024, 33000):
            x, r, w, dy, dsum = inputs(33, D, dtype, 9)
            first = ms.rms_norm(x, w, residual=r, group=128, save=True)
            for name in ("x", "residual"):
                t = dict(x=x.clone(), residual=r.clone())
                into = {k: torch.full_like(v.float(), 3).to(v.dtype) for k, v in first.items()}
                into["sum"] = t[name]
                into["y"] = t["x"] if name == "residual" else into["y"]
                res = ms.rms_norm(t["x"], w, residual=t["residual"], group=128, save=True, out=into)
                assert all(res[k] is into[k] for k in res)
                for k, v in first.items():
                    assert torch.equal(res[k].view(torch.uint8), v.view(torch.uint8)), k
            want = ms.rms_norm_backward(dy, first["sum"], w, first["rstd"], dsum=dsum)
            for name in ("dy", "dsum"):
                t = dict(dy=dy.clone(), dsum=dsum.clone())
                got = ms.rms_norm_backward(t["dy"], first["sum"], w, first["rstd"], dsum=t["dsum"], out=dict(dx=t[name], dweight=torch.empty_like(w)))
                assert got["dx"] is t[name] and all(torch.equal(got[k], want[k]) for k in want)
            scratch = torch.empty(ms.norm_scratch_bytes(33, D), dtype=torch.uint8, device="cuda")
            got = ms.rms_norm_backward(dy, first["sum"], w, first["rstd"], dsum=dsum, scratch=scratch)
            assert all(torch.equal(got[k], want[k]) for k in want)


def test_the_group_is_not_looked_at_without_an_output_in_8_bits():
    x, _, w, _, _ = inputs(5, 72, torch.bfloat16, 3)
    want, y = ms.rms_norm(x, w)["y"], torch.empty_like(x)
    for group in (2 ** 31 - 1, -5, 0):
        y.zero_()
        rc = ms.load_library().moesched_rms_norm(5, 72, 0, 1e-6, group, x.data_ptr(), None, w.data_ptr(), None, y.data_ptr(), None, None, None,
                                                 torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(y, want)


def test_no_rows_and_leading_dimensions():
    x, r, w, dy, dsum = inputs(24, 64, torch.bfloat16, 4)
    none = ms.rms_norm(x[:0], w, residual=r[:0], group=32, save=True)
    assert none["y"].shape == (0, 64) and none["scale"].shape == (0, 2) and none["rstd"].shape == (0,)
    into = dict(dx=x[:0].clone(), dweight=torch.full_like(w, 5))
    assert (ms.rms_norm_backward(dy[:0], x[:0], w, none["rstd"], out=into)["dweight"] == 0).all()
    flat = ms.rms_norm(x, w, residual=r, group=32, save=True)
    deep = ms.rms_norm(x.view(2, 3, 4, 64), w, residual=r.view(2, 3, 4, 64), group=32, save=True)
    assert deep["scale"].shape == (2, 3, 4, 2) and deep["rstd"].shape == (2, 3, 4)
    for k in flat:
        assert torch.equal(flat[k].view(torch.uint8).flatten(), deep[k].view(torch.uint8).flatten()), k
    a = ms.rms_norm_backward(dy, flat["sum"], w, flat["rstd"])
    b = ms.rms_norm_backward(dy.view(2, 3, 4, 64), deep["sum"], w, deep["rstd"])
    assert torch.equal(a["dx"], b["dx"].view(24, 64)) and torch.equal(a["dweight"], b["dweight"])


def test_captured_calls_and_another_stream():
    x, r, w, dy, dsum = inputs(700, 1032, torch.bfloat16, 6)
    want = ms.rms_norm(x, w, residual=r, group=64, save=True)
    grad = ms.rms_norm_backward(dy, want["sum"], w, want["rstd"], dsum=dsum)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = ms.rms_norm(x, w, residual=r, group=64, save=True)
            got = ms.rms_norm_backward(dy, res["sum"], w, res["rstd"], dsum=dsum)
        graphs.append((graph, res, got))
    x2 = x.clone()
    x.zero_()
    for graph, _, _ in graphs:
        graph.replay()
    x.copy_(x2)
    for stream, (graph, _, _) in zip((torch.cuda.Stream(), torch.cuda.Stream()), graphs):       # both at once
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(3):
                graph.replay()
        torch.cuda.current_stream().wait_stream(stream)
    for _, res, got in graphs:
        assert all(torch.equal(res[k].view(torch.uint8), want[k].view(torch.uint8)) for k in want) and all(torch.equal(got[k], grad[k]) for k in grad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        res = ms.rms_norm(x, w, residual=r, group=64, save=True)
        got = ms.rms_norm_backward(dy, res["sum"], w, res["rstd"], dsum=dsum)
    side.synchronize()
    assert all(torch.equal(got[k], grad[k]) for k in grad)


def test_gradients_against_differences():
    """dx along a direction is the slope of <y, dy>, in 32 bits: central differences of 64-bit forward values, off by the third derivative times t^2."""
    x, r, w, dy, _ = inputs(6, 128, torch.float32, 8)
    res = ms.rms_norm(x, w, save=True)
    got = ms.rms_norm_backward(dy, x, w, res["rstd"])
    direction = torch.randn(6, 128, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))

    def value(t, u):
        h, v = x.double() + t * direction, w.double() + u * direction[0]
        return (h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * v * dy.double()).sum().item()

    t = 1e-4
    for slope, grad in (((value(t, 0) - value(-t, 0)) / (2 * t), (got["dx"].double() * direction).sum().item()),
                        ((value(0, t) - value(0, -t)) / (2 * t), (got["dweight"].double() * direction[0]).sum().item())):
        assert abs(slope - grad) <= 1e-4 * (1 + (dy.double() * direction).abs().sum().item())
