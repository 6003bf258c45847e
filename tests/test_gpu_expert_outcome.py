"""What a call of the experts leaves behind when its offsets are out of order: NaN in every output, whether or not anybody asked for the
status. So nothing that was there before, or comes from uninitialised memory, passes for a result."""
import time

import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_expert import inputs, offsets_of, quantised

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


def wrong(R, groups):
    """Offsets of that many groups with one wrong entry each."""
    good = torch.linspace(0, R, groups + 1).int()
    for at, value in ((0, -1), (groups // 2, R + 1), (groups, R + 1), (groups // 2, -5), (groups, 2 ** 31 - 1)):
        o = good.clone()
        o[at] = value
        yield o.cuda()
    if groups > 1:
        yield good.flip(0).cuda()


def lost(tensors):
    return all(torch.isnan(t).all() for t in tensors)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,D,I,E,groups", [(20, 64, 72, 2, 2), (9, 8, 8, 1, 3), (300, 72, 40, 2, 4), (3001, 512, 384, 2, 4), (700, 64, 64, 40, 3000)])
def test_blocks_with_offsets_out_of_order(R, D, I, E, groups, dtype):
    x, wg, wu, wd, dy = inputs(R, D, I, E, dtype, R)
    good = offsets_of([R // groups] * groups)
    y, saved = ms.expert_ffn(x, wg, wu, wd, good, save=True)
    assert not torch.isnan(y[:groups * (R // groups)]).any()
    grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, good, saved)
    for offsets in wrong(R, groups):
        status = torch.full((1,), 5, dtype=torch.int32, device="cuda")
        out = torch.full_like(x, 7.0)
        bad, kept = ms.expert_ffn(x, wg, wu, wd, offsets, save=True, out=out, status=status)
        assert status.item() == ms.ST_BAD_INPUT and lost([bad, kept["gate"], kept["up"]]), offsets
        assert lost([ms.expert_ffn(x, wg, wu, wd, offsets, act="gelu")])
        into = {k: torch.full_like(v, 7.0) for k, v in grads.items()}
        status.fill_(5)
        ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved, out=into, status=status)
        assert status.item() == ms.ST_BAD_INPUT and lost(into.values()), offsets
    again, saved2 = ms.expert_ffn(x, wg, wu, wd, good, save=True)
    rows = groups * (R // groups)
    assert torch.equal(again[:rows], y[:rows])
    for k, v in ms.expert_ffn_backward(dy, x, wg, wu, wd, good, saved2).items():
        assert torch.equal(v[:rows], grads[k][:rows]) if k == "dx" else torch.equal(v, grads[k])


def test_offsets_that_name_rows_where_there_are_none():
    x, wg, wu, wd, dy = inputs(0, 64, 72, 3, torch.bfloat16, 1)
    saved = {k: torch.zeros((0, 72), device="cuda") for k in ("gate", "up")}
    for last, status in ((0, ms.ST_OK), (2, ms.ST_BAD_INPUT), (-1, ms.ST_BAD_INPUT)):
        got = torch.full((1,), 5, dtype=torch.int32, device="cuda")
        offsets = torch.tensor([0, 0, 0, last], dtype=torch.int32, device="cuda")
        assert ms.expert_ffn(x, wg, wu, wd, offsets, status=got).shape == (0, 64) and got.item() == status
        grads = ms.expert_ffn_backward(dy, x, wg, wu, wd, offsets, saved, status=got)
        assert got.item() == status
        for k in ("dw_gate", "dw_up", "dw_down"):
            assert (torch.isnan(grads[k]) if status else grads[k] == 0).all(), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K,N,E,groups", [(1, 64, 1, 1, 1), (7, 128, 33, 2, 2), (60, 192, 501, 3, 6), (41, 64, 8, 600, 1200)])
def test_4_bit_products_with_offsets_out_of_order(R, K, N, E, groups, dtype):
    x = torch.randn((R, K), device="cuda").to(dtype)
    (q, scale, _), (up, up_scale, _) = quantised(E, N, K, 32, dtype, 1), quantised(E, N, K, 32, dtype, 2)
    for offsets in wrong(R, groups):
        for second in ((None, None), (up, up_scale)):
            beyond = torch.full((R * N + 64,), 7.0, dtype=dtype, device="cuda")
            out = beyond[:R * N].view(R, N)
            ms.expert_matvec4(x, q, scale, offsets, *second, out=out)
            assert lost([out]) and (beyond[R * N:] == 7.0).all(), offsets


def test_results_are_seen_by_deterministic_mode_and_by_dispatch_modes():
    """Rows that no group has are undefined in a tensor made by the call; deterministic mode fills them (with NaN), and a dispatch mode sees
    the allocations."""
    from torch.utils._python_dispatch import TorchDispatchMode

    seen = []

    class Watching(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(func)
            return func(*args, **(kwargs or {}))

    x, wg, wu, wd, _ = inputs(40, 64, 72, 1, torch.bfloat16, 5)
    offsets = offsets_of([20], first=7)
    want = ms.expert_ffn(x, wg, wu, wd, offsets)[7:27]
    held = [torch.full_like(x, 3.0) for _ in range(4)]
    del held                                              # (what the next allocations of that size find)
    torch.use_deterministic_algorithms(True)
    try:
        y = ms.expert_ffn(x, wg, wu, wd, offsets)
    finally:
        torch.use_deterministic_algorithms(False)
    assert torch.isnan(y[:7]).all() and torch.isnan(y[27:]).all() and torch.equal(y[7:27], want)
    with Watching():
        y = ms.expert_ffn(x, wg, wu, wd, offsets)
    assert torch.ops.aten.empty_strided.default in seen and torch.equal(y[7:27], want)


def test_a_probe_times_the_gpu_and_not_the_host(monkeypatch):
    """Calls that take the host two milliseconds each leave the times of batches as they are; weights that are parameters are taken."""
    E, D, I = 2, 256, 128
    _, wg, wu, wd, _ = inputs(1, D, I, E, torch.bfloat16, 30)
    pairs = [quantised(E, n, k, 64, torch.bfloat16, n)[:2] for n, k in ((I, D), (I, D), (D, I))]
    call = ms._call

    def slow(name, *args):
        time.sleep(0.002)
        return call(name, *args)

    monkeypatch.setattr(ms, "_call", slow)
    before = torch.cuda.memory_allocated()
    for weights in ([torch.nn.Parameter(w) for w in (wg, wu, wd)], pairs):
        ns = ms.probe_expert(weights, tokens=(1, 8, 300), reps=5)["ns"]
        assert all(0 < t < 1e6 for t in ns), ns
    assert torch.cuda.memory_allocated() - before < 1 << 20
